// What the two attention kernels over pages share: arguments, the order of the work, the fold of partial results, and codes.
#pragma once

#include "segkv_pages_internal.h"
#include "segkv_ptx.cuh"

namespace segkv_impl {
namespace pages {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f;
// A column's weights are taken relative to a reference that is only moved when a score exceeds it by 2^kSlack.
constexpr float kSlack = 8.f;

struct Params {
    const char* q;
    long long q_stride;              // bytes
    char* out;
    const char *kp, *vp;
    const int32_t *table, *lens;
    const float* slopes;
    float* ws;
    int* tickets;
    int* err;
    int table_stride, n, q_len, H, Hkv, group, page_log, num_pages;
    int cols, ctiles;                // query columns of a (sequence, kv head), tiles of them
};

// ---- 4-bit rows: codes as fp16, whatever the dtype ----------------------------------------------------------------------------
// Two codes of a word, in bits 0-3 and 16-19, become fp16 numbers by or-ing them into 1024 (whose last place is 1); codes in bits 4-7 and
// 20-23 count 16.  An fp16 product takes them exactly, so the queries (scaled by a power of two per column) and the weights are
// fp16 for a bf16 cache too: 11 bits instead of 8, and half the shifts.
constexpr uint32_t kMagic = 0x64006400u;
constexpr float kLift4 = 6.f;
// (w & mask) | magic in one instruction
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(kMagic));
    return r;
}
__device__ __forceinline__ uint32_t codes_lo(uint32_t w) { return and_or(w, 0x000F000Fu); }          // 1024 + c
__device__ __forceinline__ uint32_t codes_hi(uint32_t w) { return and_or(w, 0x00F000F0u); }          // 1024 + 16 c
__device__ __forceinline__ uint32_t centred_lo(uint32_t w) {                                         // c - 8
    const uint32_t x = codes_lo(w), k = 0x64086408u;                                                 // 1032
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&k));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t centred_hi(uint32_t w) {                                         // (1024 + 16 c) / 16 - 72
    const uint32_t x = codes_hi(w), m = 0x2C002C00u, k = 0xD480D480u;
    const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&m), *reinterpret_cast<const __half2*>(&k));
    return *reinterpret_cast<const uint32_t*>(&r);
}
struct Cursor {                      // a block of keys in the grid's order
    int v, h, b, nb, klen;
    const int32_t* row;              // the sequence's pages
};

// Keys that column tile ct of sequence s reads, and how many blocks that makes (at least one: an empty sequence's output is written too).
template <int NC, int KB>
__device__ __forceinline__ void extent(const Params& p, int v, int* klen, int* nb, bool flag) {
    const int s = v / p.ctiles, ct = v - s * p.ctiles;
    const int most = (int)min((long long)p.table_stride << p.page_log, 0x7FFFFFFFLL);
    int len = __ldg(p.lens + s);
    if (len < 0 || len > most) {
        if (flag) atomicOr(p.err, SEGKV_DEV_BAD_PAGE);
        len = len < 0 ? 0 : most;
    }
    const int last = min(p.cols, (ct + 1) * NC) - 1;
    int k = len - p.q_len + last / p.group + 1;
    k = k < 0 ? 0 : k;
    *klen = k;
    *nb = k > KB ? (k + KB - 1) / KB : 1;
}

template <int NC, int KB>
__device__ __forceinline__ void enter(const Params& p, Cursor& c) {
    extent<NC, KB>(p, c.v, &c.klen, &c.nb, false);
    c.row = p.table + (long long)(c.v / p.ctiles) * p.table_stride;
}
template <int NC, int KB>
__device__ __forceinline__ void advance(const Params& p, Cursor& c, int V) {
    if (++c.b < c.nb) return;
    c.b = 0;
    if (++c.h < p.Hkv) return;
    c.h = 0;
    if (++c.v < V) enter<NC, KB>(p, c);
}

// A CTA's run of blocks: block x of all `total` is CTA c's where total*c/G <= x < total*(c+1)/G.
struct Run {
    Cursor first;
    unsigned long long x0, total;
    int V, G, blocks;
};

// By all threads of the CTA, WARPS warps of them; false (for all) where there is nothing to do.  s_scan: WARPS numbers, s_found: three.
template <int NC, int KB, int WARPS>
__device__ __forceinline__ bool find_run(const Params& p, long long* s_scan, int* s_found, Run& r) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    r.V = p.n * p.ctiles;
    r.G = gridDim.x;
    const int per = (r.V + 32 * WARPS - 1) / (32 * WARPS);
    long long mine = 0;
    const int v0 = min(tid * per, r.V), v1 = min(v0 + per, r.V);
    int klen, nb;
    for (int v = v0; v < v1; ++v) {
        extent<NC, KB>(p, v, &klen, &nb, cta == 0);
        mine += nb;
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    long long before = incl - mine, all = 0;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) before += s_scan[w];
        all += s_scan[w];
    }
    r.total = (unsigned long long)all * p.Hkv;
    if (r.total < (unsigned long long)r.G) r.G = (int)r.total;      // every CTA of a shared work group has to have a part
    if (cta >= r.G) return false;
    r.x0 = r.total * cta / r.G;
    r.blocks = (int)(r.total * (cta + 1) / r.G - r.x0);
    unsigned long long at = (unsigned long long)before * p.Hkv;
    if (mine > 0 && r.x0 >= at && r.x0 < at + (unsigned long long)mine * p.Hkv) {
        for (int v = v0;; ++v) {
            extent<NC, KB>(p, v, &klen, &nb, false);
            const unsigned long long size = (unsigned long long)nb * p.Hkv;
            if (r.x0 < at + size) {
                const unsigned rest = (unsigned)(r.x0 - at);
                s_found[0] = v;
                s_found[1] = (int)(rest / (unsigned)nb);
                s_found[2] = (int)(rest % (unsigned)nb);
                break;
            }
            at += size;
        }
    }
    __syncthreads();
    r.first.v = s_found[0];
    r.first.h = s_found[1];
    r.first.b = s_found[2];
    enter<NC, KB>(p, r.first);
    return true;
}

// floats of a partial result: NC columns of D values, their references (powers of two), their sums
template <int D, int NC> constexpr int kSlot = NC * (D + 2);

// The parts of a work group, left by CTAs c0 (in its second slot) to c1 (in their first), into the output: by 128 threads, a column of
// eight by 16 of them at a time, with the loads of several parts in flight together.
template <typename T, int D, int NC>
__device__ __forceinline__ void fold_parts(const Params& p, int s, int ct, int h, int c0, int c1, int tid) {
    constexpr int AT = D == 256 ? 4 : 8, SLOT = kSlot<D, NC>;
    const int mcol = tid >> 4, mloc = (tid & 15) * 4, parts = c1 - c0 + 1;
#pragma unroll
    for (int nt = 0; nt < (NC + 7) / 8; ++nt) {
        const int lcol = nt * 8 + mcol, col = ct * NC + lcol;
        if (NC < 8 && lcol >= NC) break;
        float top = -INFINITY, sum = 0.f;
        float4 acc[D / 64];
#pragma unroll
        for (int r = 0; r < D / 64; ++r) acc[r] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int i0 = 0; i0 < parts; i0 += AT) {
            float m[AT], l[AT];
            float4 v[AT][D / 64];
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                m[i] = -INFINITY;
                l[i] = 0.f;
#pragma unroll
                for (int r = 0; r < D / 64; ++r) v[i][r] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i0 + i >= parts) continue;
                const float* src = p.ws + ((size_t)(c0 + i0 + i) * 2 + (i0 + i == 0 ? 1 : 0)) * SLOT;
                m[i] = __ldcg(src + NC * D + lcol);
                l[i] = __ldcg(src + NC * D + NC + lcol);
#pragma unroll
                for (int r = 0; r < D / 64; ++r) v[i][r] = __ldcg(reinterpret_cast<const float4*>(src + lcol * D + 64 * r + mloc));
            }
            float mx = top;
#pragma unroll
            for (int i = 0; i < AT; ++i) mx = fmaxf(mx, m[i]);
            const float keep = top == -INFINITY ? 1.f : exp2f(top - mx);
            sum *= keep;
#pragma unroll
            for (int r = 0; r < D / 64; ++r) {
                acc[r].x *= keep; acc[r].y *= keep; acc[r].z *= keep; acc[r].w *= keep;
            }
            top = mx;
#pragma unroll
            for (int i = 0; i < AT; ++i) {
                const float fi = m[i] == -INFINITY ? 1.f : exp2f(m[i] - mx);        // (no weight: zeros, or NaN)
                sum = fmaf(l[i], fi, sum);
#pragma unroll
                for (int r = 0; r < D / 64; ++r) {
                    acc[r].x = fmaf(v[i][r].x, fi, acc[r].x);
                    acc[r].y = fmaf(v[i][r].y, fi, acc[r].y);
                    acc[r].z = fmaf(v[i][r].z, fi, acc[r].z);
                    acc[r].w = fmaf(v[i][r].w, fi, acc[r].w);
                }
            }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (col < p.cols) {
            const int row = col / p.group, hq = h * p.group + (col - row * p.group);
#pragma unroll
            for (int r = 0; r < D / 64; ++r) {
                uint2 w2;
                w2.x = Mma<T>::pack(acc[r].x * inv, acc[r].y * inv);
                w2.y = Mma<T>::pack(acc[r].z * inv, acc[r].w * inv);
                *reinterpret_cast<uint2*>(p.out + ((((size_t)s * p.q_len + row) * p.H + hq) * D + 64 * r + mloc) * 2) = w2;
            }
        }
    }
}

}  // namespace pages
}  // namespace segkv_impl
