// Attention over 4-bit pages on the fifth-generation tensor cores, for work that fills the GPU: the same work groups, runs of blocks and
// folds as in segkv_pages_sdpa.cu, one CTA per SM, blocks of 128 keys.
//
// What the warp-level kernel spends its time on is instructions: 3.5 for every code.  Here a code costs about 1.3, of them 0.1 for its
// store: eight warps turn the codes of a tile, and nothing else, into fp16 numbers c - 8 in shared memory, and scales and
// zero points never meet a code one by one:
//   * scores: S^T[128 keys, 4 groups x columns] = C_K . Q^T, where the columns of Q are the query's channels of ONE group each (zeros
//     elsewhere), so that the sum over groups of scale * S is left to the softmax, where a thread owns a key and has its four scales in
//     registers.  (M 128, N = 4 columns, so a few columns cost nothing more.)
//   * values: O^T[128 channels, 4 groups x columns] += C_V^T . P^T with the weights times each group's scale as columns (one rounding); a
//     channel's row takes its own group's column at the end and leaves the other three.  The zero points' part, sum of p * z, is
//     summed per key's thread in fp32 and added at the end.
// Codes are exact in fp16 whatever the dtype; queries are scaled by a power of two per column, scales by a power of two that only grows, as
// in the warp-level kernel, so that fp16 holds them.
//
// Order of channels: eight codes of a word come out as (0, 4, 1, 5, 2, 6, 3, 7), which is the order that the tiles keep.  Q is laid out the
// same way, and the output's rows are put right when they leave.
//
// Roles: warps 0-3 softmax (a key per thread; then a channel per thread for the output), warps 4-11 expand, warp 12 issues the MMAs.  The
// expanding and the softmax threads copy what they will read themselves (codes, scales) with cp.async, kRing tiles ahead, so that
// nobody else has to be told.  K has one tile, freed when Q.K^T has read it, V two (one at head_dim 256), S two buffers
// in tensor memory.  Every wait is bounded; when one runs out the kernel sets SEGKV_DEV_WAIT_LIMIT, leaves the output and ends.
#include <atomic>

#include "segkv_pages_sdpa.cuh"
#include "segkv_tc5.cuh"

namespace segkv_impl {
namespace {

using namespace pages;

constexpr int kSoft = 4, kExpand = 8, kWarps = kSoft + kExpand + 1, kThreads = 32 * kWarps;
constexpr int kKeys = 128;
constexpr int kBlock = kKeys * 128;                           // 64 channels of a tile's keys: 128 bytes a key, swizzled
constexpr int kTmem = 256;

template <int D, int NCOL> struct Lay {
    static constexpr int N = 4 * NCOL;
    static constexpr int CH = D / 32, IT = CH / 2;            // 16-byte chunks of a row's codes; chunks of a tile for each expanding thread
    static constexpr int BLK = D / 64, TILE = BLK * kBlock;
    static constexpr int VS = D == 256 ? 1 : 2;               // V tiles
    static constexpr int RING = D == 256 ? 2 : 4;             // tiles that are copied ahead
    static constexpr int RAW = 2 * IT * kExpand * 32 * 16;    // a tile's codes, K then V
    static constexpr int SCALES = 2 * kKeys * 16;
    // V first: at head_dim 64 its product reads 64 channels more than there are, which have to be somewhere
    static constexpr int oV = 0, oK = oV + VS * TILE, oQ = oK + (TILE < kBlock * 2 ? kBlock * 2 : TILE), oP = oQ + BLK * N * 128;
    static constexpr int oRaw = oP + 2 * N * 128, oScales = oRaw + RING * RAW, oCols = oScales + RING * SCALES;
    static constexpr int COLS = NCOL * (16 + 8 * 4) + kSoft * NCOL * 5 * 4 + 256;      // see the kernel
    static constexpr int oBars = oCols + COLS;
    static constexpr int BYTES = oBars + 16 * 8 + 16 + kWarps * 8 + 32;
    static constexpr int SMEM = BYTES > 120 * 1024 ? BYTES : 120 * 1024;               // never two CTAs with tensor memory on an SM
    static_assert(BYTES <= 232448, "shared memory");
    static_assert(2 * N + (D == 256 ? 2 : 1) * N <= kTmem, "tensor memory");
};

__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 lds128v(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a) : "memory");
    return r;
}
__device__ __forceinline__ void sts16(uint32_t a, uint32_t x) { asm volatile("st.shared.b16 [%0], %1;" ::"r"(a), "h"((uint16_t)x) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool real) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename T> constexpr int kExpShift = 10;
template <> constexpr int kExpShift<__nv_bfloat16> = 7;
template <typename T> constexpr int kExpBias = 15;
template <> constexpr int kExpBias<__nv_bfloat16> = 127;

// the channel that stands at place i of a word of eight, and its group
__device__ __forceinline__ int channel_of(int i) { return (i & ~7) + ((i & 1) << 2) + ((i & 7) >> 1); }

template <typename T, int D, int NCOL>
__global__ void __launch_bounds__(kThreads, 1) pages_tc5_kernel(const __grid_constant__ Params p) {
    using L = Lay<D, NCOL>;
    using M = Mma<T>;
    constexpr int N = L::N, IT = L::IT, RB = D / 2, VS = L::VS, R = L::RING;
    extern __shared__ __align__(1024) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, cta = blockIdx.x;
    const uint32_t base = smem_u32(smem);
    // columns: sums of q by group [NCOL][4], then {scale2, exponent of the reference}, {reference, what moves it}, slope, lim, rescale
    float* s_qsum = reinterpret_cast<float*>(smem + L::oCols);
    float2* s_sb = reinterpret_cast<float2*>(s_qsum + 4 * NCOL);
    float* s_mref = reinterpret_cast<float*>(s_sb + NCOL);
    float* s_thr = s_mref + NCOL;
    float* s_slope = s_thr + NCOL;
    int* s_lim = reinterpret_cast<int*>(s_slope + NCOL);
    float* s_al = reinterpret_cast<float*>(s_lim + NCOL);
    float* s_spare = s_al + NCOL;
    float* s_red = s_spare + NCOL;                            // [warp][NCOL][5]
    int* s_top = reinterpret_cast<int*>(s_red + kSoft * NCOL * 5);
    const uint32_t bars = base + L::oBars;
    const uint32_t kfull = bars, kempty = bars + 8, vfull = bars + 16, vempty = bars + 32, sfull = bars + 48, pfull = bars + 64, qfull = bars + 72, bend = bars + 80;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::oBars + 128);
    volatile int& s_abort = *reinterpret_cast<volatile int*>(tmem_slot + 1);
    long long* s_scan = reinterpret_cast<long long*>(smem + L::oBars + 144);
    int* s_misc = reinterpret_cast<int*>(s_scan + kWarps);

    if (tid == 0) {
        mbar_init(kfull, kExpand);
        mbar_init(kempty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(vfull + 8 * i, kExpand);
            mbar_init(vempty + 8 * i, 1);
            mbar_init(sfull + 8 * i, 1);
        }
        mbar_init(pfull, kSoft);
        mbar_init(qfull, kSoft);
        mbar_init(bend, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_proxy_async();
    }
    if (warp == kSoft + kExpand) {                            // this warp owns the tensor memory
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "n"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;                         // S buffers at columns 0 and N, O behind them
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    Run run;
    const bool busy = find_run<NCOL, kKeys, kWarps>(p, s_scan, s_misc, run);           // (the same for every thread)
    const uint32_t ps = 1u << p.page_log;
    const uint32_t head_bytes = ps * (uint32_t)(RB + 16);
    const unsigned long long page_bytes = (unsigned long long)head_bytes * p.Hkv;
    const unsigned long long limit = kWaitLimitNs;
    auto page_at = [&](int pid) -> unsigned long long {
        if ((unsigned)pid >= (unsigned)p.num_pages) {
            atomicOr(p.err, SEGKV_DEV_BAD_PAGE);
            pid = 0;
        }
        return (unsigned long long)(uint32_t)pid * page_bytes;
    };

    if (busy && warp >= kSoft && warp < kSoft + kExpand) {
        // --------------------------------------- expand ---------------------------------------
        // A lane has a row's chunk of 16 bytes; eight neighbouring lanes have eight rows, so that what they store lies in eight different
        // places of the swizzle.
        const int ew = warp - kSoft;
        int row[IT], ch[IT];
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            row[i] = D == 64 ? ew * 16 + (lane & 7) + 8 * (lane >> 4) : ((D == 256 ? i >> 1 : i) * kExpand + ew) * 8 + (lane & 7);
            ch[i] = D == 64 ? (lane >> 3) & 1 : D == 128 ? lane >> 3 : (i & 1) * 4 + (lane >> 3);
        }
        const uint32_t raw = base + L::oRaw + (ew * 32 + lane) * 16;
        Cursor ld = run.first;
        int pid[IT], copied = 0;
        auto find_pages = [&]() {
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int key = ld.b * kKeys + row[i];
                pid[i] = 0;
                if (key < ld.klen) pid[i] = __ldg(ld.row + (key >> p.page_log));
            }
        };
        auto copy_tile = [&](int slot) {
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int key = ld.b * kKeys + row[i];
                const bool real = key < ld.klen;
                unsigned long long at = 0;
                if (real) at = page_at(pid[i]) + (uint32_t)ld.h * head_bytes + ((uint32_t)key & (ps - 1)) * RB + ch[i] * 16;
                const uint32_t dst = raw + slot * L::RAW + i * (kExpand * 32 * 16);
                copy16(dst, p.kp + at, real);
                copy16(dst + IT * (kExpand * 32 * 16), p.vp + at, real);
            }
            commit_copies();
        };
        auto next = [&](int slot) {
            if (copied < run.blocks) {
                copy_tile(slot);
                if (++copied < run.blocks) {
                    advance<NCOL, kKeys>(p, ld, run.V);
                    find_pages();
                }
            } else {
                commit_copies();
            }
        };
        find_pages();
        for (int i = 0; i < R; ++i) next(i);
        // a chunk's four words to 64 bytes of fp16 numbers
        auto expand = [&](uint32_t tile, const uint4 (&x)[IT]) {
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
                const uint32_t to = tile + (ch[i] >> 1) * kBlock + row[i] * 128;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t h8 = w[j] >> 8;
                    sts128(to + (((((ch[i] & 1) * 4 + j) ^ (row[i] & 7))) << 4), centred_lo(w[j]), centred_hi(w[j]), centred_lo(h8), centred_hi(h8));
                }
            }
        };
        bool ok = true;
        int slot = 0;
        for (int i = 0; i < run.blocks && ok; ++i) {
            wait_copies<R - 1>();
            uint4 xk[IT], xv[IT];
            const uint32_t src = raw + slot * L::RAW;
#pragma unroll
            for (int c = 0; c < IT; ++c) {
                xk[c] = lds128v(src + c * (kExpand * 32 * 16));
                xv[c] = lds128v(src + (IT + c) * (kExpand * 32 * 16));
            }
            if (i > 0) ok = mbar_wait_hot(kempty, (i - 1) & 1, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            expand(base + L::oK, xk);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(kfull);
            next(slot);                                       // (this thread has read its part of the slot)
            slot = slot + 1 == R ? 0 : slot + 1;
            const int vs = VS == 2 ? i & 1 : 0;
            if (i >= VS) ok = mbar_wait_hot(vempty + 8 * vs, VS == 2 ? ((i >> 1) - 1) & 1 : (i - 1) & 1, limit);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            expand(base + L::oV + vs * L::TILE, xv);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(vfull + 8 * vs);
        }
        if (!ok) s_abort = 1;
        wait_copies<0>();
    } else if (busy && warp == kSoft + kExpand) {
        // ---------------------------------------- MMAs ----------------------------------------
        const uint32_t lead = elect_one();
        auto wait = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait_hot(bar, parity, limit)); };
        constexpr uint32_t common = (1u << 4) | ((uint32_t)(kKeys >> 4) << 24) | ((uint32_t)(N >> 3) << 17);       // fp32 sums, fp16, M 128
        constexpr uint32_t id_qk = common, id_pv = common | (1u << 15);                                            // V^T: its channels run along the rows
        const uint64_t dk = smem_desc(base + L::oK, 16, 1024), dq = smem_desc(base + L::oQ, 16, 1024);
        const uint64_t dv = smem_desc(base + L::oV, kBlock, 1024), dp = smem_desc(base + L::oP, 16, 1024);
        Cursor cur = run.first;
        bool ok = true;
        uint32_t i = 0, seg = 0;
        auto scores = [&](uint32_t t) -> bool {               // S(t) = C_K . Q^T
            if (!wait(kfull, t & 1)) return false;
            tc_fence_after();
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                tc_mma_ss_if(lead, tmem + (t & 1) * N, dk + (uint64_t)(((ks >> 2) * kBlock + (ks & 3) * 32) >> 4),
                             dq + (uint64_t)(((ks >> 2) * (N * 128) + (ks & 3) * 32) >> 4), id_qk, ks > 0);
            tc_commit_if(lead, sfull + 8 * (t & 1));
            tc_commit_if(lead, kempty);
            return true;
        };
        for (int done = 0; done < run.blocks && ok; ++seg) {
            const int count = min(cur.nb - cur.b, run.blocks - done);
            ok = wait(qfull, seg & 1);                        // the group's queries are there
            if (!ok) break;
            tc_fence_after();
            ok = scores(i);
            for (int t = 0; t < count && ok; ++t, ++i) {
                if (t + 1 < count && !(ok = scores(i + 1))) break;                     // the next tile's scores run under this one's softmax
                const uint32_t vs = VS == 2 ? i & 1 : 0;
                ok = wait(vfull + 8 * vs, VS == 2 ? (i >> 1) & 1 : i & 1) && wait(pfull, i & 1);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int hh = 0; hh < (D == 256 ? 2 : 1); ++hh)
#pragma unroll
                    for (int kk = 0; kk < kKeys / 16; ++kk)
                        tc_mma_ss_if(lead, tmem + 2 * N + hh * N, dv + (uint64_t)((vs * L::TILE + hh * 2 * kBlock + kk * 2048) >> 4),
                                     dp + (uint64_t)(((kk >> 2) * (N * 128) + (kk & 3) * 32) >> 4), id_pv, t > 0 || kk > 0);
                tc_commit_if(lead, vempty + 8 * vs);
            }
            done += count;
            cur.b += count - 1;
            if (done < run.blocks) advance<NCOL, kKeys>(p, cur, run.V);
        }
        if (!ok && lane == 0) s_abort = 1;
    } else if (busy) {
        // --------------------------------------- softmax ---------------------------------------
        constexpr float kScale2 = D == 64 ? kLog2e * 0.125f : D == 128 ? kLog2e * 0.08838834764831845f : kLog2e * 0.0625f;
        const uint32_t tm_lane = tmem + ((uint32_t)(warp * 32) << 16);
        const uint32_t scales = base + L::oScales + tid * 16;
        Cursor ld = run.first, cur = run.first;
        int pid = 0, copied = 0;
        auto find_page = [&]() {
            const int key = ld.b * kKeys + tid;
            pid = 0;
            if (key < ld.klen) pid = __ldg(ld.row + (key >> p.page_log));
        };
        auto next = [&](int slot) {
            if (copied < run.blocks) {
                const int key = ld.b * kKeys + tid;
                const bool real = key < ld.klen;              // (a key that does not exist has scales of zero and stands for 0)
                unsigned long long at = 0;
                if (real) at = page_at(pid) + (uint32_t)ld.h * head_bytes + ps * RB + ((uint32_t)key & (ps - 1)) * 16;
                copy16(scales + slot * L::SCALES, p.kp + at, real);
                copy16(scales + slot * L::SCALES + kKeys * 16, p.vp + at, real);
                if (++copied < run.blocks) {
                    advance<NCOL, kKeys>(p, ld, run.V);
                    find_page();
                }
            }
            commit_copies();
        };
        find_page();
        for (int i = 0; i < R; ++i) next(i);
        // this thread's place in the weights: key tid of rows n (its chunk of eight keys turned by n & 7)
        const uint32_t p_at = base + L::oP + (tid >> 6) * (N * 128) + (tid & 7) * 2, p_ch = (tid & 63) >> 3;
        bool ok = true;
        int slot = 0;
        uint32_t i = 0;
        unsigned long long x = run.x0;
        for (int done = 0; done < run.blocks;) {
            const int s = cur.v / p.ctiles, ct = cur.v - s * p.ctiles;
            const int count = min(cur.nb - cur.b, run.blocks - done);
            const bool whole = count == cur.nb;
            const int first_row = ct * NCOL / p.group, last_row = (min(p.cols, (ct + 1) * NCOL) - 1) / p.group;
            const int pos0 = cur.klen - 1 - last_row;         // position of row 0; below 0 where the sequence is shorter than q_len
            // ---- the group's queries: four rows a column, the channels of a group each, in the order of the tiles ------------------------
            constexpr int PC = D / 8;                         // threads of a column: eight channels each
#pragma unroll
            for (int it = 0; it < (NCOL * PC + 127) / 128; ++it) {
                const int item = it * 128 + tid;
                if (item >= NCOL * PC) break;                 // (whole warps)
                const int lcol = item / PC, c8 = item % PC, col = ct * NCOL + lcol;
                const bool real = col < p.cols;
                const int row = real ? col / p.group : first_row, hq = cur.h * p.group + (real ? col - row * p.group : 0);
                uint4 r = make_uint4(0u, 0u, 0u, 0u);
                if (real) r = __ldg(reinterpret_cast<const uint4*>(p.q + ((long long)s * p.q_len + row) * p.q_stride + (size_t)hq * (2 * D) + c8 * 16));
                const float2 e01 = M::unpack(r.x), e23 = M::unpack(r.y), e45 = M::unpack(r.z), e67 = M::unpack(r.w);
                float lo[4] = {e01.x, e01.y, e23.x, e23.y}, hi[4] = {e45.x, e45.y, e67.x, e67.y};
                float big = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) big = fmaxf(big, fmaxf(fabsf(lo[j]), fabsf(hi[j])));
#pragma unroll
                for (int o = 1; o < PC; o <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
                const int ex = min(max(__float_as_int(big) >> 23, 1), 253);
                const float down = big > 0.f ? __int_as_float((254 - ex) << 23) : 1.f, unit = big > 0.f ? __int_as_float(ex << 23) : 1.f;
                float sum[4];
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    w[j] = Mma<__half>::pack(lo[j] * down, hi[j] * down);
                    const float2 f = Mma<__half>::unpack(w[j]);
                    sum[j] = f.x + f.y;
                }
#pragma unroll
                for (int o = 1; o < PC; o <<= 1)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = lcol * 4 + j;
                    sts128(base + L::oQ + (c8 >> 3) * (N * 128) + n * 128 + (((c8 & 7) ^ (n & 7)) << 4), j == 0 ? w[0] : 0u, j == 1 ? w[1] : 0u,
                           j == 2 ? w[2] : 0u, j == 3 ? w[3] : 0u);
                }
                if (c8 == 0) {
                    *reinterpret_cast<float4*>(s_qsum + 4 * lcol) = make_float4(sum[0], sum[1], sum[2], sum[3]);
                    const float sc = kScale2 * unit;
                    s_sb[lcol] = make_float2(sc, 0.f);
                    s_mref[lcol] = s_thr[lcol] = -INFINITY;
                    s_slope[lcol] = p.slopes && real ? __ldg(p.slopes + hq) * kLog2e / sc : 0.f;
                    s_lim[lcol] = pos0 + row + 1;
                }
            }
            fence_proxy_async();
            bar_sync_n(1, 128);
            if (lane == 0) mbar_arrive(qfull);
            const int free_to = pos0 + first_row + 1;         // keys below it are seen by every row
            float l[NCOL], zacc[NCOL][4];
#pragma unroll
            for (int c = 0; c < NCOL; ++c) {
                l[c] = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) zacc[c][j] = 0.f;
            }
            int vexp = 0;
            bool gone = false;
            for (int blk = 0; blk < count; ++blk, ++i) {
                const int key0 = (cur.b + blk) * kKeys, key = key0 + tid;
                wait_copies<R - 1>();
                const uint4 ks = lds128v(scales + slot * L::SCALES), vs = lds128v(scales + slot * L::SCALES + kKeys * 16);
                next(slot);
                slot = slot + 1 == R ? 0 : slot + 1;
                if (ok) ok = mbar_wait_hot(sfull + 8 * (i & 1), (i >> 1) & 1, limit);
                ok = __all_sync(0xffffffffu, ok);
                float c[NCOL];
                {
                    tc_fence_after();
                    const float2 s0 = M::unpack(ks.x), s1 = M::unpack(ks.y), z0 = M::unpack(ks.z), z1 = M::unpack(ks.w);
#pragma unroll
                    for (int c4 = 0; c4 < NCOL; c4 += 4) {
                        uint32_t r[16];
                        tc_ld16(tm_lane + (i & 1) * N + 4 * c4, r);
                        tc_wait_ld();
                        pin<16>(r);
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const float4 qs = *reinterpret_cast<const float4*>(s_qsum + 4 * (c4 + u));
                            float v = fmaf(z0.x, qs.x, fmaf(z0.y, qs.y, fmaf(z1.x, qs.z, z1.y * qs.w)));
                            v = fmaf(s0.x, __uint_as_float(r[4 * u]), v);
                            v = fmaf(s0.y, __uint_as_float(r[4 * u + 1]), v);
                            v = fmaf(s1.x, __uint_as_float(r[4 * u + 2]), v);
                            c[c4 + u] = fmaf(s1.y, __uint_as_float(r[4 * u + 3]), v);
                        }
                    }
                }
                if (p.slopes)
#pragma unroll
                    for (int u = 0; u < NCOL; ++u) c[u] = fmaf(s_slope[u], (float)(key + 1 - s_lim[u]), c[u]);
                if (key0 + kKeys > free_to)
#pragma unroll
                    for (int u = 0; u < NCOL; ++u)
                        if (key >= s_lim[u]) c[u] = -INFINITY;
                // the values' largest scale, as an exponent; what the scales are taken relative to only grows
                uint32_t big = __vmaxu2(vs.x, vs.y);
                big = max(big & 0xFFFFu, big >> 16) >> kExpShift<T>;
                const int top = (int)min(big, (0x7FFFu >> kExpShift<T>) - 1);
                bool grow = !ok || top > vexp;
#pragma unroll
                for (int u = 0; u < NCOL; ++u) grow |= c[u] > s_thr[u];
                // P and O are free once the product before this one is done
                if (i > 0 && ok) ok = mbar_wait_hot(vempty + (VS == 2 ? 8 * ((i - 1) & 1) : 0), VS == 2 ? ((i - 1) >> 1) & 1 : (i - 1) & 1, limit);
                ok = __all_sync(0xffffffffu, ok);
                grow |= !ok;
                if (!bar_and(1, 128, !grow)) {
                    // ---- new references, by all four warps --------------------------------------------------------------------------------
                    gone = !bar_and(1, 128, ok);
                    if (gone) break;
#pragma unroll
                    for (int u = 0; u < NCOL; ++u) {
                        float mx = c[u];
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                        if (lane == 0) s_red[warp * NCOL + u] = mx;
                    }
                    const int wtop = (int)__reduce_max_sync(0xffffffffu, (unsigned)top);
                    if (lane == 0) s_top[warp] = wtop;
                    bar_sync_n(1, 128);
                    if (tid < NCOL) {
                        const float was = s_mref[tid], sc = s_sb[tid].x;
                        float mx = was;
#pragma unroll
                        for (int w = 0; w < kSoft; ++w) mx = fmaxf(mx, s_red[w * NCOL + tid]);
                        if (!(mx > s_thr[tid])) mx = was;     // (this column stays)
                        s_al[tid] = was == -INFINITY ? 1.f : exp2f((was - mx) * sc);
                        s_mref[tid] = mx;
                        s_thr[tid] = mx + kSlack / sc;
                        s_sb[tid].y = mx == -INFINITY ? 0.f : mx * sc - kLift4;
                    }
                    const int now = max(max(vexp, s_top[0]), max(max(s_top[1], s_top[2]), s_top[3]));
                    const float down = __int_as_float(max(127 + vexp - now, 0) << 23);
                    vexp = now;
                    bar_sync_n(1, 128);
#pragma unroll
                    for (int u = 0; u < NCOL; ++u) {
                        const float al = s_al[u];
                        l[u] *= al;
#pragma unroll
                        for (int j = 0; j < 4; ++j) zacc[u][j] *= al;
                    }
                    if (blk > 0) {
                        tc_fence_after();
#pragma unroll 1
                        for (int n0 = 0; n0 < (D == 256 ? 2 : 1) * N; n0 += 16) {
                            uint32_t r[16];
                            tc_ld16(tm_lane + 2 * N + n0, r);
                            tc_wait_ld();
                            pin<16>(r);
#pragma unroll
                            for (int u = 0; u < 16; ++u) r[u] = __float_as_uint(__uint_as_float(r[u]) * (s_al[((n0 & (N - 1)) + u) >> 2] * down));
                            tc_st16(tm_lane + 2 * N + n0, r);
                        }
                        tc_wait_st();
                    }
                }
                // ---- weights ------------------------------------------------------------------------------------------------------------
                {
                    const float unit = __int_as_float((127 + kExpBias<T> - vexp) << 23);
                    const float2 s0 = M::unpack(vs.x), s1 = M::unpack(vs.y), z0 = M::unpack(vs.z), z1 = M::unpack(vs.w);
                    const float su[4] = {s0.x * unit, s0.y * unit, s1.x * unit, s1.y * unit}, zz[4] = {z0.x, z0.y, z1.x, z1.y};
#pragma unroll
                    for (int u = 0; u < NCOL; ++u) {
                        const float2 sb = s_sb[u];
                        const float w = exp2f(fmaf(c[u], sb.x, -sb.y));
                        l[u] += w;
#pragma unroll
                        for (int j = 0; j < 4; ++j) zacc[u][j] = fmaf(w, zz[j], zacc[u][j]);
                        const uint32_t a = Mma<__half>::pack(w * su[0], w * su[1]), b = Mma<__half>::pack(w * su[2], w * su[3]);
                        const int n = 4 * u;
                        sts16(p_at + n * 128 + ((p_ch ^ (n & 7)) << 4), a);
                        sts16(p_at + (n + 1) * 128 + ((p_ch ^ ((n + 1) & 7)) << 4), a >> 16);
                        sts16(p_at + (n + 2) * 128 + ((p_ch ^ ((n + 2) & 7)) << 4), b);
                        sts16(p_at + (n + 3) * 128 + ((p_ch ^ ((n + 3) & 7)) << 4), b >> 16);
                    }
                }
                fence_proxy_async();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(pfull);
            }
            if (gone) break;
            // ---- the work group's end: the last product, then a channel per thread ---------------------------------------------------------
            if (ok) ok = mbar_wait_hot(vempty + (VS == 2 ? 8 * ((i - 1) & 1) : 0), VS == 2 ? ((i - 1) >> 1) & 1 : (i - 1) & 1, limit);
            ok = __all_sync(0xffffffffu, ok);
#pragma unroll
            for (int u = 0; u < NCOL; ++u) {
                float v[5] = {l[u], zacc[u][0], zacc[u][1], zacc[u][2], zacc[u][3]};
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                    for (int j = 0; j < 5; ++j) v[j] += __shfl_xor_sync(0xffffffffu, v[j], o);
                if (lane == 0)
#pragma unroll
                    for (int j = 0; j < 5; ++j) s_red[(warp * NCOL + u) * 5 + j] = v[j];
            }
            gone = !bar_and(1, 128, ok);
            if (gone) break;
            tc_fence_after();
            const unsigned long long gbase = x - (unsigned)cur.b;
            const int c0 = whole ? cta : (int)(((gbase + 1) * run.G - 1) / run.total);
            const int c1 = whole ? cta : (int)(((gbase + cur.nb) * run.G - 1) / run.total);
            float* part = p.ws + ((size_t)cta * 2 + (cta == c0 ? 1 : 0)) * kSlot<D, NCOL>;
            const float up = __int_as_float((127 + vexp - kExpBias<T>) << 23);
            const int j4 = (tid & 7) >> 1;                    // this channel's group
            if (D > 64 || tid < 64) {
#pragma unroll 1
                for (int hh = 0; hh < (D == 256 ? 2 : 1); ++hh) {
                    const int d = channel_of(hh * 128 + tid);
#pragma unroll
                    for (int c4 = 0; c4 < NCOL; c4 += 4) {
                        uint32_t r[16];
                        tc_ld16(tm_lane + 2 * N + hh * N + 4 * c4, r);
                        tc_wait_ld();
                        pin<16>(r);
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int lcol = c4 + u, col = ct * NCOL + lcol;
                            const float own = __uint_as_float(j4 & 2 ? (j4 & 1 ? r[4 * u + 3] : r[4 * u + 2]) : (j4 & 1 ? r[4 * u + 1] : r[4 * u]));
                            float zs = 0.f, ls = 0.f;
#pragma unroll
                            for (int w = 0; w < kSoft; ++w) {
                                ls += s_red[(w * NCOL + lcol) * 5];
                                zs += s_red[(w * NCOL + lcol) * 5 + 1 + j4];
                            }
                            const float v = fmaf(own, up, zs);
                            if (whole) {
                                if (col < p.cols) {
                                    const int row = col / p.group, hq = cur.h * p.group + (col - row * p.group);
                                    const float o = ls == 0.f ? 0.f : v / ls;
                                    *reinterpret_cast<T*>(p.out + ((((size_t)s * p.q_len + row) * p.H + hq) * D + d) * 2) = M::down(o);
                                }
                            } else {
                                part[lcol * D + d] = v;
                                if (tid == 0 && hh == 0) {
                                    part[NCOL * D + lcol] = s_mref[lcol] == -INFINITY ? -INFINITY : s_mref[lcol] * s_sb[lcol].x;
                                    part[NCOL * D + NCOL + lcol] = ls;
                                }
                            }
                        }
                    }
                }
            }
            tc_fence_before();
            bar_sync_n(1, 128);                               // (columns and sums are the next group's, too)
            if (!whole) {
                if (tid == 0) {
                    __threadfence();                          // (the CTA's writes, behind the barrier above)
                    s_misc[0] = atomicAdd(p.tickets + c0, 1);
                    __threadfence();
                }
                bar_sync_n(1, 128);
                if (s_misc[0] == c1 - c0) {
                    if (tid == 0) p.tickets[c0] = 0;
                    fold_parts<T, D, NCOL>(p, s, ct, cur.h, c0, c1, tid);
                }
                bar_sync_n(1, 128);
            }
            done += count;
            x += (unsigned)count;
            cur.b += count - 1;
            if (done < run.blocks) advance<NCOL, kKeys>(p, cur, run.V);
        }
        if (!ok && lane == 0) s_abort = 1;
        wait_copies<0>();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kSoft + kExpand) {
        if (s_abort && lane == 0) {
            tc_commit(bend);                                  // MMAs may be in flight: let them end before the tensor memory goes back
            (void)mbar_wait(bend, 0, limit);
            atomicOr(p.err, SEGKV_DEV_WAIT_LIMIT);
        }
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmem) : "memory");
    }
}

template <typename T, int D, int NCOL>
cudaError_t launch_variant(const Params& p, int grid, bool pdl, cudaStream_t st) {
    using L = Lay<D, NCOL>;
    auto kernel = pages_tc5_kernel<T, D, NCOL>;
    static std::atomic<bool> configured[64] = {};
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !configured[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) configured[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid, 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = L::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    if (pdl) {
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

template <typename T>
cudaError_t launch_typed(int D, int nc, const Params& p, int grid, bool pdl, cudaStream_t st) {
    if (D == 64) return nc == 4 ? launch_variant<T, 64, 4>(p, grid, pdl, st) : nc == 8 ? launch_variant<T, 64, 8>(p, grid, pdl, st) : launch_variant<T, 64, 16>(p, grid, pdl, st);
    if (D == 128) return nc == 4 ? launch_variant<T, 128, 4>(p, grid, pdl, st) : nc == 8 ? launch_variant<T, 128, 8>(p, grid, pdl, st) : launch_variant<T, 128, 16>(p, grid, pdl, st);
    return nc == 4 ? launch_variant<T, 256, 4>(p, grid, pdl, st) : launch_variant<T, 256, 8>(p, grid, pdl, st);
}

}  // namespace

cudaError_t launch_pages_tc5(const segkv_pages& h, const PageSdpaArgs& a, cudaStream_t st) {
    Params p;
    p.q = (const char*)a.q; p.q_stride = a.q_stride * 2; p.out = (char*)a.out;
    p.kp = h.kp; p.vp = h.vp; p.table = a.table; p.lens = a.lens; p.slopes = a.slopes;
    p.ws = h.ws; p.tickets = h.tickets; p.err = h.err_word;
    p.table_stride = a.table_stride; p.n = a.n; p.q_len = a.q_len; p.H = h.heads; p.Hkv = h.kv_heads; p.group = h.group;
    p.page_log = h.page_log; p.num_pages = h.num_pages;
    p.cols = a.q_len * h.group;
    const int nc = p.cols <= 4 ? 4 : p.cols <= 8 || h.head_dim == 256 ? 8 : 16;
    p.ctiles = (p.cols + nc - 1) / nc;
    return h.dtype == SEGKV_BF16 ? launch_typed<__nv_bfloat16>(h.head_dim, nc, p, h.sm_count, a.pdl, st)
                                 : launch_typed<__half>(h.head_dim, nc, p, h.sm_count, a.pdl, st);
}

}  // namespace segkv_impl
