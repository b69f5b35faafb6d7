// The paged cache's store and read-back: the newest tokens of every sequence into (from) the pages that its table lists, keys and
// queries rotated on the way, rows in 16 or in 4 bits.
#include "segkv_pages_internal.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace segkv_impl {
namespace {

template <typename T> struct Half;
template <> struct Half<__half> {
    static constexpr uint32_t kInf = 0x7C00u, kNan = 0x7FFFu;
    static __device__ __forceinline__ float2 up(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
    static __device__ __forceinline__ uint32_t down(float a, float b) {
        const __half2 t = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&t);
    }
};
template <> struct Half<__nv_bfloat16> {
    static constexpr uint32_t kInf = 0x7F80u, kNan = 0x7FFFu;
    static __device__ __forceinline__ float2 up(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
    static __device__ __forceinline__ uint32_t down(float a, float b) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&t);
    }
};

struct Place {                   // where a token's rows lie
    long long row;               // first row of the token's (page, head 0) plus its row in the page; -1: nowhere
    int pos;
};

struct TokenParams {
    int n, T, Hkv, page_log, num_pages, table_stride;
    int tokens, rows;                                             // n * T; rows of a token: key, value and query heads
    int block_log, rows_cta;                                      // a CTA's tokens (a power of two) and how many of their rows it takes
    const int32_t *table, *lens, *new_lens;
    int* err;
};

// The page row of token i of sequence s; a token that does not exist, or may not be stored, has none.
__device__ __forceinline__ Place place_of(const TokenParams& p, int s, int i, int positions, bool reading) {
    Place r;
    r.row = -1;
    r.pos = 0;
    int nw = p.new_lens ? __ldg(p.new_lens + s) : p.T;
    nw = nw < 0 ? 0 : nw > p.T ? p.T : nw;
    if (i >= nw) return r;
    const int len = __ldg(p.lens + s);
    const long long pos = (long long)len - nw + i;
    if (len < 0 || pos >= (long long)p.table_stride << p.page_log) {
        atomicOr(p.err, SEGKV_DEV_BAD_PAGE);
        return r;
    }
    if (pos < 0) return r;                       // fewer tokens than asked for: an empty slot of a padded batch, say
    if (pos >= positions) {
        atomicOr(p.err, SEGKV_DEV_BAD_POSITION);
        return r;
    }
    r.pos = (int)pos;
    int page = __ldg(p.table + (long long)s * p.table_stride + (r.pos >> p.page_log));
    if ((unsigned)page >= (unsigned)p.num_pages) {
        atomicOr(p.err, SEGKV_DEV_BAD_PAGE);
        if (!reading) return r;
        page = 0;
    }
    r.row = ((long long)page * p.Hkv << p.page_log) + (r.pos & ((1 << p.page_log) - 1));
    return r;
}

constexpr int kThreads = 256;
constexpr int kTokenBlock = 16;  // most tokens of a CTA

struct AppendParams {
    TokenParams t;
    const char *k, *v, *q;
    long long k_stride, v_stride, q_stride;       // bytes
    char *kp, *vp, *q_out;
    const float *cos, *sin;
    int H, positions;
};

// A CTA's tokens: where they go, looked up once for all of their rows.
__device__ __forceinline__ void find_places(const TokenParams& p, Place* s_place, int positions, bool reading) {
    const int tok = (blockIdx.x << p.block_log) + threadIdx.x;
    if (threadIdx.x < (1 << p.block_log)) {
        Place r;
        r.row = -1;
        r.pos = 0;
        if (tok < p.tokens) {
            const int s = tok / p.T;
            r = place_of(p, s, tok - s * p.T, positions, reading);
        }
        s_place[threadIdx.x] = r;
    }
}

// One thread's sixteen values of one row: rotated, and put where they belong.
template <typename T, int D, int BITS, int STYLE>
__device__ __forceinline__ void store_row(const AppendParams& p, const Place& at, bool ok, int kind, int head, int token, int c,
                                          uint4 lo, uint4 hi, const float* cs, const float* sn) {
    constexpr int TPR = D / 16;
    if (STYLE != 0 && kind != 1) {                            // (nothing real where !ok)
        uint32_t wl[4] = {lo.x, lo.y, lo.z, lo.w}, wh[4] = {hi.x, hi.y, hi.z, hi.w};
        if (STYLE == SEGKV_ROPE_HALF) {
            float co[8], si[8];
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                *reinterpret_cast<float4*>(co + 4 * w) = *reinterpret_cast<const float4*>(cs + c * 8 + 4 * w);
                *reinterpret_cast<float4*>(si + 4 * w) = *reinterpret_cast<const float4*>(sn + c * 8 + 4 * w);
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 a = Half<T>::up(wl[w]), b = Half<T>::up(wh[w]);
                const float c0 = co[2 * w], c1 = co[2 * w + 1], s0 = si[2 * w], s1 = si[2 * w + 1];
                wl[w] = Half<T>::down(__fsub_rn(__fmul_rn(a.x, c0), __fmul_rn(b.x, s0)), __fsub_rn(__fmul_rn(a.y, c1), __fmul_rn(b.y, s1)));
                wh[w] = Half<T>::down(__fadd_rn(__fmul_rn(b.x, c0), __fmul_rn(a.x, s0)), __fadd_rn(__fmul_rn(b.y, c1), __fmul_rn(a.y, s1)));
            }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float co[4], si[4];
                *reinterpret_cast<float4*>(co) = *reinterpret_cast<const float4*>(cs + c * 4 + u * (D / 4));
                *reinterpret_cast<float4*>(si) = *reinterpret_cast<const float4*>(sn + c * 4 + u * (D / 4));
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float2 x = Half<T>::up(u ? wh[w] : wl[w]);
                    const uint32_t y = Half<T>::down(__fsub_rn(__fmul_rn(x.x, co[w]), __fmul_rn(x.y, si[w])),
                                                     __fadd_rn(__fmul_rn(x.y, co[w]), __fmul_rn(x.x, si[w])));
                    if (u) wh[w] = y; else wl[w] = y;
                }
            }
        }
        lo = make_uint4(wl[0], wl[1], wl[2], wl[3]);
        hi = make_uint4(wh[0], wh[1], wh[2], wh[3]);
    }
    if (kind == 2) {
        if (ok) {
            char* dst = p.q_out + ((size_t)token * p.H + head) * (D * 2) + c * 16;
            *reinterpret_cast<uint4*>(dst) = lo;
            *reinterpret_cast<uint4*>(dst + D) = hi;
        }
    } else if (BITS == 16) {
        if (ok) {
            char* dst = (kind == 0 ? p.kp : p.vp) + (size_t)(at.row + ((long long)head << p.t.page_log)) * (D * 2) + c * 16;
            *reinterpret_cast<uint4*>(dst) = lo;
            *reinterpret_cast<uint4*>(dst + D) = hi;
        }
    }
    if (BITS == 4) {                                          // (every thread: the row's threads exchange)
        if (!__any_sync(0xffffffffu, ok && kind != 2)) return;
        float x[16];
        const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
        uint32_t bad = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 f = Half<T>::up(w[e]);
            x[2 * e] = f.x;
            x[2 * e + 1] = f.y;
            if ((w[e] & 0x7FFFu) >= Half<T>::kInf) bad |= 1u << ((2 * e) & 3);
            if (((w[e] >> 16) & 0x7FFFu) >= Half<T>::kInf) bad |= 1u << ((2 * e + 1) & 3);
        }
        float mn[4], mx[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            mn[j] = fminf(fminf(x[j], x[j + 4]), fminf(x[j + 8], x[j + 12]));
            mx[j] = fmaxf(fmaxf(x[j], x[j + 4]), fmaxf(x[j + 8], x[j + 12]));
        }
#pragma unroll
        for (int o = 1; o < TPR; o <<= 1) {
            bad |= __shfl_xor_sync(0xffffffffu, bad, o);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mn[j] = fminf(mn[j], __shfl_xor_sync(0xffffffffu, mn[j], o));
                mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], o));
            }
        }
        if (!ok || kind == 2) return;
        float s[4], z[4];
        uint32_t sw[2], zw[2];
        {
            float st[4], zt[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                st[j] = __fmul_rn(__fsub_rn(mx[j], mn[j]), 0x1.111112p-4f);       // 1/15, rounded
                zt[j] = __fadd_rn(mn[j], 8.f * st[j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                sw[j] = Half<T>::down(st[2 * j], st[2 * j + 1]);
                zw[j] = Half<T>::down(zt[2 * j], zt[2 * j + 1]);
#pragma unroll
                for (int u = 0; u < 2; ++u) {                 // a range that the type cannot hold is not held at all either
                    const uint32_t m = 0x7FFFu << (16 * u), inf = Half<T>::kInf << (16 * u);
                    if ((bad >> (2 * j + u) & 1u) || (sw[j] & m) >= inf || (zw[j] & m) >= inf) {
                        sw[j] |= Half<T>::kNan << (16 * u);
                        zw[j] |= Half<T>::kNan << (16 * u);
                        bad |= 1u << (2 * j + u);
                    }
                }
                const float2 a = Half<T>::up(sw[j]), b = Half<T>::up(zw[j]);
                s[2 * j] = a.x; s[2 * j + 1] = a.y;
                z[2 * j] = b.x; z[2 * j + 1] = b.y;
            }
        }
        const float inv[4] = {1.f / s[0], 1.f / s[1], 1.f / s[2], 1.f / s[3]};
        uint32_t code[2] = {0u, 0u};
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = e & 3;
            int cd = 8;
            if (s[j] > 0.f && !(bad >> j & 1u)) {
                // the quotient by a reciprocal, good to 2^-21 of it; where it stands that near a tie, by a division.  (Far outside the
                // range, where z's rounding is all there is, it may be large: clamped before it is an integer.)
                const float y = __fsub_rn(x[e], z[j]);
                float r = y * inv[j], w1 = rintf(r);
                if (fabsf(fabsf(r - w1) - 0.5f) < 1e-4f) w1 = rintf(__fdiv_rn(y, s[j]));
                cd = __float2int_rn(fminf(fmaxf(w1 + 8.f, 0.f), 15.f));
            }
            code[e >> 3] |= (uint32_t)cd << (4 * (e & 7));
        }
        const int ps = 1 << p.t.page_log;
        const long long first = at.row + ((long long)head << p.t.page_log);          // row among all rows of the pool
        const int in_page = (int)(first & (ps - 1));
        char* blk = (kind == 0 ? p.kp : p.vp) + (size_t)(first >> p.t.page_log) * ((size_t)ps * (D / 2 + 16));
        uint32_t* dst = reinterpret_cast<uint32_t*>(blk + (size_t)in_page * (D / 2));
        dst[c] = code[0];
        dst[c + D / 16] = code[1];
        if (c == 0) *reinterpret_cast<uint4*>(blk + (size_t)ps * (D / 2) + in_page * 16) = make_uint4(sw[0], sw[1], zw[0], zw[1]);
    }
}

// One row of head_dim values by D/16 threads, each with eight values of the lower half and the eight that stand D/2 behind them,
// so that a thread holds whole pairs of either rotary style and two whole code words.
//
// Rotation: products and sums rounded one by one (no contraction), so that the stored value is the one that the formula gives in
// plain fp32 arithmetic: a code of the 4-bit form depends on its last bit.
// 4 bits: the four interleaved groups' extremes go round the row's threads by shuffles (log2(D/16) steps of eight); a thread's
// eight neighbouring channels are one 32-bit word of codes.
// A CTA takes up to 16 tokens and some or all of their rows, neighbouring thread groups the same head of neighbouring tokens, whose
// page rows lie side by side; a token's page and its angles are fetched once, into shared memory.  Padding is not read.
// Bound: HBM for prompts (each value in once, each row out once), the chain length -> page -> store for a single token.
template <typename T, int D, int BITS, int STYLE>
__global__ void __launch_bounds__(kThreads) pages_append_kernel(const __grid_constant__ AppendParams p) {
    constexpr int TPR = D / 16, SLOTS = kThreads / TPR;
    __shared__ Place s_place[kTokenBlock];
    __shared__ __align__(16) float s_cos[STYLE ? kTokenBlock * (D / 2) : 4], s_sin[STYLE ? kTokenBlock * (D / 2) : 4];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    find_places(p.t, s_place, STYLE ? p.positions : 0x7FFFFFFF, false);
    __syncthreads();
    if (STYLE) {
        for (int i = threadIdx.x; i < (D / 2) << p.t.block_log; i += kThreads) {
            const Place a = s_place[i / (D / 2)];
            if (a.row >= 0) {
                s_cos[i] = __ldg(p.cos + (size_t)a.pos * (D / 2) + i % (D / 2));
                s_sin[i] = __ldg(p.sin + (size_t)a.pos * (D / 2) + i % (D / 2));
            }
        }
        __syncthreads();
    }
    const int c = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const int row0 = blockIdx.y * p.t.rows_cta, rows = min(p.t.rows_cta, p.t.rows - row0);
    const int items = rows << p.t.block_log;
    const int tok0 = blockIdx.x << p.t.block_log;
    constexpr int U = 2;                                      // rows of a thread in flight
    for (int i0 = 0; i0 < items; i0 += U * SLOTS) {
        uint4 lo_[U], hi_[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * SLOTS + slot, tl = i & ((1 << p.t.block_log) - 1), row = row0 + (i >> p.t.block_log);
            lo_[u] = hi_[u] = make_uint4(0u, 0u, 0u, 0u);
            if (i < items && s_place[tl].row >= 0) {
                const long long token = tok0 + tl;
                const char* src = row < p.t.Hkv ? p.k + token * p.k_stride + (size_t)row * (D * 2)
                                  : row < 2 * p.t.Hkv ? p.v + token * p.v_stride + (size_t)(row - p.t.Hkv) * (D * 2)
                                                      : p.q + token * p.q_stride + (size_t)(row - 2 * p.t.Hkv) * (D * 2);
                lo_[u] = *reinterpret_cast<const uint4*>(src + c * 16);
                hi_[u] = *reinterpret_cast<const uint4*>(src + c * 16 + D);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i0 + u * SLOTS >= items) break;               // (every thread)
            const int i = i0 + u * SLOTS + slot, tl = i & ((1 << p.t.block_log) - 1), row = row0 + (i >> p.t.block_log);
            const Place at = s_place[tl];
            const bool ok = i < items && at.row >= 0;
            const int kind = row < p.t.Hkv ? 0 : row < 2 * p.t.Hkv ? 1 : 2;            // key, value, query
            const int head = row - kind * p.t.Hkv;
            store_row<T, D, BITS, STYLE>(p, at, ok, kind, head, tok0 + tl, c, lo_[u], hi_[u], s_cos + tl * (D / 2), s_sin + tl * (D / 2));
        }
    }
}

struct ReadParams {
    TokenParams t;
    const char *kp, *vp;
    char *k, *v;
};

// Eight neighbouring values of a row per thread, a CTA's tokens and rows as in the append.  Bound: HBM.
template <typename T, int D, int BITS>
__global__ void __launch_bounds__(kThreads) pages_read_kernel(const __grid_constant__ ReadParams p) {
    constexpr int TPR = D / 8, SLOTS = kThreads / TPR;
    __shared__ Place s_place[kTokenBlock];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    find_places(p.t, s_place, 0x7FFFFFFF, true);
    __syncthreads();
    const int c = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const int row0 = blockIdx.y * p.t.rows_cta, rows = min(p.t.rows_cta, p.t.rows - row0);
    const int items = rows << p.t.block_log;
    const int tok0 = blockIdx.x << p.t.block_log;
    const int ps = 1 << p.t.page_log;
    constexpr int U = 4;                                      // rows of a thread in flight
    for (int i0 = 0; i0 < items; i0 += U * SLOTS) {
        uint4 x[U];
        uint32_t code[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * SLOTS + slot, tl = i & ((1 << p.t.block_log) - 1), row = row0 + (i >> p.t.block_log);
            x[u] = make_uint4(0u, 0u, 0u, 0u);
            code[u] = 0u;
            if (i >= items || s_place[tl].row < 0) continue;
            const int kind = row < p.t.Hkv ? 0 : 1, head = row - kind * p.t.Hkv;
            const long long first = s_place[tl].row + ((long long)head << p.t.page_log);
            const char* pages = kind == 0 ? p.kp : p.vp;
            if (BITS == 16) {
                x[u] = *reinterpret_cast<const uint4*>(pages + (size_t)first * (D * 2) + c * 16);
            } else {
                const int in_page = (int)(first & (ps - 1));
                const char* blk = pages + (size_t)(first >> p.t.page_log) * ((size_t)ps * (D / 2 + 16));
                code[u] = reinterpret_cast<const uint32_t*>(blk + (size_t)in_page * (D / 2))[c];
                x[u] = *reinterpret_cast<const uint4*>(blk + (size_t)ps * (D / 2) + in_page * 16);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * SLOTS + slot, tl = i & ((1 << p.t.block_log) - 1), row = row0 + (i >> p.t.block_log);
            if (i >= items || s_place[tl].row < 0) continue;
            const int kind = row < p.t.Hkv ? 0 : 1, head = row - kind * p.t.Hkv;
            uint4 out = x[u];
            if (BITS == 4) {
                const float2 s0 = Half<T>::up(x[u].x), s1 = Half<T>::up(x[u].y), z0 = Half<T>::up(x[u].z), z1 = Half<T>::up(x[u].w);
                const float s4[4] = {s0.x, s0.y, s1.x, s1.y}, z4[4] = {z0.x, z0.y, z1.x, z1.y};
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf((float)((int)(code[u] >> (4 * e) & 15u) - 8), s4[e & 3], z4[e & 3]);
                out = make_uint4(Half<T>::down(v[0], v[1]), Half<T>::down(v[2], v[3]), Half<T>::down(v[4], v[5]), Half<T>::down(v[6], v[7]));
            }
            char* dst = (kind == 0 ? p.k : p.v) + ((size_t)(tok0 + tl) * p.t.Hkv + head) * (D * 2) + c * 16;
            *reinterpret_cast<uint4*>(dst) = out;
        }
    }
}

template <typename P>
cudaError_t launch(void (*kernel)(P), P& p, int slots, int sm_count, bool pdl, cudaStream_t st) {
    // tokens of a CTA: 16, fewer where there are fewer; rows of a CTA: all, or as many fewer as give the GPU four CTAs an SM, but
    // one row for each of a CTA's thread groups at least
    p.t.block_log = 0;
    while ((1 << p.t.block_log) < kTokenBlock && (2 << p.t.block_log) <= p.t.tokens) p.t.block_log++;
    const long long blocks = ((long long)p.t.tokens + (1 << p.t.block_log) - 1) >> p.t.block_log;
    int rows = p.t.rows;
    while (rows > 1 && (rows << p.t.block_log) > slots && blocks * ((p.t.rows + rows - 1) / rows) < 4LL * sm_count) rows = (rows + 1) / 2;
    p.t.rows_cta = rows;
    const int chunks = (p.t.rows + rows - 1) / rows;
    if (chunks > 65535) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks, (unsigned)chunks, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
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

TokenParams token_params(const segkv_pages& h, const PageTokens& t, int rows) {
    TokenParams p;
    p.n = t.n; p.T = t.tokens; p.Hkv = h.kv_heads; p.page_log = h.page_log; p.num_pages = h.num_pages;
    p.table_stride = t.table_stride; p.rows = rows; p.tokens = t.n * t.tokens;
    p.table = t.table; p.lens = t.lens; p.new_lens = t.new_lens; p.err = h.err_word;
    return p;
}

template <typename T, int D, int BITS>
void (*append_of(int style))(AppendParams) {
    return style == SEGKV_ROPE_HALF ? pages_append_kernel<T, D, BITS, SEGKV_ROPE_HALF>
           : style == SEGKV_ROPE_INTERLEAVED ? pages_append_kernel<T, D, BITS, SEGKV_ROPE_INTERLEAVED> : pages_append_kernel<T, D, BITS, 0>;
}
template <typename T, int D>
void (*append_of(int bits, int style))(AppendParams) { return bits == 16 ? append_of<T, D, 16>(style) : append_of<T, D, 4>(style); }
template <typename T>
void (*append_of(int D, int bits, int style))(AppendParams) {
    return D == 64 ? append_of<T, 64>(bits, style) : D == 128 ? append_of<T, 128>(bits, style) : append_of<T, 256>(bits, style);
}
template <typename T>
void (*read_of(int D, int bits))(ReadParams) {
    if (bits == 16) return D == 64 ? pages_read_kernel<T, 64, 16> : D == 128 ? pages_read_kernel<T, 128, 16> : pages_read_kernel<T, 256, 16>;
    return D == 64 ? pages_read_kernel<T, 64, 4> : D == 128 ? pages_read_kernel<T, 128, 4> : pages_read_kernel<T, 256, 4>;
}

}  // namespace

cudaError_t launch_pages_append(const segkv_pages& h, const PageAppendArgs& a, cudaStream_t st) {
    AppendParams p;
    p.t = token_params(h, a.t, 2 * h.kv_heads + (a.q ? h.heads : 0));
    p.k = (const char*)a.k; p.v = (const char*)a.v; p.q = (const char*)a.q;
    p.k_stride = a.k_stride * 2; p.v_stride = a.v_stride * 2; p.q_stride = a.q_stride * 2;
    p.kp = h.kp; p.vp = h.vp; p.q_out = (char*)a.q_out;
    p.cos = a.cos; p.sin = a.sin; p.H = h.heads; p.positions = a.positions;
    auto kernel = h.dtype == SEGKV_BF16 ? append_of<__nv_bfloat16>(h.head_dim, h.bits, a.style) : append_of<__half>(h.head_dim, h.bits, a.style);
    return launch(kernel, p, kThreads / (h.head_dim / 16), h.sm_count, a.t.pdl, st);
}

cudaError_t launch_pages_read(const segkv_pages& h, const PageTokens& t, void* k_out, void* v_out, cudaStream_t st) {
    ReadParams p;
    p.t = token_params(h, t, 2 * h.kv_heads);
    p.kp = h.kp; p.vp = h.vp; p.k = (char*)k_out; p.v = (char*)v_out;
    auto kernel = h.dtype == SEGKV_BF16 ? read_of<__nv_bfloat16>(h.head_dim, h.bits) : read_of<__half>(h.head_dim, h.bits);
    return launch(kernel, p, kThreads / (h.head_dim / 8), h.sm_count, t.pdl, st);
}

}  // namespace segkv_impl
