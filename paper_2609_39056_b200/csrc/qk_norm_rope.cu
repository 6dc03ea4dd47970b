// What stands between the QKV linear and attention, in one pass over the QKV rows: RMS norm of every query and key
// head, rotation by the row's position, and the append of keys and values to the paged cache (bf16 or E4M3).
//
//     y = (x r) w,  r = 1 / sqrt(mean_D(x^2) + eps)           per head of D channels
//     u_i = y_i c - y_j s,  u_j = y_j c + y_i s               for the pairs (i, j) of the first `rot` channels,
//                                                             c, s = cos / sin table at (position, pair)
//     Q <- bf16(u), K <- bf16(u) or e4m3(u (1 / k_scale)), V <- x or e4m3(x (1 / v_scale))
//
// Every operation is a single correctly rounded fp32 add, multiply, divide or square root in the order written here
// (no fused multiply-add), rounded once to the output type: bit-defined like the other glue.  A head is held by D / 8 lanes of 8
// channels, two runs of four: lane l < rot / 8 has 4 l .. 4 l + 3 and the same + rot / 2 with half-split pairs (both members of its
// pairs), every other lane 8 neighbours.  A lane adds the squares of its even and of its odd places in order, then the
// two; the lanes' sums are combined by the exchange with l ^ (D / 16), ..., 2, 1.
//
// Bound by latency: by one chain of dependent loads (position -> angles) for a few rows, and for thousands of rows by what a warp does between two groups
// of four steps (nothing is in flight while it computes).  Hence two-lane arithmetic (f32x2: the same roundings, half the instructions), both members of
// a pair in one lane (no exchange), angles read once per row and thread for all its heads, and four steps of loads in flight.
// Every access of a head is one or two contiguous runs.  Measured: 4416 rows into an E4M3 cache 25.6 us = 3.4 TB/s (13.3 us are its bytes at
// the copy rate; issue slots 65 %, ALU 49 %, 38 % of the warps resident, an SM idle for a quarter of the time: the last wave), 17000 rows in bf16 79 us = 5.0 TB/s,
// 1021 rows in pairs 4.3 us, 16 rows 2.9 us.
#include "internal.cuh"
#include "paged.cuh"

#include <cuda_bf16.h>

namespace rudder {

namespace {

constexpr int QK_THREADS = 256;

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Two fp32 numbers in one register pair; each operation rounds both on their own.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 make2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 split(f32x2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// a + b as a 1 + b with a 1 that the compiler does not know (a kernel argument): a two-lane addition is merged with the
// multiplication in front of it into one operation with one rounding, .rn or not (seen: results one bf16 step off the defined bits).
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b, f32x2 one) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(one), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 widen(uint32_t w) { return make2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ f32x2 swap2(f32x2 v) { const float2 t = split(v); return make2(t.y, t.x); }
__device__ __forceinline__ uint32_t to_bf16(f32x2 v) { const float2 t = split(v); return pack_bf16(t.x, t.y); }
__device__ __forceinline__ uint32_t to_e4m3(f32x2 a, f32x2 b) {
    const float2 s = split(a), t = split(b);
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(s.y), "f"(s.x));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(t.y), "f"(t.x));
    return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
__device__ __forceinline__ void load4(const float* p, f32x2& a, f32x2& b) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    a = make2(v.x, v.y);
    b = make2(v.z, v.w);
}

// D: channels of a head; PAIRS: neighbours (2i, 2i+1) are turned together, else (i, i + rot/2); E4M3: format of the cache.
// `share` warps work on a row: warp p of them takes the steps p, p + share, ... of 32 / (D / 8) heads each.
template <int D, bool PAIRS, bool E4M3>
__global__ void __launch_bounds__(QK_THREADS, 4) qk_norm_rope_kernel(const QkArgs a, int share)
{
    constexpr int LPH = D / 8;                             // lanes of a head
    constexpr int HPW = 32 / LPH;                          // heads of a step
    constexpr int U = 4;                                   // steps in hand at once: their loads are in flight together
    __shared__ float s_inv[E4M3 ? 2 * kMaxKvHeads : 1];    // reciprocals of the cache's scales: keys, values
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31;
    const int l = tid & (LPH - 1), h0 = lane / LPH;
    pdl_wait();
    const int half = a.rot >> 1;
    const int n_qk = a.heads + a.kv_heads;
    const bool to_cache = a.slots != nullptr;
    const int n_heads = to_cache ? n_qk + a.kv_heads : n_qk;
    const bool turns = 8 * l < a.rot;
    // the two runs of four channels of this lane
    const int ca = (PAIRS || !turns) ? 8 * l : 4 * l;
    const int cb = (PAIRS || !turns) ? ca + 4 : ca + half;
    const long long n_slots = static_cast<long long>(a.cache.n_pages) << a.cache.page_shift;
    if (E4M3) {
        for (int i = tid; i < 2 * a.kv_heads; i += QK_THREADS) {
            const float* sc = i < a.kv_heads ? a.cache.k_scale : a.cache.v_scale;
            const int h = i < a.kv_heads ? i : i - a.kv_heads;
            s_inv[i] = sc != nullptr ? __fdiv_rn(1.0f, sc[h]) : 1.0f;
        }
        __syncthreads();
    }
    const uint2 zero2 = make_uint2(0, 0);
    const f32x2 one = make2(a.one, a.one);
    const int warp = blockIdx.x * (QK_THREADS / 32) + (tid >> 5), part = warp % share;

    for (int m = warp / share; m < a.M; m += gridDim.x * (QK_THREADS / 32) / share) {
        const uint16_t* xr = a.X + static_cast<size_t>(m) * a.ldx;
        // the row's data does not depend on its position: both are requested together
        uint2 xa[U], xb[U];
        auto fetch = [&](int step, int n) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = (step + u * share) * HPW + h0;
                xa[u] = h < n ? *reinterpret_cast<const uint2*>(xr + h * D + ca) : zero2;
                xb[u] = h < n ? *reinterpret_cast<const uint2*>(xr + h * D + cb) : zero2;
            }
        };
        fetch(part, n_heads);
        const int pos = a.positions != nullptr ? a.positions[m] : 0;
        long long slot = to_cache ? a.slots[m] : -1;
        if (pos < 0) continue;                             // a row of padding: left as it was
        if (a.rot > 0 && pos >= a.n_pos) {
            if (lane == 0) record_bad_data(kBadPosition);
            continue;
        }
        if (slot >= n_slots) {
            if (lane == 0) record_bad_data(kBadSlot);
            slot = -1;
        }
        const int heads = (to_cache && slot < 0) ? a.heads : n_heads;               // nothing to append: queries only
        const long long token_off = slot < 0 ? 0 : (slot >> a.cache.page_shift) * a.cache.page_stride +
                                                   (slot & ((1 << a.cache.page_shift) - 1)) * a.cache.token_stride;
        uint16_t* const q_row = a.Q + static_cast<size_t>(m) * a.ldq;
        uint16_t* const k_row = to_cache ? nullptr : a.K + static_cast<size_t>(m) * a.ldk;
        uint8_t* const k_tok = a.cache.k + (E4M3 ? 1 : 2) * token_off;
        uint8_t* const v_tok = a.cache.v + (E4M3 ? 1 : 2) * token_off;
        // half-split: c and s of the four pairs; neighbours: (c, c) and (-s, s) of the four pairs
        f32x2 c[PAIRS ? 4 : 2], s[PAIRS ? 4 : 2];
        if (turns) {
            const float* cp = a.cos + static_cast<size_t>(pos) * half + 4 * l;
            const float* sp = a.sin + static_cast<size_t>(pos) * half + 4 * l;
            if (PAIRS) {
                const float4 c4 = *reinterpret_cast<const float4*>(cp), s4 = *reinterpret_cast<const float4*>(sp);
                c[0] = make2(c4.x, c4.x); c[1] = make2(c4.y, c4.y); c[PAIRS ? 2 : 0] = make2(c4.z, c4.z); c[PAIRS ? 3 : 0] = make2(c4.w, c4.w);
                s[0] = make2(-s4.x, s4.x); s[1] = make2(-s4.y, s4.y); s[PAIRS ? 2 : 0] = make2(-s4.z, s4.z); s[PAIRS ? 3 : 0] = make2(-s4.w, s4.w);
            } else {
                load4(cp, c[0], c[1]);
                load4(sp, s[0], s[1]);
            }
        }
        // all lanes of a warp stay together (the exchanges): the loops run to the same bounds in every lane
        for (int step = part; step * HPW < heads; step += U * share) {
            if (step != part) fetch(step, heads);
            float rr[U];
            if (step * HPW < n_qk) {                       // (else only values: nothing to compute)
                float sum[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const f32x2 y[4] = {widen(xa[u].x), widen(xa[u].y), widen(xb[u].x), widen(xb[u].y)};
                    f32x2 sq = mul2(y[0], y[0]);
#pragma unroll
                    for (int i = 1; i < 4; ++i) sq = add2(mul2(y[i], y[i]), sq, one);
                    const float2 both = split(sq);
                    sum[u] = __fadd_rn(both.x, both.y);
                }
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1)
#pragma unroll
                    for (int u = 0; u < U; ++u) sum[u] = __fadd_rn(sum[u], __shfl_xor_sync(0xffffffffu, sum[u], o));
                // the division and the square root once for the four steps: lane 4 i + u of a head does the head's step u
                const float mine = (lane & 2) ? ((lane & 1) ? sum[3] : sum[2]) : ((lane & 1) ? sum[1] : sum[0]);
                const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(mine, 1.0f / D), a.eps)));
#pragma unroll
                for (int u = 0; u < U; ++u) rr[u] = __shfl_sync(0xffffffffu, r, (lane & ~3) | u);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = (step + u * share) * HPW + h0;
                if (h >= heads) break;
                f32x2 y[4] = {widen(xa[u].x), widen(xa[u].y), widen(xb[u].x), widen(xb[u].y)};
                if (h < n_qk) {
                    const f32x2 r2 = make2(rr[u], rr[u]);
                    const float* wp = h < a.heads ? a.q_weight : a.k_weight;
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], r2);
                    if (wp != nullptr) {
                        f32x2 w[4];
                        load4(wp + ca, w[0], w[1]);
                        load4(wp + cb, w[2], w[3]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = mul2(y[i], w[i]);
                    }
                    if (turns) {
                        if (PAIRS) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[i] = add2(mul2(swap2(y[i]), s[PAIRS ? i : 0]), mul2(y[i], c[PAIRS ? i : 0]), one);
                        } else {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const f32x2 p = y[i], n = y[2 + i], ns = mul2(n, s[i]);
                                const float2 t = split(ns);
                                y[i] = add2(make2(-t.x, -t.y), mul2(p, c[i]), one);
                                y[2 + i] = add2(mul2(p, s[i]), mul2(n, c[i]), one);
                            }
                        }
                    }
                    if (h < a.heads || !to_cache) {
                        uint16_t* out = h < a.heads ? q_row + h * D : k_row + (h - a.heads) * D;
                        *reinterpret_cast<uint2*>(out + ca) = make_uint2(to_bf16(y[0]), to_bf16(y[1]));
                        *reinterpret_cast<uint2*>(out + cb) = make_uint2(to_bf16(y[2]), to_bf16(y[3]));
                        continue;
                    }
                }
                const bool is_v = h >= n_qk;
                const int kvh = is_v ? h - n_qk : h - a.heads;
                const long long off = static_cast<long long>(kvh) * a.cache.head_stride;
                uint8_t* const base = is_v ? v_tok : k_tok;
                if (E4M3) {
                    const float iv = s_inv[is_v ? a.kv_heads + kvh : kvh];
                    const f32x2 inv = make2(iv, iv);
                    *reinterpret_cast<uint32_t*>(base + off + ca) = to_e4m3(mul2(y[0], inv), mul2(y[1], inv));
                    *reinterpret_cast<uint32_t*>(base + off + cb) = to_e4m3(mul2(y[2], inv), mul2(y[3], inv));
                } else {
                    uint16_t* out = reinterpret_cast<uint16_t*>(base) + off;
                    *reinterpret_cast<uint2*>(out + ca) = is_v ? xa[u] : make_uint2(to_bf16(y[0]), to_bf16(y[1]));
                    *reinterpret_cast<uint2*>(out + cb) = is_v ? xb[u] : make_uint2(to_bf16(y[2]), to_bf16(y[3]));
                }
            }
            __syncwarp();
        }
    }
}

template <int D>
cudaError_t launch_d(const QkArgs& a, bool e4m3, const cudaLaunchConfig_t& cfg, int share)
{
    if (a.pairs) return e4m3 ? cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, true, true>, a, share) : cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, true, false>, a, share);
    return e4m3 ? cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, false, true>, a, share) : cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, false, false>, a, share);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const QkArgs& a, int head_dim, bool e4m3, int sm_count, cudaStream_t st)
{
    constexpr int kWarps = QK_THREADS / 32;
    // Warps that share a row.  A row costs a warp about 4 steps before its first head; up to one warp per slot (32 per SM) everything runs
    // at once, beyond that in proportion: the share with the least (4 + steps / share) x max(1, rows x share / slots).  Measured, 48 heads of
    // 128: 1024 rows 18.7, 11.7, 7.7, 8.2 us with 1, 2, 4, 8 warps, 3000 rows 24.3, 20.5, 20.7, 24.2 us, 17000 rows 78, 79, 92, 122 us.
    const int steps = (a.heads + 2 * a.kv_heads) * head_dim / 256;
    int share = 1;
    double best = 0.0;
    for (int s = 1; s <= 32 && (s == 1 || s <= steps); s *= 2) {
        const double load = static_cast<double>(a.M) * s / (sm_count * 32.0), cost = (4.0 + static_cast<double>(steps) / s) * (load > 1.0 ? load : 1.0);
        if (s == 1 || cost < best) { best = cost; share = s; }
    }
    const long long need = (static_cast<long long>(a.M) * share + kWarps - 1) / kWarps;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(need < (1 << 20) ? need : (1 << 20)), 1, 1);
    cfg.blockDim = dim3(QK_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (head_dim == 64) return launch_d<64>(a, e4m3, cfg, share);
    if (head_dim == 128) return launch_d<128>(a, e4m3, cfg, share);
    return launch_d<256>(a, e4m3, cfg, share);
}

}  // namespace rudder
