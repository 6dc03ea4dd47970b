// What stands between the QKV linear and attention, in one pass over the QKV rows: RMS norm of every query and key
// head, rotation by the row's position, and the append of keys and values to the paged cache (bf16 or E4M3).
//
//     y = (x r) w,  r = 1 / sqrt(mean_D(x^2) + eps)           per head of D channels
//     u_i = y_i c - y_j s,  u_j = y_j c + y_i s               for the pairs (i, j) of the first `rot` channels,
//                                                             c, s = cos / sin table at (position, pair)
//     Q <- bf16(u), K <- bf16(u) or e4m3(u (1 / k_scale)), V <- x or e4m3(x (1 / v_scale))
//
// Every operation is a single correctly rounded fp32 add, multiply, divide or square root in the order written here
// (no fused multiply-add), rounded once to the output type: bit-defined like the other glue.  The head's sum of
// squares: lane l of the D / 8 lanes that hold the head adds its 8 squares in channel order, the lanes' sums are
// combined by the exchange with l ^ (D / 16), ..., 2, 1.
//
// Bound by HBM for long inputs (each row is read once and written once) and by one chain of dependent loads
// (position -> angles) for a few rows.  D / 8 lanes per head, 16 bytes per lane: every access of a head is one
// contiguous run.  A CTA takes one row at a time; a thread keeps its place l inside the head for all the heads it
// handles, so angles and norm weights are read once per row and thread, not once per head.
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
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return static_cast<uint32_t>(lo) | (static_cast<uint32_t>(hi) << 16);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// Heads of one kind that a CTA takes in one step, 8 channels per lane: see the kernel below.
struct QkLane {
    float c[8], s[8];                                      // angles of this lane's channels
    int partner;                                           // half-split pairs: the lane with the other channels
    float sign;
    bool turns;
};

// x r w of one head, its sum of squares over the LPH lanes that hold it, and the rotation.
template <int D, bool PAIRS>
__device__ __forceinline__ void norm_and_turn(float (&y)[8], const float (&x)[8], const float (&w)[8], float eps, bool rot, const QkLane& t, int l)
{
    constexpr int LPH = D / 8;
    float sum = __fmul_rn(x[0], x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) sum = __fadd_rn(sum, __fmul_rn(x[i], x[i]));
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, o));
    const float r = __fdiv_rn(1.0f, __fsqrt_rn(__fadd_rn(__fmul_rn(sum, 1.0f / D), eps)));
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(__fmul_rn(x[i], r), w[i]);
    if (!rot) return;
    if (PAIRS) {
        if (t.turns) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float u = y[2 * i], v = y[2 * i + 1];
                y[2 * i] = __fsub_rn(__fmul_rn(u, t.c[i]), __fmul_rn(v, t.s[i]));
                y[2 * i + 1] = __fadd_rn(__fmul_rn(v, t.c[i]), __fmul_rn(u, t.s[i]));
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float o = __shfl_sync(0xffffffffu, y[i], t.partner, LPH);
            if (t.turns) y[i] = __fadd_rn(__fmul_rn(y[i], t.c[i]), __fmul_rn(o, t.s[i]));     // (sign of the sine: negated where it is subtracted)
        }
    }
}

// D: channels of a head; PAIRS: neighbours (2i, 2i+1) are turned together, else (i, i + rot/2); E4M3: format of the cache.
template <int D, bool PAIRS, bool E4M3>
__global__ void __launch_bounds__(QK_THREADS, 3) qk_norm_rope_kernel(const QkArgs a)
{
    constexpr int LPH = D / 8;                             // lanes of a head
    constexpr int HPC = QK_THREADS / LPH;                  // heads a CTA has in hand at once
    constexpr int U = 4;                                   // steps whose loads are in flight together
    pdl_launch_dependents();
    const int tid = threadIdx.x;
    const int l = tid & (LPH - 1), h0 = tid / LPH;
    pdl_wait();
    const int half = a.rot >> 1;
    const int n_qk = a.heads + a.kv_heads;
    const bool to_cache = a.slots != nullptr;
    const int n_heads = to_cache ? n_qk + a.kv_heads : n_qk;
    QkLane t;
    t.turns = 8 * l < a.rot;
    t.partner = !t.turns ? l : (8 * l < half) ? l + (half >> 3) : l - (half >> 3);
    const bool first = 8 * l < half;
    const long long n_slots = static_cast<long long>(a.cache.n_pages) << a.cache.page_shift;
    const bool w_null_q = a.q_weight == nullptr, w_null_k = a.k_weight == nullptr;

    for (int m = blockIdx.x; m < a.M; m += gridDim.x) {
        const uint16_t* xr = a.X + static_cast<size_t>(m) * a.ldx + 8 * l;
        // the row's data does not depend on its position: both are requested together
        uint4 x4[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * HPC;
            x4[u] = h < n_heads ? *reinterpret_cast<const uint4*>(xr + static_cast<size_t>(h) * D) : make_uint4(0, 0, 0, 0);
        }
        const int pos = a.positions != nullptr ? a.positions[m] : 0;
        long long slot = to_cache ? a.slots[m] : -1;
        if (pos < 0) continue;                             // a row of padding: left as it was
        if (a.rot > 0 && pos >= a.n_pos) {
            if (tid == 0) record_bad_data(kBadPosition);
            continue;
        }
        if (slot >= n_slots) {
            if (tid == 0) record_bad_data(kBadSlot);
            slot = -1;
        }
        const int heads = (to_cache && slot < 0) ? a.heads : n_heads;               // nothing to append: queries only
        const long long token_off = slot < 0 ? 0 : (slot >> a.cache.page_shift) * a.cache.page_stride +
                                                   (slot & ((1 << a.cache.page_shift) - 1)) * a.cache.token_stride;
        if (t.turns) {
            const float* cp = a.cos + static_cast<size_t>(pos) * half;
            const float* sp = a.sin + static_cast<size_t>(pos) * half;
            if (PAIRS) {
                const float4 c4 = __ldg(reinterpret_cast<const float4*>(cp) + l), s4 = __ldg(reinterpret_cast<const float4*>(sp) + l);
                t.c[0] = c4.x; t.c[1] = c4.y; t.c[2] = c4.z; t.c[3] = c4.w;
                t.s[0] = s4.x; t.s[1] = s4.y; t.s[2] = s4.z; t.s[3] = s4.w;
            } else {
                const int at = first ? 8 * l : 8 * l - half;
                load8(cp + at, t.c);
                load8(sp + at, t.s);
                if (first) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) t.s[i] = -t.s[i];
                }
            }
        }
        // all lanes of a warp stay together (the exchanges): the loops run to the same bounds in every thread
        for (int hb = 0; hb < heads; hb += U * HPC) {
            if (hb > 0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int h = hb + h0 + u * HPC;
                    x4[u] = h < heads ? *reinterpret_cast<const uint4*>(xr + static_cast<size_t>(h) * D) : make_uint4(0, 0, 0, 0);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int hw = hb + u * HPC;
                if (hw >= heads) break;
                const int h = hw + h0;
                const uint32_t w4[4] = {x4[u].x, x4[u].y, x4[u].z, x4[u].w};
                float x[8], y[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = __uint_as_float(w4[i] << 16);
                    x[2 * i + 1] = __uint_as_float(w4[i] & 0xFFFF0000u);
                }
                // a warp whose heads are all values has nothing to compute
                if (__any_sync(0xffffffffu, h < n_qk)) {
                    float w[8];
                    const bool is_q = h < a.heads;
                    if (is_q ? w_null_q : w_null_k) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[i] = 1.0f;
                    } else {
                        load8((is_q ? a.q_weight : a.k_weight) + 8 * l, w);
                    }
                    norm_and_turn<D, PAIRS>(y, x, w, a.eps, a.rot > 0, t, l);
                }
                if (h >= heads) continue;
                if (h < a.heads) {
                    *reinterpret_cast<uint4*>(a.Q + static_cast<size_t>(m) * a.ldq + static_cast<size_t>(h) * D + 8 * l) =
                        make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                    continue;
                }
                const bool is_v = h >= n_qk;
                const int kvh = is_v ? h - n_qk : h - a.heads;
                if (!to_cache) {
                    *reinterpret_cast<uint4*>(a.K + static_cast<size_t>(m) * a.ldk + static_cast<size_t>(kvh) * D + 8 * l) =
                        make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                    continue;
                }
                const long long off = token_off + static_cast<long long>(kvh) * a.cache.head_stride + 8 * l;
                uint8_t* base = is_v ? a.cache.v : a.cache.k;
                if (E4M3) {
                    const float* sc = is_v ? a.cache.v_scale : a.cache.k_scale;
                    const float inv = sc != nullptr ? __fdiv_rn(1.0f, __ldg(sc + kvh)) : 1.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(is_v ? x[i] : y[i], inv);
                    *reinterpret_cast<uint2*>(base + off) = make_uint2(pack_e4m3x4(y[0], y[1], y[2], y[3]), pack_e4m3x4(y[4], y[5], y[6], y[7]));
                } else {
                    *reinterpret_cast<uint4*>(base + 2 * off) =
                        is_v ? x4[u] : make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                }
            }
        }
    }
}

template <int D>
cudaError_t launch_d(const QkArgs& a, bool e4m3, const cudaLaunchConfig_t& cfg)
{
    if (a.pairs) return e4m3 ? cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, true, true>, a) : cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, true, false>, a);
    return e4m3 ? cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, false, true>, a) : cudaLaunchKernelEx(&cfg, qk_norm_rope_kernel<D, false, false>, a);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const QkArgs& a, int head_dim, bool e4m3, int sm_count, cudaStream_t st)
{
    const int cap = sm_count * 3;                          // CTAs resident at once
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(a.M < cap ? a.M : cap), 1, 1);
    cfg.blockDim = dim3(QK_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (head_dim == 64) return launch_d<64>(a, e4m3, cfg);
    if (head_dim == 128) return launch_d<128>(a, e4m3, cfg);
    return launch_d<256>(a, e4m3, cfg);
}

}  // namespace rudder
