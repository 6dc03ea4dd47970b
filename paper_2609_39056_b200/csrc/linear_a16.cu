// Products of one to sixteen rows with 4-bit weights, activations kept in 16 bits (no activation quantisation):
//     y_mj = sum_k (x_mk dinv_k) q_jk Delta_W[j, g(k)] + b_j
// on the packed weights of rudder_pack_weights (D folded in, Eq. 6; gains cancel without a quantiser between them).
//
// Bound by the stream of packed weights (K N / 2 bytes) and, at these sizes (1 to 20 MB), as much by latency.  The
// multiply-adds run on mma.sync.m16n8k16 with the WEIGHTS as the 16-row operand, taken straight from global memory:
// 16 output channels x 16 input channels per instruction, the token side only 8 columns wide.  On the CUDA cores
// the same work is a conversion and an FMA per weight and row, 2 x the issue slots that 6.5 TB/s of nibbles leave.
//
// Precision: v = x dinv is an fp32 product (24 bits), the MMA takes bf16.  Each row of v therefore enters as TWO columns,
// hi = bf16(v) and lo = bf16(v - hi): 16 bits of v, an error of 2^-17 of each product, far below the bf16 step of y; 8
// columns hold 4 rows and the second column costs nothing up to 4 rows.  The weight operand is exact: integers in
// [-7, 7], or E2M1 x UE4M3 (2 + 4 significant bits).  Products and sums in fp32.
//
// Work split: a CTA owns 16 output channels over all of K, its 16 warps take steps of 128 input channels in turn and
// their sums are added in warp order (deterministic), no scratch in global memory.  v is computed once per CTA and
// staged in shared memory in fragment order (persistent CTAs keep it for all their tiles); where it does not fit, a cluster of four CTAs
// shares 64 output channels and splits K.  The order of the input channels
// inside a 64-channel block is free as long as both operands use the same one: each is the order in which the packed
// layout's nibbles come out of a word by one shift and one mask per pair.
//
// Measured: 1 row x 2048 x 2048 W4A8 3.0 us (an empty launch 2.0), 8 rows x 8192 x 2048 NVFP4 9.0 us = 1.1 TB/s, 1 row x 8192 x 8192 W4A8 17.5 us = 2.0 TB/s: the latency
// of the first weights, the staging of v, and for many tiles the sums over the warps between two barriers of each (issue slots 48 %, ALU 48 %, DRAM a fifth).
#include "internal.cuh"
#include "paged.cuh"

#include <cuda_bf16.h>

#include "fp4.cuh"

namespace rudder {

namespace {

enum A16Layout { A16_INT, A16_SIGNMAG, A16_NVFP4 };

struct LinearA16Params {
    const uint16_t* X; int64_t ldx;
    uint16_t* Y; int64_t ldy;
    const uint8_t* codes;
    const float* scales_t;          // INT: [K/G][N] Delta_W / 16
    const uint8_t* scales_c;        // NVFP4: UE4M3 [N][K/16]
    const float* dinv;
    const float* tensor_scale;
    const float* bias;
    int M, N, K, G;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t hsub2_bf16(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t hmul2_bf16(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Pair t (0..3) of a packed word as two bf16 weights.
//   INT: bits 4 t of both halves of the word; 0x4300 | (n ^ 8) is the bf16 number 128 + 8 + code, minus 136 exact.
//   SIGNMAG: magnitudes at 4 t of both halves, signs at bits 3 + 8 t and 7 + 8 t; 128 + magnitude, minus 128, then the signs.
//   NVFP4: the three low bits moved to bit 6 are an E2M1 magnitude in bf16's exponent range from 2^-126 on (subnormals
//   included); `mul` brings it back times the block scale (exact: 6 significant bits).
template <int LAYOUT>
__device__ __forceinline__ uint32_t weight_pair(uint32_t w, int t, uint32_t mul) {
    if (LAYOUT == A16_INT) return hsub2_bf16(((w >> (4 * t)) & 0x000F000Fu) ^ 0x43084308u, 0x43084308u);
    if (LAYOUT == A16_SIGNMAG) {
        const uint32_t mag = hsub2_bf16(((w >> (4 * t)) & 0x00070007u) | 0x43004300u, 0x43004300u);
        const uint32_t lo = (t < 2 ? (w << (12 - 8 * t)) : (w >> (8 * t - 12))) & 0x00008000u;
        const uint32_t hi = (w << (24 - 8 * t)) & 0x80000000u;
        return mag | lo | hi;
    }
    const uint32_t mag = (t < 2 ? w << (6 - 4 * t) : w >> (4 * t - 6)) & 0x01C001C0u;
    return hmul2_bf16(((w << (12 - 4 * t)) & 0x80008000u) | mag, mul);
}
// Offsets (inside the lane's channels of a 64-channel block) of the two channels of pair t of word j.
//   INT: lane q holds channels base .. base + 7 and base + 16 .. base + 23, base = 32 (q >> 1) + 8 (q & 1): byte b of the
//   run = channels b (low nibble) and 16 + b.  Word j: pair t = nibbles t and t + 4 = bytes t / 2 and t / 2 + 2.
//   As an index 0..15 into the 8 + 8 channels: 4 j + (t >> 1) + 8 (t & 1) and that + 2.
//   SIGNMAG: pair t = channels 4 j + t and 16 + 4 j + t -> indices 4 j + t, 8 + 4 j + t.
//   NVFP4: channels 16 q + 8 j + t and + 4.
template <int LAYOUT>
__device__ __forceinline__ constexpr int pair_index(int j, int t, int half) {
    if (LAYOUT == A16_INT) return 4 * j + (t >> 1) + 8 * (t & 1) + 2 * half;
    if (LAYOUT == A16_SIGNMAG) return 4 * j + t + 8 * half;
    return 8 * j + t + 4 * half;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy8(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
// The split of two fp32 values: hi and lo as packed bf16 pairs.  An infinite one is all hi: what is left over would be infinity - infinity.
// (8 rows x 8192 x 2048 8.85 -> 9.0 us; one look at the largest of 16 values and a branch 8.95, but 16 rows x 2048 x 2048 5.55 against 5.45.)
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(b), "f"(a));
    const float ha = __uint_as_float(hi << 16), hb = __uint_as_float(hi & 0xFFFF0000u);
    const float ra = fabsf(ha) == INFINITY ? 0.0f : __fsub_rn(a, ha), rb = fabsf(hb) == INFINITY ? 0.0f : __fsub_rn(b, hb);
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(rb), "f"(ra));
}

__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_dsmem(const void* local, uint32_t rank) {
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(local)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// NT: tiles of 8 columns (4 rows each).  KS: CTAs of a cluster that share 16 KS output channels, each with 1 / KS of the input
// channels.  A step = 128 input channels of 16 output channels: 1 KB of codes and 128 bytes of scales, in a ring of ST stages per
// warp filled by cp.async; the ring runs on over the tiles of a persistent CTA.  v fragments in shared memory, one block of 64
// channels = [4 steps of the MMA][NT tiles][8 columns][4 lanes q][8 bytes], padded by 32 bytes so that the blocks start on
// different banks.
template <int LAYOUT, int NT, int KS>
struct A16Cfg {
    static constexpr int WARPS = 16, THREADS = 32 * WARPS;
    static constexpr int WK = WARPS / KS;                  // warps that share a tile of 16 channels: every WK-th step each
    static constexpr int ST = NT == 4 ? 3 : 4;
    static constexpr int kStage = 1024 + 128;
    static constexpr int kBlockBytes = 4 * NT * 256 + 32;
    static constexpr int kRing = WARPS * ST * kStage;
    static constexpr int kRed = (WARPS + KS) * 4 * NT * 17 * 4;
    static constexpr int smem(int n_blocks) { return kRing + kRed + n_blocks * kBlockBytes; }
};

template <int LAYOUT, int NT, int KS>
__global__ void __launch_bounds__(A16Cfg<LAYOUT, NT, KS>::THREADS, 1) linear_a16_kernel(const LinearA16Params p)
{
    using C = A16Cfg<LAYOUT, NT, KS>;
    constexpr int WARPS = C::WARPS, THREADS = C::THREADS, WK = C::WK, ST = C::ST, kBlockBytes = C::kBlockBytes;
    extern __shared__ __align__(16) uint8_t smem_a16[];
    float (*red)[4 * NT][17] = reinterpret_cast<float (*)[4 * NT][17]>(smem_a16 + C::kRing);                  // [WARPS]: the warps' sums
    float (*part)[4 * NT][17] = red + WARPS;               // [KS]: this CTA's sums for its cluster
    uint8_t* vfrag = smem_a16 + C::kRing + C::kRed;
    pdl_launch_dependents();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, q = lane & 3;
    const int mt = warp % KS, wk = warp / KS;
    const int rank = KS > 1 ? static_cast<int>(blockIdx.x % KS) : 0;
    const int all_steps = p.K >> 7, per_cta = (all_steps + KS - 1) / KS;
    const int s_begin = min(all_steps, rank * per_cta), s_end = min(all_steps, s_begin + per_cta);
    const int n_tiles = p.N / (16 * KS), tile0 = blockIdx.x / KS, tile_step = gridDim.x / KS;
    const size_t row_bytes = static_cast<size_t>(p.K >> 1);
    const uint8_t* ring = smem_a16 + warp * (ST * C::kStage);
    const uint32_t ring_u = smem_u32(ring);

    // one step of weights into a stage: lane i copies halves of row i / 2 of both blocks, and its piece of the scales
    auto issue = [&](int tile, int step, int stage) {
        const int n0 = (tile * KS + mt) * 16;
        const uint32_t dst = ring_u + stage * C::kStage;
        const uint8_t* src = p.codes + static_cast<size_t>(n0 + (lane >> 1)) * row_bytes + static_cast<size_t>(step) * 64 + 16 * (lane & 1);
        copy16(dst + 16 * lane, src);
        copy16(dst + 512 + 16 * lane, src + 32);
        if (LAYOUT == A16_NVFP4) {
            if (lane < 16) copy8(dst + 1024 + 8 * lane, p.scales_c + static_cast<size_t>(n0 + lane) * (p.K >> 4) + 8 * step);
        } else {
            if (lane < 8) copy16(dst + 1024 + 16 * lane, p.scales_t + static_cast<size_t>(((step << 7) + ((lane >> 2) << 6)) / p.G) * p.N + n0 + 4 * (lane & 3));
        }
    };
    int f_tile = tile0, f_step = s_begin + wk;             // what is requested next
    auto issue_next = [&](int stage) {
        if (s_begin + wk < s_end && f_tile < n_tiles) {
            issue(f_tile, f_step, stage);
            f_step += WK;
            if (f_step >= s_end) { f_step = s_begin + wk; f_tile += tile_step; }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // the weights do not depend on the kernel before this one
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) issue_next(i);
    // UE4M3 scale x 2^117: together with the 2^-126 of the raw codes the weights come out times 2^-9 (448 x 2^117 is in range)
    const float out_scale = (LAYOUT == A16_NVFP4) ? 512.0f * __ldg(p.tensor_scale) : 16.0f;
    pdl_wait();
    {
        // v: item = (block, lane q), rows m, m + groups, ...: 16 channels -> 4 steps x (hi, lo) x 8 bytes
        const int items = 8 * (s_end - s_begin);
        const int groups = items > 0 && items < THREADS ? THREADS / items : 1;   // threads that share an item, every groups-th row each
        const int stride = items < THREADS ? max(items, 1) : THREADS;
        for (int r = tid % stride, m0 = tid / stride; r < items && m0 < groups; r += stride) {
            const int blk = r >> 2, qq = r & 3;
            const int ch = 128 * s_begin + 64 * blk + (LAYOUT == A16_NVFP4 ? 16 * qq : 32 * (qq >> 1) + 8 * (qq & 1));
            constexpr int second = (LAYOUT == A16_NVFP4) ? 8 : 16;
            float dd[16];
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
                const float4 d0 = __ldg(reinterpret_cast<const float4*>(p.dinv + ch + hh * second));
                const float4 d1 = __ldg(reinterpret_cast<const float4*>(p.dinv + ch + hh * second) + 1);
                dd[8 * hh] = d0.x; dd[8 * hh + 1] = d0.y; dd[8 * hh + 2] = d0.z; dd[8 * hh + 3] = d0.w;
                dd[8 * hh + 4] = d1.x; dd[8 * hh + 5] = d1.y; dd[8 * hh + 6] = d1.z; dd[8 * hh + 7] = d1.w;
            }
#pragma unroll 2
            for (int m = m0; m < p.M; m += groups) {
                float v[16];
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    const uint4 x4 = *reinterpret_cast<const uint4*>(p.X + static_cast<size_t>(m) * p.ldx + ch + hh * second);
                    const uint32_t xw[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        v[8 * hh + 2 * i] = __fmul_rn(__uint_as_float(xw[i] << 16), dd[8 * hh + 2 * i]);
                        v[8 * hh + 2 * i + 1] = __fmul_rn(__uint_as_float(xw[i] & 0xFFFF0000u), dd[8 * hh + 2 * i + 1]);
                    }
                }
                uint8_t* dst = vfrag + static_cast<size_t>(blk) * kBlockBytes + (m >> 2) * 256 + 2 * (m & 3) * 32 + qq * 8;
#pragma unroll
                for (int st = 0; st < 4; ++st) {                        // MMA step st = pairs 2 (st & 1), + 1 of word st >> 1
                    uint2 hi, lo;
                    split2(v[pair_index<LAYOUT>(st >> 1, 2 * (st & 1), 0)], v[pair_index<LAYOUT>(st >> 1, 2 * (st & 1), 1)], hi.x, lo.x);
                    split2(v[pair_index<LAYOUT>(st >> 1, 2 * (st & 1) + 1, 0)], v[pair_index<LAYOUT>(st >> 1, 2 * (st & 1) + 1, 1)], hi.y, lo.y);
                    *reinterpret_cast<uint2*>(dst + st * NT * 256) = hi;
                    *reinterpret_cast<uint2*>(dst + st * NT * 256 + 32) = lo;
                }
            }
        }
    }
    __syncthreads();

    int stage = 0;
    for (int tile = tile0; tile < n_tiles; tile += tile_step) {
        float acc[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
        for (int step = s_begin + wk; step < s_end; step += WK) {
            asm volatile("cp.async.wait_group %0;" ::"n"(ST - 2) : "memory");
            __syncwarp();
            issue_next(stage == 0 ? ST - 1 : stage - 1);   // the stage read in the step before
            const uint8_t* sp = ring + stage * C::kStage;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const uint2 wa = *reinterpret_cast<const uint2*>(sp + 512 * b + 8 * lane);            // row g, 8 q bytes in
                const uint2 wb = *reinterpret_cast<const uint2*>(sp + 512 * b + 256 + 8 * lane);      // row g + 8
                uint32_t ma = 0, mb = 0;
                float ga = 1.0f, gb = 1.0f;
                if (LAYOUT == A16_NVFP4) {
                    const float fa = ue4m3_to_f32(sp[1024 + 8 * g + 4 * b + q]) * 0x1p117f, fb = ue4m3_to_f32(sp[1024 + 64 + 8 * g + 4 * b + q]) * 0x1p117f;
                    ma = __float_as_uint(fa) >> 16; ma |= ma << 16;      // 4 significant bits: exact in bf16
                    mb = __float_as_uint(fb) >> 16; mb |= mb << 16;
                } else {
                    ga = *reinterpret_cast<const float*>(sp + 1024 + 64 * b + 4 * g);
                    gb = *reinterpret_cast<const float*>(sp + 1024 + 64 * b + 32 + 4 * g);
                }
                float c[NT][4];
#pragma unroll
                for (int t = 0; t < NT; ++t) c[t][0] = c[t][1] = c[t][2] = c[t][3] = 0.0f;
                const uint8_t* vb = vfrag + static_cast<size_t>(2 * (step - s_begin) + b) * kBlockBytes + lane * 8;
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    const uint32_t wx = st < 2 ? wa.x : wa.y, wy = st < 2 ? wb.x : wb.y;
                    const int t0 = 2 * (st & 1);
                    const uint32_t a0 = weight_pair<LAYOUT>(wx, t0, ma), a2 = weight_pair<LAYOUT>(wx, t0 + 1, ma);
                    const uint32_t a1 = weight_pair<LAYOUT>(wy, t0, mb), a3 = weight_pair<LAYOUT>(wy, t0 + 1, mb);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const uint2 v = *reinterpret_cast<const uint2*>(vb + (st * NT + t) * 256);
                        mma_bf16(c[t], a0, a1, a2, a3, v.x, v.y);
                    }
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    acc[t][0] = fmaf(c[t][0], ga, acc[t][0]);
                    acc[t][1] = fmaf(c[t][1], ga, acc[t][1]);
                    acc[t][2] = fmaf(c[t][2], gb, acc[t][2]);
                    acc[t][3] = fmaf(c[t][3], gb, acc[t][3]);
                }
            }
            stage = stage + 1 == ST ? 0 : stage + 1;
        }
        // hi and lo of row 4 t + q are the two columns this lane holds; the warps' sums in warp order, the CTAs' in rank order
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            red[warp][4 * t + q][g] = acc[t][0] + acc[t][1];
            red[warp][4 * t + q][g + 8] = acc[t][2] + acc[t][3];
        }
        __syncthreads();
        for (int o = tid; o < 16 * KS * p.M; o += THREADS) {
            const int n = o & 15, t = (o >> 4) % KS, m = (o >> 4) / KS;
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WK; ++w) sum += red[w * KS + t][m][n];
            if (KS > 1) {
                part[t][m][n] = sum;
            } else {
                const float b = p.bias != nullptr ? p.bias[tile * 16 + n] : 0.0f;
                p.Y[static_cast<size_t>(m) * p.ldy + tile * 16 + n] = __bfloat16_as_ushort(__float2bfloat16_rn(fmaf(sum, out_scale, b)));
            }
        }
        if (KS > 1) {
            cluster_sync_all();
            for (int o = tid; o < 16 * p.M; o += THREADS) {                     // rank r finishes the r-th 16 channels
                const int n = o & 15, m = o >> 4, col = (tile * KS + rank) * 16 + n;
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < KS; ++r) sum += ld_dsmem(&part[rank][m][n], r);
                const float b = p.bias != nullptr ? p.bias[col] : 0.0f;
                p.Y[static_cast<size_t>(m) * p.ldy + col] = __bfloat16_as_ushort(__float2bfloat16_rn(fmaf(sum, out_scale, b)));
            }
            cluster_sync_all();                                                 // the peers have read `part`
        } else {
            __syncthreads();                                                    // `red` has been read
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

constexpr int kMaxSmem = 226 * 1024;

template <int LAYOUT, int NT, int KS>
cudaError_t launch_one(const LinearA16Params& p, int sm_count, cudaStream_t st)
{
    using C = A16Cfg<LAYOUT, NT, KS>;
    const int n_blocks = 2 * (((p.K >> 7) + KS - 1) / KS);
    const int tiles = p.N / (16 * KS), most = sm_count / KS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((tiles < most ? tiles : most) * KS), 1, 1);
    cfg.blockDim = dim3(C::THREADS, 1, 1);
    cfg.dynamicSmemBytes = static_cast<size_t>(C::smem(n_blocks));
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = KS; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = KS > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, linear_a16_kernel<LAYOUT, NT, KS>, p);
}
template <int LAYOUT, int NT, int KS>
bool fits(int K) { return A16Cfg<LAYOUT, NT, KS>::smem(2 * (((K >> 7) + KS - 1) / KS)) <= kMaxSmem; }
// One CTA per 16 channels while v fits beside the ring (K up to 9216, 4480, 2432 for 4, 8, 16 rows); a cluster of four
// with a quarter of K each beyond that.  Measured, one / four: 1 x 2048 x 2048 2.9 / 4.0 us, 8 x 4096 x 4096 7.8 / 11.2 us (the cluster's
// two barriers per tile); where v does not fit, four against the CTA that stages it in pieces: 8 x 8192 x 2048 8.8 / 11.0 us,
// 16 x 8192 x 2048 11.1 / 17.9 us.
template <int NT, int KS>
constexpr bool widest(int K) { return A16Cfg<A16_INT, NT, KS>::smem(2 * (K / 128 / KS)) <= kMaxSmem && A16Cfg<A16_INT, NT, KS>::smem(2 * (K / 128 / KS + 1)) > kMaxSmem; }
static_assert(widest<1, 1>(9216) && widest<2, 1>(4480) && widest<4, 1>(2432) && widest<1, 4>(36864) && widest<2, 4>(17920) && widest<4, 4>(9216), "limits stated here and in rudder.h");
template <int LAYOUT, int NT>
cudaError_t launch_nt(const LinearA16Params& p, int sm_count, cudaStream_t st)
{
    if (fits<LAYOUT, NT, 1>(p.K)) return launch_one<LAYOUT, NT, 1>(p, sm_count, st);
    return launch_one<LAYOUT, NT, 4>(p, sm_count, st);
}
template <int LAYOUT>
cudaError_t launch_layout(LinearA16Params p, int sm_count, cudaStream_t st)
{
    // as many rows per pass as v fits in shared memory for: 16, 8 or 4
    const int most = fits<LAYOUT, 4, 4>(p.K) ? 16 : (fits<LAYOUT, 2, 4>(p.K) ? 8 : 4);
    for (int left = p.M; left > 0; left -= most) {
        p.M = left < most ? left : most;
        const cudaError_t e = p.M <= 4 ? launch_nt<LAYOUT, 1>(p, sm_count, st) : (p.M <= 8 ? launch_nt<LAYOUT, 2>(p, sm_count, st) : launch_nt<LAYOUT, 4>(p, sm_count, st));
        if (e != cudaSuccess) return e;
        p.X += static_cast<int64_t>(p.M) * p.ldx;
        p.Y += static_cast<int64_t>(p.M) * p.ldy;
    }
    return cudaSuccess;
}
template <int LAYOUT, int NT>
cudaError_t init_one()
{
    cudaError_t e = cudaFuncSetAttribute(linear_a16_kernel<LAYOUT, NT, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(linear_a16_kernel<LAYOUT, NT, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    return e;
}
template <int LAYOUT>
cudaError_t init_layout()
{
    cudaError_t e = init_one<LAYOUT, 1>();
    if (e == cudaSuccess) e = init_one<LAYOUT, 2>();
    if (e == cudaSuccess) e = init_one<LAYOUT, 4>();
    return e;
}

}  // namespace

cudaError_t linear_a16_init()
{
    cudaError_t e = init_layout<A16_INT>();
    if (e == cudaSuccess) e = init_layout<A16_SIGNMAG>();
    if (e == cudaSuccess) e = init_layout<A16_NVFP4>();
    return e;
}

bool linear_a16_fits(int K) { return fits<A16_NVFP4, 1, 4>(K); }

cudaError_t launch_linear_a16(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M, const float* bias, uint16_t* Y, int64_t ldy, int sm_count,
                              cudaStream_t st)
{
    LinearA16Params p;
    p.X = X; p.ldx = ldx; p.Y = Y; p.ldy = ldy;
    p.codes = w->codes; p.scales_t = w->scales_t; p.scales_c = static_cast<const uint8_t*>(w->scales_c);
    p.dinv = w->dinv; p.tensor_scale = w->tensor_scale; p.bias = bias;
    p.M = M; p.N = w->N; p.K = w->K; p.G = w->G;
    if (w->scheme == RUDDER_W4A4_NVFP4) return launch_layout<A16_NVFP4>(p, sm_count, st);
    return w->f8 ? launch_layout<A16_SIGNMAG>(p, sm_count, st) : launch_layout<A16_INT>(p, sm_count, st);
}

}  // namespace rudder
