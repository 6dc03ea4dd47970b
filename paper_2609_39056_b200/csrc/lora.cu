// Low-rank adapters of many requests beside a shared projection: each row has an adapter of its own, or none.
//
//     h_m = X_m A_a^T  (rank_a numbers, fp32),     Y_m = bf16( base_m + scale_a (h_m B_a^T) ),     a = adapters[m]
//
// What bounds it: up to a few dozen rows the read of the adapters that occur (2 rank (K + N) bytes each), for thousands of rows base and Y (4 N bytes a row)
// and X.  The products themselves are small (2 rank (K + N) operations a row), so both run on mma.sync m16n8k16.  The order in which the 32 inputs of two steps are
// handed to the tensor core does not matter as long as both operands use the same one, so lane q takes 8 neighbours of each row: 16 bytes that the lane
// itself copies to shared memory, as it will use them, several steps ahead (cp.async), without ldmatrix or a swizzle.
//
// Measured: 4416 rows, rank 64, 2048 -> 8192 49.4 us (floor 25: X, base and Y once), of which the sorting 8, shrink 13 and expand 29; 64 rows of 40 adapters of rank up to
// 64, 2048 -> 6144 15.8 us (floor 4.5); one row of rank 16 4.9 us, two launches.  Expand issues in 51 % of its slots with 14 warps to an SM: the products (hi and lo, 16 us
// at the rate of mma.sync) and some 200 instructions for every 16 x 64 numbers of base and Y.
//
// Two launches: shrink writes h (a few KB, fp32) and expand reads it; the second is launched early, fetches base and B meanwhile and waits only for
// h.  A tile is rows of ONE adapter.  Up to kWindowRows rows: windows of 16 rows, a CTA for each adapter that occurs in a window (the
// first row that has it speaks for it), rows of other adapters are left out of its loads and its writes.  Above: a third launch in front
// sorts the rows by adapter (a counting sort in one CTA) and lists tiles of 64 rows; 256 rows of 20 adapters in turn would read B 9 times from L2
// as windows, and once as sorted tiles.  A row's result does not depend on its place in a tile.
//
// Rounding: products of bf16 numbers and sums in fp32; h enters the second product as two bf16 numbers hi + lo (2^-16, see low_part); Y is rounded once.
// Numbers at or behind an adapter's rank are not used, whatever they are.
#include "internal.cuh"
#include "paged.cuh"

namespace rudder {

namespace {

constexpr int kBadAdapter = 917;           // adapter at or beyond n_adapters (or below -1), or a rank outside 0..R
// Rows up to which they are taken as they lie.  Measured, windows / sorted, us, inputs -> outputs and rank 2048 -> 6144 64; 2048 -> 8192 16; 1024 -> 4096 32; 2048 -> 2048 128:
//   four adapters in turn   64 rows 12.6 / 17.3; 11.2 / 14.5; 7.7 / 12.3; 11.5 / 20.2    128 rows 20.0 / 19.2; 18.0 / 15.3; 11.0 / 12.7; 17.1 / 23.5    256 rows 35.2 / 22.8; 31.3 / 17.0; 18.3 / 13.8; 25.9 / 29.2
//   forty                   64 rows 15.4 / 35.2; 13.1 / 30.3; 8.6 / 22.8; 15.4 / 36.4    128 rows 26.2 / 39.3; 20.9 / 31.4; 12.7 / 21.7; 24.5 / 39.9    256 rows 47.7 / 40.8; 36.4 / 32.6; 22.3 / 22.2; 36.8 / 42.2
// Up to 96 rows windows won every case; the two cross between there and some hundreds of rows, later the more adapters there are and the larger the rank.  The bound lies in front of the crossing.
constexpr int kWindowRows = 64;
constexpr int kTileRows = 64;              // rows of a sorted tile
constexpr int kSortThreads = 1024;
constexpr int kNoTile = -2;

struct LoraParams {
    LoraArgs a;
    float* h;                              // [splits][M][RP]
    int RP, splits;
    const int4* tiles;                     // sorted: adapter (-1: none), first place in `perm`, rows
    const int32_t* perm;                   // sorted: rows by adapter
    int slots;                             // windows: CTAs a window, one per row that may speak for an adapter
};

// The rows of this CTA's tile (a row or -1) and their adapter, -1 for none; false if there is nothing to do.  All threads call it.
template <int TM>
__device__ __forceinline__ bool load_tile(const LoraParams& p, int tile, int (&s_rows)[TM], int& adapter) {
    __shared__ int s_adapter;
    const int tid = threadIdx.x;
    if (p.tiles != nullptr) {
        const int4 t = __ldcg(p.tiles + tile);
        if (t.z == 0) return false;
        if (tid < TM) s_rows[tid] = tid < t.z ? __ldcg(p.perm + t.y + tid) : -1;
        adapter = t.x;
        __syncthreads();
        return true;
    }
    const int first = tile / p.slots * 16, slot = tile % p.slots;
    if (tid < 32) {
        const int row = first + tid;
        const bool in = tid < 16 && row < p.a.M;
        int a = in ? p.a.adapters[row] : -1;
        if (a < -1 || a >= p.a.n_adapters) { record_bad_data(kBadAdapter); a = -1; }
        const int mine = __shfl_sync(0xffffffffu, a, slot);
        const uint32_t same = __ballot_sync(0xffffffffu, in && a == mine);
        if (tid < 16) s_rows[tid] = (same >> tid) & 1 ? row : -1;
        if (tid == 0) s_adapter = (same & ((2u << slot) - 1)) == 1u << slot ? mine : kNoTile;                    // or another row speaks for it, or there is no such row
    }
    __syncthreads();
    adapter = s_adapter;
    return adapter != kNoTile;
}
__device__ __forceinline__ int rank_of(const LoraParams& p, int adapter) {
    if (adapter < 0) return 0;
    const int r = p.a.ranks[adapter];
    if (r < 0 || r > p.a.R) {
        if (threadIdx.x == 0) record_bad_data(kBadAdapter);
        return min(max(r, 0), p.a.R);
    }
    return r;
}

// 16 bytes to shared memory on their way, or zeros.  (Through L2 alone: nothing here is read twice by an SM.)
__device__ __forceinline__ void fetch16(uint32_t dst, const void* src, bool valid) { cp_async16(dst, src, valid); }
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}

// h of a tile of 16 MW rows, ranks 8 NT blockIdx.y .., one of `splits` parts of K.  KG groups of MW warps take 32 inputs in turn and are added in order.
// A group's MW warps share A (each fetches its part of a step) and have rows of X of their own.  A step's fragments lie in the ring as the lanes use them, 512 bytes
// after 512 bytes; RING - 1 steps are on their way.
template <int MW, int NT, int KG>
struct ShrinkCfg {
    static constexpr int RING = 4, A = NT * 512, X = 1024, STEP = A + MW * X, BYTES = KG * RING * STEP;
};
template <int MW, int NT, int KG>
__global__ void __launch_bounds__(32 * MW * KG) lora_shrink_kernel(const LoraParams p)
{
    using C = ShrinkCfg<MW, NT, KG>;
    constexpr int TM = 16 * MW, RB = 8 * NT, RING = C::RING;
    static_assert(NT % MW == 0, "each warp fetches as many pieces of A");
    extern __shared__ __align__(16) uint8_t s_ring[];
    __shared__ int s_rows[TM];
    pdl_wait();
    pdl_launch_dependents();               // (behind the wait: what expand reads in front of its own wait is complete when it starts)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mw = warp % MW, kg = warp / MW;
    const int g = lane >> 2, q = lane & 3;
    int adapter;
    if (!load_tile(p, blockIdx.x, s_rows, adapter)) return;
    const int rank = rank_of(p, adapter), r0 = blockIdx.y * RB;
    if (r0 >= rank) return;
    const int blocks = (p.a.K + 31) / 32;
    const int b0 = static_cast<int>(static_cast<long long>(blocks) * blockIdx.z / p.splits), b1 = static_cast<int>(static_cast<long long>(blocks) * (blockIdx.z + 1) / p.splits);
    const int row0 = s_rows[16 * mw + g], row1 = s_rows[16 * mw + g + 8];
    const uint16_t* x0 = p.a.X + static_cast<int64_t>(max(row0, 0)) * p.a.ldx;
    const uint16_t* x1 = p.a.X + static_cast<int64_t>(max(row1, 0)) * p.a.ldx;
    const uint16_t* w = p.a.A + static_cast<int64_t>(adapter) * p.a.a_stride + static_cast<int64_t>(r0 + g) * p.a.lda;
    const uint32_t ring = smem_u32(s_ring) + kg * (RING * C::STEP) + 16 * lane;
    auto sync_group = [&]() {
        if (MW == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + kg), "n"(32 * MW) : "memory");
    };
    auto fetch = [&](int b, int slot) {
        if (b < b1) {
            const uint32_t at = ring + slot * C::STEP;
            const int k = 32 * b + 8 * q;
            const bool in = k < p.a.K;
            fetch16(at + C::A + mw * C::X, in ? x0 + k : x0, in && row0 >= 0);
            fetch16(at + C::A + mw * C::X + 512, in ? x1 + k : x1, in && row1 >= 0);
#pragma unroll
            for (int i = 0; i < NT / MW; ++i) {
                const int t = mw * (NT / MW) + i;
                const bool live = in && r0 + 8 * t + g < rank;
                fetch16(at + 512 * t, live ? w + 8 * t * p.a.lda + k : p.a.A, live);
            }
        }
        cp_async_commit();
    };
    float acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) fetch(b0 + kg + i * KG, i);
    int slot = 0;
#pragma unroll 1
    for (int b = b0 + kg; b < b1; b += KG) {
        cp_async_wait<RING - 2>();
        sync_group();
        fetch(b + (RING - 1) * KG, slot == 0 ? RING - 1 : slot - 1);             // where all of the group have read the step before
        const uint32_t at = ring + slot * C::STEP;
        const uint4 xa = lds16(at + C::A + mw * C::X), xb = lds16(at + C::A + mw * C::X + 512);
        const uint32_t a0[4] = {xa.x, xb.x, xa.y, xb.y}, a1[4] = {xa.z, xb.z, xa.w, xb.w};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint4 wa = lds16(at + 512 * t);
            mma16<false>(acc[t], a0, wa.x, wa.y);
            mma16<false>(acc[t], a1, wa.z, wa.w);
        }
        slot = slot + 1 == RING ? 0 : slot + 1;
    }
    cp_async_wait<0>();
    __syncthreads();                       // the ring is free: the groups' sums
    float* red = reinterpret_cast<float*>(s_ring);                 // [KG][TM][RB + 4]
    constexpr int P = RB + 4;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float* at = red + (kg * TM + 16 * mw + g) * P + 8 * t + 2 * q;
        *reinterpret_cast<float2*>(at) = make_float2(acc[t][0], acc[t][1]);
        *reinterpret_cast<float2*>(at + 8 * P) = make_float2(acc[t][2], acc[t][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TM * RB; i += 32 * MW * KG) {
        const int rl = i / RB, r = i % RB, row = s_rows[rl];
        if (row < 0 || r0 + r >= rank) continue;
        float s = red[rl * P + r];
#pragma unroll
        for (int k = 1; k < KG; ++k) s += red[(k * TM + rl) * P + r];
        p.h[(static_cast<size_t>(blockIdx.z) * p.a.M + row) * p.RP + r0 + r] = s;
    }
}
template <int MW, int NT, int KG>
constexpr int shrink_smem() {
    return ShrinkCfg<MW, NT, KG>::BYTES > KG * 16 * MW * (8 * NT + 4) * 4 ? ShrinkCfg<MW, NT, KG>::BYTES : KG * 16 * MW * (8 * NT + 4) * 4;
}

// Words of 8 neighbouring numbers of which the first `n` (1..8) count.
__device__ __forceinline__ uint4 keep_first(uint4 v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = n >= 2 * i + 2 ? w[i] : (n == 2 * i + 1 ? w[i] & 0xFFFFu : 0u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What stands behind the upper half of h's bits.  hi is cut off, not rounded (rounded it would be 2^-17 instead of 2^-16, of which a bf16 output shows nothing): lo has its sign, hi of
// a number is a number, and lo of a number that is not zero is not zero (2^-24 of h, or the least number, where bf16 holds h exactly).  So hi w + lo w is infinite or no number
// exactly where h w is, for an infinite weight w too: rounded, lo is 0 or of the other sign, and 0 x infinity and infinity - infinity are no numbers.  That costs the second product
// nothing; looking through its results instead cost 2 to 7 %.
__device__ __forceinline__ float low_part(float h) {
    if (h == 0.0f || !(fabsf(h) < INFINITY)) return h;
    const float rest = h - __uint_as_float(__float_as_uint(h) & 0xFFFF0000u);
    return copysignf(fmaxf(fmaxf(fabsf(rest), fabsf(h) * 0x1p-24f), 0x1p-133f), h);
}

// Y of a tile of 16 MW rows, `iters` times 64 NW columns from blockIdx.y on.  A warp has 16 rows x 64 columns: column 32 (j / 4) + 8 (c / 2) +
// 2 (j % 4) + c % 2 of them is column c of product j, so that a lane ends up with twice 8 neighbouring columns of two rows, and four lanes with a
// whole 64 bytes of a row (with 16 neighbouring columns a lane, each store had half of every 32-byte sector: 4416 rows x 8192 46 -> 37 us).  B comes in steps of 32 ranks of the 64 columns through a
// ring as in shrink (the MW warps with the same columns share it).  BASE: base comes through a ring of each warp, as many steps of columns ahead (many columns a
// CTA); else through registers, requested in front of everything (one step of columns a CTA, more CTAs to an SM).
template <int MW, int NW, int RING, bool BASE>
struct ExpandCfg {
    static constexpr int STEP = 8 * 512, B_BYTES = NW * RING * STEP, BASE_BYTES = BASE ? MW * NW * RING * 4 * 512 : 0;
    static size_t smem(int R) { return B_BYTES + BASE_BYTES + 2 * sizeof(uint16_t) * 16 * MW * ((static_cast<size_t>(R) + 31) / 32 * 32 + 8); }
};
template <int MW, int NW, int RING, bool BASE>
__global__ void __launch_bounds__(32 * MW * NW, 4) lora_expand_kernel(const LoraParams p, int iters)
{
    using C = ExpandCfg<MW, NW, RING, BASE>;
    constexpr int TM = 16 * MW, THREADS = 32 * MW * NW, STEP = C::STEP;
    extern __shared__ __align__(16) uint8_t s_expand[];            // B, base, then h: [2][TM][pitch], hi and lo
    uint16_t* s_h = reinterpret_cast<uint16_t*>(s_expand + C::B_BYTES + C::BASE_BYTES);
    __shared__ int s_rows[TM];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mw = warp % MW, nw = warp / MW;
    const int g = lane >> 2, q = lane & 3;
    int adapter;
    if (!load_tile(p, blockIdx.x, s_rows, adapter)) { pdl_wait(); return; }
    const int rank = rank_of(p, adapter), steps = max(1, (rank + 31) / 32), pitch = (p.a.R + 31) / 32 * 32 + 8;
    const float scale = adapter >= 0 ? p.a.scales[adapter] : 0.0f;
    const int n_first = blockIdx.y * iters * (64 * NW) + 64 * nw;
    const uint16_t* bw = p.a.B + static_cast<int64_t>(max(adapter, 0)) * p.a.b_stride + static_cast<int64_t>(8 * (g >> 1) + (g & 1)) * p.a.ldb + 8 * q;
    const uint32_t ring = smem_u32(s_expand) + nw * (RING * STEP) + 16 * lane;
    auto sync_group = [&]() {
        if (MW == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + nw), "n"(32 * MW) : "memory");
    };
    // this lane's two rows: columns 8 q .. + 7 and 32 + 8 q .. of the warp's 64
    bool has[2];
    const uint16_t* base_at[2];
    uint16_t* y_at[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int row = s_rows[16 * mw + g + 8 * e];
        has[e] = row >= 0;
        base_at[e] = p.a.base != nullptr ? p.a.base + static_cast<int64_t>(max(row, 0)) * p.a.ld_base + n_first + 8 * q : p.a.B;
        y_at[e] = p.a.Y + static_cast<int64_t>(max(row, 0)) * p.a.ldy + n_first + 8 * q;
    }
    auto base_there = [&](int off, int e) { return p.a.base != nullptr && has[e >> 1] && n_first + off + 8 * q + 32 * (e & 1) < p.a.N; };
    const uint32_t base_ring = smem_u32(s_expand) + C::B_BYTES + warp * (RING * 4 * 512) + 16 * lane;
    uint4 base[BASE ? 1 : 4];
    const int n_steps = iters * steps;
    int f_off = 0, f_step = 0, f_left = n_steps, f_base = 0;       // the step that is fetched next, and where its base goes
    auto fetch = [&](int slot) {
        if (f_left > 0) {
            const uint16_t* from = bw + static_cast<int64_t>(n_first + f_off) * p.a.ldb + 32 * f_step;
            const bool ranked = 32 * f_step + 8 * q < rank;
#pragma unroll
            for (int i = 0; i < 8 / MW; ++i) {
                const int j = mw * (8 / MW) + i, col = 32 * (j >> 2) + 2 * (j & 3);
                const bool live = ranked && n_first + f_off + col + 8 * (g >> 1) + (g & 1) < p.a.N;
                fetch16(ring + slot * STEP + 512 * j, live ? from + col * p.a.ldb : p.a.B, live);
            }
            if (BASE && f_step == 0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool live = base_there(f_off, e);
                    fetch16(base_ring + f_base * (4 * 512) + 512 * e, live ? base_at[e >> 1] + f_off + 32 * (e & 1) : p.a.B, live);
                }
                f_base = f_base + 1 == RING ? 0 : f_base + 1;
            }
            --f_left;
            if (++f_step == steps) {
                f_step = 0;
                f_off += 64 * NW;
            }
        }
        cp_async_commit();
    };
    if (!BASE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) base[BASE ? 0 : e] = base_there(0, e) ? *reinterpret_cast<const uint4*>(base_at[e >> 1] + 32 * (e & 1)) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < RING - 1; ++i) fetch(i);
    pdl_wait();
    pdl_launch_dependents();
    // h of the tile, split into hi and lo; places at or behind the rank are zeros
    for (int i = threadIdx.x; i < TM * steps * 8; i += THREADS) {
        const int rl = i / (steps * 8), r = 4 * (i % (steps * 8)), row = s_rows[rl];
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (row >= 0 && r < rank) {
#pragma unroll 2
            for (int s = 0; s < p.splits; ++s) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(p.h + (static_cast<size_t>(s) * p.a.M + row) * p.RP + r));
                v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (r + e >= rank) v[e] = 0.0f;
        }
        *reinterpret_cast<uint2*>(s_h + rl * pitch + r) = make_uint2(__byte_perm(__float_as_uint(v[0]), __float_as_uint(v[1]), 0x7632),
                                                                     __byte_perm(__float_as_uint(v[2]), __float_as_uint(v[3]), 0x7632));
        *reinterpret_cast<uint2*>(s_h + (TM + rl) * pitch + r) = make_uint2(bf16x2(low_part(v[0]), low_part(v[1])), bf16x2(low_part(v[2]), low_part(v[3])));
    }
    __syncthreads();
    const uint32_t hr0 = smem_u32(s_h) + 2 * ((16 * mw + g) * pitch + 8 * q);
    float acc[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
    int off = 0, step = 0, slot = 0, base_slot = 0;                // columns behind the first ones
#pragma unroll 1
    for (int left = n_steps; left > 0; --left) {
        cp_async_wait<RING - 2>();
        sync_group();
        fetch(slot == 0 ? RING - 1 : slot - 1);
        const uint32_t at = ring + slot * STEP;
        uint32_t h[2][2][4];                                       // hi, lo; the step's two halves
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const uint32_t hr = hr0 + 2 * (part * TM * pitch + 32 * step);
            const uint4 ha = lds16(hr), hb = lds16(hr + 16 * pitch);
            h[part][0][0] = ha.x; h[part][0][1] = hb.x; h[part][0][2] = ha.y; h[part][0][3] = hb.y;
            h[part][1][0] = ha.z; h[part][1][1] = hb.z; h[part][1][2] = ha.w; h[part][1][3] = hb.w;
        }
        const int kept = rank - 32 * step - 8 * q;                 // of this lane's eight ranks
        if (kept > 0 && kept < 8) {
            // what stands behind the rank is not this adapter's.  (Warps that share the step write the same.)
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                const uint4 wb = keep_first(lds16(at + 512 * j), kept);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + 512 * j), "r"(wb.x), "r"(wb.y), "r"(wb.z), "r"(wb.w) : "memory");
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint4 wb = lds16(at + 512 * j);
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                mma16<false>(acc[j], h[part][0], wb.x, wb.y);
                mma16<false>(acc[j], h[part][1], wb.z, wb.w);
            }
        }
        slot = slot + 1 == RING ? 0 : slot + 1;
        if (++step < steps) continue;
        step = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j0 = 4 * (e & 1), c = e < 2 ? 0 : 2;
            const uint4 bb = BASE ? lds16(base_ring + base_slot * (4 * 512) + 512 * e) : base[BASE ? 0 : e];
            const uint32_t b[4] = {bb.x, bb.y, bb.z, bb.w};
            uint32_t y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y[i] = rank > 0 ? bf16x2(fmaf(scale, acc[j0 + i][c], bf16_lo(b[i])), fmaf(scale, acc[j0 + i][c + 1], bf16_hi(b[i]))) : b[i];
            if (has[e >> 1] && n_first + off + 8 * q + 32 * (e & 1) < p.a.N) *reinterpret_cast<uint4*>(y_at[e >> 1] + off + 32 * (e & 1)) = make_uint4(y[0], y[1], y[2], y[3]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
        off += 64 * NW;
        base_slot = base_slot + 1 == RING ? 0 : base_slot + 1;
        if (!BASE && left > 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) base[BASE ? 0 : e] = base_there(off, e) ? *reinterpret_cast<const uint4*>(base_at[e >> 1] + off + 32 * (e & 1)) : make_uint4(0, 0, 0, 0);
        }
    }
    cp_async_wait<0>();
}

// Rows by adapter, those without one last, and the tiles of each.
__global__ void __launch_bounds__(kSortThreads) lora_sort_kernel(const LoraArgs a, int4* tiles, int max_tiles, int32_t* perm)
{
    extern __shared__ int s_count[];                               // [n_adapters + 1] rows, then the next place of each
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, lane = tid & 31, groups = a.n_adapters + 1;
    for (int i = tid; i < groups; i += kSortThreads) s_count[i] = 0;
    __syncthreads();
    auto group_of = [&](int m, bool tell) {
        const int x = a.adapters[m];
        if (x >= 0 && x < a.n_adapters) return x;
        if (x != -1 && tell) record_bad_data(kBadAdapter);
        return a.n_adapters;
    };
    // (neighbours mostly have the same adapter: one addition for all lanes of a warp that do; 4416 rows of four adapters one by one took 9 us)
    // The first rows stay in registers for the second pass.
    constexpr int KEPT = 8;
    int kept[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const int m = tid + i * kSortThreads;
        kept[i] = m < a.M ? group_of(m, true) : -1;
    }
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
        const uint32_t same = __match_any_sync(0xffffffffu, kept[i]);
        if (kept[i] >= 0 && lane == __ffs(same) - 1) atomicAdd(&s_count[kept[i]], __popc(same));
    }
    for (int m0 = tid - lane + KEPT * kSortThreads; m0 < a.M; m0 += kSortThreads) {
        const int m = m0 + lane, g = m < a.M ? group_of(m, true) : -1;
        const uint32_t same = __match_any_sync(0xffffffffu, g);
        if (g >= 0 && lane == __ffs(same) - 1) atomicAdd(&s_count[g], __popc(same));
    }
    __syncthreads();
    const int per = (groups + kSortThreads - 1) / kSortThreads, g0 = min(groups, tid * per), g1 = min(groups, g0 + per);
    int rows = 0, n_tiles = 0;
    for (int g = g0; g < g1; ++g) {
        rows += s_count[g];
        n_tiles += (s_count[g] + kTileRows - 1) / kTileRows;
    }
    int total, at_tile, at_row;
    at_row = block_prefix<kSortThreads>(rows, total);
    at_tile = block_prefix<kSortThreads>(n_tiles, total);
    for (int g = g0; g < g1; ++g) {
        const int n = s_count[g];
        s_count[g] = at_row;
        for (int i = 0; i < n; i += kTileRows) tiles[at_tile++] = make_int4(g < a.n_adapters ? g : -1, at_row + i, min(kTileRows, n - i), 0);
        at_row += n;
    }
    for (int t = total + tid; t < max_tiles; t += kSortThreads) tiles[t] = make_int4(-1, 0, 0, 0);
    __syncthreads();
    for (int i = 0, m0 = tid - lane; m0 < a.M; ++i, m0 += kSortThreads) {
        const int m = m0 + lane;
        int g = -1;
        if (i < KEPT) {
#pragma unroll
            for (int k = 0; k < KEPT; ++k)
                if (k == i) g = kept[k];
        } else if (m < a.M) {
            g = group_of(m, false);
        }
        const uint32_t same = __match_any_sync(0xffffffffu, g);
        const int leader = __ffs(same) - 1;
        int at = 0;
        if (g >= 0 && lane == leader) at = atomicAdd(&s_count[g], __popc(same));
        at = __shfl_sync(0xffffffffu, at, leader) + __popc(same & ((1u << lane) - 1));
        if (g >= 0) perm[at] = m;
    }
}

struct LoraPlan {
    bool sorted;
    int tiles, splits, RP, rank_blocks, rank_block, columns, iters;        // columns of a step of expand; steps of one of its CTAs
    size_t h_bytes, tiles_bytes, perm_bytes;
};
LoraPlan lora_plan(int M, int K, int N, int R, int n_adapters, int sm_count)
{
    LoraPlan l;
    l.sorted = M > kWindowRows;
    const int slots = M < 16 ? M : 16;
    l.tiles = l.sorted ? static_cast<int>(std::min<long long>(M, static_cast<long long>(M) / kTileRows + n_adapters + 1)) : (M + 15) / 16 * slots;
    l.rank_block = !l.sorted ? 16 : (R <= 32 ? 32 : 64);
    l.rank_blocks = (R + l.rank_block - 1) / l.rank_block;
    // K is cut until there is a CTA for three SMs of four, but not into parts of less than 512 (the sums of the parts are read again by every CTA of expand).  Tiles
    // are counted as if all rows had one adapter: more adapters only mean more CTAs (64 rows of 40 adapters in 4 parts 8.4 us, in 2 6.6, hence no more for several windows).
    const long long sure = l.sorted ? (M + kTileRows - 1) / kTileRows : (M + 15) / 16;
    l.splits = 1;
    while (l.splits < (l.sorted || M <= 16 ? 8 : 2) && 4 * sure * l.rank_blocks * l.splits < 3 * sm_count && K / (2 * l.splits) >= 512) l.splits *= 2;
    // columns: one wave of four CTAs to an SM, each with as many steps as it takes
    l.columns = l.sorted ? 64 : 256;
    const int blocks = (N + l.columns - 1) / l.columns;
    const long long tiles = l.sorted ? sure + (n_adapters < 8 ? n_adapters : 8) : l.tiles;
    const long long side = std::max<long long>(1, std::min<long long>(blocks, 4ll * sm_count / tiles));
    l.iters = static_cast<int>((blocks + side - 1) / side);
    l.RP = (R + 7) / 8 * 8;
    l.h_bytes = (static_cast<size_t>(l.splits) * M * l.RP * sizeof(float) + 255) / 256 * 256;
    l.tiles_bytes = l.sorted ? (static_cast<size_t>(l.tiles) * sizeof(int4) + 255) / 256 * 256 : 0;
    l.perm_bytes = l.sorted ? (static_cast<size_t>(M) * sizeof(int32_t) + 255) / 256 * 256 : 0;
    return l;
}
template <int MW, int NT, int KG>
cudaError_t launch_shrink(const LoraParams& p, const LoraPlan& l, cudaStream_t st)
{
    const dim3 grid(static_cast<unsigned>(l.tiles), static_cast<unsigned>(l.rank_blocks), static_cast<unsigned>(l.splits));
    return launch_pdl(lora_shrink_kernel<MW, NT, KG>, grid, 32 * MW * KG, shrink_smem<MW, NT, KG>(), 0, st, p);
}
template <int MW, int NW, int RING, bool BASE>
cudaError_t launch_expand(const LoraParams& p, const LoraPlan& l, cudaStream_t st)
{
    const int blocks = (p.a.N + l.columns - 1) / l.columns;
    const dim3 grid(static_cast<unsigned>(l.tiles), static_cast<unsigned>((blocks + l.iters - 1) / l.iters), 1);
    return launch_pdl(lora_expand_kernel<MW, NW, RING, BASE>, grid, 32 * MW * NW, ExpandCfg<MW, NW, RING, BASE>::smem(p.a.R), 0, st, p, l.iters);
}
template <int MW, int NW, int RING, bool BASE>
cudaError_t allow_expand()
{
    return cudaFuncSetAttribute(lora_expand_kernel<MW, NW, RING, BASE>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(ExpandCfg<MW, NW, RING, BASE>::smem(kMaxRank)));
}

}  // namespace

cudaError_t lora_init()
{
    cudaError_t e = allow_expand<4, 1, 3, true>();
    if (e == cudaSuccess) e = allow_expand<1, 4, 3, false>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_shrink_kernel<1, 2, 8>, cudaFuncAttributeMaxDynamicSharedMemorySize, shrink_smem<1, 2, 8>());
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_shrink_kernel<4, 4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, shrink_smem<4, 4, 2>());
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_shrink_kernel<4, 8, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, shrink_smem<4, 8, 2>());
    return e;
}

size_t lora_workspace_bytes(int M, int K, int N, int R, int n_adapters, int sm_count)
{
    const LoraPlan l = lora_plan(M, K, N, R, n_adapters, sm_count);
    return l.h_bytes + l.tiles_bytes + l.perm_bytes;
}

cudaError_t launch_lora(const LoraArgs& a, void* workspace, int sm_count, cudaStream_t st)
{
    const LoraPlan l = lora_plan(a.M, a.K, a.N, a.R, a.n_adapters, sm_count);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    LoraParams p = {};
    p.a = a;
    p.h = reinterpret_cast<float*>(ws);
    p.RP = l.RP; p.splits = l.splits;
    if (!l.sorted) {
        p.slots = a.M < 16 ? a.M : 16;
        const cudaError_t e = launch_shrink<1, 2, 8>(p, l, st);
        return e == cudaSuccess ? launch_expand<1, 4, 3, false>(p, l, st) : e;
    }
    int4* list = reinterpret_cast<int4*>(ws + l.h_bytes);
    int32_t* perm = reinterpret_cast<int32_t*>(ws + l.h_bytes + l.tiles_bytes);
    cudaError_t e = launch_pdl(lora_sort_kernel, dim3(1, 1, 1), kSortThreads, sizeof(int) * static_cast<size_t>(a.n_adapters + 1), 0, st, a, list, l.tiles, perm);
    if (e != cudaSuccess) return e;
    p.tiles = list;
    p.perm = perm;
    e = l.rank_block <= 32 ? launch_shrink<4, 4, 2>(p, l, st) : launch_shrink<4, 8, 2>(p, l, st);
    if (e != cudaSuccess) return e;
    return launch_expand<4, 1, 3, true>(p, l, st);
}

}  // namespace rudder
