// Low-rank adapters of many requests beside a shared projection: each row has an adapter of its own, or none.
//
//     h_m = X_m A_a^T  (rank_a numbers, fp32),     Y_m = bf16( base_m + scale_a (h_m B_a^T) ),     a = adapters[m]
//
// What bounds it: up to a few dozen rows the read of the adapters that occur (2 rank (K + N) bytes each), for thousands of rows base and Y (4 N bytes a row)
// and X.  The products themselves are small (2 rank (K + N) operations a row), so both run on mma.sync m16n8k16 with operands loaded straight into
// registers, 16 bytes a lane: the order in which the 32 inputs of two steps are handed to the tensor core does not matter as long as both operands use the
// same one, so lane q takes 8 neighbours of each row.  No staging, no barrier in either main loop.
//
// Two launches: shrink writes h (a few KB, fp32) and expand reads it; the second is launched early, fetches base and B meanwhile and waits only for
// h.  A tile is rows of ONE adapter.  Up to kWindowRows rows: windows of 16 rows, a CTA for each adapter that occurs in a window (the
// first row that has it speaks for it), rows of other adapters are left out of its loads and its writes.  Above: a third launch in front
// sorts the rows by adapter (a counting sort in one CTA) and lists tiles of 64 rows; 256 rows of 20 adapters in turn would read B 9 times from L2
// as windows, and once as sorted tiles.  A row's result does not depend on its place in a tile.
//
// Rounding: products of bf16 numbers and sums in fp32; h enters the second product as two bf16 numbers hi + lo (2^-17); Y is rounded once.
// Numbers at or behind an adapter's rank are not used, whatever they are.
#include "internal.cuh"
#include "paged.cuh"

namespace rudder {

namespace {

constexpr int kBadAdapter = 917;           // adapter at or beyond n_adapters (or below -1), or a rank outside 0..R
constexpr int kWindowRows = 64;            // rows up to which they are taken as they lie
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

// h of a tile of 16 MW rows, ranks 8 NT blockIdx.y .., one of `splits` parts of K.  KG groups of MW warps take 32 inputs in turn and are added in order.
template <int MW, int NT, int KG>
__global__ void __launch_bounds__(32 * MW * KG) lora_shrink_kernel(const LoraParams p)
{
    constexpr int TM = 16 * MW, RB = 8 * NT;
    __shared__ int s_rows[TM];
    __shared__ __align__(16) float red[KG][TM][RB + 4];            // (written two at a time)
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
    float acc[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
    constexpr int U = NT <= 2 ? 4 : 2;     // blocks in flight
    const uint4 zero = make_uint4(0, 0, 0, 0);
    for (int b = b0 + kg; b < b1; b += KG * U) {
        uint4 xa[U], xb[U], wa[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = 32 * (b + u * KG) + 8 * q;
            const bool in = b + u * KG < b1 && k < p.a.K;
            xa[u] = in && row0 >= 0 ? *reinterpret_cast<const uint4*>(x0 + k) : zero;
            xb[u] = in && row1 >= 0 ? *reinterpret_cast<const uint4*>(x1 + k) : zero;
#pragma unroll
            for (int t = 0; t < NT; ++t) wa[u][t] = in && r0 + 8 * t + g < rank ? *reinterpret_cast<const uint4*>(w + 8 * t * p.a.lda + k) : zero;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t a0[4] = {xa[u].x, xb[u].x, xa[u].y, xb[u].y}, a1[4] = {xa[u].z, xb[u].z, xa[u].w, xb[u].w};
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                mma16<false>(acc[t], a0, wa[u][t].x, wa[u][t].y);
                mma16<false>(acc[t], a1, wa[u][t].z, wa[u][t].w);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        *reinterpret_cast<float2*>(&red[kg][16 * mw + g][8 * t + 2 * q]) = make_float2(acc[t][0], acc[t][1]);
        *reinterpret_cast<float2*>(&red[kg][16 * mw + g + 8][8 * t + 2 * q]) = make_float2(acc[t][2], acc[t][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TM * RB; i += 32 * MW * KG) {
        const int rl = i / RB, r = i % RB, row = s_rows[rl];
        if (row < 0 || r0 + r >= rank) continue;
        float s = red[0][rl][r];
#pragma unroll
        for (int k = 1; k < KG; ++k) s += red[k][rl][r];
        p.h[(static_cast<size_t>(blockIdx.z) * p.a.M + row) * p.RP + r0 + r] = s;
    }
}

// Words of 8 neighbouring numbers of which the first `n` (1..8) count.
__device__ __forceinline__ uint4 keep_first(uint4 v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = n >= 2 * i + 2 ? w[i] : (n == 2 * i + 1 ? w[i] & 0xFFFFu : 0u);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Y of a tile of 16 MW rows, `iters` times 64 NW columns from blockIdx.y on.  A warp has 16 rows x 64 columns: column 16 (c / 2) + 2 j + c % 2 of
// them is column c of product j, so that a lane ends up with 16 neighbouring columns of two rows.
template <int MW, int NW>
__global__ void __launch_bounds__(32 * MW * NW) lora_expand_kernel(const LoraParams p, int iters)
{
    constexpr int TM = 16 * MW, THREADS = 32 * MW * NW;
    extern __shared__ __align__(16) uint16_t s_h[];                // [2][TM][pitch]: hi, lo
    __shared__ int s_rows[TM];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mw = warp % MW, nw = warp / MW;
    const int g = lane >> 2, q = lane & 3;
    int adapter;
    if (!load_tile(p, blockIdx.x, s_rows, adapter)) { pdl_wait(); return; }
    const int rank = rank_of(p, adapter), steps = (rank + 31) / 32, pitch = (p.a.R + 31) / 32 * 32 + 8;
    const float scale = adapter >= 0 ? p.a.scales[adapter] : 0.0f;
    const int row0 = s_rows[16 * mw + g], row1 = s_rows[16 * mw + g + 8];
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const uint16_t* bw = p.a.B + static_cast<int64_t>(max(adapter, 0)) * p.a.b_stride;
    bool waited = false;
    for (int it = 0; it < iters; ++it) {
        const int n0 = (blockIdx.y * iters + it) * (64 * NW) + 64 * nw, nl = n0 + 16 * q;
        if (n0 - 64 * nw >= p.a.N) break;                          // (the whole CTA)
        uint4 base[4], wb[8];
        auto load_w = [&](int step) {
            const int r = 32 * step + 8 * q;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int n = n0 + 16 * (g >> 1) + 2 * j + (g & 1);
                wb[j] = r < rank && n < p.a.N ? *reinterpret_cast<const uint4*>(bw + static_cast<int64_t>(n) * p.a.ldb + r) : zero;
                if (r + 8 > rank && r < rank) wb[j] = keep_first(wb[j], rank - r);
            }
        };
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = e < 2 ? row0 : row1, n = nl + 8 * (e & 1);
            base[e] = p.a.base != nullptr && row >= 0 && n < p.a.N ? *reinterpret_cast<const uint4*>(p.a.base + static_cast<int64_t>(row) * p.a.ld_base + n) : zero;
        }
        load_w(0);
        if (!waited) {
            // h of the tile, split into hi and lo; places at or behind the rank are zeros
            pdl_wait();
            pdl_launch_dependents();
            waited = true;
            for (int i = threadIdx.x; i < TM * steps * 8; i += THREADS) {
                const int rl = i / (steps * 8), r = 4 * (i % (steps * 8)), row = s_rows[rl];
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (row >= 0 && r < rank) {
                    for (int s = 0; s < p.splits; ++s) {
                        const float4 t = __ldcg(reinterpret_cast<const float4*>(p.h + (static_cast<size_t>(s) * p.a.M + row) * p.RP + r));
                        v[0] += t.x; v[1] += t.y; v[2] += t.z; v[3] += t.w;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (r + e >= rank) v[e] = 0.0f;
                }
                const uint32_t h0 = bf16x2(v[0], v[1]), h1 = bf16x2(v[2], v[3]);
                *reinterpret_cast<uint2*>(s_h + rl * pitch + r) = make_uint2(h0, h1);
                const float hi[4] = {bf16_lo(h0), bf16_hi(h0), bf16_lo(h1), bf16_hi(h1)};
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fabsf(hi[e]) < INFINITY ? v[e] - hi[e] : 0.0f;        // (infinity has no low part)
                *reinterpret_cast<uint2*>(s_h + (TM + rl) * pitch + r) = make_uint2(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]));
            }
            __syncthreads();
        }
        float acc[8][4];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
        for (int step = 0; step < steps; ++step) {
            if (step > 0) load_w(step);
            const uint16_t* hr = s_h + (16 * mw + g) * pitch + 32 * step + 8 * q;
#pragma unroll
            for (int part = 0; part < 2; ++part) {                 // hi, lo
                const uint4 ha = *reinterpret_cast<const uint4*>(hr + part * TM * pitch), hb = *reinterpret_cast<const uint4*>(hr + (part * TM + 8) * pitch);
                const uint32_t a0[4] = {ha.x, hb.x, ha.y, hb.y}, a1[4] = {ha.z, hb.z, ha.w, hb.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    mma16<false>(acc[j], a0, wb[j].x, wb[j].y);
                    mma16<false>(acc[j], a1, wb[j].z, wb[j].w);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int row = e < 2 ? row0 : row1, n = nl + 8 * (e & 1), j0 = 4 * (e & 1), c = e < 2 ? 0 : 2;
            if (row < 0 || n >= p.a.N) continue;
            const uint32_t b[4] = {base[e].x, base[e].y, base[e].z, base[e].w};
            uint32_t y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y[i] = rank > 0 ? bf16x2(fmaf(scale, acc[j0 + i][c], bf16_lo(b[i])), fmaf(scale, acc[j0 + i][c + 1], bf16_hi(b[i]))) : b[i];
            *reinterpret_cast<uint4*>(p.a.Y + static_cast<int64_t>(row) * p.a.ldy + n) = make_uint4(y[0], y[1], y[2], y[3]);
        }
    }
    if (!waited) pdl_wait();
}

// Rows by adapter, those without one last, and the tiles of each.
__global__ void __launch_bounds__(kSortThreads) lora_sort_kernel(const LoraArgs a, int4* tiles, int max_tiles, int32_t* perm)
{
    extern __shared__ int s_count[];                               // [n_adapters + 1] rows, then the next place of each
    pdl_wait();
    pdl_launch_dependents();
    const int tid = threadIdx.x, groups = a.n_adapters + 1;
    for (int i = tid; i < groups; i += kSortThreads) s_count[i] = 0;
    __syncthreads();
    auto group_of = [&](int m, bool tell) {
        const int x = a.adapters[m];
        if (x >= 0 && x < a.n_adapters) return x;
        if (x != -1 && tell) record_bad_data(kBadAdapter);
        return a.n_adapters;
    };
    for (int m = tid; m < a.M; m += kSortThreads) atomicAdd(&s_count[group_of(m, true)], 1);
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
    for (int m = tid; m < a.M; m += kSortThreads) perm[atomicAdd(&s_count[group_of(m, false)], 1)] = m;
}

struct LoraPlan {
    bool sorted;
    int tiles, splits, RP, rank_blocks;
    size_t h_bytes, tiles_bytes, perm_bytes;
};
LoraPlan lora_plan(int M, int K, int R, int n_adapters, int sm_count)
{
    LoraPlan l;
    l.sorted = M > kWindowRows;
    const int slots = M < 16 ? M : 16;
    l.tiles = l.sorted ? static_cast<int>(std::min<long long>(M, static_cast<long long>(M) / kTileRows + n_adapters + 1)) : (M + 15) / 16 * slots;
    const int rb = l.sorted ? 64 : 16;
    l.rank_blocks = (R + rb - 1) / rb;
    // K is cut until there is a CTA for each SM, but not into parts of less than 512 (the sums of the parts are read again by every CTA of expand).  Tiles
    // are counted as if all rows had one adapter: more adapters only mean more CTAs.
    const long long sure = l.sorted ? (M + kTileRows - 1) / kTileRows : (M + 15) / 16;
    l.splits = 1;
    while (l.splits < 8 && sure * l.rank_blocks * l.splits < sm_count && K / (2 * l.splits) >= 512) l.splits *= 2;
    l.RP = (R + 7) / 8 * 8;
    l.h_bytes = (static_cast<size_t>(l.splits) * M * l.RP * sizeof(float) + 255) / 256 * 256;
    l.tiles_bytes = l.sorted ? (static_cast<size_t>(l.tiles) * sizeof(int4) + 255) / 256 * 256 : 0;
    l.perm_bytes = l.sorted ? (static_cast<size_t>(M) * sizeof(int32_t) + 255) / 256 * 256 : 0;
    return l;
}
size_t expand_smem(int tm, int R) { return 2 * sizeof(uint16_t) * static_cast<size_t>(tm) * ((R + 31) / 32 * 32 + 8); }

}  // namespace

cudaError_t lora_init()
{
    cudaError_t e = cudaFuncSetAttribute(lora_expand_kernel<4, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(expand_smem(64, kMaxRank)));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(lora_expand_kernel<1, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(expand_smem(16, kMaxRank)));
    return e;
}

size_t lora_workspace_bytes(int M, int K, int R, int n_adapters, int sm_count)
{
    const LoraPlan l = lora_plan(M, K, R, n_adapters, sm_count);
    return l.h_bytes + l.tiles_bytes + l.perm_bytes;
}

cudaError_t launch_lora(const LoraArgs& a, void* workspace, int sm_count, cudaStream_t st)
{
    const LoraPlan l = lora_plan(a.M, a.K, a.R, a.n_adapters, sm_count);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    LoraParams p = {};
    p.a = a;
    p.h = reinterpret_cast<float*>(ws);
    p.RP = l.RP; p.splits = l.splits;
    const unsigned tiles = static_cast<unsigned>(l.tiles), rb = static_cast<unsigned>(l.rank_blocks), ks = static_cast<unsigned>(l.splits);
    if (!l.sorted) {
        p.slots = a.M < 16 ? a.M : 16;
        const cudaError_t e = launch_pdl(lora_shrink_kernel<1, 2, 8>, dim3(tiles, rb, ks), 256, 0, 0, st, p);
        if (e != cudaSuccess) return e;
        return launch_pdl(lora_expand_kernel<1, 4>, dim3(tiles, static_cast<unsigned>((a.N + 255) / 256), 1), 128, expand_smem(16, a.R), 0, st, p, 1);
    }
    int4* list = reinterpret_cast<int4*>(ws + l.h_bytes);
    int32_t* perm = reinterpret_cast<int32_t*>(ws + l.h_bytes + l.tiles_bytes);
    cudaError_t e = launch_pdl(lora_sort_kernel, dim3(1, 1, 1), kSortThreads, sizeof(int) * static_cast<size_t>(a.n_adapters + 1), 0, st, a, list, l.tiles, perm);
    if (e != cudaSuccess) return e;
    p.tiles = list;
    p.perm = perm;
    e = launch_pdl(lora_shrink_kernel<4, 8, 2>, dim3(tiles, rb, ks), 256, 0, 0, st, p);
    if (e != cudaSuccess) return e;
    const int iters = 4;
    return launch_pdl(lora_expand_kernel<4, 2>, dim3(tiles, static_cast<unsigned>((a.N + 128 * iters - 1) / (128 * iters)), 1), 256, expand_smem(64, a.R), 0, st, p, iters);
}

}  // namespace rudder
