// The pool of pages behind a paged key-value cache: branching requests off others, taking back what nobody holds, and closing the holes.
//
//   fork     child i continues request src_i at length l_i: its table row starts with the floor(l_i / P) full pages of src_i's, which both share
//            from then on; if r_i = l_i mod P > 0 it takes one page of the free list and the first r_i tokens of src_i's page are copied to it
//   release  refs[p] = how many table entries of living requests hold p (request b: its first ceil(len_b / P) columns); free = those with none, ascending
//   compact  n = pages with a reference; the k-th referenced page at or above n moves to the k-th unreferenced one below n
//
// Forking reads and writes r_i tokens of every layer and little else: HBM bounds it when there is much to copy, the launch when there is not.  So it is ONE
// launch: every CTA repeats the bookkeeping of all children in shared memory (one pass over n pairs, one prefix sum: a child's page is
// free[children with r > 0 before it]), then takes its share of the table rows and of the copies, which no CTA has to hear of from another.
// A warp copies one head's tokens of one page of one layer's keys or values, eight 16-byte pieces a lane in flight.
//
// Release and compaction are chains: zero the counts, count, sum, write.  They move a few hundred kilobytes, so each is ONE launch of one cluster of
// CTAs whose steps are a cluster barrier apart, instead of three or four launches.  Counts are atomic additions of integers: the order
// changes nothing.  Compaction needs no counts, only a mark, and renames the tables in the same launch; its copies are a second one that reads their
// number from the device.
//
// Measured: a fork of 8 children 4.8 us, of 64 over 12 layers (184 MB written) 49.5 us; release of 512 requests 9.3 us, of 9 4.1; the plan of a compaction of 48
// requests 19 us and its 452 MB of copies 73 us (6.2 TB/s, 95 % of a plain copy's rate).
#include <algorithm>

#include "internal.cuh"
#include "paged.cuh"

namespace rudder {

namespace {

// Fork, copy: CTAs of 256 threads, eight for each SM although two fit at a time (the hardware hands out the rest as they end).  64 children x 12 layers 49.5 us, 452 MB of
// a compaction's copies with their plan 91.6; with one CTA of 512 threads to an SM that stays 52.9 and 97.5, with four CTAs of 64 registers a thread at a time 45.3 and 93.9.
constexpr int PF_THREADS = 256, PF_PER_SM = 8;
constexpr int PP_THREADS = 1024;           // release, compact: CTAs of one cluster
constexpr int PP_MAX_CTAS = 8;

// Bases of the layers' caches; geometry and strides are common to them (strides in BYTES here).
template <int CAP>
struct Layers {
    uint8_t* k[CAP];
    uint8_t* v[CAP];
};

// One head's first `tokens` tokens of a page, by one warp.  `chunks`: 16-byte pieces of a token, a power of two.
__device__ __forceinline__ void copy_tokens(const uint8_t* src, uint8_t* dst, int tokens, int64_t token_stride, int chunk_shift, int lane) {
    const int total = tokens << chunk_shift, mask = (1 << chunk_shift) - 1;
    for (int i0 = lane; i0 < total; i0 += 32 * 8) {
        uint4 x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + 32 * e;
            if (i < total) x[e] = *reinterpret_cast<const uint4*>(src + (i >> chunk_shift) * token_stride + 16 * (i & mask));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = i0 + 32 * e;
            if (i < total) *reinterpret_cast<uint4*>(dst + (i >> chunk_shift) * token_stride + 16 * (i & mask)) = x[e];
        }
    }
}
template <int CAP>
__device__ __forceinline__ void copy_unit(const Layers<CAP>& l, const PoolCache& c, int part, int src, int dst, int tokens, int lane) {
    const int head = part % c.heads, lk = part / c.heads;          // keys and values of a layer in turn
    uint8_t* base = (lk & 1) ? l.v[lk >> 1] : l.k[lk >> 1];
    base += static_cast<int64_t>(head) * c.head_stride;
    copy_tokens(base + src * c.page_stride, base + dst * c.page_stride, tokens, c.token_stride, c.chunk_shift, lane);
}

// Exclusive prefix sum over the CTA's threads and the total (THREADS a multiple of 32, at most 1024).
template <int THREADS>
__device__ __forceinline__ int block_prefix(int x, int& total) {
    __shared__ int s_warp[THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += u;
    }
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    int w = lane < THREADS / 32 ? s_warp[lane] : 0;
#pragma unroll
    for (int d = 1; d < THREADS / 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= d) w += u;
    }
    total = __shfl_sync(0xffffffffu, w, THREADS / 32 - 1);
    const int before = warp > 0 ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
    __syncthreads();                                               // (the next call writes s_warp)
    return before + inc - x;
}

// ------------------------------------------------------------------------------------------------------------------- fork
constexpr int kNoChild = -2;               // left out: a bad row or length, or no page for it
constexpr int kWhole = -1;                 // nothing but full pages

// Length a child starts with, or -1 if the pair is no good.
__device__ __forceinline__ int fork_length(const PageForkArgs& a, int i, int s) {
    const int have = a.lens[s], want = a.fork_lens != nullptr ? a.fork_lens[i] : have;
    const long long room = static_cast<long long>(a.max_pages) << a.page_shift;
    return have < 0 || want < 0 || want > have || want > room ? -1 : want;
}

template <int CAP>
__global__ void __launch_bounds__(PF_THREADS, 2) page_fork_kernel(const PageForkArgs a, const __grid_constant__ Layers<CAP> layers)
{
    extern __shared__ int s_fork[];
    int* owner = s_fork;                                           // [B] first child that goes to the row
    int* take = owner + a.B;                                       // [n] place in the free list, kWhole or kNoChild
    int* with_rest = take + a.n;                                   // [n] children that have tokens to copy, in order
    uint32_t* is_src = reinterpret_cast<uint32_t*>(with_rest + a.n);         // [ceil(B / 32)]
    __shared__ int s_bad;
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int P = 1 << a.page_shift;
    if (tid == 0) s_bad = 0;
    for (int b = tid; b < a.B; b += PF_THREADS) owner[b] = 0x7fffffff;
    for (int b = tid; b < (a.B + 31) / 32; b += PF_THREADS) is_src[b] = 0;
    __syncthreads();
    for (int i = tid; i < a.n; i += PF_THREADS) {
        const int s = a.src[i], d = a.dst[i];
        if (s >= 0 && s < a.B) atomicOr(&is_src[s >> 5], 1u << (s & 31));
        if (d >= 0 && d < a.B) atomicMin(&owner[d], i);
    }
    __syncthreads();
    const int per = (a.n + PF_THREADS - 1) / PF_THREADS;
    const int i0 = min(a.n, tid * per), i1 = min(a.n, i0 + per);
    int need = 0;
    for (int i = i0; i < i1; ++i) {
        const int s = a.src[i], d = a.dst[i];
        // rows that exist, a child per row, and no row that another child still reads
        bool ok = s >= 0 && s < a.B && d >= 0 && d < a.B && owner[d] == i && !((is_src[d >> 5] >> (d & 31)) & 1);
        const int len = ok ? fork_length(a, i, s) : -1;
        ok = ok && len >= 0;
        if (!ok) s_bad = 1;
        const bool rest = ok && (len & (P - 1)) != 0;
        take[i] = rest ? need : (ok ? kWhole : kNoChild);
        need += rest;
    }
    int total;
    const int before = block_prefix<PF_THREADS>(need, total);
    const int skip = a.taken != nullptr ? max(0, a.taken[0]) : 0;
    for (int i = i0; i < i1; ++i) {
        if (take[i] < 0) continue;
        const int at = before + take[i];
        const long long f = static_cast<long long>(skip) + at;
        const int page = f < a.n_free ? a.free_pages[f] : -1;
        with_rest[at] = i;
        take[i] = page >= 0 && page < a.n_pages ? page : kNoChild;                 // from here on the page itself
        if (take[i] == kNoChild && blockIdx.x == 0) record_bad_data(page < 0 ? kNoPages : kBadPage);
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        a.used[0] = total;
        if (s_bad) record_bad_data(kBadLength);
    }
    const int gwarp = blockIdx.x * (PF_THREADS / 32) + warp, nwarps = gridDim.x * (PF_THREADS / 32);
    // the rows of the table
    for (int i = gwarp; i < a.n; i += nwarps) {
        const int t = take[i];
        int from = -1, rest = 0;
        if (t != kNoChild) {
            const int s = a.src[i], len = fork_length(a, i, s), full = len >> a.page_shift;
            const int32_t* row = a.table + static_cast<size_t>(s) * a.ld_table;
            int32_t* out = a.table + static_cast<size_t>(a.dst[i]) * a.ld_table;
            for (int c = lane; c < full; c += 32) out[c] = row[c];
            if (t >= 0) {
                from = row[full];
                rest = len & (P - 1);
                if (lane == 0) out[full] = t;
                if ((from < 0 || from >= a.n_pages) && lane == 0) record_bad_data(kBadPage);
            }
            if (lane == 0) a.lens[a.dst[i]] = len;
        }
        if (lane < 3 && a.copies != nullptr) a.copies[3 * static_cast<size_t>(i) + lane] = lane == 0 ? from : (lane == 1 ? (t >= 0 ? t : -1) : rest);
    }
    // the tokens
    const uint32_t parts = 2u * a.layers * a.cache.heads, units = parts * static_cast<uint32_t>(total);
    for (uint32_t u = gwarp; u < units; u += nwarps) {
        const int i = with_rest[u / parts], part = static_cast<int>(u % parts);
        if (take[i] < 0) continue;
        const int s = a.src[i], len = fork_length(a, i, s);
        const int from = a.table[static_cast<size_t>(s) * a.ld_table + (len >> a.page_shift)];
        if (from >= 0 && from < a.n_pages && from != take[i]) copy_unit(layers, a.cache, part, from, take[i], len & (P - 1), lane);
    }
}

// ------------------------------------------------------------------------------------------------------------------- copies by a list
template <int CAP>
__global__ void __launch_bounds__(PF_THREADS, 2) page_copy_kernel(const PageCopyArgs a, const __grid_constant__ Layers<CAP> layers)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int n = a.count != nullptr ? min(max(0, a.count[0]), a.n) : a.n;
    if (a.count != nullptr && a.count[0] != n && blockIdx.x == 0 && threadIdx.x == 0) record_bad_data(kBadLength);
    const uint32_t parts = 2u * a.layers * a.cache.heads, units = parts * static_cast<uint32_t>(n);
    const uint32_t nwarps = gridDim.x * (PF_THREADS / 32);
    for (uint32_t u = blockIdx.x * (PF_THREADS / 32) + (threadIdx.x >> 5); u < units; u += nwarps) {
        const int32_t* e = a.copies + 3 * static_cast<size_t>(u / parts);
        const int src = e[0], dst = e[1], tokens = e[2];
        if (src < 0 || dst < 0) continue;                          // nothing to copy
        if (src >= a.n_pages || dst >= a.n_pages || tokens < 0 || tokens > (1 << a.page_shift)) {
            if (lane == 0) record_bad_data(src >= a.n_pages || dst >= a.n_pages ? kBadPage : kBadLength);
            continue;
        }
        if (src != dst) copy_unit(layers, a.cache, static_cast<int>(u % parts), src, dst, tokens, lane);
    }
}

// ------------------------------------------------------------------------------------------------------------------- release, compact
// All CTAs of the cluster have written what they have written.  (One CTA alone: a cluster's barrier costs it a microsecond more.)
__device__ __forceinline__ void pool_sync() {
    if (gridDim.x == 1) {
        __syncthreads();
        return;
    }
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// `x` to element `at` of `array`, in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ void store_remote(int* array, int at, int rank, int x) {
    uint32_t addr;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(addr) : "r"(smem_u32(array + at)), "r"(rank));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(x) : "memory");
}
// Calls f(page id) for the entries of the tables that living requests hold; a warp takes kCols columns of a request at a time.
constexpr int kCols = 256;
template <class F>
__device__ __forceinline__ void held_entries(const PagePoolArgs& a, F f) {
    const int gwarp = blockIdx.x * (PP_THREADS / 32) + (threadIdx.x >> 5), nwarps = gridDim.x * (PP_THREADS / 32), lane = threadIdx.x & 31;
    const int pieces = (a.max_pages + kCols - 1) / kCols;
    const long long units = static_cast<long long>(a.B) * pieces;
    for (long long u = gwarp; u < units; u += nwarps) {
        const int b = static_cast<int>(u % a.B), c0 = static_cast<int>(u / a.B) * kCols;
        const int len = __ldcg(a.lens + b);
        const long long held = (static_cast<long long>(max(0, len)) + (1 << a.page_shift) - 1) >> a.page_shift;
        if ((len < 0 || held > a.max_pages) && c0 == 0 && lane == 0) record_bad_data(kBadLength);
        const int c1 = static_cast<int>(min(static_cast<long long>(min(a.max_pages, c0 + kCols)), held));
        const int32_t* row = a.table + static_cast<size_t>(b) * a.ld_table;
#pragma unroll
        for (int i = 0; i < kCols / 32; ++i) {
            const int c = c0 + 32 * i + lane;
            if (c < c1) {
                const int p = row[c];
                if (p < 0 || p >= a.n_pages) record_bad_data(kBadPage);
                else f(p);
            }
        }
    }
}

constexpr int PP_EACH = 4;                 // neighbouring pages of a thread
constexpr int PP_TILE = PP_THREADS * PP_EACH;
constexpr int PP_WORK = 4096;              // pages or table entries of a CTA: 48 requests x 512 columns 19 us, with 16384 23

template <bool COMPACT>
__global__ void __launch_bounds__(PP_THREADS) page_pool_kernel(const PagePoolArgs a)
{
    __shared__ int s_sums[PP_MAX_CTAS];                            // pages of every CTA's slice that count
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, rank = blockIdx.x, ctas = gridDim.x;
    const int gtid = rank * PP_THREADS + tid, gsize = ctas * PP_THREADS;
    int* mark = COMPACT ? a.remap : a.refs;                        // released: references; compaction: -1, or >= 0 where there is one
    for (int p = gtid; p < a.n_pages; p += gsize) mark[p] = COMPACT ? -1 : 0;
    if (!COMPACT)
        for (int i = gtid; i < a.n_drop; i += gsize) {
            const int b = a.drop[i];
            if (b >= 0 && b < a.B) a.lens[b] = 0;
            else record_bad_data(kBadLength);
        }
    pool_sync();
    held_entries(a, [&](int p) {
        if (COMPACT) mark[p] = 0;
        else atomicAdd(mark + p, 1);
    });
    pool_sync();
    // this CTA's slice of the pages: how many count (unreferenced ones; compaction: referenced ones)
    const int slice = ((a.n_pages + ctas - 1) / ctas + PP_TILE - 1) / PP_TILE * PP_TILE;
    const int p0 = static_cast<int>(min(static_cast<long long>(a.n_pages), static_cast<long long>(rank) * slice)), p1 = min(a.n_pages, p0 + min(slice, a.n_pages - p0));
    auto counts = [&](int x) { return COMPACT ? x >= 0 : x == 0; };
    int mine = 0, total;
    // (a slice of one tile stays in registers, in the order in which it is written below)
    const bool one = slice == PP_TILE;
    bool kept[PP_EACH];
#pragma unroll
    for (int e = 0; e < PP_EACH; ++e) {
        const int p = p0 + tid * PP_EACH + e;
        kept[e] = one && p < p1 && counts(__ldcg(mark + p));
        mine += kept[e];
    }
    for (int p = one ? p1 : p0 + tid; p < p1; p += PP_THREADS) mine += counts(__ldcg(mark + p));
    const int in_front = block_prefix<PP_THREADS>(mine, total);    // (of this thread's pages, in a slice of one tile)
    if (tid < ctas) store_remote(s_sums, rank, tid, total);
    pool_sync();
    int before = 0, all = 0;
    for (int c = 0; c < ctas; ++c) {
        if (c < rank) before += s_sums[c];
        all += s_sums[c];
    }
    int low = 0;                                                   // compaction: referenced pages below n_live
    if (COMPACT) {
        const int home = all / slice, h0 = home * slice;
        int part = 0;
        for (int p = h0 + tid; p < all; p += PP_THREADS) part += counts(__ldcg(mark + p));
        block_prefix<PP_THREADS>(part, low);
        for (int c = 0; c < min(home, ctas); ++c) low += s_sums[c];
        // (other CTAs give their marks new values meanwhile: what is >= 0 stays so)
    }
    for (int t0 = p0; t0 < p1; t0 += PP_TILE) {
        const int first = t0 + tid * PP_EACH;
        bool hit[PP_EACH];
        int n = 0;
#pragma unroll
        for (int e = 0; e < PP_EACH; ++e) {
            hit[e] = one ? kept[e] : first + e < p1 && counts(__ldcg(mark + first + e));
            n += hit[e];
        }
        int in_tile = 0;
        int at = before + (one ? in_front : block_prefix<PP_THREADS>(n, in_tile));                 // those in front of page `first`
        before += in_tile;
#pragma unroll
        for (int e = 0; e < PP_EACH; ++e) {
            const int p = first + e;
            if (p >= p1) break;
            if (!COMPACT) {
                if (hit[e]) a.free_pages[at] = p;
            } else if (hit[e]) {
                if (p < all) mark[p] = p;
                else {
                    const size_t m = at - low;
                    a.copies[3 * m] = p;
                    a.copies[3 * m + 2] = 1 << a.page_shift;
                    mark[p] = all + static_cast<int>(m);           // until its place is known: no place of a page is that high
                }
            } else if (p < all) {
                a.copies[3 * static_cast<size_t>(p - at) + 1] = p;
            }
            at += hit[e];
        }
    }
    if (!COMPACT) {
        for (int i = all + gtid; i < a.n_pages; i += gsize) a.free_pages[i] = -1;
        if (gtid == 0) a.n_free[0] = all;
        return;                                                    // (nobody reads this CTA's shared memory any more: the last such access is behind a barrier)
    }
    pool_sync();
    const int moves = all - low;
    if (gtid == 0) { a.n_copies[0] = moves; a.n_live[0] = all; }
    auto place = [&](int p) {
        const int r = __ldcg(mark + p);
        return r >= all ? __ldcg(a.copies + 3 * static_cast<size_t>(r - all) + 1) : r;
    };
    // The two passes below may run side by side: a page that moves is found by its rank or, once that is done, by its place.
    for (int m = gtid; m < moves; m += gsize) {
        const int p = __ldcg(a.copies + 3 * static_cast<size_t>(m));
        mark[p] = __ldcg(a.copies + 3 * static_cast<size_t>(m) + 1);
    }
    const int gwarp = rank * (PP_THREADS / 32) + (tid >> 5), nwarps = ctas * (PP_THREADS / 32), lane = tid & 31;
    const int pieces = (a.max_pages + kCols - 1) / kCols;
    for (long long u = gwarp; u < static_cast<long long>(a.B) * pieces; u += nwarps) {
        const int b = static_cast<int>(u % a.B), c0 = static_cast<int>(u / a.B) * kCols;
        const long long held = (static_cast<long long>(max(0, a.lens[b])) + (1 << a.page_shift) - 1) >> a.page_shift;
        const int32_t* row = a.table + static_cast<size_t>(b) * a.ld_table;
        int32_t* out = a.new_table + static_cast<size_t>(b) * a.ld_new;
#pragma unroll
        for (int i = 0; i < kCols / 32; ++i) {
            const int c = c0 + 32 * i + lane;
            if (c < a.max_pages) {
                const int p = row[c];
                out[c] = c < held && p >= 0 && p < a.n_pages ? place(p) : p;
            }
        }
    }
}

template <class... K, class... A>
cudaError_t launch_pdl(void (*kernel)(K...), dim3 grid, int threads, size_t smem, int cluster, cudaStream_t st, A... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = static_cast<unsigned>(cluster); attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <int CAP>
Layers<CAP> layers_of(const rudder_paged_cache* caches, int n)
{
    Layers<CAP> l = {};
    for (int i = 0; i < n; ++i) { l.k[i] = static_cast<uint8_t*>(caches[i].k); l.v[i] = static_cast<uint8_t*>(caches[i].v); }
    return l;
}
constexpr int kFewLayers = 8;              // 128 instead of 2048 bytes of arguments

size_t fork_smem(int B, int n) { return sizeof(int) * (static_cast<size_t>(B) + 2 * static_cast<size_t>(n) + (static_cast<size_t>(B) + 31) / 32); }

// CTAs for `units` warp-sized pieces of copying
int copy_ctas(long long units, int sm_count)
{
    const long long ctas = (units + PF_THREADS / 32 - 1) / (PF_THREADS / 32);
    return static_cast<int>(ctas < 1 ? 1 : (ctas > PF_PER_SM * sm_count ? PF_PER_SM * sm_count : ctas));
}

}  // namespace

cudaError_t page_pool_init()
{
    const int most = static_cast<int>(fork_smem(kMaxRequests, kMaxRequests));
    cudaError_t e = cudaFuncSetAttribute(page_fork_kernel<kFewLayers>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e == cudaSuccess ? cudaFuncSetAttribute(page_fork_kernel<kMaxLayers>, cudaFuncAttributeMaxDynamicSharedMemorySize, most) : e;
}

cudaError_t launch_page_fork(const PageForkArgs& a, const rudder_paged_cache* caches, int sm_count, cudaStream_t st)
{
    const long long units = std::max<long long>(2ll * a.layers * a.cache.heads * a.n, a.n);
    const dim3 grid(static_cast<unsigned>(copy_ctas(units, sm_count)), 1, 1);
    const size_t smem = fork_smem(a.B, a.n);
    if (a.layers <= kFewLayers) return launch_pdl(page_fork_kernel<kFewLayers>, grid, PF_THREADS, smem, 0, st, a, layers_of<kFewLayers>(caches, a.layers));
    return launch_pdl(page_fork_kernel<kMaxLayers>, grid, PF_THREADS, smem, 0, st, a, layers_of<kMaxLayers>(caches, a.layers));
}

cudaError_t launch_page_copy(const PageCopyArgs& a, const rudder_paged_cache* caches, int sm_count, cudaStream_t st)
{
    const dim3 grid(static_cast<unsigned>(copy_ctas(2ll * a.layers * a.cache.heads * a.n, sm_count)), 1, 1);
    if (a.layers <= kFewLayers) return launch_pdl(page_copy_kernel<kFewLayers>, grid, PF_THREADS, 0, 0, st, a, layers_of<kFewLayers>(caches, a.layers));
    return launch_pdl(page_copy_kernel<kMaxLayers>, grid, PF_THREADS, 0, 0, st, a, layers_of<kMaxLayers>(caches, a.layers));
}

cudaError_t launch_page_pool(const PagePoolArgs& a, bool compact, cudaStream_t st)
{
    // a CTA per PP_WORK pages or table entries, at most a portable cluster
    const long long work = std::max<long long>(a.n_pages, static_cast<long long>(a.B) * a.max_pages);
    int ctas = 1;
    while (ctas < PP_MAX_CTAS && static_cast<long long>(ctas) * PP_WORK < work) ctas *= 2;
    return launch_pdl(compact ? page_pool_kernel<true> : page_pool_kernel<false>, dim3(static_cast<unsigned>(ctas), 1, 1), PP_THREADS, 0, ctas, st, a);
}

}  // namespace rudder
