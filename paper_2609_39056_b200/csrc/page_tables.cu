// Page tables and slot maps of a paged key-value cache, built on the device from the requests' lengths.
//
// Request b holds old_b tokens in pages(old_b) = ceil(old_b / P) pages and gets new_b more.  It takes
// need_b = pages(old_b + new_b) - pages(old_b) pages of the free list, requests in order:
//     first_b = sum_{i < b} need_i,   table[b][pages(old_b) + j] = free[first_b + j]
//     starts_b = sum_{i < b} new_i,   token starts_b + i: position old_b + i, slot = page * P + position % P
// Two prefix sums over the requests and two gathers: nothing here moves more than a few hundred kilobytes, so what
// it costs is the launch and one chain of dependent loads (lengths -> sums -> page -> slot).  Hence ONE launch: every
// CTA repeats the prefix sums over all requests in its shared memory (8192 requests are 64 KB of loads that hit L2)
// instead of a second launch or a grid barrier, then takes its part of the tokens and of the new pages; each
// finds its request by bisection in the sums.  A token's page is looked up in the old part of the table, which
// nobody writes, or in the free list, never in the entries other CTAs are writing: no order between CTAs.
// Sums saturate at kSumCap (addition of non-negative numbers with a common cap is associative), so lengths of any size
// cannot wrap an index.  Measured: 4 requests of a token each 2.3 us, 512 ragged ones (7000 new tokens) 4.6 us; an empty launch
// in the same place takes 2.0 us.
#include "internal.cuh"
#include "paged.cuh"

namespace rudder {

namespace {

constexpr int PT_THREADS = 512;
constexpr int kSumCap = (1 << 30) - 1;

__device__ __forceinline__ int sat_add(int a, int b) { return min(a + b, kSumCap); }
__device__ __forceinline__ int pages_of(int tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }   // tokens <= 2 kSumCap + page < 2^31 + ...

// Last r with sums[r] <= i (sums[0] = 0, non-decreasing, n + 1 entries; i < sums[n]).
__device__ __forceinline__ int owner(const int* sums, int n, int i) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (sums[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(PT_THREADS) page_tables_kernel(const PageTablesArgs a)
{
    extern __shared__ int sums[];                          // [B + 1] new tokens before, [B + 1] new pages before
    __shared__ int warp_new[PT_THREADS / 32], warp_need[PT_THREADS / 32];
    int* s_new = sums;
    int* s_need = sums + a.B + 1;
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // each thread sums a run of requests, the block scans the threads' sums, each thread writes its run's prefixes
    const int per = (a.B + PT_THREADS - 1) / PT_THREADS;
    const int b0 = min(a.B, tid * per), b1 = min(a.B, b0 + per);
    int t_new = 0, t_need = 0;
    bool bad = false;
    for (int b = b0; b < b1; ++b) {
        const int o = a.old_lens[b], n = a.new_lens[b];
        const int oc = min(max(o, 0), kSumCap), nc = min(max(n, 0), kSumCap);
        bad |= o != oc || n != nc;
        t_new = sat_add(t_new, nc);
        t_need = sat_add(t_need, pages_of(sat_add(oc, nc), a.page_shift) - pages_of(oc, a.page_shift));
    }
    int i_new = t_new, i_need = t_need;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, i_new, d), v = __shfl_up_sync(0xffffffffu, i_need, d);
        if (lane >= d) { i_new = sat_add(i_new, u); i_need = sat_add(i_need, v); }
    }
    if (lane == 31) { warp_new[warp] = i_new; warp_need[warp] = i_need; }
    int e_new = __shfl_up_sync(0xffffffffu, i_new, 1), e_need = __shfl_up_sync(0xffffffffu, i_need, 1);
    if (lane == 0) { e_new = 0; e_need = 0; }
    __syncthreads();
    for (int w = 0; w < warp; ++w) { e_new = sat_add(e_new, warp_new[w]); e_need = sat_add(e_need, warp_need[w]); }
    for (int b = b0; b < b1; ++b) {
        s_new[b] = e_new;
        s_need[b] = e_need;
        const int oc = min(max(a.old_lens[b], 0), kSumCap), nc = min(max(a.new_lens[b], 0), kSumCap);
        e_new = sat_add(e_new, nc);
        e_need = sat_add(e_need, pages_of(sat_add(oc, nc), a.page_shift) - pages_of(oc, a.page_shift));
    }
    if (b1 == a.B && (b0 < b1 || tid == 0)) { s_new[a.B] = e_new; s_need[a.B] = e_need; }     // the thread with the last request (B >= 1)
    __syncthreads();
    const int total_new = s_new[a.B], total_need = s_need[a.B];

    const int gtid = blockIdx.x * PT_THREADS + tid, gsize = gridDim.x * PT_THREADS;
    for (int b = gtid; b <= a.B; b += gsize) a.starts[b] = s_new[b];
    if (gtid == 0) {
        a.used[0] = total_need;
        if (total_new > a.capacity) record_bad_data(kNoRoom);
        if (total_need > a.n_free) record_bad_data(kNoPages);
    }
    if (blockIdx.x == 0 && bad) record_bad_data(kBadLength);
    const int P1 = (1 << a.page_shift) - 1;
    // the pages that are taken
    for (int i = gtid; i < min(total_need, a.n_free); i += gsize) {
        const int b = owner(s_need, a.B, i);
        const int held = pages_of(min(max(a.old_lens[b], 0), kSumCap), a.page_shift);
        const long long col = static_cast<long long>(held) + (i - s_need[b]);
        if (col < a.max_pages) a.table[static_cast<size_t>(b) * a.ld_table + col] = a.free_pages[i];
        else record_bad_data(kNoPages);
    }
    // the tokens
    for (int t = gtid; t < a.capacity; t += gsize) {
        int pos = -1;
        long long slot = -1;
        if (t < total_new) {
            const int b = owner(s_new, a.B, t);
            const int old = min(max(a.old_lens[b], 0), kSumCap);
            pos = min(old + (t - s_new[b]), 0x7fffffff - 1);
            const int held = pages_of(old, a.page_shift), col = pos >> a.page_shift;
            int page = -1;
            if (col >= a.max_pages) {
                if (col < held) record_bad_data(kNoPages);           // (a new page beyond the table was recorded above)
            } else if (col < held) {
                page = a.table[static_cast<size_t>(b) * a.ld_table + col];
                if (page < 0) record_bad_data(kBadPage);
            } else {
                const int f = sat_add(s_need[b], col - held);
                if (f < a.n_free) page = a.free_pages[f];
            }
            if (page >= 0) slot = (static_cast<long long>(page) << a.page_shift) + (pos & P1);
        }
        a.positions[t] = pos;
        a.slots[t] = slot;
    }
}

}  // namespace

cudaError_t page_tables_init()
{
    return cudaFuncSetAttribute(page_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * (kMaxRequests + 1) * static_cast<int>(sizeof(int)));
}

cudaError_t launch_page_tables(const PageTablesArgs& a, int sm_count, cudaStream_t st)
{
    // one CTA per 1024 tokens or 512 requests (two tokens per thread hide nothing of the sums each CTA repeats), at most one per SM
    long long blocks = (static_cast<long long>(a.capacity) + 1023) / 1024;
    blocks = blocks < (a.B + PT_THREADS - 1) / PT_THREADS ? (a.B + PT_THREADS - 1) / PT_THREADS : blocks;
    if (blocks > sm_count) blocks = sm_count;
    if (blocks < 1) blocks = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(blocks), 1, 1);
    cfg.blockDim = dim3(PT_THREADS, 1, 1);
    cfg.dynamicSmemBytes = 2 * static_cast<size_t>(a.B + 1) * sizeof(int);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, page_tables_kernel, a);
}

}  // namespace rudder
