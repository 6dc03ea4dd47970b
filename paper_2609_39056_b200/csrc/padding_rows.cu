// Rows of padding behind attention: a row with a negative position attends to nothing, so its output is zeros and, where it is one of a
// request's rows, its lse -infinity.  (Attention knows rows by their place in the request alone; to it such a row is a query like any other.)
//
// Reads 4 bytes a row and writes only where there is padding: what it costs is a launch in the chain, 0.6 us of the block's 84
// (64 rows over 4416 cached ones, width 2048).  In attention itself the check
// would sit in four places that write a row, on the path of every call.  A warp takes 32 rows: a lane looks up one position, then all of them write
// the rows that were found.
#include "internal.cuh"
#include "paged.cuh"

namespace rudder {

namespace {

constexpr int PAD_THREADS = 128;

__global__ void __launch_bounds__(PAD_THREADS) padding_rows_kernel(const AttnArgs a, const int32_t* positions)
{
    pdl_launch_dependents();
    pdl_wait();
    const int lane = threadIdx.x & 31;
    const int row0 = (blockIdx.x * PAD_THREADS + threadIdx.x) & ~31, row = row0 + lane;
    uint32_t pad = __ballot_sync(0xffffffffu, row < a.M && positions[row < a.M ? row : 0] < 0);
    if (pad == 0) return;
    // the requests' rows are one range
    const long long first = a.q_starts != nullptr ? a.q_starts[0] : 0;
    const long long end = a.q_starts != nullptr ? a.q_starts[a.B] : static_cast<long long>(a.B) * a.max_q;
    const int pieces = a.heads * a.head_dim / 8;
    for (; pad != 0; pad &= pad - 1) {
        const int m = row0 + __ffs(pad) - 1;
        uint4* o = reinterpret_cast<uint4*>(a.O + static_cast<size_t>(m) * a.ldo);
        for (int i = lane; i < pieces; i += 32) o[i] = make_uint4(0, 0, 0, 0);
        if (a.lse != nullptr && m >= first && m < end)
            for (int h = lane; h < a.heads; h += 32) a.lse[static_cast<size_t>(m) * a.heads + h] = -INFINITY;
    }
}

}  // namespace

cudaError_t launch_padding_rows(const AttnArgs& a, const int32_t* positions, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>((a.M + PAD_THREADS - 1) / PAD_THREADS), 1, 1);
    cfg.blockDim = dim3(PAD_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, padding_rows_kernel, a, positions);
}

}  // namespace rudder
