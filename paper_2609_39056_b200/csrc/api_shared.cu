// Host side of the operators for many requests that continue one context: argument checks, workspace carving, launches.
// Every check needs only the host's arguments and comes before anything is launched.
#include "internal.cuh"
#include "paged.cuh"

using namespace rudder;

namespace {

constexpr int kMaxPages = 1 << 30, kMaxRows = 1 << 20, kMaxSize = 1 << 30;

bool g_pool_ready[64] = {false};

rudder_status ensure_pool_init()
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RUDDER_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_state_mutex);
    if (!g_pool_ready[dev]) {
        if (page_pool_init() != cudaSuccess || lora_init() != cudaSuccess) return RUDDER_ERR_CUDA;
        g_pool_ready[dev] = true;
    }
    return RUDDER_OK;
}

// The layers' caches: each one sound, all in the geometry of the first.  `entries`: rows of the list of copies.
rudder_status check_layers(const rudder_paged_cache* c, int n, int page_size, int64_t entries, PoolCache* out, int* n_pages)
{
    *out = {};
    if (n < 0 || (n > 0 && !c)) return RUDDER_ERR_ARG;
    if (n > kMaxLayers) return RUDDER_ERR_SHAPE;
    for (int i = 0; i < n; ++i) {
        if (c[i].heads < 1 || !head_dim_ok(c[i].head_dim)) return RUDDER_ERR_SHAPE;
        CacheParams p;
        const rudder_status s = check_cache(c + i, c[i].heads, c[i].head_dim, &p);
        if (s != RUDDER_OK) return s;
        if (c[i].format != c[0].format || c[i].n_pages != c[0].n_pages || c[i].page_size != page_size || c[i].heads != c[0].heads || c[i].head_dim != c[0].head_dim ||
            c[i].page_stride != c[0].page_stride || c[i].head_stride != c[0].head_stride || c[i].token_stride != c[0].token_stride)
            return RUDDER_ERR_SHAPE;
    }
    if (n == 0) return RUDDER_OK;
    if (2 * static_cast<int64_t>(n) * c->heads > ((int64_t(1) << 31) - 1) / (entries > 0 ? entries : 1)) return RUDDER_ERR_SHAPE;
    const int elt = c->format == RUDDER_CACHE_BF16 ? 2 : 1;
    out->page_stride = c->page_stride * elt; out->head_stride = c->head_stride * elt; out->token_stride = c->token_stride * elt;
    out->heads = c->heads;
    while ((16 << out->chunk_shift) < c->head_dim * elt) ++out->chunk_shift;
    *n_pages = c->n_pages;
    return RUDDER_OK;
}

// What a kernel writes while other CTAs of it still read: no word in common.
struct Words {
    const int32_t* at;
    size_t n;
    bool meets(const Words& o) const
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(at), b = reinterpret_cast<uintptr_t>(o.at);
        return at != nullptr && o.at != nullptr && a < b + o.n * sizeof(int32_t) && b < a + n * sizeof(int32_t);
    }
};
bool fork_arrays_apart(const rudder_page_fork_args* a)
{
    const size_t n = static_cast<size_t>(a->n);
    const Words out[] = {{a->lens, static_cast<size_t>(a->B)}, {a->copies, 3 * n}, {a->used, 1}};
    const Words in[] = {{a->src, n}, {a->dst, n}, {a->fork_lens, n}, {a->free_pages, static_cast<size_t>(a->n_free)}, {a->taken, 1}};
    for (int i = 0; i < 3; ++i) {
        for (const Words& r : in)
            if (out[i].meets(r)) return false;
        for (int j = 0; j < i; ++j)
            if (out[i].meets(out[j])) return false;
    }
    return true;
}

rudder_status ok_or_cuda(cudaError_t e) { return e == cudaSuccess ? RUDDER_OK : RUDDER_ERR_CUDA; }

rudder_status check_shared_shape(const rudder_attention_shared_args* a)
{
    if (!a) return RUDDER_ERR_ARG;
    const rudder_status s = check_attention_shape(&a->attn);
    if (s != RUDDER_OK) return s;
    if (a->n_groups < 1 || a->n_groups > kMaxRows || a->table_rows < a->attn.B || a->group_q < 1 || a->attn.M < 1 || a->attn.M > kMaxRows / (a->attn.heads / a->attn.cache->heads))
        return RUDDER_ERR_SHAPE;
    return RUDDER_OK;
}

rudder_status check_lora_shape(const rudder_lora_args* a)
{
    if (!a) return RUDDER_ERR_ARG;
    // (2^30: the kernels step over rows, inputs and columns in 32 bits)
    if (a->M < 1 || a->M > kMaxSize || a->K < 8 || a->K > kMaxSize || a->K % 8 != 0 || a->N < 8 || a->N > kMaxSize || a->N % 8 != 0 || a->R < 8 || a->R > kMaxRank || a->R % 8 != 0 || a->n_adapters < 1 || a->n_adapters > kMaxAdapters)
        return RUDDER_ERR_SHAPE;
    return RUDDER_OK;
}

}  // namespace

extern "C" {

rudder_status rudder_page_fork(const rudder_page_fork_args* a, const rudder_paged_cache* caches, int n_caches, void* stream)
{
    if (!a || !a->page_table || !a->lens || !a->src || !a->dst || !a->used || a->n_free < 0 || (a->n_free > 0 && !a->free_pages)) return RUDDER_ERR_ARG;
    const int shift = page_shift_of(a->page_size);
    if (shift < 0 || a->B < 1 || a->B > kMaxRequests || a->n < 1 || a->n > kMaxRequests || a->max_pages < 1 || a->max_pages > kMaxPages || a->ld_table < a->max_pages) return RUDDER_ERR_SHAPE;
    PageForkArgs p = {};
    p.n_pages = 0x7fffffff;                                    // (without caches any page id is taken for one)
    rudder_status s = check_layers(caches, n_caches, a->page_size, a->n, &p.cache, &p.n_pages);
    if (s != RUDDER_OK) return s;
    if (!fork_arrays_apart(a)) return RUDDER_ERR_ARG;
    if ((s = ensure_pool_init()) != RUDDER_OK) return s;
    p.table = a->page_table; p.ld_table = a->ld_table; p.max_pages = a->max_pages; p.B = a->B; p.lens = a->lens; p.page_shift = shift;
    p.src = a->src; p.dst = a->dst; p.fork_lens = a->fork_lens; p.n = a->n;
    p.free_pages = a->free_pages; p.n_free = a->n_free; p.taken = a->taken; p.copies = a->copies; p.used = a->used;
    p.layers = n_caches;
    return ok_or_cuda(launch_page_fork(p, caches, sm_count(), static_cast<cudaStream_t>(stream)));
}

rudder_status rudder_page_copy(const rudder_page_copy_args* a, const rudder_paged_cache* caches, int n_caches, void* stream)
{
    if (!a || !a->copies || !caches || n_caches < 1) return RUDDER_ERR_ARG;
    if (a->n < 1) return RUDDER_ERR_SHAPE;
    PageCopyArgs p = {};
    rudder_status s = check_layers(caches, n_caches, caches->page_size, a->n, &p.cache, &p.n_pages);
    if (s != RUDDER_OK || (s = ensure_pool_init()) != RUDDER_OK) return s;
    p.copies = a->copies; p.count = a->count; p.n = a->n; p.page_shift = page_shift_of(caches->page_size); p.layers = n_caches;
    return ok_or_cuda(launch_page_copy(p, caches, sm_count(), static_cast<cudaStream_t>(stream)));
}

rudder_status rudder_page_release(const rudder_page_release_args* a, void* stream)
{
    if (!a || !a->page_table || !a->lens || !a->refs || !a->free_pages || !a->n_free || a->n_drop < 0 || (a->n_drop > 0 && !a->drop)) return RUDDER_ERR_ARG;
    const int shift = page_shift_of(a->page_size);
    if (shift < 0 || a->B < 1 || a->B > kMaxRows || a->max_pages < 1 || a->max_pages > kMaxPages || a->ld_table < a->max_pages || a->n_pages < 1 ||
        a->n_pages > kMaxPages)
        return RUDDER_ERR_SHAPE;
    PagePoolArgs p = {};
    p.table = a->page_table; p.ld_table = a->ld_table; p.max_pages = a->max_pages; p.B = a->B; p.lens = a->lens; p.page_shift = shift; p.n_pages = a->n_pages;
    p.drop = a->drop; p.n_drop = a->n_drop; p.refs = a->refs; p.free_pages = a->free_pages; p.n_free = a->n_free;
    return ok_or_cuda(launch_page_pool(p, false, static_cast<cudaStream_t>(stream)));
}

rudder_status rudder_page_compact(const rudder_page_compact_args* a, const rudder_paged_cache* caches, int n_caches, void* stream)
{
    if (!a || !a->page_table || !a->lens || !a->new_table || !a->remap || !a->n_copies || !a->n_live || (a->n_pages > 1 && !a->copies)) return RUDDER_ERR_ARG;
    const int shift = page_shift_of(a->page_size);
    if (shift < 0 || a->B < 1 || a->B > kMaxRows || a->max_pages < 1 || a->max_pages > kMaxPages || a->ld_table < a->max_pages || a->ld_new < a->max_pages || a->n_pages < 1 || a->n_pages > kMaxPages ||
        (a->new_table == a->page_table && a->ld_new != a->ld_table))
        return RUDDER_ERR_SHAPE;
    PageCopyArgs c = {};
    c.n_pages = a->n_pages;
    rudder_status s = check_layers(caches, n_caches, a->page_size, a->n_pages / 2, &c.cache, &c.n_pages);
    if (s != RUDDER_OK) return s;
    if (c.n_pages != a->n_pages) return RUDDER_ERR_SHAPE;
    if ((s = ensure_pool_init()) != RUDDER_OK) return s;
    PagePoolArgs p = {};
    p.table = a->page_table; p.ld_table = a->ld_table; p.max_pages = a->max_pages; p.B = a->B; p.lens = const_cast<int32_t*>(a->lens); p.page_shift = shift;
    p.n_pages = a->n_pages; p.new_table = a->new_table; p.ld_new = a->ld_new; p.remap = a->remap; p.copies = a->copies; p.n_copies = a->n_copies; p.n_live = a->n_live;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if ((s = ok_or_cuda(launch_page_pool(p, true, st))) != RUDDER_OK || n_caches == 0 || a->n_pages == 1) return s;
    c.copies = a->copies; c.count = a->n_copies; c.n = a->n_pages / 2; c.page_shift = shift; c.layers = n_caches;
    return ok_or_cuda(launch_page_copy(c, caches, sm_count(), st));
}

size_t rudder_attention_shared_workspace_bytes(const rudder_attention_shared_args* args)
{
    if (check_shared_shape(args) != RUDDER_OK) return 0;
    const rudder_attention_args& a = args->attn;
    const int group = a.heads / a.cache->heads;
    return attention_shared_workspace_bytes(shared_group_rows(args->group_q, a.M, group), a.max_q * group, a.M, a.heads, a.cache->head_dim, a.cache->format == RUDDER_CACHE_E4M3,
                                            static_cast<long long>(a.max_pages) * a.cache->page_size, sm_count());
}

rudder_status rudder_attention_shared(const rudder_attention_shared_args* args, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!args || !args->group_starts || !args->prefix_lens || !args->prefix_rows) return RUDDER_ERR_ARG;
    AttnArgs rest;
    rudder_status s = check_attention(&args->attn, &rest);
    if (s != RUDDER_OK || (s = check_shared_shape(args)) != RUDDER_OK) return s;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < rudder_attention_shared_workspace_bytes(args)) return RUDDER_ERR_WORKSPACE;
    if ((s = ensure_paged_init()) != RUDDER_OK) return s;
    const int group = rest.heads / rest.kv_heads;
    AttnArgs prefixes = rest;
    add_maps(args->attn.cache, shared_group_rows(args->group_q, rest.M, group), &prefixes);
    add_maps(args->attn.cache, rest.max_q * group, &rest);
    const SharedGroups g = {args->group_starts, args->prefix_lens, args->prefix_rows, args->n_groups, args->table_rows, args->group_q};
    return ok_or_cuda(launch_attention_shared(prefixes, rest, g, workspace, sm_count(), static_cast<cudaStream_t>(stream)));
}

size_t rudder_lora_workspace_bytes(const rudder_lora_args* a)
{
    if (check_lora_shape(a) != RUDDER_OK) return 0;
    return lora_workspace_bytes(a->M, a->K, a->N, a->R, a->n_adapters, sm_count());
}

rudder_status rudder_lora(const rudder_lora_args* a, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a || !a->X || !a->A || !a->B || !a->ranks || !a->scales || !a->adapters || !a->Y) return RUDDER_ERR_ARG;
    rudder_status s = check_lora_shape(a);
    if (s != RUDDER_OK) return s;
    if (!aligned(a->X, 16) || !aligned(a->A, 16) || !aligned(a->B, 16) || !aligned(a->Y, 16) || a->ldx % 8 != 0 || a->ldx < a->K || a->ldy % 8 != 0 || a->ldy < a->N ||
        a->lda % 8 != 0 || a->lda < a->K || a->a_stride % 8 != 0 || a->a_stride < 0 || a->ldb % 8 != 0 || a->ldb < a->R || a->b_stride % 8 != 0 || a->b_stride < 0)
        return RUDDER_ERR_ALIGN;
    if (a->base && (!aligned(a->base, 16) || a->ld_base % 8 != 0 || a->ld_base < a->N || (a->base == a->Y && a->ld_base != a->ldy))) return RUDDER_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < rudder_lora_workspace_bytes(a)) return RUDDER_ERR_WORKSPACE;
    if ((s = ensure_pool_init()) != RUDDER_OK) return s;
    LoraArgs p = {};
    p.X = a->X; p.ldx = a->ldx; p.M = a->M; p.K = a->K; p.A = a->A; p.a_stride = a->a_stride; p.lda = a->lda; p.B = a->B; p.b_stride = a->b_stride; p.ldb = a->ldb;
    p.N = a->N; p.R = a->R; p.n_adapters = a->n_adapters; p.ranks = a->ranks; p.scales = a->scales; p.adapters = a->adapters;
    p.base = a->base; p.ld_base = a->ld_base; p.Y = a->Y; p.ldy = a->ldy;
    return ok_or_cuda(launch_lora(p, workspace, sm_count(), static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
