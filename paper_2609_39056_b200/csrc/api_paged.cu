// Host side of the operators around the paged key-value cache: argument checks, workspace carving, launches.
// Every check needs only the host's arguments and comes before anything is launched.
#include "internal.cuh"
#include "paged.cuh"

using namespace rudder;

namespace {

bool g_paged_ready[64] = {false};

rudder_status ensure_paged_init()
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RUDDER_ERR_CUDA;
    std::lock_guard<std::mutex> lock(g_state_mutex);
    if (!g_paged_ready[dev]) {
        if (page_tables_init() != cudaSuccess || attention_paged_init() != cudaSuccess || linear_a16_init() != cudaSuccess) return RUDDER_ERR_CUDA;
        g_paged_ready[dev] = true;
    }
    return RUDDER_OK;
}

// log2 of a page size, or -1
int page_shift_of(int page_size)
{
    if (page_size < 1 || page_size > 1024 || (page_size & (page_size - 1)) != 0) return -1;
    int s = 0;
    while ((1 << s) < page_size) ++s;
    return s;
}

bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }

rudder_status check_cache(const rudder_paged_cache* c, int kv_heads, int head_dim, CacheParams* out)
{
    if (!c || !c->k || !c->v || c->n_pages < 1) return RUDDER_ERR_ARG;
    if (c->format != RUDDER_CACHE_BF16 && c->format != RUDDER_CACHE_E4M3) return RUDDER_ERR_UNSUPPORTED;
    const int shift = page_shift_of(c->page_size);
    if (shift < 0 || c->heads != kv_heads || c->head_dim != head_dim) return RUDDER_ERR_SHAPE;
    const int per16 = c->format == RUDDER_CACHE_BF16 ? 8 : 16;               // elements in 16 bytes
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->page_stride % per16 != 0 || c->head_stride % per16 != 0 || c->token_stride % per16 != 0)
        return RUDDER_ERR_ALIGN;
    // an axis of one element has no stride; on the others elements may not lie on top of each other
    if (c->page_stride < 0 || c->head_stride < 0 || c->token_stride < 0 || (c->n_pages > 1 && c->page_stride < head_dim) ||
        (c->heads > 1 && c->head_stride < head_dim) || (c->page_size > 1 && c->token_stride < head_dim))
        return RUDDER_ERR_ALIGN;
    out->k = static_cast<uint8_t*>(c->k); out->v = static_cast<uint8_t*>(c->v);
    out->page_stride = c->page_stride; out->head_stride = c->head_stride; out->token_stride = c->token_stride;
    out->k_scale = c->format == RUDDER_CACHE_E4M3 ? c->k_scale : nullptr;
    out->v_scale = c->format == RUDDER_CACHE_E4M3 ? c->v_scale : nullptr;
    out->n_pages = c->n_pages; out->page_shift = shift;
    return RUDDER_OK;
}

rudder_status check_qk(const rudder_qk_args* a, QkArgs* out)
{
    if (!a || !a->X || !a->Q) return RUDDER_ERR_ARG;
    const bool to_cache = a->cache != nullptr;
    if (to_cache ? (!a->slots || a->K) : (!a->K || a->slots)) return RUDDER_ERR_ARG;          // keys go to the cache or to K, not both
    if (!(a->eps >= 0.0f)) return RUDDER_ERR_ARG;
    if (a->style != RUDDER_ROPE_HALF && a->style != RUDDER_ROPE_PAIRS) return RUDDER_ERR_UNSUPPORTED;
    if (a->M < 1 || a->heads < 1 || a->kv_heads < 1 || a->heads > 1024 || a->kv_heads > kMaxKvHeads || !head_dim_ok(a->head_dim)) return RUDDER_ERR_SHAPE;
    if (a->rot < 0 || a->rot > a->head_dim || a->rot % 16 != 0) return RUDDER_ERR_SHAPE;
    if (a->rot > 0 && (!a->cos || !a->sin || !a->positions || a->n_pos < 1)) return RUDDER_ERR_ARG;
    const int64_t width = static_cast<int64_t>(a->heads + 2 * a->kv_heads) * a->head_dim;
    if (!aligned(a->X, 16) || a->ldx % 8 != 0 || a->ldx < width || !aligned(a->Q, 16) || a->ldq % 8 != 0 ||
        a->ldq < static_cast<int64_t>(a->heads) * a->head_dim)
        return RUDDER_ERR_ALIGN;
    if (a->K && (!aligned(a->K, 16) || a->ldk % 8 != 0 || a->ldk < static_cast<int64_t>(a->kv_heads) * a->head_dim)) return RUDDER_ERR_ALIGN;
    if ((a->q_weight && !aligned(a->q_weight, 16)) || (a->k_weight && !aligned(a->k_weight, 16)) || (a->rot > 0 && (!aligned(a->cos, 16) || !aligned(a->sin, 16))))
        return RUDDER_ERR_ALIGN;
    QkArgs o = {};
    if (to_cache) {
        rudder_status s = check_cache(a->cache, a->kv_heads, a->head_dim, &o.cache);
        if (s != RUDDER_OK) return s;
    }
    o.X = a->X; o.ldx = a->ldx; o.M = a->M; o.heads = a->heads; o.kv_heads = a->kv_heads;
    o.q_weight = a->q_weight; o.k_weight = a->k_weight; o.eps = a->eps; o.one = 1.0f;
    o.cos = a->cos; o.sin = a->sin; o.n_pos = a->n_pos; o.rot = a->rot; o.pairs = a->style == RUDDER_ROPE_PAIRS;
    o.positions = a->positions; o.Q = a->Q; o.ldq = a->ldq; o.K = a->K; o.ldk = a->ldk; o.slots = a->slots;
    *out = o;
    return RUDDER_OK;
}

// Tensor map over one tensor of the cache; false if the strides do not fit one.
bool make_tmap_cache(CUtensorMap* tm, const void* base, const rudder_paged_cache* c)
{
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    const bool e4m3 = c->format == RUDDER_CACHE_E4M3;
    const cuuint64_t elt = e4m3 ? 1 : 2, row = static_cast<cuuint64_t>(c->head_dim) * elt;
    cuuint64_t gdim[4] = {static_cast<cuuint64_t>(c->head_dim), static_cast<cuuint64_t>(c->page_size), static_cast<cuuint64_t>(c->heads), static_cast<cuuint64_t>(c->n_pages)};
    // (an axis of one element may have any stride)
    cuuint64_t gstride[3] = {c->page_size > 1 ? static_cast<cuuint64_t>(c->token_stride) * elt : row, c->heads > 1 ? static_cast<cuuint64_t>(c->head_stride) * elt : row,
                             c->n_pages > 1 ? static_cast<cuuint64_t>(c->page_stride) * elt : row};
    // bf16: 64 channels, swizzled as the tensor core reads them; E4M3: whole rows as they are, converted on the way
    cuuint32_t box[4] = {e4m3 ? static_cast<cuuint32_t>(c->head_dim) : 64, static_cast<cuuint32_t>(c->page_size < 64 ? c->page_size : 64), 1, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(tm, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), gdim, gstride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              e4m3 ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

rudder_status check_attention_shape(const rudder_attention_args* a)
{
    if (!a || !a->cache) return RUDDER_ERR_ARG;
    if (a->B < 1 || a->B > (1 << 20) || a->max_q < 1 || a->heads < 1 || a->heads > 1024 || a->cache->heads < 1 || a->heads % a->cache->heads != 0 ||
        !head_dim_ok(a->cache->head_dim))
        return RUDDER_ERR_SHAPE;
    if (a->max_q > (1 << 20) / (a->heads / a->cache->heads)) return RUDDER_ERR_SHAPE;
    return RUDDER_OK;
}

rudder_status check_attention(const rudder_attention_args* a, AttnArgs* out)
{
    if (!a || !a->Q || !a->O || !a->cache || !a->page_table || !a->kv_lens) return RUDDER_ERR_ARG;
    if (!(a->scale == a->scale) || a->scale - a->scale != 0.0f) return RUDDER_ERR_ARG;        // NaN, infinity
    rudder_status s = check_attention_shape(a);
    if (s != RUDDER_OK) return s;
    if (a->M < 1 || a->max_pages < 1 || a->ld_table < a->max_pages) return RUDDER_ERR_SHAPE;
    if (!a->q_starts && static_cast<int64_t>(a->B) * a->max_q > a->M) return RUDDER_ERR_SHAPE;
    AttnArgs o = {};
    s = check_cache(a->cache, a->cache->heads, a->cache->head_dim, &o.cache);
    if (s != RUDDER_OK) return s;
    if ((static_cast<int64_t>(a->max_pages) << o.cache.page_shift) > (int64_t(1) << 31) - (1 << 16)) return RUDDER_ERR_SHAPE;
    const int64_t width = static_cast<int64_t>(a->heads) * a->cache->head_dim;
    if (!aligned(a->Q, 16) || !aligned(a->O, 16) || a->ldq % 8 != 0 || a->ldo % 8 != 0 || a->ldq < width || a->ldo < width) return RUDDER_ERR_ALIGN;
    o.Q = a->Q; o.ldq = a->ldq; o.M = a->M; o.O = a->O; o.ldo = a->ldo; o.lse = a->lse;
    o.heads = a->heads; o.kv_heads = a->cache->heads; o.head_dim = a->cache->head_dim; o.e4m3 = a->cache->format == RUDDER_CACHE_E4M3;
    o.table = a->page_table; o.ld_table = a->ld_table; o.max_pages = a->max_pages; o.kv_lens = a->kv_lens; o.q_starts = a->q_starts;
    o.B = a->B; o.max_q = a->max_q; o.causal = a->causal != 0; o.scale = a->scale;
    *out = o;
    return RUDDER_OK;
}

// Where the kernel that the call runs takes the cache by TMA: the tensor maps (without them it copies row by row).
void add_maps(const rudder_paged_cache* c, AttnArgs* a)
{
    if (attention_uses_maps(a->max_q * (a->heads / a->kv_heads), a->head_dim, a->e4m3, c->page_size, static_cast<long long>(a->max_pages) * c->page_size)) a->tma = make_tmap_cache(&a->tm_k, c->k, c) && make_tmap_cache(&a->tm_v, c->v, c);
}

}  // namespace

extern "C" {

rudder_status rudder_page_tables(const rudder_page_table_args* a, void* stream)
{
    if (!a || !a->old_lens || !a->new_lens || !a->page_table || !a->slots || !a->positions || !a->starts || !a->used) return RUDDER_ERR_ARG;
    if (a->n_free < 0 || (a->n_free > 0 && !a->free_pages)) return RUDDER_ERR_ARG;
    const int shift = page_shift_of(a->page_size);
    if (shift < 0 || a->B < 1 || a->B > kMaxRequests || a->max_pages < 1 || a->ld_table < a->max_pages || a->capacity < 1 || a->capacity >= (1 << 30))
        return RUDDER_ERR_SHAPE;
    rudder_status s = ensure_paged_init();
    if (s != RUDDER_OK) return s;
    PageTablesArgs p;
    p.old_lens = a->old_lens; p.new_lens = a->new_lens; p.B = a->B; p.free_pages = a->free_pages; p.n_free = a->n_free;
    p.table = a->page_table; p.ld_table = a->ld_table; p.max_pages = a->max_pages; p.page_shift = shift;
    p.slots = a->slots; p.positions = a->positions; p.capacity = a->capacity; p.starts = a->starts; p.used = a->used;
    return launch_page_tables(p, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? RUDDER_OK : RUDDER_ERR_CUDA;
}

rudder_status rudder_qk_norm_rope(const rudder_qk_args* args, void* stream)
{
    QkArgs a;
    rudder_status s = check_qk(args, &a);
    if (s != RUDDER_OK) return s;
    const bool e4m3 = args->cache != nullptr && args->cache->format == RUDDER_CACHE_E4M3;
    return launch_qk_norm_rope(a, args->head_dim, e4m3, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? RUDDER_OK : RUDDER_ERR_CUDA;
}

size_t rudder_attention_workspace_bytes(const rudder_attention_args* args)
{
    if (check_attention_shape(args) != RUDDER_OK) return 0;
    return attention_workspace_bytes(args->max_q * (args->heads / args->cache->heads), args->cache->head_dim, sm_count());
}

rudder_status rudder_attention_paged(const rudder_attention_args* args, void* workspace, size_t workspace_bytes, void* stream)
{
    AttnArgs a;
    rudder_status s = check_attention(args, &a);
    if (s != RUDDER_OK) return s;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < rudder_attention_workspace_bytes(args)) return RUDDER_ERR_WORKSPACE;
    s = ensure_paged_init();
    if (s != RUDDER_OK) return s;
    add_maps(args->cache, &a);
    return launch_attention_paged(a, workspace, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? RUDDER_OK : RUDDER_ERR_CUDA;
}

rudder_status rudder_linear_a16(const rudder_weight* w, const uint16_t* X, int64_t ldx, int M, const float* bias, uint16_t* Y, int64_t ldy, void* stream)
{
    if (!w || !X || !Y) return RUDDER_ERR_ARG;
    if (!on_weights_device(w)) return RUDDER_ERR_ARG;
    if (M < 1 || M > 16 || !linear_a16_fits(w->K)) return RUDDER_ERR_SHAPE;
    if (!aligned(X, 16) || !aligned(Y, 16) || ldx % 8 != 0 || ldy % 8 != 0 || ldx < w->K || ldy < w->N || (bias && !aligned(bias, 16))) return RUDDER_ERR_ALIGN;
    rudder_status s = ensure_paged_init();
    if (s != RUDDER_OK) return s;
    return launch_linear_a16(w, X, ldx, M, bias, Y, ldy, sm_count(), static_cast<cudaStream_t>(stream)) == cudaSuccess ? RUDDER_OK : RUDDER_ERR_CUDA;
}

// Workspace of rudder_block_cached: the four linears, the staged GELU output, three M x H buffers, the normed queries and
// the attention output (M x heads D each), the attention's own workspace.
size_t rudder_block_cached_workspace_bytes(const rudder_block_args* args, const rudder_attention_args* attn, int M)
{
    const size_t dit = dit_workspace_bytes(args, M), att = rudder_attention_workspace_bytes(attn);
    if (dit == 0 || att == 0) return 0;
    return dit + 2 * align_up(static_cast<size_t>(M) * attn->heads * attn->cache->head_dim * 2, 256) + align_up(att, 256);
}

rudder_status rudder_block_cached(const rudder_block_args* args, const rudder_block_glue* glue, const rudder_qk_args* qk, const rudder_attention_args* attn, int M,
                                  const rudder_segments* seg, int step, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!args || !glue || !qk || !attn || !glue->norm1_weight || !glue->norm2_weight || !glue->out) return RUDDER_ERR_ARG;
    for (int l = 0; l < 4; ++l)
        if (!args->w[l] || !args->tab[l] || !args->y[l] || !on_weights_device(args->w[l])) return RUDDER_ERR_ARG;
    if (!args->x[0] || args->x[1] || args->x[2] || args->x[3]) return RUDDER_ERR_ARG;      // the block runs from x[0] alone
    if (!qk->cache || qk->cache != attn->cache || qk->heads != attn->heads || qk->kv_heads != attn->cache->heads || qk->head_dim != attn->cache->head_dim)
        return RUDDER_ERR_ARG;                                                             // attention reads the cache that the keys are appended to
    if (!(glue->eps >= 0.0f)) return RUDDER_ERR_ARG;
    rudder_status s = check_attention_shape(attn);
    if (s != RUDDER_OK) return s;
    const int H = args->w[0]->K, F = args->w[2]->N, A = attn->heads * attn->cache->head_dim;
    if (M < 1 || args->w[0]->N != A + 2 * attn->cache->heads * attn->cache->head_dim || args->w[1]->K != A || args->w[1]->N != H || args->w[2]->K != H ||
        args->w[3]->K != F || args->w[3]->N != H)
        return RUDDER_ERR_SHAPE;
    const size_t need = rudder_block_cached_workspace_bytes(args, attn, M);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need || need == 0) return RUDDER_ERR_WORKSPACE;
    if (!aligned(args->x[0], 16) || args->ldx[0] % 8 != 0 || args->ldx[0] < H || !aligned(glue->out, 16) || glue->ldout % 8 != 0 || glue->ldout < H ||
        !aligned(glue->norm1_weight, 16) || !aligned(glue->norm2_weight, 16))
        return RUDDER_ERR_ALIGN;
    for (int l = 0; l < 4; ++l) {
        SegParams sp;
        s = check_table_and_segments(seg, step, args->tab[l], M, &sp);
        if (s != RUDDER_OK) return s;
        if (!aligned(args->y[l], 16) || args->ldy[l] % 8 != 0 || args->ldy[l] < args->w[l]->N || (args->bias[l] && !aligned(args->bias[l], 16)))
            return RUDDER_ERR_ALIGN;
    }
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    size_t lin_off[4], off = 0;
    for (int l = 0; l < 4; ++l) { lin_off[l] = off; off += workspace_bytes_for(args->w[l], M); }
    const size_t row_h = align_up(static_cast<size_t>(M) * H * 2, 256), row_a = align_up(static_cast<size_t>(M) * A * 2, 256);
    uint16_t* gelu_buf = reinterpret_cast<uint16_t*>(ws + off); off += align_up(static_cast<size_t>(M) * F * 2, 256);
    uint16_t* n1 = reinterpret_cast<uint16_t*>(ws + off);       off += row_h;
    uint16_t* h1 = reinterpret_cast<uint16_t*>(ws + off);       off += row_h;
    uint16_t* n2 = reinterpret_cast<uint16_t*>(ws + off);       off += row_h;
    uint16_t* qn = reinterpret_cast<uint16_t*>(ws + off);       off += row_a;
    uint16_t* ao = reinterpret_cast<uint16_t*>(ws + off);       off += row_a;
    uint8_t* att_ws = ws + off;
    // the block supplies the rows: QKV output -> Q (normed, rotated) -> attention output
    rudder_qk_args qa = *qk;
    qa.X = args->y[0]; qa.ldx = args->ldy[0]; qa.M = M; qa.Q = qn; qa.ldq = A; qa.K = nullptr; qa.ldk = 0;
    rudder_attention_args ta = *attn;
    ta.Q = qn; ta.ldq = A; ta.M = M; ta.O = ao; ta.ldo = A;
    QkArgs qp;
    AttnArgs tp;
    if ((s = check_qk(&qa, &qp)) != RUDDER_OK || (s = check_attention(&ta, &tp)) != RUDDER_OK) return s;
    if ((s = ensure_init()) != RUDDER_OK || (s = ensure_paged_init()) != RUDDER_OK) return s;
    add_maps(ta.cache, &tp);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int sms = sm_count();
    auto lin = [&](int l, const uint16_t* x, int64_t ldx, bool gelu_first) {
        return linear_impl(args->w[l], x, ldx, M, seg, step, args->tab[l], args->bias[l], args->y[l], args->ldy[l], ws + lin_off[l],
                           workspace_bytes_for(args->w[l], M), st, nullptr, 0, 0, 0, 0, nullptr, gelu_first);
    };
    // rows outside every request are written by nobody between here and the O projection, the queries of padding are not either: zeros
    if (cudaMemsetAsync(qn, 0, 2 * row_a, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    // attention half: h = x + O(attention(QKV(norm1(x)), cache))
    if (launch_rmsnorm(args->x[0], args->ldx[0], glue->norm1_weight, glue->eps, n1, H, M, H, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    if ((s = lin(0, n1, H, false)) != RUDDER_OK) return s;
    if (launch_qk_norm_rope(qp, qa.head_dim, qa.cache->format == RUDDER_CACHE_E4M3, sms, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    if (launch_attention_paged(tp, att_ws, sms, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    // (among a request's rows a row of padding has been a query of zeros, i.e. it holds the mean of the values)
    if (qp.positions && launch_padding_rows(tp, qp.positions, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    if ((s = lin(1, ao, A, false)) != RUDDER_OK) return s;
    if (launch_add(args->x[0], args->ldx[0], args->y[1], args->ldy[1], h1, H, M, H, sms, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    // MLP half: out = h + down(gelu(up(norm2(h))))
    if (launch_rmsnorm(h1, H, glue->norm2_weight, glue->eps, n2, H, M, H, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    if ((s = lin(2, n2, H, false)) != RUDDER_OK) return s;
    if (gelu_fuses(args->w[3], args->tab[3])) {
        if ((s = lin(3, args->y[2], args->ldy[2], true)) != RUDDER_OK) return s;
    } else {
        if (launch_gelu(args->y[2], args->ldy[2], gelu_buf, F, M, F, sms, st) != cudaSuccess) return RUDDER_ERR_CUDA;
        if ((s = lin(3, gelu_buf, F, false)) != RUDDER_OK) return s;
    }
    if (launch_add(h1, H, args->y[3], args->ldy[3], glue->out, glue->ldout, M, H, sms, st) != cudaSuccess) return RUDDER_ERR_CUDA;
    return RUDDER_OK;
}

}  // extern "C"
