// Attention of a few new tokens of each request over a paged key-value cache (bf16 or E4M3), split over the cache's
// length and joined.
//
//     s_rj = scale q_r . k_j,   o_r = sum_j exp(s_rj - m_r) v_j / sum_j exp(s_rj - m_r),   lse_r = m_r + ln sum_j exp(s_rj - m_r)
//
// One pass over K and V with a running maximum and sum (fp32).  What bounds it is the read of the cache, once:
// 4 D bytes per key and key-value head in bf16.  The new tokens of a request and the query heads that share a key-value
// head are the ROWS of one product (R = tokens x heads / kv_heads), so the cache is read once for all of them.
//
// Matrix instructions: mma.sync m16n8k16 with the rows on the 16-row side.  With 1 to 64 rows the product has at most 64
// multiply-adds per cache byte; tcgen05's smallest tile has 128 (or 64) rows and walks them all, and its
// operands and the probabilities would have to go through shared memory and TMEM for every 32 keys.
//
// Data path: the keys are cut into units; in a unit each of KW warp groups of a CTA has its own tile of KT keys, its own ring of
// NST stages in shared memory filled by 16-byte cp.async (page by page, rows of D contiguous elements, swizzled so that
// ldmatrix reads without bank conflicts), and its own running maximum, sum and output: no CTA-wide barrier in the main
// loop.  RW warps of a group share the tile and own 16 rows each.  Keys at or behind the request's length are
// filled with zeros and masked, whatever the cache holds there.
//
// Work split: all units of all (request, kv head, row tile) are one sequence, cut into equal runs, one per CTA, one CTA per
// SM: every SM streams the same number of bytes however ragged the lengths are.  Each CTA finds its place by a prefix sum over the
// requests' unit counts (device data).  A run crosses items; an item that is cut leaves its parts (fp32 output, maximum,
// sum) in the workspace and a second kernel joins them in order (deterministic).  When every item is short the items are
// handed out whole and nothing is joined.
//
// Rounding: Q, K and V enter exactly.  E4M3 numbers become f16 by moving bits (value x 2^-8, subnormals included), Q is
// brought to f16 by a power of two per row.  Scores and sums are fp32.  The probabilities (<= 1) enter the second product as f16
// with E4M3 values (2^-12), and as TWO bf16 numbers hi + lo (2^-17) with bf16 values where that is free or cheap (PL).
#include "internal.cuh"
#include "paged.cuh"

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace rudder {

namespace {

constexpr float kLn2 = 0.6931471805599453f;

struct AttnParams {
    const uint16_t* Q; int64_t ldq;
    uint16_t* O; int64_t ldo;
    float* lse;
    CacheParams cache;                  // strides in BYTES here
    const int32_t* table; int64_t ld_table;
    const int32_t* kv_lens;
    const int32_t* q_starts;
    float* part_o;                      // [2 G][rows of a tile][D]
    float2* part_ml;                    // [2 G][rows of a tile]
    int* desc;                          // [G][8]
    float scale_log2;
    int max_pages, B, max_q, M, heads, kv_heads, group, causal;
    int whole_units;                    // items of at most this many units are not cut when there is a CTA for each
    int G;                              // CTAs
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool F16>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Four E4M3 bytes as f16 numbers x 2^-8: bytes 0 and 2, bytes 1 and 3.
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t& even, uint32_t& odd) {
    const uint32_t e = w << 8;
    even = (e & 0x80008000u) | ((e >> 1) & 0x3F803F80u);
    odd = (w & 0x80008000u) | ((w >> 1) & 0x3F803F80u);
}

// What the kernels know of a request.
struct Req { int len, row0, qlen; };
__device__ __forceinline__ Req load_request(const AttnParams& p, int b) {
    Req r;
    const long long cap = static_cast<long long>(p.max_pages) << p.cache.page_shift;      // below 2^31 (checked on the host)
    const int len = p.kv_lens[b];
    r.len = static_cast<int>(len < 0 ? 0 : (len > cap ? cap : len));
    if (p.q_starts != nullptr) {
        const int s0 = p.q_starts[b], s1 = p.q_starts[b + 1];
        r.row0 = min(max(s0, 0), p.M);
        const int end = min(max(s1, r.row0), p.M);
        r.qlen = min(end - r.row0, p.max_q);
        if (r.len != len || r.row0 != s0 || r.row0 + r.qlen != s1) record_bad_data(kBadLength);
    } else {
        r.row0 = b * p.max_q;
        r.qlen = p.max_q;
        if (r.len != len) record_bad_data(kBadLength);
    }
    return r;
}

// A place in the sequence of units: request, kv head, row tile, unit inside the item.
template <int ROWS, int UK>
struct Cursor {
    int b, h, rt, j, nt, n_rt;
    Req rq;
    __device__ __forceinline__ void set_request(const AttnParams& p, int bb) {
        b = bb;
        rq = load_request(p, bb);
        nt = max(1, (rq.len + UK - 1) / UK);
        n_rt = (rq.qlen * p.group + ROWS - 1) / ROWS;
    }
    __device__ __forceinline__ void next_item(const AttnParams& p) {
        j = 0;
        if (++rt < n_rt) return;
        rt = 0;
        if (++h < p.kv_heads) return;
        h = 0;
        int bb = b + 1;
        while (bb < p.B) {
            set_request(p, bb);
            if (n_rt > 0) break;
            ++bb;
        }
    }
    __device__ __forceinline__ void advance(const AttnParams& p) {
        if (++j == nt) next_item(p);
    }
};

// RB bytes per row of a tile: the 16-byte chunk c of row r sits at chunk swz(r, c).
template <int RB>
__device__ __forceinline__ uint32_t swz(int r, int c) {
    return static_cast<uint32_t>(r) * RB + (static_cast<uint32_t>(RB >= 128 ? (c ^ (r & 7)) : (c ^ ((r >> 1) & 3))) << 4);
}

// PL: 0 = probabilities once (f16, or bf16), 1 = at most 8 rows: the low parts ride in the unused rows 8..15 of the product (free),
// 2 = hi and lo as two products.
template <int D_, bool E4M3_, int RW_, int KW_, int KT_, int NST_, int PL_>
struct AttnCfg {
    static constexpr int D = D_, RW = RW_, KW = KW_, KT = KT_, NST = NST_, PL = PL_;
    static constexpr bool E4M3 = E4M3_;
    static constexpr int THREADS = 32 * RW * KW;
    static constexpr int ROWS = 16 * RW;
    static constexpr int UK = KW * KT;                     // keys of a unit
    static constexpr int RB = D * (E4M3 ? 1 : 2);          // bytes of a row of a tile
    static constexpr int STAGE = 2 * KT * RB;              // K tile, V tile
    static constexpr int RING = KW * NST * STAGE;
    static constexpr int MERGE = (KW / 2) * RW * 32 * (D / 8) * 16 + (KW / 2) * RW * 32 * 16;
    static constexpr int SMEM = RING + MERGE;
};

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) attention_paged_kernel(const AttnParams p)
{
    constexpr int D = C::D, RW = C::RW, KW = C::KW, KT = C::KT, NST = C::NST, PL = C::PL, RB = C::RB, UK = C::UK, ROWS = C::ROWS;
    constexpr bool E4M3 = C::E4M3;
    constexpr int CH = RB / 16;                            // 16-byte chunks of a row
    constexpr int KS = D / 16;                             // steps of the first product
    constexpr int NT = KT / 8;                             // key tiles of the first product
    constexpr int DT = D / 8;                              // channel tiles of the second
    constexpr int GT = 32 * RW;                            // threads of a warp group
    static_assert(KT == 16 || KT == 32, "a lane holds the place of one key of the tile");
    static_assert(GT % CH == 0 || CH % GT == 0, "rows are copied by whole groups of lanes");
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ long long s_units[C::THREADS / 32];
    __shared__ int s_items[C::THREADS / 32];
    __shared__ int s_max[C::THREADS / 32];
    __shared__ int s_place[4];

    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, q = lane & 3;
    const int kg = warp / RW, rw = warp % RW;
    const int gt = tid - kg * GT;                          // thread inside the warp group

    // ---- this CTA's run of units: sums over the requests, threads over consecutive requests
    const int per = (p.B + C::THREADS - 1) / C::THREADS;
    const int rb0 = min(p.B, tid * per), rb1 = min(p.B, rb0 + per);
    long long t_units = 0;
    int t_items = 0, t_max = 0;
    for (int b = rb0; b < rb1; ++b) {
        const Req r = load_request(p, b);
        const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = max(1, (r.len + UK - 1) / UK);
        t_units += static_cast<long long>(n_rt) * p.kv_heads * nt;
        t_items += n_rt * p.kv_heads;
        if (n_rt > 0) t_max = max(t_max, nt);
    }
    long long i_units = t_units;
    int i_items = t_items;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, i_units, d);
        const int v = __shfl_up_sync(0xffffffffu, i_items, d);
        if (lane >= d) { i_units += u; i_items += v; }
        t_max = max(t_max, __shfl_xor_sync(0xffffffffu, t_max, d));
    }
    if (lane == 31) { s_units[warp] = i_units; s_items[warp] = i_items; s_max[warp] = t_max; }
    __syncthreads();
    long long total = 0, e_units = i_units - t_units;
    int items = 0, e_items = i_items - t_items, most = 0;
    for (int w = 0; w < C::THREADS / 32; ++w) {
        if (w < warp) { e_units += s_units[w]; e_items += s_items[w]; }
        total += s_units[w];
        items += s_items[w];
        most = max(most, s_max[w]);
    }
    const bool whole = items <= p.G && most <= p.whole_units;
    const long long share = whole ? 1 : (total + p.G - 1) / p.G;
    const long long all = whole ? items : total;
    const long long u_begin = min(all, share * blockIdx.x), u_end = min(all, u_begin + share);
    if (u_begin >= u_end) {
        if (tid == 0) p.desc[8 * blockIdx.x] = 0;
        return;
    }
    {
        const long long mine0 = whole ? e_items : e_units, mine1 = mine0 + (whole ? t_items : t_units);
        if (u_begin >= mine0 && u_begin < mine1) {         // exactly one thread
            long long at = mine0;
            for (int b = rb0; b < rb1; ++b) {
                const Req r = load_request(p, b);
                const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = whole ? 1 : max(1, (r.len + UK - 1) / UK);
                const long long here = static_cast<long long>(n_rt) * p.kv_heads * nt;
                if (u_begin < at + here) {
                    const long long off = u_begin - at;
                    const int item = static_cast<int>(off / nt);
                    s_place[0] = b;
                    s_place[1] = item / n_rt;
                    s_place[2] = item % n_rt;
                    s_place[3] = static_cast<int>(off % nt);
                    break;
                }
                at += here;
            }
        }
    }
    __syncthreads();
    Cursor<ROWS, UK> cur;
    cur.set_request(p, s_place[0]);
    cur.h = s_place[1]; cur.rt = s_place[2]; cur.j = s_place[3];
    const int n_units = whole ? cur.nt : static_cast<int>(u_end - u_begin);
    if (tid == 0) {
        // the join of the item that this run starts inside belongs to its first cut, i.e. to the run behind its first owner
        int* d = p.desc + 8 * blockIdx.x;
        const long long item0 = u_begin - cur.j;
        const bool first_cut = !whole && cur.j > 0 && item0 >= share * (static_cast<long long>(blockIdx.x) - 1);
        d[1] = cur.h; d[2] = cur.rt; d[3] = cur.rq.row0; d[4] = cur.rq.qlen;
        d[5] = static_cast<int>((item0 + cur.nt - 1) / share);                   // last owner
        d[6] = item0 == share * (static_cast<long long>(blockIdx.x) - 1) ? 0 : 1;   // slot of the first owner's part
        d[0] = first_cut ? 1 : 0;
    }

    // ---- the ring of this warp group
    const uint32_t ring = smem_u32(smem) + kg * (NST * C::STAGE);
    Cursor<ROWS, UK> ld = cur;
    // page ids of the tile `at` is about to load: lane i holds the one of key i (KT <= 32)
    auto page_of_lane = [&](const Cursor<ROWS, UK>& at) -> int {
        const int key = at.j * UK + kg * KT + lane;
        return (lane < KT && key < at.rq.len) ? __ldg(p.table + static_cast<size_t>(at.b) * p.ld_table + (key >> p.cache.page_shift)) : -2;
    };
    auto issue = [&](const Cursor<ROWS, UK>& at, int page, int stage) {
        const int key0 = at.j * UK + kg * KT;
        if (key0 < at.rq.len) {
            if (page != -2 && (page < 0 || page >= p.cache.n_pages)) { record_bad_data(kBadPage); page = -2; }
            const int key = key0 + lane;
            // a key without a page gets an offset that no valid one has
            const long long off = page < 0 ? -1 : page * p.cache.page_stride + static_cast<long long>(at.h) * p.cache.head_stride +
                                                  static_cast<long long>(key & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride;
            const uint32_t base = ring + stage * C::STAGE;
#pragma unroll
            for (int i = 0; i < KT * CH / GT; ++i) {
                const int idx = gt + i * GT, r = idx / CH, c = idx % CH;
                const long long ro = __shfl_sync(0xffffffffu, off, r);
                const bool ok = ro >= 0;
                const long long src = (ok ? ro : 0) + 16 * c;
                cp_async16(base + swz<RB>(r, c), p.cache.k + src, ok);
                cp_async16(base + KT * RB + swz<RB>(r, c), p.cache.v + src, ok);
            }
        }
    };
#pragma unroll
    for (int s = 0; s < NST - 1; ++s) {
        if (s < n_units) {
            issue(ld, page_of_lane(ld), s);
            ld.advance(p);
        }
        cp_async_commit();
    }

    uint32_t qf[KS][4];
    float acc[DT][4];
    float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.0f, l1 = 0.0f;
    float f0 = p.scale_log2, f1 = p.scale_log2;            // score factors of rows g and g + 8
    int lim0 = 0, lim1 = 0;                                // keys that rows g and g + 8 see
    bool fresh = true;

    for (int i = 0; i < n_units; ++i) {
        const int stage = i % NST;
        if (fresh) {
            // ---- a new item (or the rest of one): queries, limits, empty sums
            fresh = false;
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
            m0 = m1 = -INFINITY;
            l0 = l1 = 0.0f;
            const int R = cur.rq.qlen * p.group;
            const int r0 = cur.rt * ROWS + rw * 16 + g, r1 = r0 + 8;
            const uint16_t* q0 = p.Q;
            const uint16_t* q1 = p.Q;
            lim0 = lim1 = cur.rq.len;                      // rows that do not exist: zeros, no limit of their own
            if (r0 < R) {
                const int t = r0 / p.group, hh = cur.h * p.group + r0 % p.group;
                q0 = p.Q + static_cast<size_t>(cur.rq.row0 + t) * p.ldq + static_cast<size_t>(hh) * D;
                if (p.causal) lim0 = cur.rq.len - cur.rq.qlen + t + 1;
            }
            if (r1 < R) {
                const int t = r1 / p.group, hh = cur.h * p.group + r1 % p.group;
                q1 = p.Q + static_cast<size_t>(cur.rq.row0 + t) * p.ldq + static_cast<size_t>(hh) * D;
                if (p.causal) lim1 = cur.rq.len - cur.rq.qlen + t + 1;
            }
            if (!E4M3) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    qf[ks][0] = r0 < R ? *reinterpret_cast<const uint32_t*>(q0 + 16 * ks + 2 * q) : 0u;
                    qf[ks][1] = r1 < R ? *reinterpret_cast<const uint32_t*>(q1 + 16 * ks + 2 * q) : 0u;
                    qf[ks][2] = r0 < R ? *reinterpret_cast<const uint32_t*>(q0 + 16 * ks + 2 * q + 8) : 0u;
                    qf[ks][3] = r1 < R ? *reinterpret_cast<const uint32_t*>(q1 + 16 * ks + 2 * q + 8) : 0u;
                }
            } else {
                // channels 4 q .. 4 q + 3 of every 16 (the K bytes of a lane): pairs (0, 2) and (1, 3); f16 times a power of two per row
                float x0 = 0.0f, x1 = 0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const uint2 a = r0 < R ? *reinterpret_cast<const uint2*>(q0 + 16 * ks + 4 * q) : make_uint2(0, 0);
                    const uint2 b = r1 < R ? *reinterpret_cast<const uint2*>(q1 + 16 * ks + 4 * q) : make_uint2(0, 0);
                    qf[ks][0] = a.x; qf[ks][2] = a.y; qf[ks][1] = b.x; qf[ks][3] = b.y;
                    x0 = fmaxf(x0, fmaxf(fmaxf(fabsf(bf16_lo(a.x)), fabsf(bf16_hi(a.x))), fmaxf(fabsf(bf16_lo(a.y)), fabsf(bf16_hi(a.y)))));
                    x1 = fmaxf(x1, fmaxf(fmaxf(fabsf(bf16_lo(b.x)), fabsf(bf16_hi(b.x))), fmaxf(fabsf(bf16_lo(b.y)), fabsf(bf16_hi(b.y)))));
                }
#pragma unroll
                for (int o = 1; o < 4; o <<= 1) {
                    x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, o));
                    x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, o));
                }
                // the row's largest magnitude lands in [2^14, 2^15); exponent fields outside bf16's normal range give factors of 2^+-126
                const int e0 = min(126, max(-126, 14 - (static_cast<int>((__float_as_uint(x0) >> 23) & 255u) - 127)));
                const int e1 = min(126, max(-126, 14 - (static_cast<int>((__float_as_uint(x1) >> 23) & 255u) - 127)));
                const float s0 = __uint_as_float(static_cast<uint32_t>(e0 + 127) << 23), s1 = __uint_as_float(static_cast<uint32_t>(e1 + 127) << 23);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const uint32_t ax = qf[ks][0], ay = qf[ks][2], bx = qf[ks][1], by = qf[ks][3];
                    qf[ks][0] = f16x2(bf16_lo(ax) * s0, bf16_lo(ay) * s0);
                    qf[ks][2] = f16x2(bf16_hi(ax) * s0, bf16_hi(ay) * s0);
                    qf[ks][1] = f16x2(bf16_lo(bx) * s1, bf16_lo(by) * s1);
                    qf[ks][3] = f16x2(bf16_hi(bx) * s1, bf16_hi(by) * s1);
                }
                const float ksc = (p.cache.k_scale != nullptr ? __ldg(p.cache.k_scale + cur.h) : 1.0f) * 256.0f * p.scale_log2;
                f0 = ksc * __uint_as_float(static_cast<uint32_t>(127 - e0) << 23);
                f1 = ksc * __uint_as_float(static_cast<uint32_t>(127 - e1) << 23);
            }
        }
        cp_async_wait<NST - 2>();
        if (RW == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + kg), "n"(GT) : "memory");
        // page ids of the tile that goes into the stage just freed: requested now, used after this tile's products
        const bool more = i + NST - 1 < n_units;
        const int page = more ? page_of_lane(ld) : -2;

        const int key0 = cur.j * UK + kg * KT;
        if (key0 < cur.rq.len) {
            const uint32_t kt = ring + stage * C::STAGE, vt = kt + KT * RB;
            float s[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.0f;
            // ---- S = Q K^T
            if (!E4M3) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int n = 0; n < NT; n += 2) {
                        uint32_t b[4];                     // (keys 0..7, 8..15) x (two chunks of the step)
                        ldsm_x4(b, kt + swz<RB>(8 * n + ((lane >> 4) << 3) + (lane & 7), 2 * ks + ((lane >> 3) & 1)));
                        mma16<false>(s[n], qf[ks], b[0], b[1]);
                        mma16<false>(s[n + 1], qf[ks], b[2], b[3]);
                    }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2)
#pragma unroll
                    for (int n = 0; n < NT; n += 2) {
                        uint32_t b[4], ev, od;             // (keys 0..7, 8..15) x (two steps, one chunk each)
                        ldsm_x4(b, kt + swz<RB>(8 * n + ((lane >> 4) << 3) + (lane & 7), ks + ((lane >> 3) & 1)));
                        e4m3_to_f16(b[0], ev, od); mma16<true>(s[n], qf[ks], ev, od);
                        e4m3_to_f16(b[1], ev, od); mma16<true>(s[n], qf[ks + 1], ev, od);
                        e4m3_to_f16(b[2], ev, od); mma16<true>(s[n + 1], qf[ks], ev, od);
                        e4m3_to_f16(b[3], ev, od); mma16<true>(s[n + 1], qf[ks + 1], ev, od);
                    }
            }
            // ---- running maximum and sum (base 2)
            float x0 = -INFINITY, x1 = -INFINITY;
            const bool edge = key0 + KT > min(lim0, lim1);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                s[n][0] *= f0; s[n][1] *= f0; s[n][2] *= f1; s[n][3] *= f1;
                if (edge) {
                    const int k = key0 + 8 * n + 2 * q;
                    if (k >= lim0) s[n][0] = -INFINITY;
                    if (k + 1 >= lim0) s[n][1] = -INFINITY;
                    if (k >= lim1) s[n][2] = -INFINITY;
                    if (k + 1 >= lim1) s[n][3] = -INFINITY;
                }
                x0 = fmaxf(x0, fmaxf(s[n][0], s[n][1]));
                x1 = fmaxf(x1, fmaxf(s[n][2], s[n][3]));
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, o));
                x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, o));
            }
            const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1);
            const float u0 = n0 == -INFINITY ? 0.0f : n0, u1 = n1 == -INFINITY ? 0.0f : n1;      // an empty row so far: exp2(-inf - 0) = 0
            const float c0 = exp2_approx(m0 - u0), c1 = PL == 1 ? c0 : exp2_approx(m1 - u1);
            m0 = n0; m1 = n1;
            l0 *= c0; l1 *= c1;
            if (__any_sync(0xffffffffu, c0 != 1.0f || c1 != 1.0f)) {
#pragma unroll
                for (int t = 0; t < DT; ++t) { acc[t][0] *= c0; acc[t][1] *= c0; acc[t][2] *= c1; acc[t][3] *= c1; }
            }
            uint32_t ph[NT / 2][4], pl[PL == 2 ? NT / 2 : 1][4];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int kk = n >> 1, e = (n & 1) << 1;   // a0, a1 from the even key tile, a2, a3 from the odd one
                const float e0 = exp2_approx(s[n][0] - u0), e1 = exp2_approx(s[n][1] - u0);
                l0 += e0 + e1;
                if (E4M3) {
                    const float e2 = exp2_approx(s[n][2] - u1), e3 = exp2_approx(s[n][3] - u1);
                    l1 += e2 + e3;
                    ph[kk][e] = f16x2(e0, e1);
                    ph[kk][e + 1] = f16x2(e2, e3);
                } else if (PL == 1) {
                    const uint32_t hi = bf16x2(e0, e1);
                    ph[kk][e] = hi;
                    ph[kk][e + 1] = bf16x2(e0 - bf16_lo(hi), e1 - bf16_hi(hi));
                } else {
                    const float e2 = exp2_approx(s[n][2] - u1), e3 = exp2_approx(s[n][3] - u1);
                    l1 += e2 + e3;
                    const uint32_t h0 = bf16x2(e0, e1), h1 = bf16x2(e2, e3);
                    ph[kk][e] = h0;
                    ph[kk][e + 1] = h1;
                    if (PL == 2) {
                        pl[kk][e] = bf16x2(e0 - bf16_lo(h0), e1 - bf16_hi(h0));
                        pl[kk][e + 1] = bf16x2(e2 - bf16_lo(h1), e3 - bf16_hi(h1));
                    }
                }
            }
            // ---- O += P V
#pragma unroll
            for (int kk = 0; kk < KT / 16; ++kk) {
                if (!E4M3) {
#pragma unroll
                    for (int t = 0; t < DT; t += 2) {
                        uint32_t b[4];                     // (keys 0..7, 8..15) of two channel tiles
                        ldsm_x4_t(b, vt + swz<RB>(16 * kk + (((lane >> 3) & 1) << 3) + (lane & 7), t + (lane >> 4)));
                        mma16<false>(acc[t], ph[kk], b[0], b[1]);
                        mma16<false>(acc[t + 1], ph[kk], b[2], b[3]);
                        if (PL == 2) {
                            mma16<false>(acc[t], pl[PL == 2 ? kk : 0], b[0], b[1]);
                            mma16<false>(acc[t + 1], pl[PL == 2 ? kk : 0], b[2], b[3]);
                        }
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < DT; t += 4) {
                        uint32_t b[4], e0, o0, e1, o1;     // two chunks of 16 channels; a register = 2 keys x channels (2 g, 2 g + 1)
                        ldsm_x4_t(b, vt + swz<RB>(16 * kk + (((lane >> 3) & 1) << 3) + (lane & 7), (t >> 1) + (lane >> 4)));
                        e4m3_to_f16(b[0], e0, o0);
                        e4m3_to_f16(b[1], e1, o1);
                        mma16<true>(acc[t], ph[kk], e0, e1);
                        mma16<true>(acc[t + 1], ph[kk], o0, o1);
                        e4m3_to_f16(b[2], e0, o0);
                        e4m3_to_f16(b[3], e1, o1);
                        mma16<true>(acc[t + 2], ph[kk], e0, e1);
                        mma16<true>(acc[t + 3], ph[kk], o0, o1);
                    }
                }
            }
        }
        if (more) {
            issue(ld, page, (i + NST - 1) % NST);
            ld.advance(p);
        }
        cp_async_commit();

        const bool item_end = cur.j + 1 == cur.nt;
        if (item_end || i + 1 == n_units) {
            // ---- end of an item or of this run: join the warp groups, write the rows or the part
            if (!E4M3 && PL == 1) {
#pragma unroll
                for (int t = 0; t < DT; ++t) { acc[t][0] += acc[t][2]; acc[t][1] += acc[t][3]; }
            }
#pragma unroll
            for (int o = 1; o < 4; o <<= 1) {
                l0 += __shfl_xor_sync(0xffffffffu, l0, o);
                l1 += __shfl_xor_sync(0xffffffffu, l1, o);
            }
            float4* box = reinterpret_cast<float4*>(smem + C::RING);
            float4* box_ml = box + (KW / 2) * RW * 32 * DT;
#pragma unroll
            for (int step = KW / 2; step >= 1; step >>= 1) {
                __syncthreads();                           // readers of the box before
                if (kg >= step && kg < 2 * step) {
                    const int at = (kg - step) * RW + rw;
#pragma unroll
                    for (int t = 0; t < DT; ++t) box[(at * DT + t) * 32 + lane] = make_float4(acc[t][0], acc[t][1], acc[t][2], acc[t][3]);
                    box_ml[at * 32 + lane] = make_float4(m0, m1, l0, l1);
                }
                __syncthreads();
                if (kg < step) {
                    const int at = kg * RW + rw;
                    const float4 o = box_ml[at * 32 + lane];
                    const float n0 = fmaxf(m0, o.x), n1 = fmaxf(m1, o.y);
                    const float u0 = n0 == -INFINITY ? 0.0f : n0, u1 = n1 == -INFINITY ? 0.0f : n1;
                    const float a0 = exp2_approx(m0 - u0), a1 = exp2_approx(m1 - u1), b0 = exp2_approx(o.x - u0), b1 = exp2_approx(o.y - u1);
                    m0 = n0; m1 = n1;
                    l0 = l0 * a0 + o.z * b0;
                    l1 = l1 * a1 + o.w * b1;
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        const float4 v = box[(at * DT + t) * 32 + lane];
                        acc[t][0] = acc[t][0] * a0 + v.x * b0;
                        acc[t][1] = acc[t][1] * a0 + v.y * b0;
                        acc[t][2] = acc[t][2] * a1 + v.z * b1;
                        acc[t][3] = acc[t][3] * a1 + v.w * b1;
                    }
                }
            }
            if (kg == 0) {
                const int R = cur.rq.qlen * p.group;
                const int seg_units = i + 1 < cur.j + 1 ? i + 1 : cur.j + 1;     // units of this item in this run so far
                const bool entire = item_end && seg_units == cur.nt;
                const int slot = 2 * blockIdx.x + (seg_units == i + 1 ? 0 : 1);  // part at the start of the run, or at its end
                const float vs = E4M3 ? (p.cache.v_scale != nullptr ? __ldg(p.cache.v_scale + cur.h) : 1.0f) * 256.0f : 1.0f;
#pragma unroll
                for (int half = 0; half < (PL == 1 && !E4M3 ? 1 : 2); ++half) {
                    const int rl = rw * 16 + g + 8 * half, r = cur.rt * ROWS + rl;
                    if (r >= R) continue;
                    const float m = half ? m1 : m0, l = half ? l1 : l0;
                    const float f = entire ? (l > 0.0f ? vs / l : 0.0f) : vs;
                    const int t_row = r / p.group, hh = cur.h * p.group + r % p.group;
                    uint16_t* orow = p.O + static_cast<size_t>(cur.rq.row0 + t_row) * p.ldo + static_cast<size_t>(hh) * D;
                    float* prow = p.part_o + (static_cast<size_t>(slot) * ROWS + rl) * D;
                    if (!E4M3) {
#pragma unroll
                        for (int t = 0; t < DT; ++t) {
                            const float a = acc[t][2 * half] * f, b = acc[t][2 * half + 1] * f;
                            if (entire) *reinterpret_cast<uint32_t*>(orow + 8 * t + 2 * q) = bf16x2(a, b);
                            else *reinterpret_cast<float2*>(prow + 8 * t + 2 * q) = make_float2(a, b);
                        }
                    } else {
#pragma unroll
                        for (int t = 0; t < DT; t += 2) {  // even and odd channels of a chunk of 16: a lane holds 4 q .. 4 q + 3
                            const float a = acc[t][2 * half] * f, b = acc[t + 1][2 * half] * f, c = acc[t][2 * half + 1] * f, d = acc[t + 1][2 * half + 1] * f;
                            if (entire) *reinterpret_cast<uint2*>(orow + 8 * t + 4 * q) = make_uint2(bf16x2(a, b), bf16x2(c, d));
                            else *reinterpret_cast<float4*>(prow + 8 * t + 4 * q) = make_float4(a, b, c, d);
                        }
                    }
                    if (q == 0) {
                        if (entire) {
                            if (p.lse != nullptr)
                                p.lse[static_cast<size_t>(cur.rq.row0 + t_row) * p.heads + hh] = l > 0.0f ? (m + log2f(l)) * kLn2 : -INFINITY;
                        } else {
                            p.part_ml[static_cast<size_t>(slot) * ROWS + rl] = make_float2(m, l);
                        }
                    }
                }
            }
            fresh = true;
        }
        cur.advance(p);
    }
    cp_async_wait<0>();
}

// The parts of the items that were cut, joined in the order of their runs: CTA (c, y) the item that run c starts inside, rows
// JOIN_ROWS y .. + JOIN_ROWS - 1 of its tile.  JOIN_SPLIT warps per row take the parts in turn.
constexpr int JOIN_THREADS = 256, JOIN_ROWS = 2, JOIN_SPLIT = JOIN_THREADS / 32 / JOIN_ROWS;

template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) attention_join_kernel(const AttnParams p, int rows_of_tile)
{
    __shared__ float s_o[JOIN_ROWS][JOIN_SPLIT][D];
    __shared__ float2 s_ml[JOIN_ROWS][JOIN_SPLIT];
    pdl_launch_dependents();
    pdl_wait();
    const int c = blockIdx.x;
    const int* d = p.desc + 8 * c;
    if (d[0] == 0) return;
    const int h = d[1], rt = d[2], row0 = d[3], qlen = d[4], last = d[5], slot_first = d[6];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ry = warp / JOIN_SPLIT, part = warp % JOIN_SPLIT;
    const int rl = blockIdx.y * JOIN_ROWS + ry, r = rt * rows_of_tile + rl;
    const bool live = r < qlen * p.group;
    constexpr int V = D / 32;                              // channels of a lane
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    if (live) {
        const int n = last - (c - 1) + 1;
        for (int s = part; s < n; s += JOIN_SPLIT) {
            const int slot = 2 * (c - 1 + s) + (s == 0 ? slot_first : 0);
            const size_t at = static_cast<size_t>(slot) * rows_of_tile + rl;
            const float2 ml = __ldcg(p.part_ml + at);
            const float* src = p.part_o + at * D + lane * V;
            float v[V];
            if (V == 2) { const float2 x = __ldcg(reinterpret_cast<const float2*>(src)); v[0] = x.x; v[1] = x.y; }
            else {
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float4 x = __ldcg(reinterpret_cast<const float4*>(src + i));
                    v[i] = x.x; v[i + 1] = x.y; v[i + 2] = x.z; v[i + 3] = x.w;
                }
            }
            const float nm = fmaxf(m, ml.x), u = nm == -INFINITY ? 0.0f : nm;
            const float a = exp2_approx(m - u), b = exp2_approx(ml.x - u);
            m = nm;
            l = l * a + ml.y * b;
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = o[i] * a + v[i] * b;
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s_o[ry][part][lane * V + i] = o[i];
    if (lane == 0) s_ml[ry][part] = make_float2(m, l);
    __syncthreads();
    if (part != 0 || !live) return;
    float mm = -INFINITY, ll = 0.0f, w[JOIN_SPLIT];
#pragma unroll
    for (int s = 0; s < JOIN_SPLIT; ++s) mm = fmaxf(mm, s_ml[ry][s].x);
    const float u = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int s = 0; s < JOIN_SPLIT; ++s) {
        w[s] = exp2_approx(s_ml[ry][s].x - u);
        ll += s_ml[ry][s].y * w[s];
    }
    const float inv = ll > 0.0f ? 1.0f / ll : 0.0f;
    const int t_row = r / p.group, hh = h * p.group + r % p.group;
    uint16_t* orow = p.O + static_cast<size_t>(row0 + t_row) * p.ldo + static_cast<size_t>(hh) * D + lane * V;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int s = 0; s < JOIN_SPLIT; ++s) {
            a += s_o[ry][s][lane * V + i] * w[s];
            b += s_o[ry][s][lane * V + i + 1] * w[s];
        }
        *reinterpret_cast<uint32_t*>(orow + i) = bf16x2(a * inv, b * inv);
    }
    if (lane == 0 && p.lse != nullptr)
        p.lse[static_cast<size_t>(row0 + t_row) * p.heads + hh] = ll > 0.0f ? (mm + log2f(ll)) * kLn2 : -INFINITY;
}

// ---- variants: warps over rows (RW) and keys (KW), keys per tile, stages.  The ring is about 130 to 200 KB: it is what keeps
// enough of the cache in flight with one CTA per SM.
template <int D, bool E4M3, int RWS, int PL>
struct Pick;
template <bool E4M3, int PL> struct Pick<64, E4M3, 1, PL> { using C = AttnCfg<64, E4M3, 1, 4, 32, 5, PL>; };
template <bool E4M3, int PL> struct Pick<64, E4M3, 2, PL> { using C = AttnCfg<64, E4M3, 2, 4, 32, 5, PL>; };
template <bool E4M3, int PL> struct Pick<64, E4M3, 4, PL> { using C = AttnCfg<64, E4M3, 4, 2, 32, 5, PL>; };
template <bool E4M3, int PL> struct Pick<128, E4M3, 1, PL> { using C = AttnCfg<128, E4M3, 1, 4, 32, E4M3 ? 5 : 3, PL>; };
template <bool E4M3, int PL> struct Pick<128, E4M3, 2, PL> { using C = AttnCfg<128, E4M3, 2, 2, 32, 5, PL>; };
template <bool E4M3, int PL> struct Pick<128, E4M3, 4, PL> { using C = AttnCfg<128, E4M3, 4, 2, 32, 5, PL>; };
template <bool E4M3, int PL> struct Pick<256, E4M3, 1, PL> { using C = AttnCfg<256, E4M3, 1, 4, 16, 3, PL>; };
template <bool E4M3, int PL> struct Pick<256, E4M3, 2, PL> { using C = AttnCfg<256, E4M3, 2, 2, 16, 4, PL>; };
template <bool E4M3, int PL> struct Pick<256, E4M3, 4, PL> { using C = AttnCfg<256, E4M3, 4, 2, 16, 4, PL>; };

int row_warps(int max_rows) { return max_rows <= 16 ? 1 : (max_rows <= 32 ? 2 : 4); }

template <class C>
cudaError_t launch_main(const AttnParams& p, cudaStream_t st)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.G), 1, 1);
    cfg.blockDim = dim3(C::THREADS, 1, 1);
    cfg.dynamicSmemBytes = C::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_paged_kernel<C>, p);
}
template <int D>
cudaError_t launch_join(const AttnParams& p, int rows_of_tile, int max_rows, cudaStream_t st)
{
    const int rows = max_rows < rows_of_tile ? max_rows : rows_of_tile;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.G), static_cast<unsigned>((rows + JOIN_ROWS - 1) / JOIN_ROWS), 1);
    cfg.blockDim = dim3(JOIN_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_join_kernel<D>, p, rows_of_tile);
}
template <class C>
cudaError_t run_one(AttnParams p, int max_rows, long long max_kv, cudaStream_t st)
{
    p.whole_units = kAttnWholeKeys / C::UK;
    cudaError_t e = launch_main<C>(p, st);
    if (e != cudaSuccess) return e;
    // no item can be cut: there is a CTA for each and the table has no room for a longer one
    const long long items = static_cast<long long>(p.B) * p.kv_heads * ((max_rows + C::ROWS - 1) / C::ROWS);
    if (items <= p.G && (max_kv + C::UK - 1) / C::UK <= p.whole_units) return cudaSuccess;
    return launch_join<C::D>(p, C::ROWS, max_rows, st);
}
template <int D>
cudaError_t run_d(const AttnParams& p, bool e4m3, int max_rows, long long max_kv, cudaStream_t st)
{
    const int rw = row_warps(max_rows);
    if (e4m3) {
        if (rw == 1) return run_one<typename Pick<D, true, 1, 0>::C>(p, max_rows, max_kv, st);
        if (rw == 2) return run_one<typename Pick<D, true, 2, 0>::C>(p, max_rows, max_kv, st);
        return run_one<typename Pick<D, true, 4, 0>::C>(p, max_rows, max_kv, st);
    }
    if (max_rows <= 8) return run_one<typename Pick<D, false, 1, 1>::C>(p, max_rows, max_kv, st);
    if (rw == 1) return run_one<typename Pick<D, false, 1, 2>::C>(p, max_rows, max_kv, st);
    if (rw == 2) return run_one<typename Pick<D, false, 2, 2>::C>(p, max_rows, max_kv, st);
    return run_one<typename Pick<D, false, 4, 2>::C>(p, max_rows, max_kv, st);
}
template <class C>
cudaError_t init_one_attn() { return cudaFuncSetAttribute(attention_paged_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); }
template <int D>
cudaError_t init_d()
{
    cudaError_t e = init_one_attn<typename Pick<D, true, 1, 0>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, true, 2, 0>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, true, 4, 0>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, false, 1, 1>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, false, 1, 2>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, false, 2, 2>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, false, 4, 2>::C>();
    return e;
}

}  // namespace

cudaError_t attention_paged_init()
{
    cudaError_t e = init_d<64>();
    if (e == cudaSuccess) e = init_d<128>();
    if (e == cudaSuccess) e = init_d<256>();
    return e;
}

// Workspace: descriptors, (maximum, sum) and fp32 outputs of at most two parts per CTA.
size_t attention_workspace_bytes(int max_rows, int head_dim, int sm_count)
{
    const size_t rows = 2 * static_cast<size_t>(sm_count) * 16 * row_warps(max_rows);
    const size_t desc = (static_cast<size_t>(sm_count) * 32 + 255) / 256 * 256;
    return desc + (rows * sizeof(float2) + 255) / 256 * 256 + rows * head_dim * sizeof(float);
}

cudaError_t launch_attention_paged(const AttnArgs& a, void* workspace, int sm_count, cudaStream_t st)
{
    AttnParams p;
    const int elt = a.e4m3 ? 1 : 2;
    p.Q = a.Q; p.ldq = a.ldq; p.O = a.O; p.ldo = a.ldo; p.lse = a.lse;
    p.cache = a.cache;
    p.cache.page_stride *= elt; p.cache.head_stride *= elt; p.cache.token_stride *= elt;
    p.table = a.table; p.ld_table = a.ld_table; p.kv_lens = a.kv_lens; p.q_starts = a.q_starts;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.max_pages = a.max_pages; p.B = a.B; p.max_q = a.max_q; p.M = a.M; p.heads = a.heads; p.kv_heads = a.kv_heads;
    p.group = a.heads / a.kv_heads; p.causal = a.causal;
    p.G = sm_count;
    const int max_rows = a.max_q * p.group;
    const size_t rows = 2 * static_cast<size_t>(sm_count) * 16 * row_warps(max_rows);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    p.desc = reinterpret_cast<int*>(ws);
    ws += (static_cast<size_t>(sm_count) * 32 + 255) / 256 * 256;
    p.part_ml = reinterpret_cast<float2*>(ws);
    ws += (rows * sizeof(float2) + 255) / 256 * 256;
    p.part_o = reinterpret_cast<float*>(ws);
    const long long max_kv = static_cast<long long>(a.max_pages) << a.cache.page_shift;
    if (a.head_dim == 64) return run_d<64>(p, a.e4m3, max_rows, max_kv, st);
    if (a.head_dim == 128) return run_d<128>(p, a.e4m3, max_rows, max_kv, st);
    return run_d<256>(p, a.e4m3, max_rows, max_kv, st);
}

}  // namespace rudder
