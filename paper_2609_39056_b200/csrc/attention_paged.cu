// Attention of a few new tokens of each request over a paged key-value cache (bf16 or E4M3), split over the cache's
// length and joined.
//
//     s_rj = scale q_r . k_j,   o_r = sum_j exp(s_rj - m_r) v_j / sum_j exp(s_rj - m_r),   lse_r = m_r + ln sum_j exp(s_rj - m_r)
//
// One pass over K and V with a running maximum and sum (fp32).  What bounds it is the read of the cache, once:
// 4 D bytes per key and key-value head in bf16.  The new tokens of a request and the query heads that share a key-value
// head are the ROWS of one product (R = tokens x heads / kv_heads), so the cache is read once for all of them.
//
// Up to 32 rows run here (more, and some of 17 to 32: attention_rows.cu), on mma.sync m16n8k16 with the KEYS (then V's channels) on the 16-row
// side and the rows on the 8 columns: S^T = K Q^T, O^T += V^T P^T.  Decoding has 1 to 8 rows, so 8 columns waste less than 16, and the cache's tiles are
// read by ldmatrix as they lie; tcgen05's smallest tile would walk 64 or 128 rows and move scores and probabilities through tensor memory
// for every tile.  P leaves the first product row-major and is transposed in registers, 8 x 8 at a time.
//
// Data path: the keys are cut into units; in a unit each of KW warp groups of a CTA has its own tile of KT keys, its own ring of
// NST stages in shared memory filled by 16-byte cp.async (page by page, rows of D contiguous elements, swizzled so that
// ldmatrix reads without bank conflicts), and its own running maximum, sum and output: no CTA-wide barrier in the main
// loop.  RW warps of a group share the tile and own 8 NB rows each.  Keys at or behind the request's length are
// filled with zeros and masked, whatever the cache holds there.
//
// Work split: all units of all (request, kv head, row tile) are one sequence, cut into equal runs, one per CTA, one CTA per
// SM: every SM streams the same number of bytes however ragged the lengths are.  Each CTA finds its place by a prefix sum over the
// requests' unit counts (device data).  A run crosses items; an item that is cut leaves its parts (fp32 output, maximum,
// sum) in the workspace and a second kernel joins them in order (deterministic).  When every item is short the items are
// handed out whole and nothing is joined.
//
// Rounding: K and V enter exactly, and so does Q with a bf16 cache.  E4M3 numbers are f16 numbers, Q is brought to f16
// by a power of two per row: exact down to 2^-28 of the row's largest element, below that off by at most 2^-39 of it.
// Scores and sums are fp32.  With bf16 values the probabilities enter the second product as TWO bf16 numbers hi + lo (2^-17): for up to 4 rows in
// the columns that would be empty, for more as a second product (LO).  With E4M3 values they enter as one f16 number, and f16 has few exponents: the
// reference of a row is its maximum less kTop, so that the largest probability is 2^kTop instead of 1 and 2^-11 holds for every key down to 2^-29 of the
// largest, 2^-40 of the largest below that.  (With the maximum as the reference a key 2^20 below the largest kept four bits: what
// is left of a row when its largest key is a sink with a small value.)  Sums and parts are relative to the same reference: nothing else changes.
//
// Measured (one new token, 8 query heads per key-value head unless said): 4 x 126k keys bf16 158 us = 6.6 TB/s, D = 64 86 us = 6.1, E4M3 86 us = 6.1;
// 48 requests of up to 16384 keys in E4M3 57.5 us = 4.9 TB/s; one request of 333 keys 6.6 us, of which a launch is 2, the place of the run 1,
// the pages and the first tile 1.2, the products 1.3 and the output 1.
#include "attention_rows.cu"

namespace rudder {

namespace {

__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool F16>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (F16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 x 8 block of 16-bit numbers, a row per 4 lanes: transposed.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
// RB bytes per row of a tile: the 16-byte chunk c of row r sits at chunk swz(r, c).
template <int RB>
__device__ __forceinline__ uint32_t swz(int r, int c) {
    return static_cast<uint32_t>(r) * RB + (static_cast<uint32_t>(RB >= 128 ? (c ^ (r & 7)) : (c ^ ((r >> 1) & 3))) << 4);
}

// LO: 0 = probabilities once (f16, or bf16), 1 = at most 4 rows: columns 4..7 repeat the queries of 0..3 and carry the
// low parts of the probabilities (free), 2 = hi and lo as two products.
template <int D_, bool E4M3_, int NB_, int RW_, int KW_, int KT_, int NST_, int LO_>
struct AttnCfg {
    static constexpr int D = D_, NB = NB_, RW = RW_, KW = KW_, KT = KT_, NST = NST_, LO = LO_;
    static constexpr bool E4M3 = E4M3_;
    static constexpr int THREADS = 32 * RW * KW;
    static constexpr int ROWS = 8 * NB * RW;               // rows of a tile
    static constexpr int UK = KW * KT;                     // keys of a unit
    static constexpr int RB = D * (E4M3 ? 1 : 2);          // bytes of a row of a tile
    static constexpr int STAGE = 2 * KT * RB;              // K tile, V tile
    static constexpr int RING = KW * NST * STAGE;
    // the box in which the warp groups' outputs are added, [KW][ROWS][channels of a round + 4]: as many rounds as make it fit behind the ring
    static constexpr int ML = KW * ROWS * 8;
    static constexpr int box_bytes(int rounds) { return KW * ROWS * (D / rounds + 4) * 4; }
    static constexpr int rounds() {
        int r = 1;
        while (r < D / 32 && (RING + ML + box_bytes(r) > 226 * 1024 || box_bytes(r) > 36 * 1024)) r *= 2;
        return r;
    }
    static constexpr int ROUNDS = rounds();
    static constexpr int DC = D / ROUNDS;
    static constexpr int BOX = box_bytes(ROUNDS);
    static constexpr int SMEM = RING + BOX + ML;
    static_assert(DC % 16 == 0 && DC >= 32, "a round is whole channel tiles");
    static_assert(SMEM <= 226 * 1024, "shared memory of an SM");
};

// CAUSAL: the rows of an item may see different numbers of keys.
template <class C, bool CAUSAL>
__global__ void __launch_bounds__(C::THREADS, 1) attention_paged_kernel(const AttnParams p)
{
    constexpr int D = C::D, NB = C::NB, RW = C::RW, KW = C::KW, KT = C::KT, NST = C::NST, LO = C::LO, RB = C::RB, UK = C::UK, ROWS = C::ROWS, DC = C::DC;
    constexpr bool E4M3 = C::E4M3;
    constexpr int CH = RB / 16;                            // 16-byte chunks of a row
    constexpr int KS = D / 16;                             // steps of the first product
    constexpr int MT = KT / 16;                            // key tiles of the first product
    constexpr int DT = D / 16;                             // channel tiles of the second
    constexpr int GT = 32 * RW;                            // threads of a warp group
    constexpr float kTop = E4M3 ? 15.0f : 0.0f;            // log2 of the largest probability: f16 ends at 2^16
    static_assert(KT == 16 || KT == 32, "a lane holds the place of one key of the tile");
    static_assert(GT % CH == 0 || CH % GT == 0, "rows are copied by whole groups of lanes");
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint32_t s_dropped[RW * KW];                // per warp: see drop_nonfinite
    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int g = lane >> 2, q = lane & 3;
    const int kg = warp / RW, rw = warp % RW;
    const int gt = tid - kg * GT;                          // thread inside the warp group

    Cursor<ROWS, UK> cur;
    if (!start_of_run<ROWS, UK, C::THREADS>(p, cur)) return;

    // ---- the ring of this warp group
    const uint32_t ring = smem_u32(smem) + kg * (NST * C::STAGE);
    Cursor<ROWS, UK> ld = cur;
    // page ids of the tile `at` is about to load: lane i holds the one of key i (KT <= 32)
    auto page_of_lane = [&](const Cursor<ROWS, UK>& at) -> int {
        const int key = at.j * UK + kg * KT + lane;
        return (lane < KT && key < at.rq.len) ? p.table[static_cast<size_t>(at.b) * p.ld_table + (key >> p.cache.page_shift)] : -2;
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
    int pages[NST - 1];                                    // of the first tiles: one wait for all of them
    {
        Cursor<ROWS, UK> ahead = cur;
#pragma unroll
        for (int s = 0; s < NST - 1; ++s) {
            pages[s] = ahead.left > 0 ? page_of_lane(ahead) : -2;
            if (ahead.left > 0) ahead.advance(p);
        }
    }
#pragma unroll
    for (int s = 0; s < NST - 1; ++s) {
        if (ld.left > 0) {
            issue(ld, pages[s], s);
            ld.advance(p);
        }
        cp_async_commit();
    }

    uint32_t qf[KS][NB][2];
    float acc[DT][NB][4];                                  // output, transposed: channels on the 16-row side, rows on the 8 columns
    float mx[NB][2], sum[NB][2], fac[NB][2];               // of rows 2 q and 2 q + 1 of every 8: reference (running maximum - kTop) and sum, score factor
    int lim[NB][2];                                        // keys the rows see
    int tail = 0;                                          // keys that all rows of the tile see: len where it is the same for all
    bool fresh = true, first_part = true, dropped = false;
    int part_j = 0;                                        // the unit of the item this run starts it with
    int stage = 0;

    while (cur.left > 0) {
        if (fresh) {
            // ---- a new item (or the rest of one): queries, limits, empty sums
            fresh = false;
            part_j = cur.j;
            tail = CAUSAL ? tail_of(cur.rq.len, cur.rq.qlen, row_of(p, cur.rt * ROWS).token) : cur.rq.len;
            dropped = false;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int n = 0; n < NB; ++n) acc[t][n][0] = acc[t][n][1] = acc[t][n][2] = acc[t][n][3] = 0.0f;
            const int R = cur.rq.qlen * p.group, first_row = cur.rt * ROWS + rw * 8 * NB;
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                mx[n][0] = mx[n][1] = -INFINITY;
                sum[n][0] = sum[n][1] = 0.0f;
                // rows that do not exist: zeros, no limit of their own
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = first_row + 8 * n + (LO == 1 ? (2 * q + e) & 3 : 2 * q + e);
                    lim[n][e] = (CAUSAL && r < R) ? cur.rq.len - cur.rq.qlen + row_of(p, r).token + 1 : cur.rq.len;
                    fac[n][e] = p.scale_log2;
                }
                const int r = first_row + 8 * n + (LO == 1 ? g & 3 : g);
                const bool live = r < R;
                const uint16_t* qr = p.Q;
                const RowOf at = row_of(p, r);
                if (live) qr += static_cast<size_t>(cur.rq.row0 + at.token) * p.ldq + static_cast<size_t>(cur.h * p.group + at.head) * D;
                if (!E4M3) {
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        qf[ks][n][0] = live ? *reinterpret_cast<const uint32_t*>(qr + 16 * ks + 2 * q) : 0u;
                        qf[ks][n][1] = live ? *reinterpret_cast<const uint32_t*>(qr + 16 * ks + 2 * q + 8) : 0u;
                    }
                } else {
                    // channels 4 q .. 4 q + 3 of every 16 (the K bytes of a lane); f16 times a power of two per row
                    float x = 0.0f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        const uint2 a = live ? *reinterpret_cast<const uint2*>(qr + 16 * ks + 4 * q) : make_uint2(0, 0);
                        qf[ks][n][0] = a.x; qf[ks][n][1] = a.y;
                        x = fmaxf(x, fmaxf(fmaxf(fabsf(bf16_lo(a.x)), fabsf(bf16_hi(a.x))), fmaxf(fabsf(bf16_lo(a.y)), fabsf(bf16_hi(a.y)))));
                    }
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                    x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                    // the row's largest magnitude lands in [2^14, 2^15), as far as a factor of 2^+-126 brings it
                    const int ex = min(126, max(-126, 14 - (static_cast<int>((__float_as_uint(x) >> 23) & 255u) - 127)));
                    const float sc = __uint_as_float(static_cast<uint32_t>(ex + 127) << 23);
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        const uint32_t ax = qf[ks][n][0], ay = qf[ks][n][1];
                        qf[ks][n][0] = f16x2(bf16_lo(ax) * sc, bf16_hi(ax) * sc);
                        qf[ks][n][1] = f16x2(bf16_lo(ay) * sc, bf16_hi(ay) * sc);
                    }
                    const float back = (p.cache.k_scale != nullptr ? p.cache.k_scale[cur.h] : 1.0f) * p.scale_log2 *
                                       __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
                    fac[n][0] = __shfl_sync(0xffffffffu, back, 8 * q);         // row 2 q of the tile is lane g = 2 q
                    fac[n][1] = __shfl_sync(0xffffffffu, back, 8 * q + 4);
                }
            }
        }
        cp_async_wait<NST - 2>();
        if (RW == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + kg), "n"(GT) : "memory");
        // page ids of the tile that goes into the stage just freed: requested now, used after this tile's products
        const bool more = ld.left > 0;
        const int page = more ? page_of_lane(ld) : -2;

        const int key0 = cur.j * UK + kg * KT;
        if (key0 < cur.rq.len) {
            const uint32_t kt = ring + stage * C::STAGE, vt = kt + KT * RB;
            const bool edge = key0 + KT > tail;
            if (CAUSAL && edge && tail < cur.rq.len) {
                const int r0 = max(0, tail - key0), r1 = min(KT, cur.rq.len - key0);
                for (int i = r0 * CH + gt; i < r1 * CH; i += GT) dropped |= drop_nonfinite<E4M3 ? kExpE4m3 : kExpBf16>(vt + 16 * i);
                if (RW == 1) __syncwarp();
                else asm volatile("bar.sync %0, %1;" ::"r"(1 + kg), "n"(GT) : "memory");
            }
            float s[MT][NB][4];                            // scores, transposed: keys on the 16-row side
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int n = 0; n < NB; ++n) s[t][n][0] = s[t][n][1] = s[t][n][2] = s[t][n][3] = 0.0f;
            // ---- S^T = K Q^T
            if (!E4M3) {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        uint32_t a[4];                     // keys (0..7, 8..15) x the step's two chunks
                        ldsm_x4(a, kt + swz<RB>(16 * t + (lane & 15), 2 * ks + (lane >> 4)));
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16<false>(s[t][n], a, qf[ks][n][0], qf[ks][n][1]);
                    }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2)
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        uint32_t r[4], a[4];               // keys (0..7, 8..15) x two chunks, a step each
                        ldsm_x4(r, kt + swz<RB>(16 * t + (lane & 15), ks + (lane >> 4)));
                        e4m3_to_f16(r[0], a[0], a[2]);
                        e4m3_to_f16(r[1], a[1], a[3]);
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16<true>(s[t][n], a, qf[ks][n][0], qf[ks][n][1]);
                        e4m3_to_f16(r[2], a[0], a[2]);
                        e4m3_to_f16(r[3], a[1], a[3]);
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16<true>(s[t][n], a, qf[ks + 1][n][0], qf[ks + 1][n][1]);
                    }
            }
            // ---- running maximum and sum (base 2)
            uint32_t ph[MT][NB][2], pl[LO == 2 ? MT : 1][NB][2];
            bool moved = false;
            float cor[NB][2];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    s[t][n][0] *= fac[n][0]; s[t][n][1] *= fac[n][1]; s[t][n][2] *= fac[n][0]; s[t][n][3] *= fac[n][1];
                    if (edge) {
                        const int k = key0 + 16 * t + g;
                        if (k >= lim[n][0]) s[t][n][0] = -INFINITY;
                        if (k >= lim[n][1]) s[t][n][1] = -INFINITY;
                        if (k + 8 >= lim[n][0]) s[t][n][2] = -INFINITY;
                        if (k + 8 >= lim[n][1]) s[t][n][3] = -INFINITY;
                    }
                    x0 = fmaxf(x0, fmaxf(s[t][n][0], s[t][n][2]));
                    x1 = fmaxf(x1, fmaxf(s[t][n][1], s[t][n][3]));
                }
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, o));
                    x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, o));
                }
                if (E4M3) { x0 -= kTop; x1 -= kTop; }
                const float n0 = fmaxf(mx[n][0], x0), n1 = fmaxf(mx[n][1], x1);
                const float u0 = n0 == -INFINITY ? 0.0f : n0, u1 = n1 == -INFINITY ? 0.0f : n1;  // an empty row so far: exp2(-inf - 0) = 0
                cor[n][0] = exp2_approx(mx[n][0] - u0);
                cor[n][1] = exp2_approx(mx[n][1] - u1);
                moved |= cor[n][0] != 1.0f || cor[n][1] != 1.0f;
                mx[n][0] = n0; mx[n][1] = n1;
                float l0 = 0.0f, l1 = 0.0f;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    const float e0 = exp2_approx(s[t][n][0] - u0), e1 = exp2_approx(s[t][n][1] - u1);
                    const float e2 = exp2_approx(s[t][n][2] - u0), e3 = exp2_approx(s[t][n][3] - u1);
                    l0 += e0 + e2;
                    l1 += e1 + e3;
                    if (E4M3) {
                        ph[t][n][0] = f16x2(e0, e1);
                        ph[t][n][1] = f16x2(e2, e3);
                    } else {
                        const uint32_t h0 = bf16x2(e0, e1), h1 = bf16x2(e2, e3);
                        ph[t][n][0] = h0;
                        ph[t][n][1] = h1;
                        if (LO != 0) {
                            const uint32_t w0 = bf16x2(e0 - bf16_lo(h0), e1 - bf16_hi(h0)), w1 = bf16x2(e2 - bf16_lo(h1), e3 - bf16_hi(h1));
                            if (LO == 1) {
                                if (q >= 2) { ph[t][n][0] = w0; ph[t][n][1] = w1; }
                            } else {
                                pl[LO == 2 ? t : 0][n][0] = transpose8x8(w0);
                                pl[LO == 2 ? t : 0][n][1] = transpose8x8(w1);
                            }
                        }
                    }
                    ph[t][n][0] = transpose8x8(ph[t][n][0]);
                    ph[t][n][1] = transpose8x8(ph[t][n][1]);
                }
                sum[n][0] = sum[n][0] * cor[n][0] + l0;
                sum[n][1] = sum[n][1] * cor[n][1] + l1;
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int t = 0; t < DT; ++t)
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        acc[t][n][0] *= cor[n][0]; acc[t][n][1] *= cor[n][1]; acc[t][n][2] *= cor[n][0]; acc[t][n][3] *= cor[n][1];
                    }
            }
            // ---- O^T += V^T P^T
#pragma unroll
            for (int kk = 0; kk < MT; ++kk) {
                if (!E4M3) {
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        uint32_t a[4];                     // channels (0..7, 8..15) x keys (0..7, 8..15)
                        ldsm_x4_t(a, vt + swz<RB>(16 * kk + ((lane >> 4) << 3) + (lane & 7), 2 * t + ((lane >> 3) & 1)));
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            mma16<false>(acc[t][n], a, ph[kk][n][0], ph[kk][n][1]);
                            if (LO == 2) mma16<false>(acc[t][n], a, pl[LO == 2 ? kk : 0][n][0], pl[LO == 2 ? kk : 0][n][1]);
                        }
                    }
                } else {
#pragma unroll
                    for (int t = 0; t < DT; t += 2) {
                        uint32_t r[4], a[4];               // keys (0..7, 8..15) of two chunks; a register = 2 keys x channels (2 g, 2 g + 1)
                        ldsm_x4_t(r, vt + swz<RB>(16 * kk + (lane & 15), t + (lane >> 4)));
                        e4m3_to_f16_split(r[0], a[0], a[1]);     // row g of the product is channel 2 g, row g + 8 channel 2 g + 1
                        e4m3_to_f16_split(r[1], a[2], a[3]);
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16<true>(acc[t][n], a, ph[kk][n][0], ph[kk][n][1]);
                        e4m3_to_f16_split(r[2], a[0], a[1]);
                        e4m3_to_f16_split(r[3], a[2], a[3]);
#pragma unroll
                        for (int n = 0; n < NB; ++n) mma16<true>(acc[t + 1][n], a, ph[kk][n][0], ph[kk][n][1]);
                    }
                }
            }
        }
        if (more) {
            issue(ld, page, stage == 0 ? NST - 1 : stage - 1);
            ld.advance(p);
        }
        cp_async_commit();
        stage = stage + 1 == NST ? 0 : stage + 1;

        const bool item_end = cur.j + 1 == cur.nt;
        if (item_end || cur.left == 1) {
            // ---- end of an item or of this run: add the warp groups, write the rows or the part
            float* box = reinterpret_cast<float*>(smem + C::RING);
            float2* ml = reinterpret_cast<float2*>(smem + C::RING + C::BOX);
            const bool entire = item_end && part_j == 0;
            const int slot = 2 * blockIdx.x + (first_part ? 0 : 1);              // part at the start of the run, or at its end
            const int R = cur.rq.qlen * p.group;
            const float vs = E4M3 ? (p.cache.v_scale != nullptr ? p.cache.v_scale[cur.h] : 1.0f) : 1.0f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float l = sum[n][e];
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
                    if (g == 0) ml[kg * ROWS + rw * 8 * NB + 8 * n + 2 * q + e] = make_float2(mx[n][e], l);
                }
            if (CAUSAL && tail < cur.rq.len) {
                dropped = __any_sync(0xffffffffu, dropped);
                if (lane == 0) s_dropped[warp] = dropped;
            }
            __syncthreads();
            if (CAUSAL && tail < cur.rq.len)
                for (int w = 0; w < RW * KW; ++w) dropped |= s_dropped[w] != 0;
            float wgt[NB][2];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int rl = rw * 8 * NB + 8 * n + 2 * q + e;
                    float m = mx[n][e], l = 0.0f;
#pragma unroll
                    for (int w = 0; w < KW; ++w) m = fmaxf(m, ml[w * ROWS + rl].x);
                    const float u = m == -INFINITY ? 0.0f : m;
#pragma unroll
                    for (int w = 0; w < KW; ++w) {
                        const float2 o = ml[w * ROWS + rl];
                        l += o.y * exp2_approx(o.x - u);
                    }
                    wgt[n][e] = exp2_approx(mx[n][e] - u) * vs * (entire ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f);
                    if (kg == 0 && g == 0) {
                        const int r = cur.rt * ROWS + rl;
                        if (r < R) {
                            if (!entire) p.part_ml[static_cast<size_t>(slot) * ROWS + rl] = make_float2(m, l);
                            else if (p.lse != nullptr) {
                                const RowOf at = row_of(p, r);
                                p.lse[static_cast<size_t>(cur.rq.row0 + at.token) * p.heads + cur.h * p.group + at.head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
                            }
                        }
                    }
                }
            const int rows_here = min(ROWS, R - cur.rt * ROWS);
#pragma unroll
            for (int round = 0; round < C::ROUNDS; ++round) {
                if (round > 0) __syncthreads();
                float* mine = box + (kg * ROWS + rw * 8 * NB) * (DC + 4);
#pragma unroll
                for (int t = 0; t < DC / 16; ++t)
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        const float* c = acc[round * (DC / 16) + t][n];
                        float* b0 = mine + (8 * n + 2 * q) * (DC + 4) + 16 * t;
                        float* b1 = b0 + DC + 4;
                        if (E4M3) {
                            *reinterpret_cast<float2*>(b0 + 2 * g) = make_float2(c[0] * wgt[n][0], c[2] * wgt[n][0]);
                            *reinterpret_cast<float2*>(b1 + 2 * g) = make_float2(c[1] * wgt[n][1], c[3] * wgt[n][1]);
                        } else {
                            b0[g] = c[0] * wgt[n][0]; b0[g + 8] = c[2] * wgt[n][0];
                            b1[g] = c[1] * wgt[n][1]; b1[g + 8] = c[3] * wgt[n][1];
                        }
                    }
                __syncthreads();
                for (int i = tid; i < rows_here * (DC / 4); i += C::THREADS) {
                    const int rl = i / (DC / 4), d = 4 * (i % (DC / 4));
                    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < KW; ++w) {
                        const float4 v = *reinterpret_cast<const float4*>(box + (w * ROWS + rl) * (DC + 4) + d);
                        o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
                        if (LO == 1) {                     // the low parts of row rl are row rl + 4
                            const float4 x = *reinterpret_cast<const float4*>(box + (w * ROWS + rl + 4) * (DC + 4) + d);
                            o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
                        }
                    }
                    const RowOf at = row_of(p, cur.rt * ROWS + rl);
                    if (entire)
                        *reinterpret_cast<uint2*>(p.O + static_cast<size_t>(cur.rq.row0 + at.token) * p.ldo + static_cast<size_t>(cur.h * p.group + at.head) * D +
                                                  round * DC + d) = make_uint2(bf16x2(o.x, o.y), bf16x2(o.z, o.w));
                    else
                        *reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(slot) * ROWS + rl) * D + round * DC + d) = o;
                }
            }
            if (CAUSAL && dropped) {
                // each thread goes over what it has written
                for (int round = 0; round < C::ROUNDS; ++round)
                    for (int i = tid; i < rows_here * (DC / 4); i += C::THREADS) {
                        const int rl = i / (DC / 4), d = round * DC + 4 * (i % (DC / 4));
                        const RowOf at = row_of(p, cur.rt * ROWS + rl);
                        const float4 z = nonfinite_values<E4M3>(p, cur.b, cur.h, max(tail, part_j * UK), min(cur.rq.len - cur.rq.qlen + at.token + 1, (cur.j + 1) * UK), d);
                        if (entire) {
                            uint2* o = reinterpret_cast<uint2*>(p.O + static_cast<size_t>(cur.rq.row0 + at.token) * p.ldo + static_cast<size_t>(cur.h * p.group + at.head) * D + d);
                            const uint2 v = *o;
                            *o = make_uint2(bf16x2(bf16_lo(v.x) + z.x, bf16_hi(v.x) + z.y), bf16x2(bf16_lo(v.y) + z.z, bf16_hi(v.y) + z.w));
                        } else {
                            float4* o = reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(slot) * ROWS + rl) * D + d);
                            const float4 v = *o;
                            *o = make_float4(v.x + z.x, v.y + z.y, v.z + z.z, v.w + z.w);
                        }
                    }
            }
            fresh = true;
            first_part = false;
            // (the next item's end writes `ml` only after every thread has read it: each reads before the barrier above)
        }
        cur.advance(p);
    }
    cp_async_wait<0>();
}

// The parts of the items that were cut, joined in the order of their runs: CTA (c, y) the item that run c starts inside, rows
// JOIN_ROWS y .. + JOIN_ROWS - 1 of its tile.  JOIN_SPLIT warps per row take the parts in turn.
constexpr int JOIN_THREADS = 256, JOIN_ROWS = 2, JOIN_SPLIT = JOIN_THREADS / 32 / JOIN_ROWS;

// The item that run c starts inside; false if its join is another CTA's or there is none.
struct Cut { int h, rt, row0, qlen, first, n, slot_first; };
__device__ __forceinline__ bool load_cut(const AttnParams& p, int c, Cut& x) {
    const int4 a = __ldcg(reinterpret_cast<const int4*>(p.desc + 8 * c)), b = __ldcg(reinterpret_cast<const int4*>(p.desc + 8 * c + 4));
    x.h = a.y; x.rt = a.z; x.row0 = a.w; x.qlen = b.x; x.first = c - 1; x.n = b.y - (c - 1) + 1; x.slot_first = b.z;
    return a.x != 0;
}

template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) attention_join_kernel(const AttnParams p, int rows_of_tile)
{
    __shared__ float s_o[JOIN_ROWS][JOIN_SPLIT][D];
    __shared__ float2 s_ml[JOIN_ROWS][JOIN_SPLIT];
    pdl_launch_dependents();
    pdl_wait();
    Cut x;
    if (!load_cut(p, blockIdx.x, x)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int ry = warp / JOIN_SPLIT, part = warp % JOIN_SPLIT;
    const int rl = blockIdx.y * JOIN_ROWS + ry, r = x.rt * rows_of_tile + rl;
    const bool live = r < x.qlen * p.group;
    constexpr int V = D / 32;                              // channels of a lane
    float o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    if (live) {
        for (int s = part; s < x.n; s += JOIN_SPLIT) {
            const size_t at = (2 * static_cast<size_t>(x.first + s) + (s == 0 ? x.slot_first : 0)) * rows_of_tile + rl;
            const float2 ml = __ldcg(p.part_ml + at);
            const float* src = p.part_o + at * D + lane * V;
            float v[V];
            if (V == 2) { const float2 t = __ldcg(reinterpret_cast<const float2*>(src)); v[0] = t.x; v[1] = t.y; }
            else {
#pragma unroll
                for (int i = 0; i < V; i += 4) {
                    const float4 t = __ldcg(reinterpret_cast<const float4*>(src + i));
                    v[i] = t.x; v[i + 1] = t.y; v[i + 2] = t.z; v[i + 3] = t.w;
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
    const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
    const RowOf at = row_of(p, r);
    const int hh = x.h * p.group + at.head;
    uint16_t* orow = p.O + static_cast<size_t>(x.row0 + at.token) * p.ldo + static_cast<size_t>(hh) * D + lane * V;
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
    if (lane == 0 && p.lse != nullptr) p.lse[static_cast<size_t>(x.row0 + at.token) * p.heads + hh] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * kLn2;
}

// The same for many rows: a lane per row, as the parts lie; a warp has 32 rows x 8 channels, a CTA 64 channels, y = row block x channel block.
template <int D>
__global__ void __launch_bounds__(JOIN_THREADS) attention_join_rows_kernel(const AttnParams p, int rows_of_tile)
{
    pdl_launch_dependents();
    pdl_wait();
    Cut x;
    if (!load_cut(p, blockIdx.x, x)) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rl = blockIdx.y / (D / 64) * 32 + lane, ch = blockIdx.y % (D / 64) * 64 + warp * 8;
    const int r = x.rt * rows_of_tile + rl;
    if (r >= x.qlen * p.group) return;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = 0.0f;
    float m = -INFINITY, l = 0.0f;
#pragma unroll 4
    for (int s = 0; s < x.n; ++s) {
        const size_t slot = 2 * static_cast<size_t>(x.first + s) + (s == 0 ? x.slot_first : 0);
        const float2 ml = __ldcg(p.part_ml + slot * rows_of_tile + rl);
        const float* src = p.part_o + slot * rows_of_tile * D + (static_cast<size_t>(ch / 4) * rows_of_tile + rl) * 4;
        const float4 v0 = __ldcg(reinterpret_cast<const float4*>(src)), v1 = __ldcg(reinterpret_cast<const float4*>(src + 4 * rows_of_tile));
        const float nm = fmaxf(m, ml.x), u = nm == -INFINITY ? 0.0f : nm;
        const float a = exp2_approx(m - u), b = exp2_approx(ml.x - u);
        m = nm;
        l = l * a + ml.y * b;
        o[0] = o[0] * a + v0.x * b; o[1] = o[1] * a + v0.y * b; o[2] = o[2] * a + v0.z * b; o[3] = o[3] * a + v0.w * b;
        o[4] = o[4] * a + v1.x * b; o[5] = o[5] * a + v1.y * b; o[6] = o[6] * a + v1.z * b; o[7] = o[7] * a + v1.w * b;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const RowOf at = row_of(p, r);
    const int hh = x.h * p.group + at.head;
    *reinterpret_cast<uint4*>(p.O + static_cast<size_t>(x.row0 + at.token) * p.ldo + static_cast<size_t>(hh) * D + ch) =
        make_uint4(bf16x2(o[0] * inv, o[1] * inv), bf16x2(o[2] * inv, o[3] * inv), bf16x2(o[4] * inv, o[5] * inv), bf16x2(o[6] * inv, o[7] * inv));
    if (ch == 0 && p.lse != nullptr) p.lse[static_cast<size_t>(x.row0 + at.token) * p.heads + hh] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// ---- variants: warps over rows (RW) and keys (KW), keys per tile, stages.  The ring is about 130 to 200 KB: it is what keeps
// enough of the cache in flight with one CTA per SM.
// CLS: rows of an item up to 4, 8, 16, 32 (more: attention_rows.cu)
template <int D, bool E4M3, int CLS>
struct Pick;
template <int CLS> constexpr int kLo = CLS == 0 ? 1 : 2;
template <int CLS> struct Pick<64, false, CLS> { using C = AttnCfg<64, false, CLS <= 1 ? 1 : 2, 1, 8, 32, 3, kLo<CLS>>; };
template <int CLS> struct Pick<64, true, CLS> { using C = AttnCfg<64, true, CLS <= 1 ? 1 : 2, 1, CLS <= 1 ? 16 : 8, 32, CLS <= 1 ? 3 : 5, 0>; };
template <int CLS> struct Pick<128, false, CLS> { using C = AttnCfg<128, false, CLS <= 1 ? 1 : 2, 1, 8, 16, 3, kLo<CLS>>; };
template <int CLS> struct Pick<128, true, CLS> { using C = AttnCfg<128, true, CLS <= 1 ? 1 : 2, 1, 8, 32, 3, 0>; };
template <int CLS> struct Pick<256, false, CLS> { using C = AttnCfg<256, false, CLS <= 1 ? 1 : 2, 1, 4, 16, 3, kLo<CLS>>; };
template <int CLS> struct Pick<256, true, CLS> { using C = AttnCfg<256, true, CLS <= 1 ? 1 : 2, 1, 8, 16, 3, 0>; };
template <> struct Pick<64, false, 3> { using C = AttnCfg<64, false, 2, 2, 4, 32, 5, 2>; };
template <> struct Pick<64, true, 3> { using C = AttnCfg<64, true, 2, 2, 4, 32, 5, 0>; };
template <> struct Pick<128, false, 3> { using C = AttnCfg<128, false, 2, 2, 4, 16, 5, 2>; };
template <> struct Pick<128, true, 3> { using C = AttnCfg<128, true, 2, 2, 4, 32, 5, 0>; };
template <> struct Pick<256, false, 3> { using C = AttnCfg<256, false, 2, 2, 4, 16, 3, 2>; };
template <> struct Pick<256, true, 3> { using C = AttnCfg<256, true, 2, 2, 4, 16, 5, 0>; };

int rows_class(int max_rows) { return max_rows <= 4 ? 0 : (max_rows <= 8 ? 1 : (max_rows <= 16 ? 2 : (max_rows <= 32 ? 3 : 4))); }
// The tcgen05 kernel (attention_rows.cu): above 32 rows always; 17 to 32 rows in bf16 with D = 128 and a table of 4096 tokens or more (the lengths
// themselves are device data).  Measured, this kernel / that one, 4 requests x 4 key-value heads unless said:
//   bf16, D = 128: 32 rows x 1000 keys 13.1 / 14.4 us, 1 request x 16 heads of 32 x 4480 22.6 / 21.5, 20 x 8000 30.4 / 30.9, 32 x 126k 293 / 210, 64 x 126k 429 / 218;
//   D = 64: 20 rows, 9 requests of up to 2500 keys 10.5 / 13.6, 32 x 126k 155 to 193 / 220 to 250, 64 x 126k 299 / 197; D = 256: 32 x 1500 21.1 / 20.0, 32 x 60k 265 / 278;
//   E4M3, D = 128: 20 x 1000 12.1 / 15.9, 32 x 8000 25 / 36, 32 x 60k 96 / 144, 32 x 126k 189 / 282, 64 x 126k 353 / 295; D = 64: 20 x 8000 18.3 / 25.5, 32 x 126k 143 / 227,
//   64 x 126k 269 / 227; D = 256: 32 x 1500 19.1 / 21.4, 32 x 60k 219 / 244.
bool many_rows(int max_rows, int head_dim, bool e4m3, long long max_kv) { return max_rows > 32 || (max_rows > 16 && head_dim == 128 && !e4m3 && max_kv >= 4096); }
// Rows of a part in the workspace (whichever kernel runs: the size depends on the shapes alone)
int tile_rows(int max_rows) { return max_rows <= 8 ? 8 : (max_rows <= 16 ? 16 : 128); }

template <int D, bool E4M3>
cudaError_t launch_main(const AttnParams& p, const AttnArgs& a, cudaStream_t st, RowsCfg<D, E4M3>) { return launch_rows<RowsCfg<D, E4M3>>(p, &a.tm_k, &a.tm_v, st); }
template <class C>
cudaError_t launch_main(const AttnParams& p, const AttnArgs&, cudaStream_t st, C)
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
    return cudaLaunchKernelEx(&cfg, p.causal ? attention_paged_kernel<C, true> : attention_paged_kernel<C, false>, p);
}
template <int D>
cudaError_t launch_join(const AttnParams& p, int rows_of_tile, int max_rows, cudaStream_t st)
{
    const int rows = max_rows < rows_of_tile ? max_rows : rows_of_tile;
    const bool many = rows_of_tile == 128;                 // the parts of attention_rows.cu
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(p.G), static_cast<unsigned>(many ? (rows + 31) / 32 * (D / 64) : (rows + JOIN_ROWS - 1) / JOIN_ROWS), 1);
    cfg.blockDim = dim3(JOIN_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return many ? cudaLaunchKernelEx(&cfg, attention_join_rows_kernel<D>, p, rows_of_tile) : cudaLaunchKernelEx(&cfg, attention_join_kernel<D>, p, rows_of_tile);
}
template <class C>
cudaError_t run_one(AttnParams p, const AttnArgs& a, int max_rows, long long max_kv, cudaStream_t st)
{
    const long long items = static_cast<long long>(p.B) * p.kv_heads * ((max_rows + C::ROWS - 1) / C::ROWS);
    // Short items are handed out whole: a join costs about 1.2 us, a unit of 128 keys in one CTA as much.  Measured, whole / cut: 16 items of 200 keys
    // 6.2 / 7.4 us, 333 7.4 / 7.4, 500 8.7 / 7.5; 64 items of 333 7.6 / 9.7, 500 9.0 / 10.1, 1000 14.0 / 12.6.
    p.whole_units = (4 * items > p.G ? 512 : 384) / C::UK;
    cudaError_t e = launch_main(p, a, st, C());
    if (e != cudaSuccess) return e;
    // no item can be cut: there is a CTA for each and the table has no room for a longer one
    if (items <= p.G && (max_kv + C::UK - 1) / C::UK <= p.whole_units) return cudaSuccess;
    return launch_join<C::D>(p, C::ROWS, max_rows, st);
}
template <int D, bool E4M3>
cudaError_t run_df(const AttnParams& p, const AttnArgs& a, int max_rows, long long max_kv, cudaStream_t st)
{
    static_assert(Pick<D, E4M3, 0>::C::ROWS == 8 && Pick<D, E4M3, 2>::C::ROWS == 16 && RowsCfg<D, E4M3>::ROWS == 128, "tile_rows()");
    switch (rows_class(max_rows)) {
        case 0: return run_one<typename Pick<D, E4M3, E4M3 ? 1 : 0>::C>(p, a, max_rows, max_kv, st);
        case 1: return run_one<typename Pick<D, E4M3, 1>::C>(p, a, max_rows, max_kv, st);
        case 2: return run_one<typename Pick<D, E4M3, 2>::C>(p, a, max_rows, max_kv, st);
        case 3: if (!many_rows(max_rows, D, E4M3, max_kv)) return run_one<typename Pick<D, E4M3, 3>::C>(p, a, max_rows, max_kv, st); [[fallthrough]];
        default: return run_one<RowsCfg<D, E4M3>>(p, a, max_rows, max_kv, st);
    }
}
template <int D>
cudaError_t run_d(const AttnParams& p, const AttnArgs& a, bool e4m3, int max_rows, long long max_kv, cudaStream_t st)
{
    return e4m3 ? run_df<D, true>(p, a, max_rows, max_kv, st) : run_df<D, false>(p, a, max_rows, max_kv, st);
}
template <class C>
cudaError_t init_one_attn()
{
    const cudaError_t e = cudaFuncSetAttribute(attention_paged_kernel<C, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    return e == cudaSuccess ? cudaFuncSetAttribute(attention_paged_kernel<C, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) : e;
}
template <int D, bool E4M3>
cudaError_t init_df()
{
    cudaError_t e = init_one_attn<typename Pick<D, E4M3, E4M3 ? 1 : 0>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, E4M3, 1>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, E4M3, 2>::C>();
    if (e == cudaSuccess) e = init_one_attn<typename Pick<D, E4M3, 3>::C>();
    if (e == cudaSuccess) e = init_rows<RowsCfg<D, E4M3>>();
    return e;
}
template <int D>
cudaError_t init_d()
{
    cudaError_t e = init_df<D, false>();
    return e == cudaSuccess ? init_df<D, true>() : e;
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
bool attention_uses_maps(int max_rows, int head_dim, bool e4m3, int page_size, long long max_kv)
{
    return many_rows(max_rows, head_dim, e4m3, max_kv) && page_size >= 8;
}

size_t attention_workspace_bytes(int max_rows, int head_dim, int sm_count)
{
    const size_t rows = 2 * static_cast<size_t>(sm_count) * tile_rows(max_rows);
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
    p.group = a.heads / a.kv_heads; p.causal = a.causal && a.max_q > 1;
    p.group_inv = p.group == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + p.group - 1) / p.group);
    p.G = sm_count;
    p.tma = a.tma;
    const int max_rows = a.max_q * p.group;
    const size_t rows = 2 * static_cast<size_t>(sm_count) * tile_rows(max_rows);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    p.desc = reinterpret_cast<int*>(ws);
    ws += (static_cast<size_t>(sm_count) * 32 + 255) / 256 * 256;
    p.part_ml = reinterpret_cast<float2*>(ws);
    ws += (rows * sizeof(float2) + 255) / 256 * 256;
    p.part_o = reinterpret_cast<float*>(ws);
    const long long max_kv = static_cast<long long>(a.max_pages) << a.cache.page_shift;
    if (a.head_dim == 64) return run_d<64>(p, a, a.e4m3, max_rows, max_kv, st);
    if (a.head_dim == 128) return run_d<128>(p, a, a.e4m3, max_rows, max_kv, st);
    return run_d<256>(p, a, a.e4m3, max_rows, max_kv, st);
}

}  // namespace rudder
