// Attention over the paged cache for more than 16 rows per key-value head (an action chunk): the same definition, work split and join as
// attention_paged.cu, the products on tcgen05.
//
// With 17 to 128 rows the two products cost 4 rows D operations per key and head: on the register-level path (mma.sync) 64 rows ran at
// 180 TFLOP/s, two thirds of the time in the latency of ldmatrix and mma chains.  Here one thread issues
//     S = Q K^T    128 rows x KT keys,  operands in shared memory,  S in tensor memory (two buffers)
//     O += P V     P read from tensor memory,  V in shared memory as it lies in the cache (its channels are the contiguous axis: the
//                  operand is "MN-major", no transposition anywhere),  O in tensor memory
// and the read of the cache is the bound again.
//
// Warps: 0..3 softmax, a thread per row (no exchange between lanes); 4 issues the MMAs; the others load, half of them K, half V.
//   Loading: 16-byte cp.async per row piece, page by page, straight into the 128-byte-swizzled layout the tensor core reads; keys at or
//     behind the request's length become zeros.  E4M3 goes through registers and becomes f16 (exact; Q as in attention_paged.cu).
//   Softmax: pass 1 takes the maximum of the row's KT scores, pass 2 turns them into probabilities and writes them over the scores they
//     came from: f16, or bf16 hi in the first and lo in the second half of every 32 columns (two products; see attention_paged.cu on the
//     rounding).  The reference the exponent is taken from is raised only when the maximum exceeds it by 2^8: O is rescaled
//     (read, multiplied, written) a few times per item instead of once per tile; sums stay fp32 and exact either way.
//
// Every wait is bounded; a role that gives up records the wait and makes the others leave (see ptx.cuh).
#include "attention_common.cuh"

namespace rudder {

namespace {

enum RowsWhere { W_R_Q_EMPTY = 1001, W_R_KV_EMPTY = 1002, W_R_Q_FULL = 1101, W_R_K_FULL = 1102, W_R_V_FULL = 1103, W_R_P_FULL = 1104, W_R_O_FREE = 1105,
                 W_R_S_FULL = 1201, W_R_PV_DONE = 1202, W_R_DRAIN = 1301 };

template <int D_, bool E4M3_>
struct RowsCfg {
    static constexpr int D = D_;
    static constexpr bool E4M3 = E4M3_;
    static constexpr int ROWS = 128;
    static constexpr int UK = D <= 128 ? 128 : 64;
    static constexpr int KT = UK;                          // keys of a tile: a unit of the work split
    static constexpr int ST = D == 64 ? 4 : (D == 128 ? 3 : 2);
    static constexpr int LW = E4M3 ? 4 : 2;                // loading warps per operand
    static constexpr int THREADS = 32 * (5 + 2 * LW);
    static constexpr int BLK = KT * 128;                   // a tile is D / 64 blocks of [KT keys][64 channels]
    static constexpr int TILE = D / 64 * BLK;
    static constexpr int QBLK = ROWS * 128;
    static constexpr int QBYTES = D / 64 * QBLK;
    static constexpr int SMEM = 1024 + QBYTES + 2 * ST * TILE;
    static constexpr int O_COL = 2 * KT;                   // tensor memory columns: two S / P buffers, O
    static_assert(O_COL + D <= 512 && SMEM <= 226 * 1024, "tensor memory and shared memory");
};

// kind::f16, A and B both f16 or both bf16, fp32 accumulators; b_mn: B with its N axis contiguous.
__device__ __forceinline__ uint32_t umma_idesc_f16(int m, int n, bool bf16, bool b_mn) {
    uint32_t d = 1u << 4;                                  // D format: F32
    if (bf16) d |= (1u << 7) | (1u << 10);                 // A, B formats: BF16 (0 = F16)
    if (b_mn) d |= 1u << 16;
    d |= static_cast<uint32_t>(n >> 3) << 17;
    d |= static_cast<uint32_t>(m >> 4) << 24;
    return d;
}
// N-contiguous operand with the 128-byte swizzle: blocks of 64 N values x 8 K rows of 128 bytes; the next 8 K rows 1024 bytes on, the next
// 64 N values `block` bytes on.
__device__ __forceinline__ uint64_t umma_desc_sw128_mn(uint32_t smem_addr, uint32_t block) {
    uint64_t d = umma_desc_sw128(smem_addr) & ~(0x3FFFull << 16);
    return d | (static_cast<uint64_t>(block >> 4) << 16);
}
__device__ __forceinline__ void umma_f16_ss(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}\n" ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_f16_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}\n" ::"r"(tmem_d), "r"(tmem_a), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
          "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) attention_rows_kernel(const AttnParams p)
{
    constexpr int D = C::D, KT = C::KT, ST = C::ST, LW = C::LW, ROWS = C::ROWS;
    constexpr bool E4M3 = C::E4M3;
    extern __shared__ uint8_t smem_raw_rows[];
    __shared__ __align__(8) uint64_t bars[4 * ST + 8];
    __shared__ float s_fac[ROWS];                          // E4M3: what the row's power of two has to be undone by
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;

    pdl_launch_dependents();
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    Cursor<ROWS, KT> cur;
    if (!start_of_run<ROWS, KT, C::THREADS>(p, cur)) return;

    const uint32_t base = (smem_u32(smem_raw_rows) + 1023u) & ~1023u;
    const uint32_t q_s = base, k_s = base + C::QBYTES, v_s = k_s + ST * C::TILE;
    const uint32_t bar0 = smem_u32(bars);
    auto k_full = [&](int i) { return bar0 + 8u * i; };
    auto k_empty = [&](int i) { return bar0 + 8u * (ST + i); };
    auto v_full = [&](int i) { return bar0 + 8u * (2 * ST + i); };
    auto v_empty = [&](int i) { return bar0 + 8u * (3 * ST + i); };
    auto s_full = [&](int i) { return bar0 + 8u * (4 * ST + i); };
    auto p_full = [&](int i) { return bar0 + 8u * (4 * ST + 2 + i); };
    const uint32_t pv_done = bar0 + 8u * (4 * ST + 4), o_free = pv_done + 8u, q_full = pv_done + 16u, q_empty = pv_done + 24u;
    if (tid == 0) {
        abort_word = 0;
        for (int i = 0; i < ST; ++i) {
            mbar_init(k_full(i), LW); mbar_init(k_empty(i), 1);
            mbar_init(v_full(i), LW); mbar_init(v_empty(i), 1);
        }
        for (int i = 0; i < 2; ++i) { mbar_init(s_full(i), 1); mbar_init(p_full(i), 4); }
        mbar_init(pv_done, 1); mbar_init(o_free, 4);
        mbar_init(q_full, LW); mbar_init(q_empty, 5);      // the last S of the item, and the four softmax warps
        fence_mbar_init();
    }
    if (warp == 4) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_word;
    auto wait_all = [&](uint32_t bar, uint32_t parity, int where) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abortp, where)) != 0; };

    if (warp < 4) {
        // ---------------------------------------------------------------------------------------- softmax and output
        const int row = 32 * warp + lane;
        const uint32_t lanes = static_cast<uint32_t>(32 * warp) << 16;
        const float vs_base = 1.0f;
        int t = 0, item = 0, part_j = 0;
        bool ok = true, fresh = true, first_part = true, live_warp = false, first_tile = false;
        int lim = 0, lim_warp = 0, R = 0, r = 0;
        float f = 0.0f, m = -INFINITY, l = 0.0f;
        while (cur.left > 0) {
            if (fresh) {
                fresh = false;
                first_tile = true;
                part_j = cur.j;
                R = cur.rq.qlen * p.group;
                r = cur.rt * ROWS + row;
                live_warp = cur.rt * ROWS + 32 * warp < R;
                lim = (p.causal && r < R) ? cur.rq.len - cur.rq.qlen + r / p.group + 1 : cur.rq.len;
                lim_warp = __reduce_min_sync(0xffffffffu, lim);
                m = -INFINITY;
                l = 0.0f;
                f = p.scale_log2;
                ok = wait_all(q_full, item & 1, W_R_Q_FULL);
                if (!ok) break;
                if (E4M3) f *= s_fac[row] * (p.cache.k_scale != nullptr ? __ldg(p.cache.k_scale + cur.h) : 1.0f);
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty);
                ++item;
            }
            const int buf = t & 1;
            ok = wait_all(s_full(buf), (t >> 1) & 1, W_R_S_FULL);
            if (!ok) break;
            const bool item_end = cur.j + 1 == cur.nt, ends = item_end || cur.left == 1;
            if (live_warp) {
                tcgen05_fence_after_sync();
                const uint32_t s_t = tmem + lanes + buf * KT;
                const int key0 = cur.j * KT;
                const bool edge = key0 + KT > lim_warp;    // some row of this warp does not see all keys
                // pass 1: the maximum
                float mx = -INFINITY;
#pragma unroll
                for (int c = 0; c < KT / 32; ++c) {
                    uint32_t x[32];
                    tmem_ld_32x32b_x32(s_t + 32 * c, x);
                    tmem_wait_ld();
                    if (edge) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            const float v = __uint_as_float(x[i]) * f;
                            mx = fmaxf(mx, key0 + 32 * c + i < lim ? v : -INFINITY);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) mx = fmaxf(mx, __uint_as_float(x[i]) * f);
                    }
                }
                if (first_tile) {
                    m = mx;
                } else if (__any_sync(0xffffffffu, mx > m + 8.0f)) {
                    // raise the reference: O so far must be complete, then it is rescaled
                    ok = wait_all(pv_done, (t - 1) & 1, W_R_PV_DONE);
                    if (!ok) break;
                    tcgen05_fence_after_sync();
                    const float n = fmaxf(m, mx), cor = n == -INFINITY ? 1.0f : exp2_approx(m - n);
                    m = n;
                    l *= cor;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld_32x32b_x16(tmem + lanes + C::O_COL + 16 * c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * cor);
                        tmem_st_x16(tmem + lanes + C::O_COL + 16 * c, o);
                    }
                    tmem_wait_st();
                }
                const float u = m == -INFINITY ? 0.0f : m;
                // pass 2: probabilities over the scores
#pragma unroll
                for (int c = 0; c < KT / 32; ++c) {
                    uint32_t x[32], hi[16], lo[16];
                    tmem_ld_32x32b_x32(s_t + 32 * c, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float a = exp2_approx(fmaf(__uint_as_float(x[2 * i]), f, -u)), b = exp2_approx(fmaf(__uint_as_float(x[2 * i + 1]), f, -u));
                        if (edge) {
                            if (key0 + 32 * c + 2 * i >= lim) a = 0.0f;
                            if (key0 + 32 * c + 2 * i + 1 >= lim) b = 0.0f;
                        }
                        l += a + b;
                        if (E4M3) {
                            hi[i] = f16x2(a, b);
                        } else {
                            hi[i] = bf16x2(a, b);
                            lo[i] = bf16x2(a - bf16_lo(hi[i]), b - bf16_hi(hi[i]));
                        }
                    }
                    tmem_st_x16(s_t + 32 * c, hi);
                    if (!E4M3) tmem_st_x16(s_t + 32 * c + 16, lo);
                }
                tmem_wait_st();
                tcgen05_fence_before_sync();
            }
            first_tile = false;
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full(buf));
            if (ends) {
                if (live_warp) {
                    ok = wait_all(pv_done, t & 1, W_R_PV_DONE);
                    if (!ok) break;
                    tcgen05_fence_after_sync();
                    const bool entire = item_end && part_j == 0;
                    const float vs = E4M3 && p.cache.v_scale != nullptr ? __ldg(p.cache.v_scale + cur.h) : vs_base;
                    const float w = entire ? (l > 0.0f ? vs / l : 0.0f) : vs;
                    const int slot = 2 * blockIdx.x + (first_part ? 0 : 1);
                    const int tok = r / p.group, hh = cur.h * p.group + r % p.group;
                    uint16_t* orow = p.O + static_cast<size_t>(cur.rq.row0 + tok) * p.ldo + static_cast<size_t>(hh) * D;
                    float* prow = p.part_o + (static_cast<size_t>(slot) * ROWS + row) * D;
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld_32x32b_x16(tmem + lanes + C::O_COL + 16 * c, o);
                        tmem_wait_ld();
                        if (r < R) {
                            float v[16];
#pragma unroll
                            for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(o[i]) * w;
                            if (entire) {
                                *reinterpret_cast<uint4*>(orow + 16 * c) = make_uint4(bf16x2(v[0], v[1]), bf16x2(v[2], v[3]), bf16x2(v[4], v[5]), bf16x2(v[6], v[7]));
                                *reinterpret_cast<uint4*>(orow + 16 * c + 8) =
                                    make_uint4(bf16x2(v[8], v[9]), bf16x2(v[10], v[11]), bf16x2(v[12], v[13]), bf16x2(v[14], v[15]));
                            } else {
#pragma unroll
                                for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(prow + 16 * c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                            }
                        }
                    }
                    if (r < R) {
                        if (!entire) p.part_ml[static_cast<size_t>(slot) * ROWS + row] = make_float2(m, l);
                        else if (p.lse != nullptr)
                            p.lse[static_cast<size_t>(cur.rq.row0 + tok) * p.heads + hh] = l > 0.0f ? (m + log2f(l)) * kLn2 : -INFINITY;
                    }
                    tcgen05_fence_before_sync();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(o_free);
                fresh = true;
                first_part = false;
            }
            ++t;
            cur.advance(p);
        }
    } else if (warp == 4) {
        // ---------------------------------------------------------------------------------------- MMA issue
        const bool leader = elect_one();
        const uint32_t idesc_s = umma_idesc_f16(ROWS, KT, !E4M3, false), idesc_o = umma_idesc_f16(ROWS, D, !E4M3, true);
        int t = 0, item = 0, outs = 0;
        bool ok = true, fresh = true, prev_first = false;
        // O += P V of tile `pt`
        auto pv = [&](int pt, bool first) -> bool {
            const int buf = pt & 1, slot = pt % ST;
            if (!wait_all(p_full(buf), (pt >> 1) & 1, W_R_P_FULL)) return false;
            if (!wait_all(v_full(slot), (pt / ST) & 1, W_R_V_FULL)) return false;
            if (first && outs > 0 && !wait_all(o_free, (outs - 1) & 1, W_R_O_FREE)) return false;     // the item before has been read out
            if (first) ++outs;
            tcgen05_fence_after_sync();
            if (leader) {
                const uint32_t v0 = v_s + slot * C::TILE;
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk) {
                    const uint64_t db = umma_desc_sw128_mn(v0 + kk * 2048, C::BLK);
                    const uint32_t pa = tmem + buf * KT + 32 * (kk >> 1) + 8 * (kk & 1);
                    umma_f16_ts(tmem + C::O_COL, pa, db, idesc_o, (first && kk == 0) ? 0u : 1u);
                    if (!E4M3) umma_f16_ts(tmem + C::O_COL, pa + 16, db, idesc_o, 1u);
                }
                umma_commit(v_empty(slot));
                umma_commit(pv_done);
            }
            __syncwarp();
            return true;
        };
        while (cur.left > 0) {
            const bool first = fresh;
            if (fresh) {
                fresh = false;
                ok = wait_all(q_full, item & 1, W_R_Q_FULL);
                if (!ok) break;
                ++item;
            }
            const bool ends = cur.j + 1 == cur.nt || cur.left == 1;
            const int slot = t % ST;
            ok = wait_all(k_full(slot), (t / ST) & 1, W_R_K_FULL);
            // S goes over the probabilities of two tiles ago: their product must be complete (products into different accumulators are not ordered)
            if (ok && t >= 2) ok = wait_all(pv_done, t & 1, W_R_PV_DONE);
            if (!ok) break;
            tcgen05_fence_after_sync();
            if (leader) {
                const uint32_t k0 = k_s + slot * C::TILE;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_f16_ss(tmem + (t & 1) * KT, umma_desc_sw128(q_s + (ks >> 2) * C::QBLK) + 2u * (ks & 3),
                                umma_desc_sw128(k0 + (ks >> 2) * C::BLK) + 2u * (ks & 3), idesc_s, ks > 0 ? 1u : 0u);
                umma_commit(s_full(t & 1));
                umma_commit(k_empty(slot));
                if (ends) umma_commit(q_empty);
            }
            __syncwarp();
            if (t > 0) {
                ok = pv(t - 1, prev_first);
                if (!ok) break;
            }
            prev_first = first;
            fresh = ends;
            ++t;
            cur.advance(p);
        }
        if (ok && t > 0) pv(t - 1, prev_first);
    } else {
        // ---------------------------------------------------------------------------------------- loading
        const int lw = warp - 5;
        const bool is_v = lw >= LW;
        const int w = is_v ? lw - LW : lw;
        constexpr int RPW = KT / LW;                       // keys of a warp
        static_assert(RPW % 32 == 0 || RPW == 16, "a lane holds the place of whole keys");
        constexpr int OFFS = (RPW + 31) / 32;
        const uint32_t ring = is_v ? v_s : k_s;
        const uint8_t* cache = is_v ? p.cache.v : p.cache.k;
        int t = 0, item = 0, pending = -1;
        bool ok = true, fresh = true;
        auto full = [&](int i) { return is_v ? v_full(i) : k_full(i); };
        // the tile before this one has landed (bf16: its copies are the group before the last)
        auto signal = [&](int slot) {
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(full(slot));
        };
        while (cur.left > 0) {
            const bool ends = cur.j + 1 == cur.nt || cur.left == 1;
            const int slot = t % ST;
            const bool new_item = fresh;
            fresh = ends;
            // places of this warp's keys: lane i of run k holds key w RPW + 32 k + i
            long long off[OFFS];
#pragma unroll
            for (int k = 0; k < OFFS; ++k) {
                const int key = cur.j * KT + w * RPW + 32 * k + lane;
                off[k] = -1;
                if ((RPW >= 32 || lane < RPW) && key < cur.rq.len) {
                    const int page = __ldg(p.table + static_cast<size_t>(cur.b) * p.ld_table + (key >> p.cache.page_shift));
                    if (page < 0 || page >= p.cache.n_pages) record_bad_data(kBadPage);
                    else
                        off[k] = page * p.cache.page_stride + static_cast<long long>(cur.h) * p.cache.head_stride +
                                 static_cast<long long>(key & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride;
                }
            }
            if (!E4M3 && pending >= 0 && !__all_sync(0xffffffffu, mbar_try_wait(is_v ? v_empty(slot) : k_empty(slot), ((t / ST) & 1) ^ 1))) {
                // about to wait for a free stage: hand over what has landed meanwhile
                cp_async_wait<0>();
                signal(pending);
                pending = -1;
            }
            ok = wait_all(is_v ? v_empty(slot) : k_empty(slot), ((t / ST) & 1) ^ 1, W_R_KV_EMPTY);
            if (!ok) break;
            const uint32_t dst = ring + slot * C::TILE;
            if (!E4M3) {
                constexpr int CH = D / 8;                  // 16-byte pieces of a key
                constexpr int STEP = 32 / CH > 0 ? 32 / CH : 1;                  // keys per instruction of the warp (CH = 32: one)
#pragma unroll
                for (int k = 0; k < OFFS; ++k)
#pragma unroll 8
                    for (int i = 0; i < (RPW < 32 ? RPW : 32); i += STEP) {
                        const int rr = i + lane / CH, c = lane % CH;
                        const long long o = __shfl_sync(0xffffffffu, off[k], rr);
                        const int key = w * RPW + 32 * k + rr;
                        cp_async16(dst + (c >> 3) * C::BLK + key * 128 + (((c & 7) ^ (key & 7)) << 4), cache + (o >= 0 ? o : 0) + 16 * c, o >= 0);
                    }
                cp_async_commit();
            } else {
                constexpr int CH = D / 16;                 // 16-byte pieces of a key, 16 numbers each
                constexpr int STEP = 32 / CH;
                constexpr int N = (RPW < 32 ? RPW : 32) / STEP, B = N < 8 ? N : 8;
#pragma unroll
                for (int k = 0; k < OFFS; ++k)
#pragma unroll
                    for (int i0 = 0; i0 < N; i0 += B) {
                        uint4 x[B];
#pragma unroll
                        for (int i = 0; i < B; ++i) {
                            const long long o = __shfl_sync(0xffffffffu, off[k], (i0 + i) * STEP + lane / CH);
                            x[i] = make_uint4(0, 0, 0, 0);
                            if (o >= 0) x[i] = __ldcg(reinterpret_cast<const uint4*>(cache + o + 16 * (lane % CH)));
                        }
#pragma unroll
                        for (int i = 0; i < B; ++i) {
                            const int key = w * RPW + 32 * k + (i0 + i) * STEP + lane / CH, c = 2 * (lane % CH);
                            uint32_t h[8];
                            e4m3_to_f16(x[i].x, h[0], h[1]); e4m3_to_f16(x[i].y, h[2], h[3]);
                            e4m3_to_f16(x[i].z, h[4], h[5]); e4m3_to_f16(x[i].w, h[6], h[7]);
                            const uint32_t at = dst + (c >> 3) * C::BLK + key * 128;
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + (((c & 7) ^ (key & 7)) << 4)), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + ((((c & 7) + 1) ^ (key & 7)) << 4)), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
                        }
                    }
            }
            if (new_item && !is_v) {
                // the item's queries, rows w 128 / LW .. of the tile; rows that do not exist become zeros.  The item before must be through its
                // last S: hand its last tile over first.
                if (pending >= 0) {
                    cp_async_wait<1>();
                    signal(pending);
                    pending = -1;
                }
                if (item > 0) {
                    ok = wait_all(q_empty, (item - 1) & 1, W_R_Q_EMPTY);
                    if (!ok) break;
                }
                ++item;
                constexpr int QR = ROWS / LW;
                const int R = cur.rq.qlen * p.group;
                constexpr int CH = D / 8, STEP = 32 / CH;
#pragma unroll 4
                for (int i = 0; i < QR; i += STEP) {
                    const int rl = w * QR + i + lane / CH, c = lane % CH, r = cur.rt * ROWS + rl;
                    const bool live = r < R;
                    const uint16_t* src = p.Q + 8 * c;
                    if (live) src += static_cast<size_t>(cur.rq.row0 + r / p.group) * p.ldq + static_cast<size_t>(cur.h * p.group + r % p.group) * D;
                    const uint32_t at = q_s + (c >> 3) * C::QBLK + rl * 128 + (((c & 7) ^ (rl & 7)) << 4);
                    if (!E4M3) {
                        cp_async16(at, src, live);
                    } else {
                        uint4 x = make_uint4(0, 0, 0, 0);
                        if (live) x = *reinterpret_cast<const uint4*>(src);
                        const uint32_t xw[4] = {x.x, x.y, x.z, x.w};
                        float mx = 0.0f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, fmaxf(fabsf(bf16_lo(xw[e])), fabsf(bf16_hi(xw[e]))));
#pragma unroll
                        for (int o = CH / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                        const int ex = min(126, max(-126, 14 - (static_cast<int>((__float_as_uint(mx) >> 23) & 255u) - 127)));
                        const float sc = __uint_as_float(static_cast<uint32_t>(ex + 127) << 23);
                        uint32_t h[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) h[e] = f16x2(bf16_lo(xw[e]) * sc, bf16_hi(xw[e]) * sc);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
                        if (c == 0) s_fac[rl] = __uint_as_float(static_cast<uint32_t>(127 - ex) << 23);
                    }
                }
                if (!E4M3) {
                    cp_async_commit();
                    cp_async_wait<0>();                    // queries and this tile together
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(q_full);
                if (!E4M3) signal(slot);
            } else if (!E4M3) {
                if (pending >= 0) {
                    cp_async_wait<1>();
                    signal(pending);
                }
                pending = slot;
            }
            if (E4M3) signal(slot);
            ++t;
            cur.advance(p);
        }
        if (!E4M3) {
            cp_async_wait<0>();
            if (ok && pending >= 0) signal(pending);
        }
    }

    // ---- teardown: no MMA of this CTA is in flight when its tensor memory goes (the softmax warps have waited for the last product; after an
    // aborted wait the issuing thread waits for its own, bounded)
    if (warp == 4 && abort_word != 0) {
        if (elect_one()) umma_commit(pv_done);
        for (uint32_t it = 0; it < (1u << 14); ++it) { __nanosleep(100); if (abort_word == 0) break; }
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == 4) {
        __syncwarp();
        tcgen05_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

template <class C>
cudaError_t launch_rows(const AttnParams& p, cudaStream_t st)
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
    return cudaLaunchKernelEx(&cfg, attention_rows_kernel<C>, p);
}
template <class C>
cudaError_t init_rows() { return cudaFuncSetAttribute(attention_rows_kernel<C>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM); }

}  // namespace

}  // namespace rudder
