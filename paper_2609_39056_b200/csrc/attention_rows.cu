// Attention over the paged cache for many rows per key-value head (an action chunk; from 17 or 33 on, see many_rows): the same definition, work split and join as
// attention_paged.cu, the products on tcgen05.
//
// The two products cost 4 rows D operations per key and head: on the register-level path (mma.sync) 64 rows x 4 x 126k keys took 429 us
// (156 TFLOP/s), two thirds of it the latency of ldmatrix and mma chains.  Here one thread issues
//     S = Q K^T    128 rows x KT keys,  operands in shared memory,  S in tensor memory (two buffers)
//     O += P V     P read from tensor memory,  V in shared memory as it lies in the cache (its channels are the contiguous axis: the
//                  operand is "MN-major", no transposition anywhere),  O in tensor memory
// The same case takes 205 to 220 us, 128 rows run at 565 to 590 TFLOP/s.  No pipe is full (64 rows x 4 x 30k keys: tensor 39 %, DRAM 42 %, issue slots 27 %,
// exponentials 13 %): what bounds it is the chain of a tile, scores -> tensor memory -> softmax, a thread per row -> P -> product, with two tiles in hand.
// E4M3 295 us (64 rows x 4 x 30k keys 92 us; converted by the warps that also fetched it 111 us): tensor 18 %, issue slots 22 %, exponentials 9 %; the conversion adds a
// step in front of that chain (shared memory -> registers -> shared memory, fence, barrier) with two stages to cover it.
//
// Warps: two sets of four softmax warps that take half of a tile's keys each, a thread per row (no exchange between lanes; one set for D = 256), each
// set with its own reference, sum and O; then one warp that issues the MMAs; three load (E4M3: four convert, one more loads).
//   Loading: 16-byte cp.async per row piece, page by page, straight into the 128-byte-swizzled layout the tensor core reads; keys at or
//     behind the request's length become zeros.  Whole tiles in pages of 8 tokens or more come by TMA instead; E4M3 as it lies in the cache into a
//     ring of its own, from where the loading warps convert it to f16 (exact; Q as in attention_paged.cu).
//   Softmax: pass 1 takes the maximum of the row's KT scores, pass 2 turns them into probabilities and writes them over the scores they
//     came from: f16, or bf16 hi in the first and lo in the second half of every 32 columns (two products; see attention_paged.cu on the
//     rounding).  The reference the exponent is taken from is raised only when the maximum has grown by a factor of 2^8 (E4M3: 2^4): O is
//     rescaled (read, multiplied, written) a few times per item instead of once per tile; sums stay fp32 either way.  With E4M3 it lies 2^11 below the
//     maximum, so that f16 holds probabilities down to 2^-25 of the largest with all its bits (2^8 and 2^-21 took 0.3 % less time).
//   At the end of an item the first set adds the two O (in that order) and writes the rows or the part.
//
// Every wait is bounded; a role that gives up records the wait and makes the others leave (see ptx.cuh).
#include "attention_common.cuh"

namespace rudder {

namespace {

enum RowsWhere { W_R_Q_EMPTY = 1001, W_R_KV_EMPTY = 1002, W_R_RAW_FULL = 1003, W_R_RAW_EMPTY = 1004, W_R_Q_FULL = 1101, W_R_KV_FULL = 1102, W_R_P_FULL = 1104, W_R_O_FREE = 1105,
                 W_R_S_FULL = 1201, W_R_PV_DONE = 1202, W_R_ML_FULL = 1203 };

// PAIR: two tiles of 128 rows over the same keys, a set of softmax warps for each (prefixes that many rows share).
template <int D_, bool E4M3_, bool PAIR_ = false>
struct RowsCfg {
    static constexpr int D = D_;
    static constexpr bool E4M3 = E4M3_, PAIR = PAIR_;
    static constexpr int ROWS = PAIR ? 256 : 128;
    static constexpr int UK = D <= 128 ? 128 : 64;
    static constexpr int KT = UK;                          // keys of a tile: a unit of the work split
    static constexpr int ST = D == 64 ? 4 : (D == 128 && !E4M3 && !PAIR ? 3 : 2);
    static constexpr int SETS = D <= 128 ? 2 : 1;          // sets of four softmax warps: each takes its share of a tile's keys, with an O of its own
    static constexpr int HALF = PAIR ? KT : KT / SETS;     // keys of a tile that a set takes
    static constexpr int LW = E4M3 ? 4 : 3;                // loading warps (12 warps in all: 168 registers a thread),
    static constexpr int TW = E4M3 ? 1 : 0;                // with E4M3 they convert, and one more issues the TMA loads (14 warps: 144)
    // The reference is the maximum less TOP when it is taken and is raised when the maximum less TOP exceeds it by RAISE: probabilities up to 2^(TOP + RAISE),
    // for E4M3 as high in f16 as they can be (see attention_paged.cu on the rounding)
    static constexpr float RAISE = E4M3 ? 4.0f : 8.0f, TOP = E4M3 ? 15.0f - RAISE : 0.0f;
    static constexpr int QW = 2;                           // of them, those that load the queries (the first issues the TMA loads and waits for nothing else)
    static constexpr int MMA_WARP = 4 * SETS;
    static constexpr int THREADS = 32 * (MMA_WARP + 1 + LW + TW);
    static constexpr int BLK = KT * 128;                   // a tile is D / 64 blocks of [KT keys][64 channels]
    static constexpr int TILE = D / 64 * BLK;
    static constexpr int QBLK = ROWS * 128;
    static constexpr int QBYTES = D / 64 * QBLK;
    static constexpr int RAW = KT * D;                     // E4M3: a K or a V tile as it lies in the cache,
    static constexpr int RU = E4M3 ? (D == 64 ? 8 : (D == 128 && !PAIR ? 4 : 2)) : 0;     // and how many of them are on their way
    static constexpr int SMEM = 1024 + QBYTES + 2 * ST * TILE + RU * RAW;
    static constexpr int O_COL = 2 * KT;                   // tensor memory columns: two S / P buffers, O
    static_assert(!PAIR || SETS == 2, "a set of softmax warps for each tile of rows");
    static_assert(O_COL + SETS * D <= 512 && SMEM <= 226 * 1024, "tensor memory and shared memory");
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
__device__ __forceinline__ void tmem_st_x32(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
          "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
          "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st_x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
          "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Tiled load of [rows of a page][64 channels] of one head, 128-byte swizzle: coordinates channel, token of the page, head, page.
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, int w, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
                 : "memory");
}
// Sixteen E4M3 numbers as two pieces of eight f16 numbers in shared memory.
__device__ __forceinline__ void store_f16(uint32_t at0, uint32_t at1, uint4 v) {
    uint32_t h[8];
    e4m3_to_f16(v.x, h[0], h[1]); e4m3_to_f16(v.y, h[2], h[3]);
    e4m3_to_f16(v.z, h[4], h[5]); e4m3_to_f16(v.w, h[6], h[7]);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at0), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at1), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
}

// Two 32-bit numbers in one register pair: arithmetic on both at the price of one instruction, each rounded on its own.
__device__ __forceinline__ uint64_t pair(uint32_t a, uint32_t b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint64_t pair(float a, float b) { return pair(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ float2 unpair(uint64_t x) {
    uint32_t a, b;
    asm("mov.b64 {%0, %1}, %2;" : "=r"(a), "=r"(b) : "l"(x));
    return make_float2(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t exp2_pair(uint64_t x) {
    const float2 v = unpair(x);
    return pair(exp2_approx(v.x), exp2_approx(v.y));
}
// Two probabilities as bf16 hi + lo without a conversion instruction: those share a pipe of a sixteenth of a warp per clock with the exponentials, and that pipe bounded
// this pass (64 probabilities a thread 2300 -> 1500 clocks).  x (2^16 + 1) - (x (2^16 + 1) - x) is x rounded to 8 bits (Dekker's splitting, Numer. Math. 18, 1971), what is
// left is exact, and the upper half of its bits plus half a step is its bf16 number: |x - hi - lo| <= 2^-17 x.  (Cut off instead it is 2^-16: 32 requests of 16 rows x
// 16 heads over 4416 shared tokens 68.0 instead of 68.3 us, D = 64 43.0 instead of 44.3.)
__device__ __forceinline__ void split_bf16(uint64_t x, uint32_t& hi, uint32_t& lo) {
    const uint64_t neg = pair(-1.0f, -1.0f);
    const uint64_t c = mul2(x, pair(65537.0f, 65537.0f));
    const uint64_t d = fma2(x, neg, c);                    // c - x
    const uint64_t h = fma2(d, neg, c), l = fma2(h, neg, x);
    const float2 hv = unpair(h), lv = unpair(l);
    hi = __byte_perm(__float_as_uint(hv.x), __float_as_uint(hv.y), 0x7632);
    lo = __byte_perm(__float_as_uint(lv.x) + 0x8000u, __float_as_uint(lv.y) + 0x8000u, 0x7632);
}

template <class C, bool SHARED>
__global__ void __launch_bounds__(C::THREADS, 1) attention_rows_kernel(const ParamsOf<SHARED> p, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v)
{
    constexpr int D = C::D, KT = C::KT, ST = C::ST, RU = C::RU, LW = C::LW, ROWS = C::ROWS, SETS = C::SETS, HALF = C::HALF, MMA_WARP = C::MMA_WARP;
    constexpr bool E4M3 = C::E4M3;
    extern __shared__ uint8_t smem_raw_rows[];
    __shared__ __align__(8) uint64_t bars[2 * ST + 12 + 2 * C::RU];
    __shared__ float2 s_ml[C::PAIR ? 1 : ROWS];                          // (reference, sum) of the second set's rows
    __shared__ int8_t s_exp[E4M3 ? ROWS : 1];              // E4M3: the power of two that a row of Q was multiplied by
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word;
    __shared__ int s_dropped[2];                           // [item & 1]: the item, if values were dropped (see drop_nonfinite)

    start_pass(p);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    using Cur = Cursor<ROWS, KT, SHARED>;
    Cur cur;
    if (!start_of_run<ROWS, KT, C::THREADS, SHARED>(p, cur)) {
        if (SHARED) pdl_wait();
        return;
    }

    const uint32_t base = (smem_u32(smem_raw_rows) + 1023u) & ~1023u;
    const uint32_t q_s = base, k_s = base + C::QBYTES, v_s = k_s + ST * C::TILE;
    const uint32_t bar0 = smem_u32(bars);
    auto kv_full = [&](int i) { return bar0 + 8u * i; };
    auto kv_empty = [&](int i) { return bar0 + 8u * (ST + i); };
    auto s_full = [&](int i) { return bar0 + 8u * (2 * ST + i); };
    auto p_full = [&](int buf, int set) { return bar0 + 8u * (2 * ST + 2 + buf + 2 * set); };
    auto pv_done = [&](int set) { return bar0 + 8u * (2 * ST + 6 + set); };
    const uint32_t ml_full = bar0 + 8u * (2 * ST + 8), o_free = ml_full + 8u,                 // (PAIR: the first is the second set's o_free)
                    q_full = ml_full + 16u, q_empty = ml_full + 24u;
    const uint32_t raw_s = v_s + ST * C::TILE;
    auto raw_full = [&](int i) { return bar0 + 8u * (2 * ST + 12 + i); };
    auto raw_empty = [&](int i) { return bar0 + 8u * (2 * ST + 12 + RU + i); };
    // an item's queries, two warps (PAIR: for the first item all warps) their share each of the rows that exist (the others never matter)
    auto load_queries = [&](int part, int parts) {
                        const int rows_here = min(ROWS, cur.rq.qlen * p.group - cur.rt * ROWS);
                        constexpr int QCH = D / 8, QSTEP = 32 / QCH;
#pragma unroll 4
                        for (int i = part * QSTEP; i < rows_here; i += parts * QSTEP) {
                            const int rl = i + lane / QCH, qc = lane % QCH, r = cur.rt * ROWS + rl;
                            const bool live = rl < rows_here;
                            const uint16_t* src = p.Q + 8 * qc;
                            const RowOf qa = row_of(p, r);
                            if (live) src += static_cast<size_t>(cur.rq.row0 + qa.token) * p.ldq + static_cast<size_t>(cur.h * p.group + qa.head) * D;
                            const uint32_t at = q_s + (qc >> 3) * C::QBLK + rl * 128 + (((qc & 7) ^ (rl & 7)) << 4);
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
                                for (int o = QCH / 2; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                                const int ex = min(126, max(-126, 14 - (static_cast<int>((__float_as_uint(mx) >> 23) & 255u) - 127)));
                                const float sc = __uint_as_float(static_cast<uint32_t>(ex + 127) << 23);
                                uint32_t h[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e) h[e] = f16x2(bf16_lo(xw[e]) * sc, bf16_hi(xw[e]) * sc);
                                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
                                if (qc == 0) s_exp[rl] = static_cast<int8_t>(ex);
                            }
                        }
    };
    if (C::PAIR) load_queries(warp, C::THREADS / 32);      // (256 rows by two warps take 3 us)
    else if (warp > MMA_WARP + LW - C::QW && warp <= MMA_WARP + LW) load_queries(warp - 1 - MMA_WARP - (LW - C::QW), C::QW);
    if (tid == 0) {
        abort_word = 0;
        s_dropped[0] = s_dropped[1] = -1;
        for (int i = 0; i < ST; ++i) { mbar_init(kv_full(i), LW); mbar_init(kv_empty(i), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(s_full(i), 1); mbar_init(p_full(i, 0), 4); mbar_init(p_full(i, 1), 4); mbar_init(pv_done(i), 1); }
        mbar_init(ml_full, 4); mbar_init(o_free, 4);
        for (int i = 0; i < RU; ++i) { mbar_init(raw_full(i), 1); mbar_init(raw_empty(i), LW); }
        mbar_init(q_full, C::QW); mbar_init(q_empty, 1 + 4 * SETS);                 // the last S of the item, and the softmax warps
        fence_mbar_init();
    }
    if (warp == MMA_WARP) {
        tmem_alloc(smem_u32(&tmem_slot), 512);
        tmem_relinquish();
    }
    if (C::PAIR) {
        // the first item's queries, visible to the tensor core (the loading warps say so below)
        if (!E4M3) asm volatile("cp.async.wait_all;" ::: "memory");
        fence_proxy_async_smem();
        __syncwarp();
    }
    tcgen05_fence_before_sync();
    __syncthreads();
    tcgen05_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    volatile int* abortp = &abort_word;
    auto wait_all = [&](uint32_t bar, uint32_t parity, int where) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abortp, where)) != 0; };

    if (C::PAIR && warp < MMA_WARP) {
        // ---------------------------------------------------------------------------------------- softmax and output, a set of warps for each tile of rows
        // Rows of shared prefixes: each sees every key of its item.  A set has its own scores, probabilities (over them), O and counts of what it did; the two run at
        // their own pace, so that the products of one fall under the softmax of the other.  In one tile of rows the two sets wait for the same products:
        // 16 heads x 512 rows x 4416 keys 56 -> 48 us (a tile of 256 rows x 128 keys
        // 5700 clocks, one of 128 rows 3600; of the 48 us 14 are the start: place of the run, queries, and code that comes from L2 for the first time).  Tried without gain:
        // issuing whatever product is ready by polling (8200 clocks a tile); one pass with the maximum checked 32 keys at a time (52 us).
        const int set = warp >> 2, quad = warp & 3;
        const int row = 128 * set + 32 * quad + lane;
        const uint32_t lanes = static_cast<uint32_t>(32 * quad) << 16;
        const uint32_t s_t = tmem + lanes + set * KT, o_t = tmem + lanes + C::O_COL + set * D, done = set == 0 ? o_free : ml_full;
        int t = 0, item = 0, part_j = 0, R = 0, r = 0;
        bool ok = true, fresh = true, first_part = true, active = false, live_warp = false, first_tile = false;
        float f = 0.0f, m = -INFINITY, l = 0.0f;
        while (cur.left > 0) {
            if (fresh) {
                fresh = false;
                first_tile = true;
                part_j = cur.j;
                R = cur.rq.qlen * p.group;
                r = cur.rt * ROWS + row;
                active = cur.rt * ROWS + 128 * set < R;
                live_warp = cur.rt * ROWS + 128 * set + 32 * quad < R;
                m = -INFINITY;
                l = 0.0f;
                f = r < R ? p.scale_log2 : 0.0f;           // rows that do not exist hold whatever the buffer held: nothing is read from them
                ok = wait_all(q_full, item & 1, W_R_Q_FULL);
                if (!ok) break;
                if (E4M3 && r < R) f *= __uint_as_float(static_cast<uint32_t>(127 - s_exp[row]) << 23) * (p.cache.k_scale != nullptr ? p.cache.k_scale[cur.h] : 1.0f);
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty);
                ++item;
            }
            const bool item_end = cur.j + 1 == cur.nt, ends = item_end || cur.left == 1;
            if (active) {
                ok = wait_all(s_full(set), t & 1, W_R_S_FULL);
                if (!ok) break;
                if (live_warp) {
                    tcgen05_fence_after_sync();            // (the product before is complete, too: these scores lie over its probabilities)
                    const int live = cur.rq.len - cur.j * KT;                      // keys of the tile that there are
                    const bool edge = live < KT;
                    const float gone = f < 0.0f ? INFINITY : -INFINITY;
                    float fs = f;
                    if (edge && f == 0.0f) fs = 1.0f;      // (a factor of zero makes no -infinity: scores of zero with a factor of one)
                    uint32_t x[32];
                    auto load = [&](int c, uint32_t (&to)[32]) { tmem_ld_32x32b_x32(s_t + 32 * c, to); };
                    auto cut = [&](int c, uint32_t (&to)[32]) {
                        if (edge) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) to[i] = 32 * c + i < live ? (f == 0.0f ? 0u : to[i]) : __float_as_uint(gone);
                        }
                    };
                    float q[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    auto most = [&](const uint32_t (&v)[32]) {
                        if (f >= 0.0f) {
#pragma unroll
                            for (int i = 0; i < 32; i += 2) q[(i >> 1) & 3] = fmaxf(q[(i >> 1) & 3], fmaxf(__uint_as_float(v[i]), __uint_as_float(v[i + 1])));
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i) q[i & 3] = fmaxf(q[i & 3], -__uint_as_float(v[i]));
                        }
                    };
                    // pass 1: the maximum of s f
#pragma unroll 1                                           // (four times the code costs more at the start, instruction by instruction from L2, than it saves later)
                    for (int c = 0; c < KT / 32; ++c) {
                        load(c, x);
                        tmem_wait_ld();
                        cut(c, x);
                        most(x);
                    }
                    float mx = fmaxf(fmaxf(q[0], q[1]), fmaxf(q[2], q[3]));
                    mx = mx == -INFINITY ? mx : mx * fabsf(f) - C::TOP;
                    __syncwarp();
                    if (first_tile) {
                        m = mx;
                    } else if (__any_sync(0xffffffffu, r < R && mx > m + C::RAISE)) {
                        const float n = mx > m + C::RAISE ? mx : m;
                        const float cor = n == -INFINITY ? 1.0f : exp2_approx(m - n);
                        m = n;
                        l *= cor;
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            tmem_ld_32x32b_x16(o_t + 16 * c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * cor);
                            tmem_st_x16(o_t + 16 * c, o);
                        }
                        tmem_wait_st();
                    }
                    // pass 2: probabilities over the scores they come from
                    const float u = m == -INFINITY ? 0.0f : m;
                    uint64_t l01 = 0;
                    auto weigh = [&](int c, const uint32_t (&v)[32]) {
                        uint32_t w[32];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint64_t e = exp2_pair(fma2(pair(v[2 * i], v[2 * i + 1]), pair(fs, fs), pair(-u, -u)));
                            l01 = add2(l01, e);
                            if (E4M3) {
                                const float2 z = unpair(e);
                                w[i] = f16x2(z.x, z.y);
                            } else {
                                split_bf16(e, w[i], w[16 + i]);
                            }
                        }
                        __syncwarp();
                        if (E4M3) tmem_st_x16(s_t + 32 * c, reinterpret_cast<const uint32_t (&)[16]>(w));
                        else tmem_st_x32(s_t + 32 * c, w);
                    };
#pragma unroll 1
                    for (int c = 0; c < KT / 32; ++c) {
                        load(c, x);
                        tmem_wait_ld();
                        cut(c, x);
                        weigh(c, x);
                    }
                    const float2 z = unpair(l01);
                    l += z.x + z.y;
                    tmem_wait_st();
                    tcgen05_fence_before_sync();
                }
                first_tile = false;
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(0, set));
                ++t;
                if (ends) {
                    ok = wait_all(pv_done(set), (t - 1) & 1, W_R_PV_DONE);
                    if (!ok) break;
                    if (live_warp) {
                        tcgen05_fence_after_sync();
                        const bool entire = item_end && part_j == 0;
                        const float vs = E4M3 && p.cache.v_scale != nullptr ? p.cache.v_scale[cur.h] : 1.0f;
                        const int slot = 2 * blockIdx.x + (first_part ? 0 : 1);
                        float* out = p.part_o + static_cast<size_t>(slot) * ROWS * D + 4 * row;                  // [channels / 4][rows][4]: coalesced
                        int step = 4 * ROWS;
                        if constexpr (SHARED) {
                            if (entire && r < R) {
                                out = p.sh.base_o + prefix_row(p, cur.rq.row0, cur.h, r) * D;
                                step = 4;
                            }
                        }
                        __syncwarp();
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t o[32];
                            tmem_ld_32x32b_x32(o_t + 32 * c, o);
                            tmem_wait_ld();
                            if (r < R) {
#pragma unroll
                                for (int i = 0; i < 32; i += 4)
                                    *reinterpret_cast<float4*>(out + (8 * c + i / 4) * step) = make_float4(__uint_as_float(o[i]) * vs, __uint_as_float(o[i + 1]) * vs,
                                                                                                         __uint_as_float(o[i + 2]) * vs, __uint_as_float(o[i + 3]) * vs);
                            }
                            __syncwarp();
                        }
                        if (r < R) {
                            if (!entire) p.part_ml[static_cast<size_t>(slot) * ROWS + row] = make_float2(m, l);
                            else store_prefix_ml(p, cur.rq.row0, cur.h, r, m, l);
                        }
                        tcgen05_fence_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(done);
                }
            }
            if (ends) {
                fresh = true;
                first_part = false;
            }
            cur.advance(p);
        }
    } else if (C::PAIR && warp == MMA_WARP) {
        // ---------------------------------------------------------------------------------------- MMA issue for a pair: first set, second set, in turn
        const bool leader = elect_one();
        const uint32_t idesc_s = umma_idesc_f16(128, KT, !E4M3, false), idesc_o = umma_idesc_f16(128, D, !E4M3, true);
        // Bit `set` of each: whether scores were issued for the set, and whether an odd number of them; the same of its items.  (Not arrays: both products stand in a
        // loop over the sets, once each, because code that runs for the first time comes instruction by instruction from L2.)
        uint32_t scored = 0, scored_odd = 0, begun = 0, begun_odd = 0, read_out = 0;
        int t = 0, item = 0;
        bool ok = true;
        // scores of tile `of`, over the probabilities of the set's tile before: its product must be complete (products into different accumulators are not ordered)
        auto scores = [&](int set, int of) -> bool {
            if (!wait_all(kv_full(of % ST), (of / ST) & 1, W_R_KV_FULL)) return false;
            if ((scored >> set & 1) && !wait_all(pv_done(set), scored_odd >> set & 1 ^ 1, W_R_PV_DONE)) return false;
            tcgen05_fence_after_sync();
            if (leader) {
                const uint32_t k0 = k_s + (of % ST) * C::TILE, q0 = q_s + set * 128 * 128;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_f16_ss(tmem + set * KT, umma_desc_sw128(q0 + (ks >> 2) * C::QBLK) + 2u * (ks & 3), umma_desc_sw128(k0 + (ks >> 2) * C::BLK) + 2u * (ks & 3), idesc_s,
                                ks > 0 ? 1u : 0u);
                umma_commit(s_full(set));
            }
            __syncwarp();
            scored |= 1u << set;
            scored_odd ^= 1u << set;
            return true;
        };
        // O += P V of tile `of`; the item's first product starts its O, once the set's item before has been read out
        auto product = [&](int set, int of, bool first, bool last_user) -> bool {
            if (!wait_all(p_full(0, set), scored_odd >> set & 1 ^ 1, W_R_P_FULL)) return false;
            if (first && (read_out >> set & 1) && !wait_all(set == 0 ? o_free : ml_full, begun_odd >> set & 1, W_R_O_FREE)) return false;
            tcgen05_fence_after_sync();
            if (leader) {
                const uint32_t v0 = v_s + (of % ST) * C::TILE, o = tmem + C::O_COL + set * D;
#pragma unroll
                for (int kk = 0; kk < KT / 16; ++kk) {
                    const uint64_t db = umma_desc_sw128_mn(v0 + kk * 2048, C::BLK);
                    const uint32_t pa = tmem + set * KT + 32 * (kk >> 1) + 8 * (kk & 1);
                    umma_f16_ts(o, pa, db, idesc_o, (first && kk == 0) ? 0u : 1u);
                    if (!E4M3) umma_f16_ts(o, pa + 16, db, idesc_o, 1u);
                }
                umma_commit(pv_done(set));
                if (last_user) umma_commit(kv_empty(of % ST));
            }
            __syncwarp();
            return true;
        };
        auto last_of_item = [&]() { return cur.j + 1 == cur.nt || cur.left == 1; };
        auto second_has_rows = [&]() { return cur.rt * ROWS + 128 < cur.rq.qlen * p.group; };
        while (ok && cur.left > 0) {
            // an item: its first scores, then tile by tile product and the next scores, set by set
            const uint32_t sets = second_has_rows() ? 3 : 1;
            ok = wait_all(q_full, item & 1, W_R_Q_FULL);
            ++item;
            read_out = begun;                              // (of an earlier item)
            begun |= sets;
            begun_odd ^= sets;
            bool ends = false;
            for (int k = -1; ok; ++k) {
                const bool next = k < 0 || !ends, next_ends = next && last_of_item();
#pragma unroll 1
                for (int set = 0; ok && (sets >> set) != 0; ++set) {
                    if (k >= 0) ok = product(set, t, k == 0, (sets >> set) == 1);
                    if (ok && next) ok = scores(set, k < 0 ? t : t + 1);
                }
                if (ok && next_ends && leader) umma_commit(q_empty);
                __syncwarp();
                if (k >= 0) {
                    ++t;
                    if (ends) break;
                }
                ends = next_ends;
                cur.advance(p);
            }
        }
    } else if (warp < MMA_WARP) {
        // ---------------------------------------------------------------------------------------- softmax and output
        const int set = warp >> 2, quad = warp & 3;
        const int row = 32 * quad + lane;
        const uint32_t lanes = static_cast<uint32_t>(32 * quad) << 16;
        const uint32_t o_t = tmem + lanes + C::O_COL;
        int t = 0, item = 0, part_j = 0;
        bool ok = true, fresh = true, first_part = true, live_warp = false, first_tile = false;
        int lim = 0, lim_warp = 0, R = 0, r = 0, tail = 0;
        float f = 0.0f, m = -INFINITY, l = 0.0f;
        while (cur.left > 0) {
            if (fresh) {
                fresh = false;
                first_tile = true;
                part_j = cur.j;
                R = cur.rq.qlen * p.group;
                r = cur.rt * ROWS + row;
                live_warp = cur.rt * ROWS + 32 * quad < R;
                lim = (p.causal && r < R) ? cur.rq.len - cur.rq.qlen + row_of(p, r).token + 1 : cur.rq.len;
                lim_warp = __reduce_min_sync(0xffffffffu, lim);
                tail = p.causal ? tail_of(cur.rq.len, cur.rq.qlen, row_of(p, cur.rt * ROWS).token) : cur.rq.len;
                m = -INFINITY;
                l = 0.0f;
                f = r < R ? p.scale_log2 : 0.0f;           // rows that do not exist hold whatever the buffer held: weight 0, nothing read from them
                ok = wait_all(q_full, item & 1, W_R_Q_FULL);
                if (!ok) break;
                if (E4M3 && r < R) f *= __uint_as_float(static_cast<uint32_t>(127 - s_exp[row]) << 23) * (p.cache.k_scale != nullptr ? p.cache.k_scale[cur.h] : 1.0f);
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty);
                ++item;
            }
            const int buf = t & 1;
            const bool item_end = cur.j + 1 == cur.nt, ends = item_end || cur.left == 1;
            ok = wait_all(s_full(buf), (t >> 1) & 1, W_R_S_FULL);
            if (!ok) break;
            {
                if (live_warp) {
                    tcgen05_fence_after_sync();
                    const uint32_t s_t = tmem + lanes + buf * KT + set * HALF;
                    const int key0 = cur.j * KT + set * HALF;
                    const bool edge = key0 + HALF > lim_warp;                      // some row of this warp does not see all keys
                    // pass 1: the maximum of s f
                    uint32_t x[HALF / 32][32];
#pragma unroll
                    for (int c = 0; c < HALF / 32; ++c) tmem_ld_32x32b_x32(s_t + 32 * c, x[c]);
                    tmem_wait_ld();
                    float fs = f;
                    if (edge) {
                        const uint32_t gone = __float_as_uint(f < 0.0f ? INFINITY : -INFINITY);
#pragma unroll
                        for (int c = 0; c < HALF / 32; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i) x[c][i] = key0 + 32 * c + i < lim ? (SHARED && f == 0.0f ? 0u : x[c][i]) : gone;
                        // (a factor of zero, which makes no -infinity of a key that is not seen: scores of zero instead, with a factor of one)
                        if (SHARED && f == 0.0f) fs = 1.0f;
                    }
                    float mx;
                    {
                        float q[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                        if (f >= 0.0f) {
#pragma unroll
                            for (int c = 0; c < HALF / 32; ++c)
#pragma unroll
                                for (int i = 0; i < 32; i += 2) q[(i >> 1) & 3] = fmaxf(q[(i >> 1) & 3], fmaxf(__uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1])));
                        } else {
#pragma unroll
                            for (int c = 0; c < HALF / 32; ++c)
#pragma unroll
                                for (int i = 0; i < 32; ++i) q[i & 3] = fmaxf(q[i & 3], -__uint_as_float(x[c][i]));
                        }
                        mx = fmaxf(fmaxf(q[0], q[1]), fmaxf(q[2], q[3]));
                        mx = mx == -INFINITY ? mx : mx * fabsf(f) - C::TOP;      // (no key seen stays -inf whatever f is)
                    }
                    __syncwarp();                          // (the tensor memory instructions below want the whole warp together)
                    if (first_tile) {
                        m = mx;
                    } else if (__any_sync(0xffffffffu, r < R && mx > m + C::RAISE)) {
                        // raise the reference: O so far must be complete, then it is rescaled
                        ok = wait_all(pv_done(set), (t - 1) & 1, W_R_PV_DONE);
                        if (!ok) break;
                        tcgen05_fence_after_sync();
                        const float n = mx > m + C::RAISE ? mx : m;                // (row by row: what a row becomes does not depend on its neighbours)
                        const float cor = n == -INFINITY ? 1.0f : exp2_approx(m - n);
                        m = n;
                        l *= cor;
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {                       // (rare: small code before speed)
                            uint32_t o[16];
                            tmem_ld_32x32b_x16(o_t + set * D + 16 * c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * cor);
                            tmem_st_x16(o_t + set * D + 16 * c, o);
                        }
                        tmem_wait_st();
                    }
                    // pass 2: probabilities over the scores they come from
                    const float u = m == -INFINITY ? 0.0f : m;
                    float l0 = 0.0f, l1 = 0.0f;
                    uint64_t l01 = 0;                      // two zeros
#pragma unroll
                    for (int c = 0; c < HALF / 32; ++c) {
                        uint32_t w[32];                    // hi (or f16) in the first half, lo in the second
                        if constexpr (SHARED && !E4M3) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const uint64_t e = exp2_pair(fma2(pair(x[c][2 * i], x[c][2 * i + 1]), pair(fs, fs), pair(-u, -u)));
                                l01 = add2(l01, e);
                                split_bf16(e, w[i], w[16 + i]);
                            }
                        } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float a = exp2_approx(fmaf(__uint_as_float(x[c][2 * i]), fs, -u)), b = exp2_approx(fmaf(__uint_as_float(x[c][2 * i + 1]), fs, -u));
                            if (!SHARED && edge && f == 0.0f) {       // (0 x infinity)
                                if (key0 + 32 * c + 2 * i >= lim) a = 0.0f;
                                if (key0 + 32 * c + 2 * i + 1 >= lim) b = 0.0f;
                            }
                            l0 += a;
                            l1 += b;
                            if (E4M3) {
                                w[i] = f16x2(a, b);
                            } else {
                                w[i] = bf16x2(a, b);
                                w[16 + i] = bf16x2(a - bf16_lo(w[i]), b - bf16_hi(w[i]));
                            }
                        }
                        }
                        __syncwarp();
                        if (E4M3) tmem_st_x16(s_t + 32 * c, reinterpret_cast<const uint32_t (&)[16]>(w));
                        else tmem_st_x32(s_t + 32 * c, w);
                    }
                    if constexpr (SHARED && !E4M3) {
                        const float2 z = unpair(l01);
                        l0 = z.x; l1 = z.y;
                    }
                    l += l0 + l1;
                    tmem_wait_st();
                    tcgen05_fence_before_sync();
                }
                first_tile = false;
                if (tail < cur.rq.len) {
                    const int key0 = cur.j * KT + set * HALF, r0 = max(0, tail - key0), r1 = min(HALF, cur.rq.len - key0);
                    if (r0 < r1) {
                        ok = wait_all(kv_full(t % ST), (t / ST) & 1, W_R_KV_FULL);           // (complete: the scores are; this thread has to have seen it)
                        if (!ok) break;
                        const uint32_t v0 = v_s + (t % ST) * C::TILE + set * HALF * 128;
                        bool dropped = false;
#pragma unroll 1
                        for (int blk = 0; blk < D / 64; ++blk)
                            for (int i = r0 * 8 + row; i < r1 * 8; i += 128) dropped |= drop_nonfinite<E4M3 ? kExpF16 : kExpBf16>(v0 + blk * C::BLK + 16 * i);
                        if (dropped) {
                            fence_proxy_async_smem();
                            s_dropped[item & 1] = item;    // (no warp is more than an item behind another: they all release every item's queries)
                        }
                    }
                }
                // The product before must be complete before this one can begin: a barrier is waited for phase by phase (a wait for phase t while
                // phase t - 1 is open would take phase t - 2 for it, and the rows would be read out too early).
                if (t > 0) {
                    ok = wait_all(pv_done(set), (t - 1) & 1, W_R_PV_DONE);
                    if (!ok) break;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(buf, set));
            }
            if (ends) {
                if (SETS == 2 && set == 1) {
                    // the second set leaves its references and sums to the first, once that has read those of the item before
                    if (item > 1) {
                        ok = wait_all(o_free, (item - 2) & 1, W_R_O_FREE);
                        if (!ok) break;
                    }
                    s_ml[row] = make_float2(m, l);
                    __syncwarp();
                    if (lane == 0) mbar_arrive(ml_full);
                } else {
                    // (every warp of the set waits, those without rows too: one that ran ahead would arrive twice at o_free in one phase)
                    ok = wait_all(pv_done(0), t & 1, W_R_PV_DONE) &&
                         (SETS == 1 || (wait_all(ml_full, (item - 1) & 1, W_R_ML_FULL) && wait_all(pv_done(1), t & 1, W_R_PV_DONE)));
                    if (!ok) break;
                    if (SHARED) pdl_wait();
                    if (live_warp) {
                        float w0 = 1.0f, w1 = 0.0f, mm = m, ll = l;
                        if (SETS == 2) {
                            const float2 o = s_ml[row];
                            mm = fmaxf(m, o.x);
                            const float u = mm == -INFINITY ? 0.0f : mm;
                            w0 = exp2_approx(m - u);
                            w1 = exp2_approx(o.x - u);
                            ll = l * w0 + o.y * w1;
                        }
                        tcgen05_fence_after_sync();
                        const bool entire = item_end && part_j == 0;
                        const bool prefix_pass = SHARED && shared_prefixes(p), final = entire && !prefix_pass;      // final: O and lse, not a part of them
                        const float vs = E4M3 && p.cache.v_scale != nullptr ? p.cache.v_scale[cur.h] : 1.0f;
                        float* pre = nullptr;              // the prefix's part of the row: written, or added with weight wp
                        float wp = 0.0f;
                        if constexpr (SHARED) {
                            if (entire && r < R && (prefix_pass || cur.first_key() > 0)) {
                                const size_t at_row = prefix_row(p, cur.rq.row0, cur.h, r);
                                pre = p.sh.base_o + at_row * D;
                                if (!prefix_pass) {
                                    const JoinWeights j = join_weights(make_float2(mm, ll), __ldcg(p.sh.base_ml + at_row));
                                    mm = j.m; ll = j.l;
                                    w0 *= j.own; w1 *= j.own;
                                    wp = ll == 0.0f ? 0.0f : j.prefix / ll;
                                }
                            }
                            __syncwarp();
                        }
                        const float w = final ? (ll == 0.0f ? 0.0f : vs / ll) : vs;
                        w0 *= w;
                        w1 *= w;
                        const int slot = 2 * blockIdx.x + (first_part ? 0 : 1);
                        const RowOf at = row_of(p, r);
                        const int tok = at.token, hh = cur.h * p.group + at.head;
                        uint16_t* orow = p.O + static_cast<size_t>(cur.rq.row0 + tok) * p.ldo + static_cast<size_t>(hh) * D;
                        float* prow = p.part_o + static_cast<size_t>(slot) * ROWS * D + 4 * row;             // [channels / 4][rows][4]: coalesced
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            uint32_t o[32], o2[32];
                            tmem_ld_32x32b_x32(o_t + 32 * c, o);
                            if (SETS == 2) tmem_ld_32x32b_x32(o_t + D + 32 * c, o2);
                            tmem_wait_ld();
                            float v[32];
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                v[i] = __uint_as_float(o[i]) * w0;
                                if (SETS == 2) v[i] = fmaf(__uint_as_float(o2[i]), w1, v[i]);
                            }
                            if (r < R) {
                                if constexpr (SHARED) {
                                    if (pre != nullptr) {
#pragma unroll
                                        for (int i = 0; i < 32; i += 4) {
                                            float4* at4 = reinterpret_cast<float4*>(pre + 32 * c + i);
                                            if (prefix_pass) {
                                                *at4 = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                                            } else {
                                                const float4 x = __ldcg(at4);
                                                v[i] = fmaf(x.x, wp, v[i]); v[i + 1] = fmaf(x.y, wp, v[i + 1]); v[i + 2] = fmaf(x.z, wp, v[i + 2]); v[i + 3] = fmaf(x.w, wp, v[i + 3]);
                                            }
                                        }
                                    }
                                }
                                if (SHARED && entire && prefix_pass) {
                                    // (written)
                                } else if (entire) {
#pragma unroll
                                    for (int i = 0; i < 32; i += 8)
                                        *reinterpret_cast<uint4*>(orow + 32 * c + i) = make_uint4(bf16x2(v[i], v[i + 1]), bf16x2(v[i + 2], v[i + 3]),
                                                                                                  bf16x2(v[i + 4], v[i + 5]), bf16x2(v[i + 6], v[i + 7]));
                                } else {
#pragma unroll
                                    for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(prow + (8 * c + i / 4) * (4 * ROWS)) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                                }
                            }
                            __syncwarp();                  // (lanes without a row come back together before the next load)
                        }
                        if (*const_cast<volatile int*>(&s_dropped[item & 1]) == item && r < R) {
#pragma unroll 1
                            for (int d = 0; d < D; d += 4) {
                                const float4 z = nonfinite_values<E4M3>(p, cur.table_row(), cur.h, cur.first_key() + max(tail, part_j * KT), cur.first_key() + min(lim, (cur.j + 1) * KT), d);
                                const float zz[4] = {z.x, z.y, z.z, z.w};
                                for (int e = 0; e < 4; ++e) {
                                    if (entire) orow[d + e] = static_cast<uint16_t>(bf16x2(__uint_as_float(static_cast<uint32_t>(orow[d + e]) << 16) + zz[e], 0.0f) & 0xFFFFu);
                                    else prow[(d / 4) * (4 * ROWS) + e] += zz[e];
                                }
                            }
                        }
                        if (r < R) {
                            if (!entire) p.part_ml[static_cast<size_t>(slot) * ROWS + row] = make_float2(mm, ll);
                            else if (prefix_pass) store_prefix_ml(p, cur.rq.row0, cur.h, r, mm, ll);
                            else if (p.lse != nullptr)
                                p.lse[static_cast<size_t>(cur.rq.row0 + tok) * p.heads + hh] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * kLn2;
                        }
                        tcgen05_fence_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(o_free);
                }
                fresh = true;
                first_part = false;
            }
            ++t;
            cur.advance(p);
        }
    } else {
    // (keys of an item count from its first one; their places in pages and pages in the table from the request's first)
    auto page_at = [&](const Cur& at, int key) -> int {
        return key < at.rq.len ? p.table[static_cast<size_t>(at.table_row()) * p.ld_table + ((key + at.first_key()) >> p.cache.page_shift)] : -1;
    };
    const int box_rows = min(64, 1 << p.cache.page_shift), boxes = KT / box_rows;
    if (E4M3 && warp > MMA_WARP + LW) {
        // ---------------------------------------------------------------------------------------- E4M3: whole K and V tiles as they lie in the cache
        int issued = 0;
        bool ok = p.tma != 0;
        while (ok && cur.left > 0) {
            if (cur.j * KT + KT <= cur.rq.len) {
                int page = lane < boxes ? page_at(cur, cur.j * KT + box_rows * lane) : 0;
                if (page < 0 || page >= p.cache.n_pages) { record_bad_data(kBadPage); page = p.cache.n_pages; }                // out of range: zeros
                const int tok = (cur.first_key() + cur.j * KT + box_rows * lane) & ((1 << p.cache.page_shift) - 1);
#pragma unroll
                for (int half = 0; half < 2; ++half, ++issued) {
                    const int at = issued % max(RU, 1);
                    ok = wait_all(raw_empty(at), ((issued / max(RU, 1)) & 1) ^ 1, W_R_RAW_EMPTY);
                    if (!ok) break;
                    if (lane == 0) mbar_expect_tx(raw_full(at), C::RAW);
                    __syncwarp();
                    if (lane < boxes) tma_load_4d(raw_s + at * C::RAW + box_rows * lane * D, half ? &tm_v : &tm_k, 0, tok, cur.h, page, raw_full(at));
                    __syncwarp();
                }
            }
            cur.advance(p);
        }
    } else if (warp == MMA_WARP) {
        // ---------------------------------------------------------------------------------------- MMA issue
        const bool leader = elect_one();
        const uint32_t idesc_s = umma_idesc_f16(ROWS, KT, !E4M3, false), idesc_o = umma_idesc_f16(ROWS, D, !E4M3, true);
        int t = 0, item = 0, prev_item = 0;
        bool ok = true, fresh = true, prev_first = false;
        // O += P V of tile `pt` of item `it`, a set's keys each; the first tile of an item starts its O
        auto pv = [&](int pt, bool first, int it) -> bool {
            const int buf = pt & 1, slot = pt % ST;
            if (first && it > 0 && !wait_all(o_free, (it - 1) & 1, W_R_O_FREE)) return false;         // the item before has been read out
#pragma unroll
            for (int set = 0; set < SETS; ++set) {
                if (!wait_all(p_full(buf, set), (pt >> 1) & 1, W_R_P_FULL)) return false;
                tcgen05_fence_after_sync();
                if (leader) {
                    const uint32_t v0 = v_s + slot * C::TILE + set * HALF * 128, o = tmem + C::O_COL + set * D;
#pragma unroll
                    for (int kk = 0; kk < HALF / 16; ++kk) {
                        const uint64_t db = umma_desc_sw128_mn(v0 + kk * 2048, C::BLK);
                        const uint32_t pa = tmem + buf * KT + set * HALF + 32 * (kk >> 1) + 8 * (kk & 1);
                        umma_f16_ts(o, pa, db, idesc_o, (first && kk == 0) ? 0u : 1u);
                        if (!E4M3) umma_f16_ts(o, pa + 16, db, idesc_o, 1u);
                    }
                    if (set == SETS - 1) umma_commit(kv_empty(slot));            // (and the S of this stage, issued before)
                    umma_commit(pv_done(set));
                }
                __syncwarp();
            }
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
            ok = wait_all(kv_full(slot), (t / ST) & 1, W_R_KV_FULL);
            // S goes over the probabilities of two tiles ago: their product must be complete (products into different accumulators are not ordered)
            if (ok && t >= 2) ok = wait_all(pv_done(0), t & 1, W_R_PV_DONE) && (SETS == 1 || wait_all(pv_done(1), t & 1, W_R_PV_DONE));
            if (!ok) break;
            tcgen05_fence_after_sync();
            if (leader) {
                const uint32_t k0 = k_s + slot * C::TILE;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    umma_f16_ss(tmem + (t & 1) * KT, umma_desc_sw128(q_s + (ks >> 2) * C::QBLK) + 2u * (ks & 3),
                                umma_desc_sw128(k0 + (ks >> 2) * C::BLK) + 2u * (ks & 3), idesc_s, ks > 0 ? 1u : 0u);
                umma_commit(s_full(t & 1));
                if (ends) umma_commit(q_empty);
            }
            __syncwarp();
            if (t > 0) {
                ok = pv(t - 1, prev_first, prev_item);
                if (!ok) break;
            }
            prev_first = first;
            prev_item = item - 1;
            fresh = ends;
            ++t;
            cur.advance(p);
        }
        if (ok && t > 0) pv(t - 1, prev_first, prev_item);
    } else {
        // ---------------------------------------------------------------------------------------- loading
        const int w = warp - MMA_WARP - 1;
        // The keys of a tile in runs of 8, every LW-th run a warp's, K and V alike: in pages of 8 tokens or more a run lies in one page, and its
        // rows are one stride apart.  Lane i keeps the page of the warp's i-th run, requested a tile ahead.
        constexpr int RUN = 8, NRUN = KT / RUN, MINE = (NRUN + LW - 1) / LW;
        constexpr int CH = E4M3 ? D / 16 : D / 8;          // 16-byte pieces of a key
        constexpr int STEP = 32 / CH, N = RUN / STEP;      // keys per instruction of the warp, instructions per run and operand
        static_assert(STEP <= RUN, "a run is whole instructions");
        const int c = lane % CH, sub = lane / CH;
        const int64_t key_step = static_cast<int64_t>(STEP) * p.cache.token_stride;
        const bool run_in_page = p.cache.page_shift >= 3;
        int t = 0, item = 0;
        bool ok = true, fresh = true;
        // this warp's share has landed and is visible to the tensor core.  (The proxy fence waits for every copy of the thread that is still in flight: with
        // whole tiles copied this way the loading warps held one tile at a time and bounded the kernel, hence TMA for those.)
        auto signal = [&](uint32_t bar) {
            if (!E4M3) asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        auto page_of = [&](int key) -> int { return page_at(cur, key); };
        auto place = [&](int page, int key) -> long long {
            return page * p.cache.page_stride + static_cast<long long>(cur.h) * p.cache.head_stride +
                   static_cast<long long>((key + cur.first_key()) & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride;
        };
        auto run_pages = [&]() -> int {
            const int run = w + lane * LW;
            return run_in_page && lane < MINE && run < NRUN ? page_of(cur.j * KT + RUN * run) : -1;
        };
        int pages = run_pages();
        // TMA boxes of a tile, and the page of lane i's, requested a tile ahead as well
        auto box_page_of = [&]() -> int { return !E4M3 && w == 0 && lane < boxes ? page_at(cur, cur.j * KT + box_rows * lane) : -1; };
        int box_page = box_page_of();
        int taken = 0;                                     // E4M3: K and V tiles converted from where TMA left them
        while (cur.left > 0) {
            const bool ends = cur.j + 1 == cur.nt || cur.left == 1;
            const int slot = t % ST;
            const bool new_item = fresh;
            fresh = ends;
            ok = wait_all(kv_empty(slot), ((t / ST) & 1) ^ 1, W_R_KV_EMPTY);
            if (!ok) break;
            const uint32_t k_dst = k_s + slot * C::TILE, v_dst = v_s + slot * C::TILE;
            const int tile0 = cur.j * KT;
            // a whole tile in pages of 8 tokens or more: TMA, one box per page and 64 channels.  Its rows land where the copies below put them.
            const bool by_tma = !E4M3 && p.tma && tile0 + KT <= cur.rq.len;
            if (E4M3 && p.tma && tile0 + KT <= cur.rq.len) {
#pragma unroll 1
                for (int half = 0; half < 2; ++half, ++taken) {
                    const int at = taken % max(RU, 1);
                    ok = wait_all(raw_full(at), (taken / max(RU, 1)) & 1, W_R_RAW_FULL);
                    if (!ok) break;
                    const uint32_t src = raw_s + at * C::RAW + sub * D + 16 * c, dst = half ? v_dst : k_dst;
                    uint4 x[MINE * N];
#pragma unroll
                    for (int k = 0; k < MINE; ++k)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const int run = w + k * LW;
                            if (run < NRUN)
                                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[k * N + i].x), "=r"(x[k * N + i].y), "=r"(x[k * N + i].z), "=r"(x[k * N + i].w)
                                             : "r"(src + (RUN * run + i * STEP) * D) : "memory");
                        }
#pragma unroll
                    for (int k = 0; k < MINE; ++k)
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            const int run = w + k * LW;
                            if (run < NRUN) {
                                const int kr = i * STEP + sub, c2 = 2 * c;
                                const uint32_t row = (c2 >> 3) * C::BLK + (RUN * run + kr) * 128;
                                store_f16(dst + row + (((c2 & 7) ^ (kr & 7)) << 4), dst + row + ((((c2 & 7) + 1) ^ (kr & 7)) << 4), x[k * N + i]);
                            }
                        }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(raw_empty(at));
                }
                if (!ok) break;
                signal(kv_full(slot));
            } else if (by_tma) {
                if (w == 0) {
                    if (lane == 0) mbar_expect_tx(kv_full(slot), 2 * C::TILE);
                    __syncwarp();
                    if (lane < boxes) {
                        int page = box_page;
                        if (page < 0 || page >= p.cache.n_pages) { record_bad_data(kBadPage); page = p.cache.n_pages; }      // out of range: zeros
                        const int tok = (cur.first_key() + tile0 + box_rows * lane) & ((1 << p.cache.page_shift) - 1);
#pragma unroll
                        for (int blk = 0; blk < D / 64; ++blk) {
                            tma_load_4d(k_dst + blk * C::BLK + box_rows * lane * 128, &tm_k, 64 * blk, tok, cur.h, page, kv_full(slot));
                            tma_load_4d(v_dst + blk * C::BLK + box_rows * lane * 128, &tm_v, 64 * blk, tok, cur.h, page, kv_full(slot));
                        }
                    }
                } else if (lane == 0) {
                    mbar_arrive(kv_full(slot));
                }
            } else {
#pragma unroll 1
            for (int half = 0; half < (E4M3 ? 2 : 1); ++half) {
            uint4 x[E4M3 ? MINE * N : 1];                  // E4M3: this warp's share of the K or V tile, all in flight together
            const uint8_t* from = half ? p.cache.v : p.cache.k;
#pragma unroll
            for (int k = 0; k < MINE; ++k) {
                const int run = w + k * LW;
                if (run >= NRUN) break;
                const int key0 = cur.j * KT + RUN * run;
                const int page = __shfl_sync(0xffffffffu, pages, k);
                // place of this lane's first key in the run, and whether the others follow at a stride
                const bool whole = run_in_page && key0 + RUN <= cur.rq.len && page >= 0 && page < p.cache.n_pages;
                long long off = 0;
                if (whole) {
                    off = place(page, key0 + sub) + 16 * c;
                } else {
                    // the end of the request, pages of less than 8 tokens, or a bad page: lane i looks up key i
                    const int key = key0 + lane, pg = lane < RUN ? page_of(key) : -1;
                    off = -1;
                    if (lane < RUN && key < cur.rq.len) {
                        if (pg < 0 || pg >= p.cache.n_pages) record_bad_data(kBadPage);
                        else off = place(pg, key);
                    }
                }
                const uint32_t row = (E4M3 ? 0 : (c >> 3) * C::BLK) + (RUN * run + sub) * 128;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    long long o = off + i * key_step;
                    bool valid = true;
                    if (!whole) {
                        o = __shfl_sync(0xffffffffu, off, i * STEP + sub);
                        valid = o >= 0;
                        o = valid ? o + 16 * c : 0;
                    }
                    if (!E4M3) {
                        const uint32_t at = row + i * STEP * 128 + ((((c & 7) ^ sub) ^ ((i * STEP) & 7)) << 4);
                        cp_async16(k_dst + at, p.cache.k + o, valid);
                        cp_async16(v_dst + at, p.cache.v + o, valid);
                    } else {
                        x[E4M3 ? k * N + i : 0] = make_uint4(0, 0, 0, 0);
                        if (valid) x[E4M3 ? k * N + i : 0] = __ldcg(reinterpret_cast<const uint4*>(from + o));
                    }
                }
            }
            if (E4M3) {
#pragma unroll
                for (int k = 0; k < MINE; ++k) {
                    const int run = w + k * LW;
                    if (run >= NRUN) break;
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int kr = i * STEP + sub, c2 = 2 * c;               // key of the run, first of its two 16-byte pieces of f16
                        const uint32_t row = (c2 >> 3) * C::BLK + (RUN * run + kr) * 128;
                        const uint32_t at0 = row + (((c2 & 7) ^ (kr & 7)) << 4), at1 = row + ((((c2 & 7) + 1) ^ (kr & 7)) << 4);
                        const uint32_t dst = half ? v_dst : k_dst;
                        store_f16(dst + at0, dst + at1, x[E4M3 ? k * N + i : 0]);
                    }
                }
            }
            }
            signal(kv_full(slot));
            }
            if (new_item && w >= LW - C::QW) {
                // (the first item's are already on their way)
                if (item > 0) {
                    ok = wait_all(q_empty, (item - 1) & 1, W_R_Q_EMPTY);
                    if (!ok) break;
                    load_queries(w - (LW - C::QW), C::QW);
                }
                ++item;
                signal(q_full);
            }
            ++t;
            cur.advance(p);
            if (cur.left > 0) {
                if (!E4M3 || !p.tma || cur.j * KT + KT > cur.rq.len) pages = run_pages();
                box_page = box_page_of();
            }
        }
    }
    }

    // ---- teardown: no MMA of this CTA is in flight when its tensor memory goes (the first softmax set has waited for the last products; after
    // an aborted wait the issued ones get a millisecond, a thousand times what they take)
    if (warp == MMA_WARP && *abortp != 0)
        for (int it = 0; it < 1000; ++it) __nanosleep(1000);
    tcgen05_fence_before_sync();
    __syncthreads();
    if (warp == MMA_WARP) {
        __syncwarp();
        tcgen05_fence_after_sync();
        tmem_dealloc(tmem, 512);
    }
}

template <class C, bool SHARED>
cudaError_t launch_rows(const ParamsOf<SHARED>& p, const CUtensorMap* tm_k, const CUtensorMap* tm_v, cudaStream_t st)
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
    return cudaLaunchKernelEx(&cfg, attention_rows_kernel<C, SHARED>, p, *tm_k, *tm_v);
}
template <class C>
cudaError_t init_rows()
{
    if constexpr (C::PAIR) return cudaFuncSetAttribute(attention_rows_kernel<C, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    else {
    const cudaError_t e = cudaFuncSetAttribute(attention_rows_kernel<C, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    return e == cudaSuccess ? cudaFuncSetAttribute(attention_rows_kernel<C, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) : e;
    }
}

}  // namespace

}  // namespace rudder
