// What the two attention kernels share: parameters, the sequence of work units and its split into runs, small helpers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "internal.cuh"
#include "paged.cuh"

namespace rudder {

namespace {

constexpr float kLn2 = 0.6931471805599453f;

// Requests in groups that share a prefix: the prefixes are a pass in which a GROUP stands in a request's place (its rows are those of all its requests, its
// keys the prefix) and whose rows end as parts in `base`; what stands behind the prefixes is a second pass that joins these parts to its own.  A prefix is read once for its
// group this way, and its rows fill the tensor core's tiles.  Measured: 32 requests of 16 rows x 16 heads over 4416 shared and up to 80 own tokens 69 us (the prefixes 47, the join
// of their parts 8, the second pass 16), 64 requests over four prefixes of 17k to 28k tokens in E4M3, 8 key-value heads, 175 us (132, 7, 33); one by one, by
// rudder_attention_paged, 198 and 553 us.  A few requests over a short prefix take longer this way (8 of one token over 320: 13.7 against 7.0 us): three launches, of which each waits for
// the one in front.
struct SharedPass {
    const int32_t* group_starts; const int32_t* prefix_lens; const int32_t* prefix_rows;
    int n_groups, table_rows, requests;
    int key_mask;                       // a prefix is cut down to a multiple of 64 where the second pass takes its tiles by TMA
    int prefixes;                       // this pass is the first
    int causal;                         // of the call (the first pass has no causal limits of its own)
    float* base_o;                      // [M x heads][D], relative to ...
    float2* base_ml;                    // [M x heads]: reference and sum
};

struct AttnParams {
    const uint16_t* Q; int64_t ldq;
    uint16_t* O; int64_t ldo;
    float* lse;
    CacheParams cache;                  // strides in BYTES here
    const int32_t* table; int64_t ld_table;
    const int32_t* kv_lens;
    const int32_t* q_starts;
    float* part_o;                      // [2 G][rows of a tile][D]; many rows: [2 G][D / 4][rows of a tile][4]
    float2* part_ml;                    // [2 G][rows of a tile]
    int* desc;                          // [G][8]
    float scale_log2;
    int max_pages, B, max_q, M, heads, kv_heads, group, causal;
    uint32_t group_inv;                 // ceil(2^32 / group), 0 for a group of one: see row_of
    int whole_units;                    // items of at most this many units are not cut when there is a CTA for each
    int G;                              // CTAs
    int tma;                            // many rows: tensor maps over the cache are there
};
struct SharedParams : AttnParams {
    SharedPass sh;
};
template <bool SHARED>
using ParamsOf = std::conditional_t<SHARED, SharedParams, AttnParams>;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
    const int n = valid ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
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
// Four E4M3 bytes as f16 numbers (exact): bytes 0 and 1, bytes 2 and 3.  (The conversion instruction: moving the bits by shifts and masks is
// 7 operations instead of 2 and cost 101 instead of 86 us on 4 x 126k keys.)
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
}
// The same for bytes 0 and 2, bytes 1 and 3.
__device__ __forceinline__ void e4m3_to_f16_split(uint32_t w, uint32_t& even, uint32_t& odd) { e4m3_to_f16(__byte_perm(w, 0, 0x3120), even, odd); }

// Row r of an item: which of the request's new tokens, which head of its group.  r < 2^20 and a group of at most 1024 heads make the
// product exact: r (ceil(2^32 / g) g - 2^32) < 2^32.
struct RowOf { int token, head; };
__device__ __forceinline__ RowOf row_of(const AttnParams& p, int r) {
    RowOf o;
    o.token = p.group_inv ? static_cast<int>(__umulhi(static_cast<uint32_t>(r), p.group_inv)) : r;
    o.head = r - o.token * p.group;
    return o;
}

// Keys that all rows of a tile see whose first row is of new token `token`.
__device__ __forceinline__ int tail_of(int len, int qlen, int token) { return min(len, max(0, len - qlen + token + 1)); }
// Values that are infinite or no number, of 16-bit numbers (EXP: their exponent's bits in both halves) or E4M3 numbers: replaced by zero; true if there were any.
// Among the keys that only some rows see they stay out of the product (to a row that does not see the key it would add 0 x infinity) and are
// added by nonfinite_values to the rows that do.
constexpr uint32_t kExpBf16 = 0x7F807F80u, kExpF16 = 0x7C007C00u, kExpE4m3 = 0x7F7F7F7Fu;
template <uint32_t EXP>
__device__ __forceinline__ bool drop_nonfinite(uint32_t addr) {
    uint32_t w[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr) : "memory");
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t gone = EXP == kExpE4m3 ? __vcmpeq4(w[i] & EXP, EXP) : __vcmpeq2(w[i] & EXP, EXP);
        any |= gone;
        w[i] &= ~gone;
    }
    if (any) asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
    return any != 0;
}
// What was dropped of keys [k0, k1) of row b of the page table, channels d .. d + 3, summed.  (A handful of new tokens at most, and only when there was something.)
template <bool E4M3>
__device__ __forceinline__ float4 nonfinite_values(const AttnParams& p, int b, int h, int k0, int k1, int d) {
    float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int k = k0; k < k1; ++k) {
        const int page = p.table[static_cast<size_t>(b) * p.ld_table + (k >> p.cache.page_shift)];
        if (page < 0 || page >= p.cache.n_pages) continue;
        const uint8_t* v = p.cache.v + page * p.cache.page_stride + static_cast<long long>(h) * p.cache.head_stride +
                           static_cast<long long>(k & ((1 << p.cache.page_shift) - 1)) * p.cache.token_stride + d * (E4M3 ? 1 : 2);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = E4M3 ? ((v[e] & 0x7F) == 0x7F ? NAN : 0.0f) : __uint_as_float(static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(v)[e]) << 16);
            if (!(fabsf(x) < INFINITY)) z[e] += x;
        }
    }
    return make_float4(z[0], z[1], z[2], z[3]);
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

// With shared prefixes: its keys begin at key0 (behind the prefix that is joined to it, or 0), and its pages stand in row `trow` of the table.
struct SharedReq : Req { int key0, trow; };
// The group of a request: requests [begin, end) and the part of the prefix that is read for all of them; begin .. begin + 1 and 0 for a request of no group.
struct Group { int begin, end, prefix; };

__device__ __forceinline__ int prefix_of(const SharedParams& p, int g) {
    const long long cap = static_cast<long long>(p.max_pages) << p.cache.page_shift;
    const int len = p.sh.prefix_lens[g], row = p.sh.prefix_rows[g];
    const int n = static_cast<int>(len < 0 ? 0 : (len > cap ? cap : len));
    if (n != len || row < 0 || row >= p.sh.table_rows) record_bad_data(kBadLength);
    return row < 0 || row >= p.sh.table_rows ? 0 : n & p.sh.key_mask;
}
__device__ __forceinline__ Group find_group(const SharedParams& p, int b) {
    int lo = -1, hi = p.sh.n_groups;                       // last group that starts at or before b
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.sh.group_starts[mid] <= b) lo = mid; else hi = mid;
    }
    if (lo < 0) return Group{b, b + 1, 0};
    const int end = p.sh.group_starts[lo + 1];
    if (b >= end) return Group{b, b + 1, 0};
    return Group{p.sh.group_starts[lo], end, prefix_of(p, lo)};
}
// Group g in a request's place.
__device__ __forceinline__ SharedReq load_group(const SharedParams& p, int g) {
    SharedReq r;
    r.len = prefix_of(p, g);
    r.key0 = 0;
    r.trow = p.sh.prefix_rows[g];                          // (a bad one has no keys)
    const int s0 = p.sh.group_starts[g], s1 = p.sh.group_starts[g + 1];
    const int b0 = min(max(s0, 0), p.sh.requests), b1 = min(max(s1, b0), p.sh.requests);
    if (b0 != s0 || b1 != s1) record_bad_data(kBadLength);
    r.row0 = min(max(p.q_starts != nullptr ? p.q_starts[b0] : b0 * p.max_q, 0), p.M);
    const int end = min(max(p.q_starts != nullptr ? p.q_starts[b1] : b1 * p.max_q, r.row0), p.M);
    r.qlen = r.len > 0 ? end - r.row0 : 0;                 // without a prefix there is nothing to join
    return r;
}
// Request b of a group with this prefix: it reads what stands behind the prefix if each of its rows sees all of that.
__device__ __forceinline__ SharedReq load_member(const SharedParams& p, int b, int prefix) {
    SharedReq r;
    static_cast<Req&>(r) = load_request(p, b);
    r.trow = b;
    r.key0 = r.len - (p.sh.causal ? r.qlen - 1 : 0) >= prefix ? prefix : 0;
    r.len -= r.key0;
    return r;
}

// Request (or group) b by this lane, the whole warp together; b at or beyond the last one has no rows.
__device__ __forceinline__ void load_by_lane(const SharedParams& p, int b, int lane, SharedReq& r, Group& grp) {
    if (p.sh.prefixes) {
        if (b < p.B) r = load_group(p, b);
        return;
    }
    if (p.sh.n_groups <= 32) {
        // a group per lane: no search, its loads beside those of the requests
        const bool is = lane < p.sh.n_groups;
        const int s0 = is ? p.sh.group_starts[lane] : 0x7fffffff, s1 = is ? p.sh.group_starts[lane + 1] : 0, pre = is ? prefix_of(p, lane) : 0;
        int at = -1;
        for (int i = 0; i < p.sh.n_groups; ++i) at = __shfl_sync(0xffffffffu, s0, i) <= b ? i : at;
        const int from = max(at, 0);
        grp = Group{__shfl_sync(0xffffffffu, s0, from), __shfl_sync(0xffffffffu, s1, from), __shfl_sync(0xffffffffu, pre, from)};
        if (at < 0 || b >= grp.end) grp = Group{b, b + 1, 0};
    } else if (b < p.B) {
        grp = find_group(p, b);
    }
    if (b < p.B) r = load_member(p, b, grp.prefix);
}

// A place in the sequence of units: request, kv head, row tile, unit inside the item, and what is left of the run from there on.
// What starting and ending an item costs, in units (queries, merge of the warp groups, output): an item counts as its units + kItemCost,
// the cost in front.  A cut inside the cost leaves the item whole to the run behind.
// 48 requests of up to 16384 keys 56 us, without a cost 172 us, with 6 59 us.  (Units of 16 or 32 keys, a warp's: see PickSolo.)
template <int UNIT_KEYS>
constexpr int kItemCost = UNIT_KEYS >= 64 ? 2 : 4;

template <int ROWS, int UK, bool SHARED = false>
struct Cursor {
    int b, h, rt, j, nt, n_rt;
    long long left;
    std::conditional_t<SHARED, SharedReq, Req> rq;
    Group grp;                                             // SHARED, second pass: of request b
    __device__ __forceinline__ void set_request(const ParamsOf<SHARED>& p, int bb) {
        b = bb;
        if constexpr (SHARED) {
            if (p.sh.prefixes) {
                rq = load_group(p, bb);
            } else {
                if (bb < grp.begin || bb >= grp.end) grp = find_group(p, bb);
                rq = load_member(p, bb, grp.prefix);
            }
        } else {
            rq = load_request(p, bb);
        }
        nt = max(1, (rq.len + UK - 1) / UK);
        n_rt = (rq.qlen * p.group + ROWS - 1) / ROWS;
    }
    // the item's row of the page table, and what its first key is in the request's count
    __device__ __forceinline__ int table_row() const { if constexpr (SHARED) return rq.trow; else return b; }
    __device__ __forceinline__ int first_key() const { if constexpr (SHARED) return rq.key0; else return 0; }
    __device__ __forceinline__ void next_item(const ParamsOf<SHARED>& p) {
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
    __device__ __forceinline__ void advance(const ParamsOf<SHARED>& p) {
        ++j;
        if (--left <= 0 || j < nt) return;
        left -= kItemCost<UK>;
        if (left > 0) next_item(p);
    }
};

__device__ __forceinline__ bool shared_prefixes(const AttnParams&) { return false; }
__device__ __forceinline__ bool shared_prefixes(const SharedParams& p) { return p.sh.prefixes != 0; }
// The start of a pass in a chain of early launches.  The prefixes' pass lets the next launch begin only when everything in front of the call is complete; so the
// pass behind it (and what may come between them) may begin while prefixes are still read, and waits for them in front of its first output.  It begins where its CTAs find room: beside
// those of the kernel for few rows.  The kernel for many rows takes all registers of an SM (12 x 32 threads x 168), so behind that one it begins beside the join, 3 us after the prefixes.
__device__ __forceinline__ void start_pass(const AttnParams&) {
    pdl_launch_dependents();
    pdl_wait();
}
__device__ __forceinline__ void start_pass(const SharedParams& p) {
    if (p.sh.prefixes) pdl_wait();
    pdl_launch_dependents();
}
// Row `r` of an item whose rows begin at row0: its place in base_o and base_ml.
__device__ __forceinline__ size_t prefix_row(const AttnParams& p, int row0, int h, int r) {
    const RowOf at = row_of(p, r);
    return static_cast<size_t>(row0 + at.token) * p.heads + h * p.group + at.head;
}
__device__ __forceinline__ void store_prefix_ml(const AttnParams&, int, int, int, float, float) {}
__device__ __forceinline__ void store_prefix_ml(const SharedParams& p, int row0, int h, int r, float m, float l) { p.sh.base_ml[prefix_row(p, row0, h, r)] = make_float2(m, l); }
template <int D>
__device__ __forceinline__ void store_prefix_o(const AttnParams&, int, int, int, int, float4) {}
template <int D>
__device__ __forceinline__ void store_prefix_o(const SharedParams& p, int row0, int h, int r, int d, float4 o) {
    *reinterpret_cast<float4*>(p.sh.base_o + prefix_row(p, row0, h, r) * D + d) = o;
}
// A row's own (reference, sum) and those of its prefix: both together, and the factors of the two weighted sums of values.
struct JoinWeights { float m, l, own, prefix; };
__device__ __forceinline__ JoinWeights join_weights(float2 own, float2 pre) {
    JoinWeights j;
    j.m = fmaxf(own.x, pre.x);
    const float u = j.m == -INFINITY ? 0.0f : j.m;
    j.own = exp2_approx(own.x - u);
    j.prefix = exp2_approx(pre.x - u);
    j.l = own.y * j.own + pre.y * j.prefix;
    return j;
}

// Quotient of non-negative numbers, in 32 bits where they fit (they nearly always do; a 64-bit division is a hundred instructions of latency).
__device__ __forceinline__ long long quotient(long long a, long long b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// This CTA's run of units: sums over the requests (threads over consecutive requests), the place of its first unit, and the descriptor that
// the join reads.  All threads call it; false = nothing to do.
template <int ROWS, int UK, int THREADS, bool SHARED>
__device__ __forceinline__ bool start_of_run(const ParamsOf<SHARED>& p, Cursor<ROWS, UK, SHARED>& cur)
{
    using R = decltype(cur.rq);
    if constexpr (SHARED) cur.grp = Group{0, 0, 0};
    __shared__ long long s_units[THREADS / 32];
    __shared__ int s_items[THREADS / 32];
    __shared__ int s_max[THREADS / 32];
    __shared__ int s_place[4];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    long long total, share, u_begin, u_end;
    bool whole;
    int place;
    if constexpr (SHARED && UK < 64) {
        // CTAs of a warp or two: every warp for itself, 32 requests at a time (a thread after another's requests, as below, would be a chain of loads for each)
        const int chunks = (p.B + 31) / 32;
        R r = {};
        Group grp = {0, 0, 0};
        int n_rt = 0, nt = 0;
        auto load = [&](int c) {
            r = {};
            load_by_lane(p, 32 * c + lane, lane, r, grp);
            n_rt = (r.qlen * p.group + ROWS - 1) / ROWS;
            nt = max(1, (r.len + UK - 1) / UK);
        };
        long long units = 0, n_items = 0;
        int most = 0;
#pragma unroll 2
        for (int c = 0; c < chunks; ++c) {
            load(c);
            units += static_cast<long long>(n_rt) * p.kv_heads * (nt + kItemCost<UK>);
            n_items += static_cast<long long>(n_rt) * p.kv_heads;
            if (n_rt > 0) most = max(most, nt);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            units += __shfl_xor_sync(0xffffffffu, units, d);
            n_items += __shfl_xor_sync(0xffffffffu, n_items, d);
        }
        total = units;
        whole = n_items <= p.G && __reduce_max_sync(0xffffffffu, most) <= p.whole_units;
        share = whole ? 1 : quotient(total + p.G - 1, p.G);
        const long long all = whole ? n_items : total;
        u_begin = min(all, share * blockIdx.x);
        u_end = min(all, u_begin + share);
        if (u_begin >= u_end) {
            if (tid == 0) p.desc[8 * blockIdx.x] = 0;
            return false;
        }
        long long carry = 0, before = 0;
        int at = -1;
        for (int c = 0;; ++c) {
            if (chunks > 1) load(c);
            const long long mine = static_cast<long long>(n_rt) * p.kv_heads * (whole ? 1 : nt + kItemCost<UK>);
            long long inc = mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, inc, d);
                if (lane >= d) inc += u;
            }
            before = carry + inc - mine;
            const uint32_t hit = __ballot_sync(0xffffffffu, u_begin >= before && u_begin < before + mine);          // at most one lane
            if (hit != 0 || c + 1 >= chunks) {
                at = max(0, __ffs(hit) - 1);
                cur.b = 32 * c + at;
                break;
            }
            carry += __shfl_sync(0xffffffffu, inc, 31);
        }
        cur.rq.len = __shfl_sync(0xffffffffu, r.len, at);
        cur.rq.row0 = __shfl_sync(0xffffffffu, r.row0, at);
        cur.rq.qlen = __shfl_sync(0xffffffffu, r.qlen, at);
        cur.rq.key0 = __shfl_sync(0xffffffffu, r.key0, at);
        cur.rq.trow = __shfl_sync(0xffffffffu, r.trow, at);
        cur.grp = Group{__shfl_sync(0xffffffffu, grp.begin, at), __shfl_sync(0xffffffffu, grp.end, at), __shfl_sync(0xffffffffu, grp.prefix, at)};
        cur.nt = __shfl_sync(0xffffffffu, nt, at);
        cur.n_rt = __shfl_sync(0xffffffffu, n_rt, at);
        const long long off = u_begin - __shfl_sync(0xffffffffu, before, at);
        const int size = whole ? 1 : cur.nt + kItemCost<UK>;
        const uint32_t item = static_cast<uint32_t>(quotient(off, size));
        cur.h = static_cast<int>(item / static_cast<uint32_t>(cur.n_rt));
        cur.rt = static_cast<int>(item % static_cast<uint32_t>(cur.n_rt));
        place = whole ? kItemCost<UK> : static_cast<int>(off - static_cast<long long>(item) * size);
    } else if (p.B <= 32) {
        // a request per lane, every warp for itself: no barrier, nothing loaded twice (one request of 333 keys: 3200 -> 1900 clocks)
        R r = {};
        Group grp = {0, 0, 0};
        if constexpr (SHARED) load_by_lane(p, lane, lane, r, grp);
        else if (lane < p.B) r = load_request(p, lane);
        const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = max(1, (r.len + UK - 1) / UK);
        const long long t_units = static_cast<long long>(n_rt) * p.kv_heads * (nt + kItemCost<UK>);
        const int t_items = n_rt * p.kv_heads;
        long long i_units = t_units;
        int i_items = t_items;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const long long u = __shfl_up_sync(0xffffffffu, i_units, d);
            const int v = __shfl_up_sync(0xffffffffu, i_items, d);
            if (lane >= d) { i_units += u; i_items += v; }
        }
        total = __shfl_sync(0xffffffffu, i_units, 31);
        const int items = __shfl_sync(0xffffffffu, i_items, 31);
        whole = items <= p.G && __reduce_max_sync(0xffffffffu, n_rt > 0 ? nt : 0) <= p.whole_units;
        share = whole ? 1 : quotient(total + p.G - 1, p.G);
        const long long all = whole ? items : total;
        u_begin = min(all, share * blockIdx.x);
        u_end = min(all, u_begin + share);
        if (u_begin >= u_end) {
            if (tid == 0) p.desc[8 * blockIdx.x] = 0;
            return false;
        }
        const long long before = whole ? i_items - t_items : i_units - t_units, mine = whole ? t_items : t_units;
        const int b = __ffs(__ballot_sync(0xffffffffu, u_begin >= before && u_begin < before + mine)) - 1;       // exactly one lane
        cur.b = b;
        cur.rq.len = __shfl_sync(0xffffffffu, r.len, b);
        cur.rq.row0 = __shfl_sync(0xffffffffu, r.row0, b);
        cur.rq.qlen = __shfl_sync(0xffffffffu, r.qlen, b);
        if constexpr (SHARED) {
            cur.rq.key0 = __shfl_sync(0xffffffffu, r.key0, b);
            cur.rq.trow = __shfl_sync(0xffffffffu, r.trow, b);
            cur.grp = Group{__shfl_sync(0xffffffffu, grp.begin, b), __shfl_sync(0xffffffffu, grp.end, b), __shfl_sync(0xffffffffu, grp.prefix, b)};
        }
        cur.nt = __shfl_sync(0xffffffffu, nt, b);
        cur.n_rt = __shfl_sync(0xffffffffu, n_rt, b);
        const long long off = u_begin - __shfl_sync(0xffffffffu, before, b);
        const int size = whole ? 1 : cur.nt + kItemCost<UK>;
        const uint32_t item = static_cast<uint32_t>(quotient(off, size));
        cur.h = static_cast<int>(item / static_cast<uint32_t>(cur.n_rt));
        cur.rt = static_cast<int>(item % static_cast<uint32_t>(cur.n_rt));
        place = whole ? kItemCost<UK> : static_cast<int>(off - static_cast<long long>(item) * size);
    } else {
    const int per = (p.B + THREADS - 1) / THREADS;
    const int rb0 = min(p.B, tid * per), rb1 = min(p.B, rb0 + per);
    long long t_units = 0;
    int t_items = 0, t_max = 0;
    auto request = [&](int b) {
        if constexpr (SHARED) { cur.set_request(p, b); return cur.rq; }        // (the cursor remembers the group)
        else return load_request(p, b);
    };
    for (int b = rb0; b < rb1; ++b) {
        const R r = request(b);
        const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = max(1, (r.len + UK - 1) / UK);
        t_units += static_cast<long long>(n_rt) * p.kv_heads * (nt + kItemCost<UK>);
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
    long long e_units = i_units - t_units;
    total = 0;
    int items = 0, e_items = i_items - t_items, most = 0;
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) { e_units += s_units[w]; e_items += s_items[w]; }
        total += s_units[w];
        items += s_items[w];
        most = max(most, s_max[w]);
    }
    whole = items <= p.G && most <= p.whole_units;
    share = whole ? 1 : quotient(total + p.G - 1, p.G);
    const long long all = whole ? items : total;
    u_begin = min(all, share * blockIdx.x);
    u_end = min(all, u_begin + share);
    if (u_begin >= u_end) {
        if (tid == 0) p.desc[8 * blockIdx.x] = 0;
        return false;
    }
    {
        const long long mine0 = whole ? e_items : e_units, mine1 = mine0 + (whole ? t_items : t_units);
        if (u_begin >= mine0 && u_begin < mine1) {         // exactly one thread
            long long at = mine0;
            for (int b = rb0; b < rb1; ++b) {
                const R r = request(b);
                const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = whole ? 1 : max(1, (r.len + UK - 1) / UK) + kItemCost<UK>;
                const long long here = static_cast<long long>(n_rt) * p.kv_heads * nt;
                if (u_begin < at + here) {
                    const long long off = u_begin - at;
                    const uint32_t item = static_cast<uint32_t>(quotient(off, nt));         // below kv_heads x n_rt
                    s_place[0] = b;
                    s_place[1] = static_cast<int>(item / static_cast<uint32_t>(n_rt));
                    s_place[2] = static_cast<int>(item % static_cast<uint32_t>(n_rt));
                    s_place[3] = static_cast<int>(off - static_cast<long long>(item) * nt); // place inside the item, its cost included
                    break;
                }
                at += here;
            }
        }
    }
    __syncthreads();
    cur.set_request(p, s_place[0]);
    cur.h = s_place[1]; cur.rt = s_place[2];
    place = whole ? kItemCost<UK> : s_place[3];
    }
    cur.j = max(0, place - kItemCost<UK>);
    cur.left = whole ? cur.nt : (u_end - u_begin) - max(0, kItemCost<UK> - place);      // of this run, from unit cur.j on
    if (cur.left <= 0) {                                       // nothing but a part of an item's cost
        if (tid == 0) p.desc[8 * blockIdx.x] = 0;
        return false;
    }
    if (tid == 0) {
        // the join of the item that this run starts inside belongs to its first cut, i.e. to the run behind its first owner
        int* d = p.desc + 8 * blockIdx.x;
        const long long unit0 = u_begin - cur.j;           // place of the item's first unit
        const long long before = share * (static_cast<long long>(blockIdx.x) - 1);
        const bool first_cut = !whole && cur.j > 0 && unit0 >= before;
        d[1] = cur.h; d[2] = cur.rt; d[3] = cur.rq.row0; d[4] = cur.rq.qlen;
        d[5] = static_cast<int>(quotient(unit0 + cur.nt - 1, share));            // last owner
        d[6] = unit0 <= before + kItemCost<UK> ? 0 : 1;        // slot of the first owner's part: its run starts with this item (or inside its cost)
        d[0] = first_cut ? 1 : 0;
        if constexpr (SHARED) d[7] = cur.rq.key0 > 0;       // the join adds the prefix's part
    }
    return true;
}

}  // namespace

}  // namespace rudder
