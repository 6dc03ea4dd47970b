// What the two attention kernels share: parameters, the sequence of work units and its split into runs, small helpers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.cuh"
#include "paged.cuh"

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
// What was dropped of keys [k0, k1) of request b, channels d .. d + 3, summed.  (A handful of new tokens at most, and only when there was something.)
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

// A place in the sequence of units: request, kv head, row tile, unit inside the item, and what is left of the run from there on.
// What starting and ending an item costs, in units (queries, merge of the warp groups, output): an item counts as its units + kItemCost,
// the cost in front.  A cut inside the cost leaves the item whole to the run behind.
constexpr int kItemCost = 2;                               // 48 requests of up to 16384 keys 56 us, without a cost 172 us, with 6 59 us

template <int ROWS, int UK>
struct Cursor {
    int b, h, rt, j, nt, n_rt;
    long long left;
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
        ++j;
        if (--left <= 0 || j < nt) return;
        left -= kItemCost;
        if (left > 0) next_item(p);
    }
};

// Quotient of non-negative numbers, in 32 bits where they fit (they nearly always do; a 64-bit division is a hundred instructions of latency).
__device__ __forceinline__ long long quotient(long long a, long long b) {
    if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// This CTA's run of units: sums over the requests (threads over consecutive requests), the place of its first unit, and the descriptor that
// the join reads.  All threads call it; false = nothing to do.
template <int ROWS, int UK, int THREADS>
__device__ __forceinline__ bool start_of_run(const AttnParams& p, Cursor<ROWS, UK>& cur)
{
    __shared__ long long s_units[THREADS / 32];
    __shared__ int s_items[THREADS / 32];
    __shared__ int s_max[THREADS / 32];
    __shared__ int s_place[4];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    long long total, share, u_begin, u_end;
    bool whole;
    int place;
    if (p.B <= 32) {
        // a request per lane, every warp for itself: no barrier, nothing loaded twice (one request of 333 keys: 3200 -> 1900 clocks)
        Req r = {0, 0, 0};
        if (lane < p.B) r = load_request(p, lane);
        const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = max(1, (r.len + UK - 1) / UK);
        const long long t_units = static_cast<long long>(n_rt) * p.kv_heads * (nt + kItemCost);
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
        cur.nt = __shfl_sync(0xffffffffu, nt, b);
        cur.n_rt = __shfl_sync(0xffffffffu, n_rt, b);
        const long long off = u_begin - __shfl_sync(0xffffffffu, before, b);
        const int size = whole ? 1 : cur.nt + kItemCost;
        const uint32_t item = static_cast<uint32_t>(quotient(off, size));
        cur.h = static_cast<int>(item / static_cast<uint32_t>(cur.n_rt));
        cur.rt = static_cast<int>(item % static_cast<uint32_t>(cur.n_rt));
        place = whole ? kItemCost : static_cast<int>(off - static_cast<long long>(item) * size);
    } else {
    const int per = (p.B + THREADS - 1) / THREADS;
    const int rb0 = min(p.B, tid * per), rb1 = min(p.B, rb0 + per);
    long long t_units = 0;
    int t_items = 0, t_max = 0;
    for (int b = rb0; b < rb1; ++b) {
        const Req r = load_request(p, b);
        const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = max(1, (r.len + UK - 1) / UK);
        t_units += static_cast<long long>(n_rt) * p.kv_heads * (nt + kItemCost);
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
                const Req r = load_request(p, b);
                const int n_rt = (r.qlen * p.group + ROWS - 1) / ROWS, nt = whole ? 1 : max(1, (r.len + UK - 1) / UK) + kItemCost;
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
    place = whole ? kItemCost : s_place[3];
    }
    cur.j = max(0, place - kItemCost);
    cur.left = whole ? cur.nt : (u_end - u_begin) - max(0, kItemCost - place);      // of this run, from unit cur.j on
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
        d[6] = unit0 <= before + kItemCost ? 0 : 1;        // slot of the first owner's part: its run starts with this item (or inside its cost)
        d[0] = first_cut ? 1 : 0;
    }
    return true;
}

}  // namespace

}  // namespace rudder
