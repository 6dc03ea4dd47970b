// What the operators around the paged key-value cache share: the parameters of the cache and the record of bad
// indices that only the device can see.
#pragma once

#include <stdint.h>

#include "ptx.cuh"

namespace rudder {

// Codes of what a kernel found in the caller's device data (second word of rudder_device_status; the first is RUDDER_ERR_ARG).
constexpr int kBadPage = 911;        // page id outside [0, n_pages), or a cached page that was never assigned
constexpr int kBadLength = 912;      // length negative, beyond the page table, or more query rows than max_q / M
constexpr int kBadPosition = 913;    // position at or beyond n_pos
constexpr int kBadSlot = 914;        // slot at or beyond n_pages * page_size
constexpr int kNoPages = 915;        // more pages needed than the free list holds, or more columns than the table
constexpr int kNoRoom = 916;         // more new tokens than the slot map holds

// The access with the bad index is skipped; the context stays usable and the host reads the word.
__device__ __forceinline__ void record_bad_data(int what) {
    atomicExch(&g_device_status[1], what);
    atomicExch(&g_device_status[0], 1);   // RUDDER_ERR_ARG
}

// The cache as the kernels see it: strides in elements, page_size = 1 << page_shift.
struct CacheParams {
    uint8_t* k;
    uint8_t* v;
    int64_t page_stride, head_stride, token_stride;
    const float* k_scale;
    const float* v_scale;
    int n_pages, page_shift;
};

constexpr int kMaxKvHeads = 1024;

struct QkArgs {
    const uint16_t* X; int64_t ldx; int M;
    int heads, kv_heads;
    const float* q_weight; const float* k_weight; float eps;
    float one;                            // 1, see add2 in qk_norm_rope.cu
    const float* cos; const float* sin; int n_pos, rot;
    bool pairs;
    const int32_t* positions;             // or nullptr: every row is real (rot = 0)
    uint16_t* Q; int64_t ldq;
    uint16_t* K; int64_t ldk;             // keys to a buffer of their own, or ...
    CacheParams cache;                    // ... keys and values to the cache (slots != nullptr)
    const int64_t* slots;
};
struct AttnArgs {
    const uint16_t* Q; int64_t ldq; int M;
    uint16_t* O; int64_t ldo;
    float* lse;
    int heads, kv_heads, head_dim;
    CacheParams cache; bool e4m3;
    const int32_t* table; int64_t ld_table; int max_pages;
    const int32_t* kv_lens; const int32_t* q_starts;
    int B, max_q, causal;
    float scale;
    bool tma;                             // tensor maps over K and V: see attention_rows.cu
    CUtensorMap tm_k, tm_v;               // [pages][heads][tokens][channels], box of min(64, page size) tokens: bf16 64 channels, 128-byte swizzle; E4M3 whole rows as they lie
};

// A kernel that is launched early lives while the kernels in front of it still write.  Behind pdl_wait it sees what they wrote, but only by ordinary
// loads: what a caller may write on the stream (tables, lengths, scales, biases, angles) is not read through __ldg, which asks for memory that nobody
// writes while the kernel lives.  (Packed weights are complete when rudder_pack_weights returns.)
__device__ __forceinline__ void pdl_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

}  // namespace rudder
