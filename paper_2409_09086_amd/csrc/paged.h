// Internal launch interface of the rotary and paged-cache kernels.  Everything is asynchronous on the given HIP stream.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace infmllm {

struct RotaryFrequencies { double base, factor, trained, low, high, magnitude; };

// One launch over tokens x (query heads, key heads, value heads with pages); see rotary.hip.  T: uint16_t (bf16) or float.
template <typename T>
struct RotaryArgs {
    const T *q, *k, *v;                            // strides in elements between tokens
    T *q_out, *k_out;
    const T *q_weight, *k_weight;                  // null: no norm
    int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
    const int32_t* positions;                      // without pages
    const float2* table_cs;                        // [max_positions][dims / 2] (cos, sin)
    int tokens, heads, kv_heads, dims, half, max_positions;   // dims 0: nothing is turned; half: pairs (i, i + dims / 2)
    float eps;
    // with pages (see infmllm_batch_t)
    const int32_t *starts, *lens, *table;
    T *K, *V;
    int seqs, pages_per_seq, pages, page_shift;
};
template <typename T>
hipError_t launch_rotary(const RotaryArgs<T>& a, int head_dim, bool paged, hipStream_t st);
hipError_t launch_rotary_table(float* tab, int half_dims, int positions, const RotaryFrequencies& f, hipStream_t st);

// Attention over pages.
template <typename T>
struct PagedArgs {
    const T* q;                                    // [tokens][..]: q_stride elements between tokens
    const T *K, *V;                                // [pages][Hkv][1 << page_shift][D]
    T* out;                                        // [tokens][Hq][D]
    float* lse;                                    // [tokens][Hq] natural, or null
    const int32_t *starts, *lens, *table;
    int64_t q_stride;
    int seqs, tokens, pages_per_seq, pages, page_shift, Hq, Hkv, G, window;   // window 0: none
    uint32_t inv_g;                                // 2^32 / G + 1, rounded down (G > 1): see Unit::token
    float c;                                       // scale * log2(e)
};
// Partial results of units that several teams share (paged_work.h): two slots a team, and 2 * PAGED_TEAMS tickets, zero between launches.
struct PagedScratch { float* part; int* arrived; };
constexpr int PAGED_CUS = 256;                     // compute units: teams of a launch with one a CU
constexpr int PAGED_TEAMS = 8 * PAGED_CUS;         // most teams of a launch

// Few rows a unit: 16 or 32; max_new, max_len: the caller's bounds.
template <typename T>
hipError_t launch_paged_rows(const PagedArgs<T>& a, const PagedScratch& sc, int head_dim, int max_new, int max_len, hipStream_t st);
size_t paged_rows_scratch(int head_dim, int elt);  // bytes of PagedScratch::part
// The same for bf16 chunks of many rows, 256 a unit.
hipError_t launch_paged_fwd(const PagedArgs<uint16_t>& a, const PagedScratch& sc, int head_dim, hipStream_t st);
size_t paged_fwd_scratch(int head_dim);
// Both in one launch: the sequences of at most `few` rows (16), and the others.
hipError_t launch_paged_mixed(const PagedArgs<uint16_t>& a, const PagedScratch& sc, int head_dim, int few, hipStream_t st);
size_t paged_mixed_scratch(int head_dim);

}  // namespace infmllm
