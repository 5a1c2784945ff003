// Device helpers shared by the attention kernels over pages (paged_rows.hip, paged_fwd.hip).
#pragma once
#include "attn_rows.h"
#include "paged_work.h"

namespace infmllm {
namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef const __attribute__((address_space(4))) int32_t const_i32;   // uniform loads of it are scalar: they don't wait for tiles in flight

__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float to_float(float x) { return x; }

constexpr float LN2 = 0.6931471805599453f;
__device__ __forceinline__ float natural_lse(float m, float l) { return l == 0.f ? -__builtin_inff() : LN2 * (m + __builtin_log2f(l)); }
// what a sum of weights divides the output by: rows that see no key become 0
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.0f / l; }

template <typename T>
__device__ __forceinline__ int page_of(const PagedArgs<T>& a, int seq, int key)
{
    return ((const_i32*)a.table)[(int64_t)seq * a.pages_per_seq + (key >> a.page_shift)];
}
// elements ahead of row `key` of its page, which is `page`
template <typename T, int D>
__device__ __forceinline__ int64_t row_at(const PagedArgs<T>& a, int page, int h, int key)
{
    return ((((int64_t)page * a.Hkv + h) << a.page_shift) + (key & ((1 << a.page_shift) - 1))) * D;
}

// One row over keys k0 .. k1 - 1 in plain arithmetic, 64 keys at a time, a key to a lane: what a piece does over whose sums are not
// finite, or which met a page that does not exist.  Matrix products multiply hidden values by 0, which leaves no trace of
// them unless they are not finite; here nothing hidden is touched.  References in base 2.
template <typename T, int D>
__device__ __forceinline__ void plain_row(const PagedArgs<T>& a, int seq, int h, const T* q, int k0, int k1, int lane, float& m,
                                          float& l, float (&o)[D / 64])
{
    constexpr int E = 16 / (int)sizeof(T);
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) o[e] = 0.f;
#pragma nounroll
    for (int j0 = k0; j0 < k1; j0 += 64) {
        const int j = j0 + lane;
        int page = -1;
        if (j < k1) page = a.table[(int64_t)seq * a.pages_per_seq + (j >> a.page_shift)];
        const bool seen = (unsigned)page < (unsigned)a.pages;
        const int64_t row = row_at<T, D>(a, seen ? page : 0, h, j);
        float s = -__builtin_inff();
        if (seen) {
            s = 0.f;
#pragma nounroll
            for (int d = 0; d < D; d += E) {
                const u32x4 kx = *(const u32x4*)(a.K + row + d), qx = *(const u32x4*)(q + d);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const uint32_t kw = kx[e * sizeof(T) / 4], qw = qx[e * sizeof(T) / 4];
                    if constexpr (sizeof(T) == 2) s = __builtin_fmaf(to_float((uint16_t)(kw >> (16 * (e & 1)))), to_float((uint16_t)(qw >> (16 * (e & 1)))), s);
                    else s = __builtin_fmaf(__uint_as_float(kw), __uint_as_float(qw), s);
                }
            }
            s *= a.c;
        }
        float mx = s;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) mx = fmaxf(mx, __shfl_xor(mx, x));
        const float mn = fmaxf(m, mx), mu = mn == -__builtin_inff() ? 0.f : mn;
        const float alpha = fast_exp2(m - mu), p = seen ? fast_exp2(s - mu) : 0.f;
        float sum = p;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        m = mn;
        l = l * alpha + sum;
#pragma unroll
        for (int e = 0; e < D / 64; ++e) o[e] *= alpha;
#pragma nounroll
        for (uint64_t left = __ballot(seen); left; left &= left - 1) {
            const int i = __builtin_ctzll(left);
            const float w = __shfl(p, i);
            const int64_t r = __shfl(row, i);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) o[e] = __builtin_fmaf(w, to_float(a.V[r + 64 * e + lane]), o[e]);
        }
    }
}

// The query of row r of a unit.
template <typename T, int D>
__device__ __forceinline__ const T* query_of(const PagedArgs<T>& a, const Unit& u, int r)
{
    int head;
    const int tok = u.token(r, head);
    return a.q + (int64_t)(u.first + tok) * a.q_stride + (int64_t)(u.h * u.G + head) * D;
}
// The same row of out and lse: its number among [tokens][Hq].
template <typename T>
__device__ __forceinline__ int64_t result_of(const PagedArgs<T>& a, const Unit& u, int r)
{
    int head;
    const int tok = u.token(r, head);
    return (int64_t)(u.first + tok) * a.Hq + u.h * u.G + head;
}
// Keys of runs r0 .. r1 - 1 of a unit that its row r sees: k0 .. k1 - 1.
template <int RUN>
__device__ __forceinline__ void visible(const Unit& u, int window, int r, int& k0, int& k1)
{
    const int pos = u.pos(r), at = u.kb & ~(RUN - 1);
    k0 = max(max(window > 0 ? pos + 1 - window : 0, at + u.r0 * RUN), u.kb);
    k1 = min(min(pos + 1, at + u.r1 * RUN), u.ke);
}

// Memory of a team's slot, past the caches of the XCDs (see buffer_to_lds).
__device__ __forceinline__ auto slot_rsrc(const float* part, int slot, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((char*)part + (size_t)slot * bytes, 0, bytes, 0x00020000);
}
constexpr int SC1 = 16;

}  // namespace
}  // namespace infmllm
