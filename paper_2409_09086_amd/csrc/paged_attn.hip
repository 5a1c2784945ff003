// Attention of new tokens over a paged cache for gfx950, in plain arithmetic: one wavefront per (token, query head), 64 keys
// at a time, one pass with the running maximum and sum of the softmax.
#include "attn_rows.h"
#include "paged.h"

namespace infmllm {

namespace {

__device__ __forceinline__ float to_float(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ void from_float(uint16_t* p, float x) { *(__bf16*)p = (__bf16)x; }
__device__ __forceinline__ void from_float(float* p, float x) { *p = x; }

template <typename T, int D>
__device__ void plain_row(const PagedArgs<T>& a, int seq, int h, const T* q, int k0, int k1, int lane, float& m, float& l,
                          float (&o)[D / 64])
{
    constexpr int E = 16 / (int)sizeof(T);
    m = -__builtin_inff();
    l = 0.f;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) o[e] = 0.f;
    for (int j0 = k0; j0 < k1; j0 += 64) {
        const int j = j0 + lane;
        int page = -1;
        if (j < k1) page = a.table[(int64_t)seq * a.pages_per_seq + (j >> a.page_shift)];
        const bool seen = (unsigned)page < (unsigned)a.pages;
        const int64_t row = ((((int64_t)(seen ? page : 0) * a.Hkv + h) << a.page_shift) + (j & ((1 << a.page_shift) - 1))) * D;
        float s = -__builtin_inff();
        if (seen) {
            s = 0.f;
            for (int d = 0; d < D; d += E) {
                const u32x4 kx = *(const u32x4*)(a.K + row + d), qx = *(const u32x4*)(q + d);
                const T *kp = (const T*)&kx, *qp = (const T*)&qx;
#pragma unroll
                for (int e = 0; e < E; ++e) s = __builtin_fmaf(to_float(kp[e]), to_float(qp[e]), s);
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
        for (uint64_t left = __ballot(seen); left; left &= left - 1) {
            const int i = __builtin_ctzll(left);
            const float w = __shfl(p, i);
            const int64_t r = __shfl(row, i);
#pragma unroll
            for (int e = 0; e < D / 64; ++e) o[e] = __builtin_fmaf(w, to_float(a.V[r + 64 * e + lane]), o[e]);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(64)
paged_plain_kernel(PagedArgs<T> a)
{
    const int tok = blockIdx.x, hq = blockIdx.y, lane = threadIdx.x;
    int seq = 0;
    for (int s0 = 0; s0 < a.seqs; s0 += 64) {
        const int end = s0 + lane < a.seqs ? a.starts[s0 + lane + 1] : INT32_MAX;
        seq += __popcll(__ballot(end <= tok));
    }
    if (seq >= a.seqs) return;
    const int pos = max(a.lens[seq], 0) - (a.starts[seq + 1] - tok);
    const int64_t most = (int64_t)a.pages_per_seq << a.page_shift;
    const int k1 = (int)min((int64_t)max(pos + 1, 0), most), k0 = a.window > 0 ? max(0, pos + 1 - a.window) : 0;
    float m, l, o[D / 64];
    plain_row<T, D>(a, seq, hq / a.G, a.q + tok * a.q_stride + (int64_t)hq * D, k0, k1, lane, m, l, o);
    const int64_t at = (int64_t)tok * a.Hq + hq;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) from_float(a.out + at * D + 64 * e + lane, l == 0.f ? 0.f : o[e] / l);
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : 0.6931471805599453f * (m + __builtin_log2f(l));
}

}  // namespace

template <typename T>
hipError_t launch_paged_attend(const PagedArgs<T>& a, int head_dim, int max_new, int max_len, hipStream_t st)
{
    if (a.tokens <= 0) return hipSuccess;
    const dim3 grid((unsigned)a.tokens, (unsigned)a.Hq), block(64);
    if (head_dim == 128) hipLaunchKernelGGL((paged_plain_kernel<T, 128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((paged_plain_kernel<T, 64>), grid, block, 0, st, a);
    return hipGetLastError();
}
template hipError_t launch_paged_attend<uint16_t>(const PagedArgs<uint16_t>&, int, int, int, hipStream_t);
template hipError_t launch_paged_attend<float>(const PagedArgs<float>&, int, int, int, hipStream_t);

}  // namespace infmllm
