// Rotary positions, head norms and the append to a paged cache for gfx950.
//
// One pass over the rows: a head's row of x is normed (y = x w / sqrt(mean x^2 + eps)), its pairs (a, b) are turned by
// p f[i] and the row is written where it belongs: beside the input, or, for a new token's keys and values, into its page.
// Nothing is computed twice and nothing but the rows moves, so the pass is bound by memory.
//
// D / 16 lanes share a row, two runs of eight elements each, such that a pair never leaves its lane, the norm's sum is two or
// three lane exchanges, and the lanes' runs stand side by side in memory (sixteen elements in a row a lane, every other 16
// bytes an instruction, took 31.2 us for the neighbouring pairs of 4099 tokens of 64 heads of 128; so 29.5, now 26.3 = 5.1 TB/s).
// Half-split: the runs lie in the two halves of the turned part, or of what passes behind it; neighbouring pairs: of the row,
// four pairs in each.  A thread goes through HPT heads of its token, all requested before the first is used, with the one
// set of cosines.
//
// The table holds every position ((cos, sin) in floats, computed in doubles): 512 bytes a token beside the 20 KB that a
// token of 32 + 8 heads of 128 reads and writes.
#include <algorithm>

#include "attn_rows.h"
#include "paged.h"

namespace infmllm {

namespace {

// PAST: past the caches, which a large pass would only sweep
template <bool PAST>
__device__ __forceinline__ void store16(void* p, u32x4 v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, (u32x4*)p);
    else *(u32x4*)p = v;
}

// eight consecutive elements
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
    u32x4 raw;
    __device__ __forceinline__ void load(const uint16_t* p) { raw = *(const u32x4*)p; }
    template <bool PAST> __device__ __forceinline__ void store(uint16_t* p) const { store16<PAST>(p, raw); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            v[2 * w] = __uint_as_float(raw[w] << 16);
            v[2 * w + 1] = __uint_as_float(raw[w] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = (__bf16)v[e];
        raw = __builtin_bit_cast(u32x4, b);
    }
};
template <> struct Eight<float> {
    f32x4 lo, hi;
    __device__ __forceinline__ void load(const float* p) { lo = *(const f32x4*)p; hi = *(const f32x4*)(p + 4); }
    template <bool PAST> __device__ __forceinline__ void store(float* p) const
    {
        store16<PAST>(p, __builtin_bit_cast(u32x4, lo));
        store16<PAST>(p + 4, __builtin_bit_cast(u32x4, hi));
    }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[e] = lo[e]; v[4 + e] = hi[e]; }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) { lo[e] = v[e]; hi[e] = v[4 + e]; }
    }
};

// Sum over the 4 or 8 consecutive lanes of a row, in all of them.
template <int N>
__device__ __forceinline__ float row_sum(float x)
{
    x += dpp<0xB1>(x);                             // quad_perm [1,0,3,2]
    x += dpp<0x4E>(x);                             // quad_perm [2,3,0,1]
    if (N == 8) x += dpp<0x141>(x);                // row_half_mirror
    return x;
}

// PAGED: positions come from the batch, keys go to their pages and values with them.
template <typename T, int D, int HPT, bool PAGED>
__global__ void __launch_bounds__(256)
rotary_kernel(RotaryArgs<T> a)
{
    constexpr int LPR = D / 16;                    // lanes per row
    const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int tok = (int)min(idx / LPR, (int64_t)a.tokens), c = threadIdx.x % LPR;
    // which tensor, which heads
    const int qg = (a.heads + HPT - 1) / HPT, kg = (a.kv_heads + HPT - 1) / HPT;
    int grp = blockIdx.y, what = 0, heads = a.heads;
    if (grp >= qg) { grp -= qg; what = 1; heads = a.kv_heads; }
    if (PAGED && what == 1 && grp >= kg) { grp -= kg; what = 2; }
    const int h0 = grp * HPT;
    const bool exists = tok < a.tokens;

    const T* src = what == 0 ? a.q + (int64_t)tok * a.q_stride : what == 1 ? a.k + (int64_t)tok * a.k_stride : a.v + (int64_t)tok * a.v_stride;
    const T* weight = what == 0 ? a.q_weight : what == 1 ? a.k_weight : nullptr;
    // the lane's two runs of eight elements, and which of them are turned
    const int part = a.half ? (16 * c < a.dims ? a.dims : D - a.dims) : D, at0 = a.half && 16 * c >= a.dims ? a.dims : 0;
    const int ea = at0 + 8 * (a.half ? c - at0 / 16 : c), eb = ea + part / 2;
    const bool turn_a = what < 2 && ea < a.dims, turn_b = what < 2 && eb < a.dims;

    Eight<T> xa[HPT], xb[HPT];
    if (exists) {
#pragma unroll
        for (int u = 0; u < HPT; ++u) {
            const int h = min(h0 + u, heads - 1);
            xa[u].load(src + h * D + ea);
            xb[u].load(src + h * D + eb);
        }
    }
    int pos = 0, seq = 0;
    if constexpr (PAGED) {
        // the sequences that end at or before a token: a wavefront's tokens are a few consecutive ones
        const int lane = threadIdx.x & 63, t0 = __builtin_amdgcn_readfirstlane(tok);
        for (int s0 = 0; s0 < a.seqs; s0 += 64) {
            const int end = s0 + lane < a.seqs ? a.starts[s0 + lane + 1] : INT32_MAX;
#pragma unroll
            for (int i = 0; i < 64 / LPR; ++i) {
                const int n = __popcll(__ballot(end <= t0 + i));
                if (tok == t0 + i) seq += n;
            }
        }
        if (!exists || seq >= a.seqs) return;
        pos = max(a.lens[seq], 0) - (a.starts[seq + 1] - tok);
        if (pos < 0) return;                       // more new tokens than the cache holds
    } else {
        if (!exists) return;
        pos = a.positions[tok];
    }
    T* dst;
    int64_t hstride = D;
    if (what == 0) {
        dst = a.q_out + (int64_t)tok * a.q_out_stride;
    } else if constexpr (PAGED) {
        const int at = pos >> a.page_shift;
        if (at >= a.pages_per_seq) return;
        const int page = a.table[(int64_t)seq * a.pages_per_seq + at];
        if ((unsigned)page >= (unsigned)a.pages) return;
        hstride = (int64_t)D << a.page_shift;
        dst = (what == 1 ? a.K : a.V) + (int64_t)page * a.kv_heads * hstride + (int64_t)(pos & ((1 << a.page_shift) - 1)) * D;
    } else {
        dst = a.k_out + (int64_t)tok * a.k_out_stride;
    }
    // half-split: of pairs ea .. ea + 7; neighbouring pairs: of ea / 2 .. + 3 and eb / 2 .. + 3
    float cs[8], sn[8];
    if (turn_a || turn_b) {
        const bool known = (unsigned)pos < (unsigned)a.max_positions;
        const float2* row = a.table_cs + (int64_t)(known ? pos : 0) * (a.dims / 2);
        const f32x4 *ta = (const f32x4*)(row + (a.half ? ea : ea / 2)), *tb = a.half ? ta + 2 : (const f32x4*)(row + (turn_b ? eb / 2 : ea / 2));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 v = i < 2 ? ta[i] : tb[i - 2];
            cs[2 * i] = v[0]; sn[2 * i] = v[1]; cs[2 * i + 1] = v[2]; sn[2 * i + 1] = v[3];
        }
        if (!known) cs[0] = cs[1] = cs[2] = cs[3] = cs[4] = cs[5] = cs[6] = cs[7] = __builtin_nanf("");
    }
    float wa[8], wb[8];
    if (weight) {
        Eight<T> w;
        w.load(weight + ea);
        w.get(wa);
        w.load(weight + eb);
        w.get(wb);
    }
#pragma unroll
    for (int u = 0; u < HPT; ++u) {
        if (HPT > 1 && h0 + u >= heads) break;
        Eight<T> ra = xa[u], rb = xb[u];
        if (weight || turn_a || turn_b) {
            float x[8], y[8];
            ra.get(x);
            rb.get(y);
            if (weight) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], x[e], __builtin_fmaf(y[e], y[e], sum));
                const float r = rsqrtf(__builtin_fmaf(row_sum<LPR>(sum), 1.0f / D, a.eps));
#pragma unroll
                for (int e = 0; e < 8; ++e) { x[e] = x[e] * r * wa[e]; y[e] = y[e] * r * wb[e]; }
            }
            auto turn = [&](float& p, float& q, int i) {
                const float p0 = p, q0 = q;
                p = __builtin_fmaf(p0, cs[i], -(q0 * sn[i]));
                q = __builtin_fmaf(q0, cs[i], p0 * sn[i]);
            };
            if (a.half) {
                if (turn_a) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) turn(x[e], y[e], e);
                }
            } else {
                if (turn_a) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) turn(x[2 * e], x[2 * e + 1], e);
                }
                if (turn_b) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) turn(y[2 * e], y[2 * e + 1], 4 + e);
                }
            }
            ra.set(x);
            rb.set(y);
        }
        ra.template store<(HPT > 1)>(dst + (h0 + u) * hstride + ea);
        rb.template store<(HPT > 1)>(dst + (h0 + u) * hstride + eb);
    }
}

__global__ void __launch_bounds__(256)
rotary_table_kernel(float2* __restrict__ tab, int half_dims, int64_t entries, RotaryFrequencies f)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= entries) return;
    const double pair = (double)(i % half_dims), pos = (double)(i / half_dims);
    double w = pow(f.base, -pair / half_dims), g = 0.0;
    if (f.trained > 0.0) g = fmin(fmax((f.trained * w * (0.5 / M_PI) - f.low) / (f.high - f.low), 0.0), 1.0);
    w *= g + (1.0 - g) / f.factor;
    double s, c;
    sincos(pos * w, &s, &c);
    tab[i] = float2{(float)(f.magnitude * c), (float)(f.magnitude * s)};
}

template <typename T, int D, bool PAGED>
hipError_t launch(const RotaryArgs<T>& a, hipStream_t st)
{
    const dim3 block(256);
    const unsigned gx = (unsigned)(((int64_t)a.tokens * (D / 16) + 255) / 256);
    auto groups = [&](int hpt) { return (unsigned)((a.heads + hpt - 1) / hpt + (PAGED ? 2 : 1) * ((a.kv_heads + hpt - 1) / hpt)); };
    // Heads a thread: few tokens want threads, many want their cosines read once and their loads in a row.  us with 1 / 4 / 8 heads, the
    // latter two with stores past the caches: 4099 tokens of 64 heads of 128 normed and turned 31.7 / 27.9 / 26.0, 8192 of 40 turned 39.2 / 33.3 / 33.8,
    // 4236 into their pages 25.1 / 19.0 / 19.3 (22.2 with stores into the caches; the attention that follows takes as
    // long).  The kernel alone with 1 / 8, 40 heads of 128: 2000 tokens (315 workgroups of 8) turned 10.3 / 9.8, normed too 11.0 / 10.6, into their pages
    // 11.6 / 10.8; 1000 (160) 6.3 / 6.2, 7.0 / 7.2, 7.6 / 7.1; 500 (80) 4.5 / 5.7, 4.7 / 6.4, 4.9 / 5.9.  In single precision a head is as many loads as two,
    // and one a thread is enough: 2000 17.5 / 25.9, 18.8 / 23.3, 22.1 / 28.1; 4096 35.4 / 41.1, 37.6 / 49.0, 42.0 / 55.4; 16000 160 / 177, 151 / 180, 189 / 230.
    if constexpr (sizeof(T) == 2) {
        if ((int64_t)gx * groups(8) >= 256) {
            hipLaunchKernelGGL((rotary_kernel<T, D, 8, PAGED>), dim3(gx, groups(8)), block, 0, st, a);
            return hipGetLastError();
        }
    }
    hipLaunchKernelGGL((rotary_kernel<T, D, 1, PAGED>), dim3(gx, groups(1)), block, 0, st, a);
    return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t launch_rotary(const RotaryArgs<T>& a, int head_dim, bool paged, hipStream_t st)
{
    if (a.tokens <= 0) return hipSuccess;
    if (head_dim == 128) return paged ? launch<T, 128, true>(a, st) : launch<T, 128, false>(a, st);
    return paged ? launch<T, 64, true>(a, st) : launch<T, 64, false>(a, st);
}
template hipError_t launch_rotary<uint16_t>(const RotaryArgs<uint16_t>&, int, bool, hipStream_t);
template hipError_t launch_rotary<float>(const RotaryArgs<float>&, int, bool, hipStream_t);

hipError_t launch_rotary_table(float* tab, int half_dims, int positions, const RotaryFrequencies& f, hipStream_t st)
{
    const int64_t n = (int64_t)half_dims * positions;
    hipLaunchKernelGGL(rotary_table_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (float2*)tab, half_dims, n, f);
    return hipGetLastError();
}

}  // namespace infmllm
