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
    l = -0.0f;                                                 // see NONE
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
        if (__any(seen)) l = l * alpha + sum;
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

// A sum of weights of 0 is one of none or one of weights that all are exp(-inf).  Rows that see no key become 0, those that see only logits of -inf
// NaN, as every softmax of them is: the sum of a row that sees no key is -0, which weights of the one kind leave as it is
// and those of the other kind make +0, piece by piece.
constexpr float NONE = -0.0f;
__device__ __forceinline__ float inverse(float l) { return __float_as_uint(l) == 0x80000000u ? 0.f : 1.0f / l; }   // of +0: 0 * inf
// the sum of row r over a piece whose pages all exist (hidden keys have added +0)
template <int RUN>
__device__ __forceinline__ float sum_of(const Unit& u, int window, int r, float l)
{
    if (__builtin_expect(l != 0.f, 1)) return l;
    int k0, k1;
    visible<RUN>(u, window, r, k0, k1);
    return k0 < k1 ? 0.f : NONE;
}

// Memory of a team's slot, past the caches of the XCDs (see buffer_to_lds).
__device__ __forceinline__ auto slot_rsrc(const float* part, int slot, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((char*)part + (size_t)slot * bytes, 0, bytes, 0x00020000);
}
constexpr int SC1 = 16;

// ---- few query rows: see paged_rows.hip

// A wavefront's direct loads of a run of keys into `dst` (K) and `dst` + RUN bytes (V).
template <typename T, int D, int KEYS>
struct PageRuns {
    static constexpr int ROWB = D * (int)sizeof(T), RUN = KEYS * ROWB, HALVES = KEYS / 16, HALF = 16 * ROWB, NL = HALF / 1024,
                         RPL = 1024 / ROWB, LOADS = 2 * HALVES * NL;
    typedef Tile<T, D> Swz;
    const PagedArgs<T>& a;
    int seq, h, kb, ke, lrow, lpos;
    int page[HALVES];
    bool bad = false;
    __device__ __forceinline__ PageRuns(const PagedArgs<T>& a_, int lane) : a(a_), lrow(lane / (ROWB / 16)), lpos(lane % (ROWB / 16)) {}
    __device__ __forceinline__ void start(const Unit& u) { seq = u.seq; h = u.h; kb = u.kb; ke = u.ke; bad = false; }
    // the half's first key, moved to the nearest half that holds a key of the unit
    __device__ __forceinline__ int half_key(int k0, int i) const { return min(max(k0 + 16 * i, kb & ~15), (ke - 1) & ~15); }
    __device__ __forceinline__ void look_up(int k0)
    {
#pragma unroll
        for (int i = 0; i < HALVES; ++i) page[i] = page_of(a, seq, half_key(k0, i));
    }
    __device__ __forceinline__ void load(int k0, char* dst)    // of the run that was looked up last
    {
        const bool whole = k0 >= kb && k0 + KEYS <= ke;
#pragma unroll
        for (int i = 0; i < HALVES; ++i) {
            const bool there = (unsigned)page[i] < (unsigned)a.pages;
            bad |= !there;
            const int key = half_key(k0, i);
            const int64_t at = row_at<T, D>(a, there ? page[i] : 0, h, key);
            const T *kp = a.K + at, *vp = a.V + at;
            char* to = dst + i * HALF;
            if (whole) {
#pragma unroll
                for (int u = 0; u < NL; ++u)
                    buffer_to_lds(kp, HALF, to + u * 1024, lrow * ROWB + Swz::k(u * RPL + lrow, lpos) * 16, u * RPL * ROWB);
#pragma unroll
                for (int u = 0; u < NL; ++u)
                    buffer_to_lds(vp, HALF, to + RUN + u * 1024, lrow * ROWB + Swz::v(u * RPL + lrow, lpos) * 16, u * RPL * ROWB);
            } else {
#pragma unroll
                for (int u = 0; u < NL; ++u) {
                    const int r = u * RPL + lrow, from = min(max(k0 + 16 * i + r, kb), ke - 1) - key;
                    buffer_to_lds(kp, HALF, to + u * 1024, from * ROWB + Swz::k(r, lpos) * 16);
                    buffer_to_lds(vp, HALF, to + RUN + u * 1024, from * ROWB + Swz::v(r, lpos) * 16);
                }
            }
        }
    }
};

template <typename T, int D, int NRB> struct RowsKernel;

// bf16
template <int D, int NRB>
struct RowsKernel<uint16_t, D, NRB> {
    typedef uint16_t T;
    static constexpr int KEYS = 32, ROWS = 16 * NRB;
    typedef PageRuns<T, D, KEYS> Runs;
    typedef RowsCfg<D, NRB> C;
    static constexpr int STAGE = 2 * Runs::RUN;

    f32x4 o[NRB][C::NC];
    float m_ref[NRB], m_use[NRB], lsum[NRB];

    // np runs of KEYS keys from k_first on, `step` keys apart, through NST buffers of STAGE bytes
    template <int NST>
    __device__ __forceinline__ void sweep(const PagedArgs<T>& a, const Unit& u, Runs& runs, char* mine, int k_first, int np, int step, int lane)
    {
        const int c16 = lane & 15, g4 = lane >> 4;
        if (np > 0) {
            runs.look_up(k_first);
            runs.load(k_first, mine);
            if (np > 1) runs.look_up(k_first + step);
            if (NST == 2 && np > 1) {
                runs.load(k_first + step, mine + STAGE);
                if (np > 2) runs.look_up(k_first + 2 * step);
            }
        }
        bf16x8 qf[NRB][C::NS];
        int hi[NRB], lo[NRB];
#pragma unroll
        for (int x = 0; x < NRB; ++x) {
            const int row = min(16 * x + c16, u.rows - u.row0 - 1);
            const T* qp = query_of<T, D>(a, u, row) + 8 * g4;
            const int pos = u.pos(row);
            hi[x] = min(pos, u.ke - 1);                        // a table may end ahead of it
            lo[x] = a.window > 0 ? pos + 1 - a.window : 0;
#pragma unroll
            for (int s = 0; s < C::NS; ++s) qf[x][s] = as_bf16x8(*(const u32x4*)(qp + 32 * s));
#pragma unroll
            for (int b = 0; b < C::NC; ++b) o[x][b] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_ref[x] = -__builtin_inff(); m_use[x] = 0.f; lsum[x] = 0.f;
        }
        const int hi0 = __builtin_amdgcn_readfirstlane(hi[0]);                        // of the unit's first row
        const int lo1 = __builtin_amdgcn_readlane(lo[NRB - 1], 15);                   // of its last
        uint32_t kaddr[C::NS], vaddr[C::NC];                   // see attn_rows_kernel
        {
            const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)mine;
            const int vkey = 4 * g4 + (c16 >> 2), q4 = c16 & 3;
#pragma unroll
            for (int s = 0; s < C::NS; ++s) kaddr[s] = base + c16 * C::ROWB + (((4 * s + g4) ^ swz_k<D>(c16)) * 16);
#pragma unroll
            for (int b = 0; b < C::NC; ++b)
                vaddr[b] = base + C::RUN + vkey * C::ROWB + (((2 * b + (q4 >> 1)) ^ swz_v<D>(vkey)) * 16) + 8 * (q4 & 1);
        }
        for (int p = 0; p < np; ++p) {
            const int k0 = k_first + p * step;
            const uint32_t stage = NST == 2 && (p & 1) ? STAGE : 0;
            if (NST == 2 && p + 1 < np) wait_loads<Runs::LOADS>();             // this run has landed, the next one may be on its way
            else wait_loads<0>();
            bf16x8 kf[2][C::NS];
            bf16x4 vlo[C::NC], vhi[C::NC];
#pragma unroll
            for (int s = 0; s < C::NS; ++s) {
                kf[0][s] = rw_read_b128<0>(kaddr[s] + stage);
                kf[1][s] = rw_read_b128<16 * C::ROWB>(kaddr[s] + stage);
            }
#pragma unroll
            for (int b = 0; b < C::NC; ++b) {
                vlo[b] = rw_read_tr16<0>(vaddr[b] + stage);
                vhi[b] = rw_read_tr16<16 * C::ROWB>(vaddr[b] + stage);
            }
            // reads return in order: K has arrived when at most the V reads are outstanding (the counter ends at 15)
            asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(kf[0][0]), "+v"(kf[1][0]), "+v"(kf[0][1]), "+v"(kf[1][1])
                         : "n"(2 * C::NC < 15 ? 2 * C::NC : 15));
            if constexpr (C::NS == 4) asm volatile("" : "+v"(kf[0][2]), "+v"(kf[1][2]), "+v"(kf[0][3]), "+v"(kf[1][3]));
            f32x4 S[NRB][2];
#pragma unroll
            for (int s = 0; s < C::NS; ++s)
#pragma unroll
                for (int x = 0; x < NRB; ++x)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
                        S[x][kb] = mfma16(kf[kb][s], qf[x][s], s == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : S[x][kb]);
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vlo[0]), "+v"(vhi[0]), "+v"(vlo[1]), "+v"(vhi[1]), "+v"(vlo[2]), "+v"(vhi[2]),
                         "+v"(vlo[3]), "+v"(vhi[3])::"memory");
            if constexpr (C::NC == 8)
                asm volatile("" : "+v"(vlo[4]), "+v"(vhi[4]), "+v"(vlo[5]), "+v"(vhi[5]), "+v"(vlo[6]), "+v"(vhi[6]), "+v"(vlo[7]), "+v"(vhi[7]));
            // the stage has been read: its next run goes there
            if (p + NST < np) {
                runs.load(k0 + NST * step, mine + stage);
                if (p + NST + 1 < np) runs.look_up(k0 + (NST + 1) * step);
            }
            bf16x8 pf[NRB][2];
            const bool masked = k0 + KEYS - 1 > hi0 || k0 < lo1;
#pragma unroll
            for (int x = 0; x < NRB; ++x) {
                if (masked) {
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = k0 + 16 * kb + 4 * g4 + i;
                            if (key > hi[x] || key < lo[x]) S[x][kb][i] = -__builtin_inff();
                        }
                }
                float mx = fmaxf(fmaxf(fmaxf(S[x][0][0], S[x][0][1]), fmaxf(S[x][0][2], S[x][0][3])),
                                 fmaxf(fmaxf(S[x][1][0], S[x][1][1]), fmaxf(S[x][1][2], S[x][1][3])));
                mx = groups_max(mx) * a.c;
                if (__any(mx > m_ref[x] + RESCALE_TAU)) {
                    const float m_new = fmaxf(m_ref[x], mx);
                    const float mu = (m_new == -__builtin_inff()) ? 0.f : m_new;
                    const float alpha = fast_exp2(m_ref[x] - mu);          // m_ref = -inf gives 0
                    m_ref[x] = m_new;
                    m_use[x] = mu;
                    lsum[x] *= alpha;
#pragma unroll
                    for (int b = 0; b < C::NC; ++b) o[x][b] *= alpha;
                }
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = fast_exp2(__builtin_fmaf(S[x][kb][i], a.c, -m_use[x]));
                        lsum[x] += w;
                        const __bf16 first = (__bf16)w;
                        pf[x][0][4 * kb + i] = first;
                        pf[x][1][4 * kb + i] = (__bf16)(w - (float)first);
                    }
            }
#pragma unroll
            for (int b = 0; b < C::NC; ++b) {
                const bf16x8 vf = __builtin_shufflevector(vlo[b], vhi[b], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                for (int term = 0; term < 2; ++term)
#pragma unroll
                    for (int x = 0; x < NRB; ++x) o[x][b] = mfma16(vf, pf[x][term], o[x][b]);
            }
        }
    }
    __device__ __forceinline__ bool finite() const
    {
        float z = 0.f;
#pragma unroll
        for (int x = 0; x < NRB; ++x)
#pragma unroll
            for (int b = 0; b < C::NC; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = __builtin_fmaf(o[x][b][i], 0.f, z);
        return !__any(z != 0.f);
    }
    // put(row of the unit, 16-byte piece of its output, value); stat(row, m, l)
    template <class P, class S> __device__ __forceinline__ void leave(int rows, int lane, P put, S stat) const
    {
        const int c16 = lane & 15, g4 = lane >> 4;
#pragma unroll
        for (int x = 0; x < NRB; ++x) {
            const float l = groups_sum(lsum[x]);
            if (16 * x + c16 < rows) {
                if (g4 == 0) stat(16 * x + c16, m_ref[x], l);
#pragma unroll
                for (int b = 0; b < C::NC; ++b) put(16 * x + c16, 4 * b + g4, o[x][b]);
            }
        }
    }
};

// single precision: 16x16x4 products; step e of piece j contracts head dimensions 16j + 4g + e of lane group g, step i of the
// second product keys 4g + i, and a lane's bytes of a V row are its operands of D / 16 column blocks (see attn_f32.hip)
template <int D, int NRB>
struct RowsKernel<float, D, NRB> {
    typedef float T;
    static constexpr int KEYS = 16, ROWS = 16 * NRB;
    typedef PageRuns<T, D, KEYS> Runs;
    static constexpr int ROWB = Runs::ROWB, STAGE = 2 * Runs::RUN;
    static constexpr int NJ = D / 16, VW = D / 16, VP = VW / 4;

    f32x4 o[NRB][NJ];                                          // block b: lane (row c16, group g4) holds columns VW (4 g4 + i) + b
    float m_ref[NRB], m_use[NRB], lsum[NRB];

    static __device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

    template <int NST>
    __device__ __forceinline__ void sweep(const PagedArgs<T>& a, const Unit& u, Runs& runs, char* mine, int k_first, int np, int step, int lane)
    {
        static_assert(NST == 1, "one buffer");
        const int c16 = lane & 15, g4 = lane >> 4;
        if (np > 0) {
            runs.look_up(k_first);
            runs.load(k_first, mine);
            if (np > 1) runs.look_up(k_first + step);
        }
        f32x4 qf[NRB][NJ];
        int hi[NRB], lo[NRB];
#pragma unroll
        for (int x = 0; x < NRB; ++x) {
            const int row = min(16 * x + c16, u.rows - u.row0 - 1), pos = u.pos(row);
            hi[x] = min(pos, u.ke - 1);                        // a table may end ahead of it
            lo[x] = a.window > 0 ? pos + 1 - a.window : 0;
            const float* qp = query_of<T, D>(a, u, row) + 4 * g4;
#pragma unroll
            for (int j = 0; j < NJ; ++j) qf[x][j] = *(const f32x4*)(qp + 16 * j);
#pragma unroll
            for (int b = 0; b < NJ; ++b) o[x][b] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_ref[x] = -__builtin_inff(); m_use[x] = 0.f; lsum[x] = 0.f;
        }
        const int hi0 = __builtin_amdgcn_readfirstlane(hi[0]), lo1 = __builtin_amdgcn_readlane(lo[NRB - 1], 15);
        const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)mine;
        uint32_t kaddr[NJ], vaddr[VP];
#pragma unroll
        for (int j = 0; j < NJ; ++j) kaddr[j] = base + c16 * ROWB + Runs::Swz::k(c16, 4 * j + g4) * 16;
#pragma unroll
        for (int x = 0; x < VP; ++x) vaddr[x] = base + Runs::RUN + 4 * g4 * ROWB + Runs::Swz::v(0, VP * c16 + x) * 16;
        for (int p = 0; p < np; ++p) {
            const int k0 = k_first + p * step;
            wait_loads<0>();
            f32x4 kf[NJ], vf[4][VP];
#pragma unroll
            for (int j = 0; j < NJ; ++j) kf[j] = rw_read_f32x4<0>(kaddr[j]);
            static_for<0, 4>([&](auto I) {
                constexpr int i = decltype(I)::value;
#pragma unroll
                for (int x = 0; x < VP; ++x) vf[i][x] = rw_read_f32x4<i * ROWB>(vaddr[x]);
            });
            asm volatile("s_waitcnt lgkmcnt(%4)" : "+v"(kf[0]), "+v"(kf[1]), "+v"(kf[2]), "+v"(kf[3]) : "n"(4 * VP));
            if constexpr (NJ == 8) asm volatile("" : "+v"(kf[4]), "+v"(kf[5]), "+v"(kf[6]), "+v"(kf[7]));
            f32x4 S[NRB][2];
#pragma unroll
            for (int j = 0; j < NJ; j += 2)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int x = 0; x < NRB; ++x)
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            S[x][t] = mfma(kf[j + t][e], qf[x][j + t][e], j == 0 && e == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : S[x][t]);
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vf[0][0]), "+v"(vf[1][0]), "+v"(vf[2][0]), "+v"(vf[3][0])::"memory");
            if constexpr (VP == 2) asm volatile("" : "+v"(vf[0][VP - 1]), "+v"(vf[1][VP - 1]), "+v"(vf[2][VP - 1]), "+v"(vf[3][VP - 1]));
            if (p + 1 < np) {
                runs.load(k0 + step, mine);
                if (p + 2 < np) runs.look_up(k0 + 2 * step);
            }
            const bool masked = k0 + KEYS - 1 > hi0 || k0 < lo1;
            float w[NRB][4];
#pragma unroll
            for (int x = 0; x < NRB; ++x) {
                float s[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = (S[x][0][i] + S[x][1][i]) * a.c;
                if (masked) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = k0 + 4 * g4 + i;
                        if (key > hi[x] || key < lo[x]) s[i] = -__builtin_inff();
                    }
                }
                const float mx = groups_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
                if (__any(mx > m_ref[x] + RESCALE_TAU)) {
                    const float m_new = fmaxf(m_ref[x], mx);
                    const float mu = (m_new == -__builtin_inff()) ? 0.f : m_new;
                    const float alpha = fast_exp2(m_ref[x] - mu);
                    m_ref[x] = m_new;
                    m_use[x] = mu;
                    lsum[x] *= alpha;
#pragma unroll
                    for (int b = 0; b < NJ; ++b) o[x][b] *= alpha;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[x][i] = fast_exp2(s[i] - m_use[x]);
                    lsum[x] += w[x][i];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < NJ; ++b)
#pragma unroll
                    for (int x = 0; x < NRB; ++x) o[x][b] = mfma(vf[i][b / 4][b % 4], w[x][i], o[x][b]);
        }
    }
    __device__ __forceinline__ bool finite() const
    {
        float z = 0.f;
#pragma unroll
        for (int x = 0; x < NRB; ++x)
#pragma unroll
            for (int b = 0; b < NJ; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = __builtin_fmaf(o[x][b][i], 0.f, z);
        return !__any(z != 0.f);
    }
    template <class P, class S> __device__ __forceinline__ void leave(int rows, int lane, P put, S stat) const
    {
        const int c16 = lane & 15, g4 = lane >> 4;
#pragma unroll
        for (int x = 0; x < NRB; ++x) {
            const float l = groups_sum(lsum[x]);
            const int r = 16 * x + c16;
            if (r < rows) {
                if (g4 == 0) stat(r, m_ref[x], l);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int y = 0; y < VP; ++y)
                        put(r, VP * (4 * g4 + i) + y, f32x4{o[x][4 * y][i], o[x][4 * y + 1][i], o[x][4 * y + 2][i], o[x][4 * y + 3][i]});
            }
        }
    }
};


template <class W, int TW, int ROWS>
struct RowsShared {
    float m[TW][ROWS], l[TW][ROWS];
    int flag[TW + 1];
    W place[TW];               // a wavefront's place in its share: the loop over the keys wants the registers
    SeqWindow win[TW];
};
// What a unit costs beside its keys, in keys: us with 96 / 128 / 192 / 256 / 384, 64 tokens over 256..8192 keys of 8 kv-heads 199.1 / 197.2 /
// 197.1 / 196.1 / 196.8; with 16 / 32 / 64 / 96 / 128, 512 tokens over 10..300, a wavefront a team, 83.6 / 82.0 / 81.7 / 83.9 / 81.3.
// TW = 4: see paged_mixed.hip.
template <typename T, int D, int NRB, int TW>
using RowsWork = Work<16 * NRB, RowsKernel<T, D, NRB>::KEYS, TW == 1 ? 32 : TW == 4 ? 384 : 192>;

// A team's share, from where sh.place says: TW wavefronts with NST buffers of a run each, at smem.
template <typename T, int D, int NRB, int TW, int NST>
__device__ __forceinline__ void rows_body(const PagedArgs<T>& a, float* part, int* arrived, char* smem, RowsShared<RowsWork<T, D, NRB, TW>, TW, 16 * NRB>& sh)
{
    typedef RowsKernel<T, D, NRB> Kern;
    typedef RowsWork<T, D, NRB, TW> Work_;
    constexpr int STAGE = NST * Kern::STAGE, KEYS = Kern::KEYS, ROWS = Kern::ROWS, NT = 64 * TW, P4 = D / 4;
    static_assert(ROWS * D * 4 <= STAGE, "the merge reuses the buffers of the runs");
    constexpr int SLOT = ROWS * (D + 2) * 4;                   // [ROWS][D] outputs, then [ROWS] (m, l)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    auto sync = [&]() {
        if constexpr (TW > 1) __syncthreads();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    char* const mine = smem + wave * STAGE;
    // 16-byte piece p of row r of wavefront w's share lies in slot p ^ ((r ^ w) & 7) of the row
    auto share = [&](int w, int r, int p) -> f32x4* { return (f32x4*)(smem + w * STAGE + r * (D * 4) + ((p ^ ((r ^ w) & 7)) * 16)); };
    typename Kern::Runs runs(a, lane);
    Unit u;
    auto next = [&](Unit& u) -> bool {
        Work_ work = sh.place[wave];
        if (!work.next(u, lane)) return false;
        sh.place[wave] = work;
        return true;
    };
    while (next(u)) {
        const int rows = min(ROWS, u.rows - u.row0), k_first = (u.kb & ~(KEYS - 1)) + (u.r0 + wave) * KEYS;
        const int np = max(u.r1 - u.r0 - wave + TW - 1, 0) / TW;
        Kern k;
        runs.start(u);
        k.template sweep<NST>(a, u, runs, mine, k_first, np, TW * KEYS, lane);
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                          // the compiler would keep what the rest makes of it through the loop over the keys
        const int lane = tid & 63;
        const bool fine = k.finite() && !runs.bad;
        if (lane == 0) sh.flag[wave] = fine ? 0 : 1;
        // the wavefronts' shares, in their own buffers (all their loads have been waited for)
        k.leave(rows, lane, [&](int r, int p, f32x4 v) { *share(wave, r, p) = v; },
                [&](int r, float m, float l) { sh.m[wave][r] = m; sh.l[wave][r] = l; });
        sync();
        int flags = 0;
#pragma unroll
        for (int w = 0; w < TW; ++w) flags |= sh.flag[w];
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(flags), 0)) {
            // over again, row by row: the share of wavefront 0 is the piece's, the others' are empty
            sync();
            for (int r = wave; r < rows; r += TW) {
                int k0, k1;
                visible<KEYS>(u, a.window, r, k0, k1);
                float m, l, o[D / 64];
                plain_row<T, D>(a, u.seq, u.h, query_of<T, D>(a, u, r), k0, k1, lane, m, l, o);
                if (lane < TW) { sh.m[lane][r] = lane == 0 ? m : -__builtin_inff(); sh.l[lane][r] = lane == 0 ? l : NONE; }
#pragma unroll
                for (int e = 0; e < D / 64; ++e) {
                    const int d = 64 * e + lane;
                    ((float*)share(0, r, d / 4))[d % 4] = o[e];
#pragma unroll
                    for (int w = 1; w < TW; ++w) ((float*)share(w, r, d / 4))[d % 4] = 0.f;
                }
            }
            sync();
        }
        auto finish = [&](int r, int p, const PieceSum& s) {
            const float inv = inverse(s.l);
            const int64_t at = result_of(a, u, r);
            store_out4(a.out + at * D + 4 * p, f32x4{s.o[0] * inv, s.o[1] * inv, s.o[2] * inv, s.o[3] * inv});
            if (a.lse && p == 0) a.lse[at] = natural_lse(s.m, s.l);
        };
        const auto own = slot_rsrc(part, Work_::slot(u, u.piece), SLOT);
        for (int x = tid; x < rows * P4; x += NT) {
            const int r = x / P4, p = x % P4;
            PieceSum ps[TW];
#pragma unroll
            for (int w = 0; w < TW; ++w) ps[w] = PieceSum{sh.m[w][r], sh.l[w][r], *share(w, r, p)};
            PieceSum s = add_tree(ps);
            if (!flags) s.l = sum_of<KEYS>(u, a.window, r, s.l);
            if (u.pieces == 1) {
                finish(r, p, s);
            } else {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, s.o), own, (r * D + 4 * p) * 4, 0, SC1);
                if (p == 0) __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(s.m), __float_as_uint(s.l)}, own, (ROWS * D + 2 * r) * 4, 0, SC1);
            }
        }
        if (u.pieces > 1) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            sync();
            int n = 0;
            if (tid == 0) n = __hip_atomic_fetch_add(arrived + u.team0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if constexpr (TW > 1) {
                if (tid == 0) sh.flag[TW] = n;
                __syncthreads();
                n = sh.flag[TW];
            }
            n = __builtin_amdgcn_readfirstlane(n);
            if (n == u.pieces - 1) {                           // the last to arrive merges, in the pieces' order
                if (tid == 0) __hip_atomic_store(arrived + u.team0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
                const auto all = __builtin_amdgcn_make_buffer_rsrc((char*)part + (size_t)(2 * u.team0) * SLOT, 0, 2 * u.pieces * SLOT, 0x00020000);
                // few rows: groups of threads take every ng-th piece, and their sums are added through LDS
                const int items = rows * P4;
                int ng = 1;
                while (2 * ng * items <= NT && 2 * ng <= 16 && 2 * ng <= u.pieces) ng *= 2;
                const int span = ng > 1 ? items : NT, grp = tid / span;
                for (int x = tid % span; x < items; x += span) {
                    if (grp >= ng) break;
                    const int r = x / P4, p = x % P4;
                    PieceSum s{-__builtin_inff(), NONE, f32x4{0.f, 0.f, 0.f, 0.f}};
                    for (int i0 = grp; i0 < u.pieces; i0 += 4 * ng) {
                        u32x4 v[4];
                        u32x2 ml[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int i = min(i0 + e * ng, u.pieces - 1), at = (2 * i + (i == 0)) * SLOT;
                            v[e] = __builtin_amdgcn_raw_buffer_load_b128(all, at + (r * D + 4 * p) * 4, 0, SC1);
                            ml[e] = __builtin_amdgcn_raw_buffer_load_b64(all, at + (ROWS * D + 2 * r) * 4, 0, SC1);
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (i0 + e * ng < u.pieces) s.absorb(float2{__uint_as_float(ml[e][0]), __uint_as_float(ml[e][1])}, __builtin_bit_cast(f32x4, v[e]));
                    }
                    if (ng == 1) {
                        finish(r, p, s);
                    } else {
                        f32x4* to = (f32x4*)smem + 2 * (grp * items + x);
                        to[0] = s.o;
                        to[1] = f32x4{s.m, s.l, 0.f, 0.f};
                    }
                }
                if (ng > 1) {
                    sync();
                    if (tid < items) {
                        PieceSum s{-__builtin_inff(), NONE, f32x4{0.f, 0.f, 0.f, 0.f}};
                        for (int g = 0; g < ng; ++g) {
                            const f32x4* from = (const f32x4*)smem + 2 * (g * items + tid);
                            const f32x4 ml = from[1];
                            s.absorb(float2{ml[0], ml[1]}, from[0]);
                        }
                        finish(tid / P4, tid % P4, s);
                    }
                }
            }
        }
        sync();                                                // the buffers are free
    }
}

}  // namespace
}  // namespace infmllm
