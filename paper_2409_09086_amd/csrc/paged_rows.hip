// Attention over pages for few query rows (decoded tokens, drafted runs, short prompts) on the matrix cores of gfx950, and all of it in single precision.
//
// Bound by the keys and values that it reads.  A wavefront goes through runs of 32 keys (16 in single precision) with an online
// softmax of its own; K and V come from memory straight into LDS, into a buffer only this wavefront uses, and the next
// run is requested as soon as the fragments of a run are in registers: no barrier in the loop, 16 KB a wavefront on their way.
// S^T = K.Q^T on 16x16x32 products leaves four consecutive keys of one query row in a lane, two such blocks are the B operand
// of O^T += V^T.P^T as they stand.  In bf16 a weight enters the product as two terms, its rounding and the rounded rest (16
// bits), which costs nothing: the matrix cores have the time.
//
// A run lies in one page or, with pages of 16 rows, in two: it is fetched in halves of 16 rows, each from its page, whose number
// was read a run ahead by a scalar load.  Rows outside the keys that the unit's queries see are replaced by the nearest one
// that is seen, so that pages nobody is meant to read (freed ones in front of a window, rows past the end) are not read.
//
// A team (see paged_work.h) is a workgroup of 8 wavefronts that take a unit's runs in turn and merge in LDS, or a single
// wavefront: see the launch for which.
#include <algorithm>

#include "paged_rows.h"

namespace infmllm {

namespace {

// A wavefront's direct loads of a run of keys into `dst` (K) and `dst` + RUN bytes (V).
template <typename T, int D, int KEYS>
struct PageRuns {
    static constexpr int ROWB = D * (int)sizeof(T), RUN = KEYS * ROWB, HALVES = KEYS / 16, HALF = 16 * ROWB, NL = HALF / 1024,
                         RPL = 1024 / ROWB;
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

    // np runs of KEYS keys from k_first on, `step` keys apart
    __device__ __forceinline__ void sweep(const PagedArgs<T>& a, const Unit& u, Runs& runs, char* mine, int k_first, int np, int step, int lane)
    {
        const int c16 = lane & 15, g4 = lane >> 4;
        if (np > 0) {
            runs.look_up(k_first);
            runs.load(k_first, mine);
            if (np > 1) runs.look_up(k_first + step);
        }
        bf16x8 qf[NRB][C::NS];
        int hi[NRB], lo[NRB];
#pragma unroll
        for (int x = 0; x < NRB; ++x) {
            const int row = min(16 * x + c16, u.rows - u.row0 - 1);
            const T* qp = query_of<T, D>(a, u, row) + 8 * g4;
            hi[x] = u.pos(row);
            lo[x] = a.window > 0 ? hi[x] + 1 - a.window : 0;
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
            wait_loads<0>();
            bf16x8 kf[2][C::NS];
            bf16x4 vlo[C::NC], vhi[C::NC];
#pragma unroll
            for (int s = 0; s < C::NS; ++s) {
                kf[0][s] = rw_read_b128<0>(kaddr[s]);
                kf[1][s] = rw_read_b128<16 * C::ROWB>(kaddr[s]);
            }
#pragma unroll
            for (int b = 0; b < C::NC; ++b) {
                vlo[b] = rw_read_tr16<0>(vaddr[b]);
                vhi[b] = rw_read_tr16<16 * C::ROWB>(vaddr[b]);
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
            // the stage has been read: the next run goes there
            if (p + 1 < np) {
                runs.load(k0 + step, mine);
                if (p + 2 < np) runs.look_up(k0 + 2 * step);
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
template <int D>
struct RowsKernel<float, D, 1> {
    typedef float T;
    static constexpr int KEYS = 16, ROWS = 16;
    typedef PageRuns<T, D, KEYS> Runs;
    static constexpr int ROWB = Runs::ROWB, STAGE = 2 * Runs::RUN;
    static constexpr int NJ = D / 16, VW = D / 16, VP = VW / 4;

    f32x4 o[NJ];                                               // block b: lane (row c16, group g4) holds columns VW (4 g4 + i) + b
    float m_ref, m_use, lsum;

    static __device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

    __device__ __forceinline__ void sweep(const PagedArgs<T>& a, const Unit& u, Runs& runs, char* mine, int k_first, int np, int step, int lane)
    {
        const int c16 = lane & 15, g4 = lane >> 4;
        if (np > 0) {
            runs.look_up(k_first);
            runs.load(k_first, mine);
            if (np > 1) runs.look_up(k_first + step);
        }
        f32x4 qf[NJ];
        const int row = min(c16, u.rows - u.row0 - 1), hi = u.pos(row), lo = a.window > 0 ? hi + 1 - a.window : 0;
        {
            const float* qp = query_of<T, D>(a, u, row) + 4 * g4;
#pragma unroll
            for (int j = 0; j < NJ; ++j) qf[j] = *(const f32x4*)(qp + 16 * j);
        }
#pragma unroll
        for (int b = 0; b < NJ; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
        m_ref = -__builtin_inff(); m_use = 0.f; lsum = 0.f;
        const int hi0 = __builtin_amdgcn_readfirstlane(hi), lo1 = __builtin_amdgcn_readlane(lo, 15);
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
            f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NJ; j += 2)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s0 = mfma(kf[j][e], qf[j][e], s0);
                    s1 = mfma(kf[j + 1][e], qf[j + 1][e], s1);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vf[0][0]), "+v"(vf[1][0]), "+v"(vf[2][0]), "+v"(vf[3][0])::"memory");
            if constexpr (VP == 2) asm volatile("" : "+v"(vf[0][VP - 1]), "+v"(vf[1][VP - 1]), "+v"(vf[2][VP - 1]), "+v"(vf[3][VP - 1]));
            if (p + 1 < np) {
                runs.load(k0 + step, mine);
                if (p + 2 < np) runs.look_up(k0 + 2 * step);
            }
            float s[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = (s0[i] + s1[i]) * a.c;
            if (k0 + KEYS - 1 > hi0 || k0 < lo1) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int key = k0 + 4 * g4 + i;
                    if (key > hi || key < lo) s[i] = -__builtin_inff();
                }
            }
            const float mx = groups_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
            if (__any(mx > m_ref + RESCALE_TAU)) {
                const float m_new = fmaxf(m_ref, mx);
                const float mu = (m_new == -__builtin_inff()) ? 0.f : m_new;
                const float alpha = fast_exp2(m_ref - mu);
                m_ref = m_new;
                m_use = mu;
                lsum *= alpha;
#pragma unroll
                for (int b = 0; b < NJ; ++b) o[b] *= alpha;
            }
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = fast_exp2(s[i] - m_use);
                lsum += w[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int b = 0; b < NJ; ++b) o[b] = mfma(vf[i][b / 4][b % 4], w[i], o[b]);
        }
    }
    __device__ __forceinline__ bool finite() const
    {
        float z = 0.f;
#pragma unroll
        for (int b = 0; b < NJ; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) z = __builtin_fmaf(o[b][i], 0.f, z);
        return !__any(z != 0.f);
    }
    template <class P, class S> __device__ __forceinline__ void leave(int rows, int lane, P put, S stat) const
    {
        const int c16 = lane & 15, g4 = lane >> 4;
        const float l = groups_sum(lsum);
        if (c16 < rows) {
            if (g4 == 0) stat(c16, m_ref, l);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int x = 0; x < VP; ++x) put(c16, VP * (4 * g4 + i) + x, f32x4{o[4 * x][i], o[4 * x + 1][i], o[4 * x + 2][i], o[4 * x + 3][i]});
        }
    }
};

// TW: wavefronts of a team.
template <typename T, int D, int NRB, int TW>
__global__ void __launch_bounds__(64 * TW, 2)
paged_rows_kernel(PagedArgs<T> a, PagedScratch sc, int least, int row_lo, int row_hi)
{
    typedef RowsKernel<T, D, NRB> Kern;
    constexpr int STAGE = Kern::STAGE, KEYS = Kern::KEYS, ROWS = Kern::ROWS, NT = 64 * TW, P4 = D / 4;
    static_assert(ROWS * D * 4 <= STAGE, "the merge reuses the buffers of the runs");
    constexpr int SLOT = ROWS * (D + 2) * 4;                   // [ROWS][D] outputs, then [ROWS] (m, l)
    __shared__ __attribute__((aligned(1024))) char smem[TW * STAGE];
    __shared__ float s_m[TW][ROWS], s_l[TW][ROWS];
    __shared__ int s_flag[TW + 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    auto sync = [&]() {
        if constexpr (TW > 1) __syncthreads();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    char* const mine = smem + wave * STAGE;
    // 16-byte piece p of row r of wavefront w's share lies in slot p ^ ((r ^ w) & 7) of the row
    auto share = [&](int w, int r, int p) -> f32x4* { return (f32x4*)(smem + w * STAGE + r * (D * 4) + ((p ^ ((r ^ w) & 7)) * 16)); };

    // a wavefront's place in its share is in LDS, the loop over the keys wants the registers
    // What a unit costs beside its keys, in keys: us with 16 / 64 / 128 / 256, 64 tokens over 256..8192 keys of 8 kv-heads 205.7 / 202.3 / 198.7 /
    // 196.9, 16 over 2000..6000 61.9 / 54.2 / 54.5 / 53.7, 512 over 10..300 90.3 / 80.8 / 80.7 / 81.5.
    constexpr int OVERHEAD = TW == 1 ? 32 : 192;
    typedef Work<ROWS, KEYS, OVERHEAD> W;
    __shared__ __attribute__((aligned(16))) char s_work[TW][(sizeof(W) + 15) / 16 * 16];
    W* const place = (W*)s_work[wave];
    *place = W(a, blockIdx.x, gridDim.x, least, row_lo, row_hi, lane);
    typename Kern::Runs runs(a, lane);
    auto next = [&](Unit& u) -> bool {
        W work = *place;
        if (!work.next(u)) return false;
        *place = work;
        return true;
    };
    Unit u;
    while (next(u)) {
        const int rows = min(ROWS, u.rows - u.row0), k_first = (u.kb & ~(KEYS - 1)) + (u.r0 + wave) * KEYS;
        const int np = max(u.r1 - u.r0 - wave + TW - 1, 0) / TW;
        Kern k;
        runs.start(u);
        k.sweep(a, u, runs, mine, k_first, np, TW * KEYS, lane);
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));                          // the compiler would keep what the rest makes of it through the loop over the keys
        const int lane = tid & 63;
        const bool fine = k.finite() && !runs.bad;
        if (lane == 0) s_flag[wave] = fine ? 0 : 1;
        // the wavefronts' shares, in their own buffers (all their loads have been waited for)
        k.leave(rows, lane, [&](int r, int p, f32x4 v) { *share(wave, r, p) = v; },
                [&](int r, float m, float l) { s_m[wave][r] = m; s_l[wave][r] = l; });
        sync();
        int flags = 0;
#pragma unroll
        for (int w = 0; w < TW; ++w) flags |= s_flag[w];
        if (__builtin_expect(__builtin_amdgcn_readfirstlane(flags), 0)) {
            // over again, row by row: the share of wavefront 0 is the piece's, the others' are empty
            sync();
            for (int r = wave; r < rows; r += TW) {
                int k0, k1;
                visible<KEYS>(u, a.window, r, k0, k1);
                float m, l, o[D / 64];
                plain_row<T, D>(a, u.seq, u.h, query_of<T, D>(a, u, r), k0, k1, lane, m, l, o);
                if (lane < TW) { s_m[lane][r] = lane == 0 ? m : -__builtin_inff(); s_l[lane][r] = lane == 0 ? l : 0.f; }
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
        const auto own = slot_rsrc(sc.part, W::slot(u, u.piece), SLOT);
        for (int x = tid; x < rows * P4; x += NT) {
            const int r = x / P4, p = x % P4;
            PieceSum ps[TW];
#pragma unroll
            for (int w = 0; w < TW; ++w) ps[w] = PieceSum{s_m[w][r], s_l[w][r], *share(w, r, p)};
            const PieceSum s = add_tree(ps);
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
            if (tid == 0) n = __hip_atomic_fetch_add(sc.arrived + u.team0, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if constexpr (TW > 1) {
                if (tid == 0) s_flag[TW] = n;
                __syncthreads();
                n = s_flag[TW];
            }
            n = __builtin_amdgcn_readfirstlane(n);
            if (n == u.pieces - 1) {                           // the last to arrive merges, in the pieces' order
                if (tid == 0) __hip_atomic_store(sc.arrived + u.team0, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
                const auto all = __builtin_amdgcn_make_buffer_rsrc((char*)sc.part + (size_t)(2 * u.team0) * SLOT, 0, 2 * u.pieces * SLOT, 0x00020000);
                // few rows: groups of threads take every ng-th piece, and their sums are added through LDS
                const int items = rows * P4;
                int ng = 1;
                while (2 * ng * items <= NT && 2 * ng <= 16 && 2 * ng <= u.pieces) ng *= 2;
                const int span = ng > 1 ? items : NT, grp = tid / span;
                for (int x = tid % span; x < items; x += span) {
                    if (grp >= ng) break;
                    const int r = x / P4, p = x % P4;
                    PieceSum s{-__builtin_inff(), 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
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
                        PieceSum s{-__builtin_inff(), 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
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

template <typename T, int D, int NRB, int TW>
hipError_t launch(const PagedArgs<T>& a, const PagedScratch& sc, int teams, int least, int row_lo, int row_hi, hipStream_t st)
{
    hipLaunchKernelGGL((paged_rows_kernel<T, D, NRB, TW>), dim3(teams), dim3(64 * TW), 0, st, a, sc, least, row_lo, row_hi);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_d(const PagedArgs<T>& a, const PagedScratch& sc, int max_new, int row_lo, int row_hi, hipStream_t st)
{
    constexpr int KEYS = RowsKernel<T, D, 1>::KEYS;
    const int64_t rows = (int64_t)std::max(1, std::min(max_new, a.tokens)) * a.G;
    const int64_t units = (int64_t)std::min(a.seqs, a.tokens) * a.Hkv * ((rows + 15) / 16);
    if constexpr (sizeof(T) == 2) {
        if (rows > 16 && row_hi > 16) return launch<T, D, 2, 8>(a, sc, PAGED_CUS, 4 * KEYS, row_lo, row_hi, st);
    }
    if (units >= 4 * PAGED_CUS) return launch<T, D, 1, 1>(a, sc, 8 * PAGED_CUS, 2 * KEYS, row_lo, row_hi, st);
    return launch<T, D, 1, 8>(a, sc, PAGED_CUS, 4 * KEYS, row_lo, row_hi, st);
}

}  // namespace

template <typename T>
hipError_t launch_paged_rows(const PagedArgs<T>& a, const PagedScratch& sc, int head_dim, int max_new, int row_lo, int row_hi, hipStream_t st)
{
    if (head_dim == 128) return launch_d<T, 128>(a, sc, max_new, row_lo, row_hi, st);
    return launch_d<T, 64>(a, sc, max_new, row_lo, row_hi, st);
}
template hipError_t launch_paged_rows<uint16_t>(const PagedArgs<uint16_t>&, const PagedScratch&, int, int, int, int, hipStream_t);
template hipError_t launch_paged_rows<float>(const PagedArgs<float>&, const PagedScratch&, int, int, int, int, hipStream_t);

size_t paged_rows_scratch(int head_dim, int elt)
{
    const size_t row = (size_t)(head_dim + 2) * 4;
    return std::max<size_t>((size_t)2 * 8 * PAGED_CUS * 16 * row, elt == 2 ? (size_t)2 * PAGED_CUS * 32 * row : 0);
}

}  // namespace infmllm
