// Device side of the attention of chunks over pages: see paged_fwd.hip.
#pragma once
#include "paged_rows.h"

namespace infmllm {
namespace {

constexpr int PF_NT = 256, PF_ROWS = 256, PF_TILE = 64, PF_NBUF = 4;
template <int D> constexpr int PF_VECS = D / 4 + 1;            // 16-byte vectors of a lane's partial results: o of two blocks, then (m, l) of both
template <int D> constexpr int PF_SLOT = 4 * PF_VECS<D> * 1024;

// LDS fragment reads as assembly, waited for by hand: see attn_mfma64.hip
template <int OFF>
__device__ __forceinline__ bf16x8 lds_read_b128(uint32_t addr)
{
    bf16x8 v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF>
__device__ __forceinline__ bf16x4 lds_read_tr16_b64(uint32_t addr)
{
    bf16x4 v;
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
    return v;
}
template <int OFF>                                             // into accumulation registers
__device__ __forceinline__ bf16x8 lds_read_b128_acc(uint32_t addr)
{
    bf16x8 v;
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=a"(v) : "v"(addr), "n"(OFF));
    return v;
}
// Every LDS read issued so far is waited for; the registers are named so that what reads them stays behind.
template <int N>
__device__ __forceinline__ void lds_wait(bf16x8 (&f)[N])
{
    if constexpr (N == 8)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]), "+v"(f[4]), "+v"(f[5]), "+v"(f[6]), "+v"(f[7]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(f[0]), "+v"(f[1]), "+v"(f[2]), "+v"(f[3]));
}
// Two weights into one register, left in the slot it is written in.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t v;
    asm volatile("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(v) : "v"(lo), "v"(hi));
    return v;
}
__device__ __forceinline__ uint32_t pack_bf16_after_nop(float lo, float hi)   // right behind the transcendental that made hi
{
    uint32_t v;
    asm volatile("s_nop 0\n\tv_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(v) : "v"(lo), "v"(hi));
    return v;
}
// S^T += K Q^T into ordinary registers (the compiler would give a kernel of more than 256 registers results in accumulation
// registers).  What it would check is checked here: the products of a chain follow each other with the same accumulators,
// and a block's logits are first read at least four products after its last one.
__device__ __forceinline__ void mfma_qk_first(f32x16& S, bf16x8 k, bf16x8 q)
{
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(S) : "v"(k), "a"(q));
}
__device__ __forceinline__ void mfma_qk(f32x16& S, bf16x8 k, bf16x8 q)
{
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(S) : "v"(k), "a"(q));
}

template <bool B> using Flag = std::integral_constant<bool, B>;

// What a unit costs beside its keys (queries, first tiles, output), in keys: us with 256 / 384 / 512 / 640 / 768, 512 tokens over 4206 keys of 32
// heads on 8 59.4 / 58.7 / 55.9 / 55.2 / 55.1, four chunks of 300..700 over up to 3000 96.4 / 96.9 / 95.9 / 99.9 / 98.7.
constexpr int FWD_OVERHEAD = 512;
typedef Work<PF_ROWS, PF_TILE, FWD_OVERHEAD> FwdWork;
struct FwdShared {
    FwdWork place[4];          // a wavefront's place in its share: the loop wants the registers
    SeqWindow win[4];
    int flag[5];
};
// The tiles of K, those of V, 1 KB a wavefront for loads past the last tile.
template <int D> constexpr int PF_LDS = 2 * PF_NBUF * PF_TILE * D * 2 + 4 * 1024;

// A team's share, from where sh.place says.
template <int D, bool BIG>
__device__ __forceinline__ void fwd_body(const PagedArgs<uint16_t>& a, float* part, int* arrived, char* smem, FwdShared& sh, int team)
{
    constexpr int ROWB = D * 2, TBYTES = PF_TILE * ROWB, NBUF = PF_NBUF;
    constexpr int KREG = 0, VREG = NBUF * TBYTES, DUMP = 2 * NBUF * TBYTES;    // the K tiles, the V tiles, 1 KB a wavefront for loads past the last tile
    constexpr int RPL = 1024 / ROWB, NLD = PF_TILE / RPL / 4;  // rows of a load; loads of K (and of V) a wavefront issues for a tile
    constexpr int NS = D / 16, NB = D / 32, SLOTS = D / 8, PER = 32 / SLOTS;   // products along D, column blocks; slots of half a period, logits of a slot
    constexpr int VECS = PF_VECS<D>, SLOT = PF_SLOT<D>;
    static_assert(NBUF * TBYTES <= 65536, "a region must be addressable with a 16-bit instruction offset");
    typedef FwdWork W;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    Unit u;
    for (;;) {
        {
            FwdWork work = sh.place[wave];
            if (!work.next(u, (int)threadIdx.x & 63)) break;
            sh.place[wave] = work;
        }
        int lane = threadIdx.x & 63;
        asm volatile("" : "+v"(lane));                         // else what every unit makes of it stays in registers from unit to unit
        const int l32 = lane & 31, hh = lane >> 5;
        const int rows = min(PF_ROWS, u.rows - u.row0);        // of the unit
        const bool active = 64 * wave < rows;                  // else the wavefront only takes its share of the loads
        const int kal = u.kb & ~(PF_TILE - 1);
        const int t0 = u.r0, t1 = u.r1;                        // tiles
        int hi[2], lo[2];                                      // a lane's rows see the keys lo .. lo + span
        uint32_t span[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int pos = u.pos(min(64 * wave + 32 * x + l32, rows - 1));
            hi[x] = min(pos, u.ke - 1);                        // a table may end ahead of it
            lo[x] = a.window > 0 ? max(pos + 1 - a.window, 0) : 0;
            if (hi[x] < lo[x]) hi[x] = lo[x] = INT32_MAX;      // none
            span[x] = (uint32_t)(hi[x] - lo[x]);
        }
        // tiles that hold a key which some row of the wavefront does not see
        const int hi_first = min(u.pos(min(64 * wave, rows - 1)), u.ke - 1), hi_last = u.pos(min(64 * wave + 63, rows - 1));
        const int full0 = a.window > 0 ? (max(hi_last + 1 - a.window, 0) - kal + PF_TILE - 1) / PF_TILE : 0;
        const int full1 = hi_first + 1 > kal ? (hi_first + 1 - kal) / PF_TILE : 0;

        f32x16 o[2][NB], S[2];
        bf16x8 qf[2][NS], kf[NS], vf[2 * NB];
        u32x4 pf[2][2];
        float m_ref[2], m_use[2], lsum[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[x][b][i] = 0.f;
            m_ref[x] = -__builtin_inff(); m_use[x] = 0.f; lsum[x] = 0.f;
        }
        bool bad = false;

        // ---- tiles: memory -> LDS.  A load moves 16 bytes a lane into 1 KB: RPL rows.  Wavefront w issues loads 4k + w of a tile's K
        // and V: rows (4k + w) RPL + lane / (64 / RPL), which lie in group (4k + w) RPL / 16 of 16 rows.  Rows are not padded, their 16-byte
        // pieces are permuted instead (Tile in attn_rows.h).
        constexpr int LPR = 64 / RPL;                          // lanes of a row
        const int drow = wave * RPL + lane / LPR;              // row of this lane in the wavefront's first load
        const int grow = drow & 15;                            // ... in its group (the others lie multiples of 16 further on)
        const uint32_t pieceK = (uint32_t)(Tile<uint16_t, D>::k(grow, lane % LPR) * 16), pieceV = (uint32_t)(Tile<uint16_t, D>::v(grow, lane % LPR) * 16);
        const uint32_t page_bytes = (uint32_t)a.Hkv << (a.page_shift + (D == 128 ? 8 : 7));
        const int64_t head_at = ((int64_t)u.h << a.page_shift) * D;
        const char *Kh = (const char*)(a.K + head_at), *Vh = (const char*)(a.V + head_at);
        const int g_lo = u.kb & ~15, g_hi = max(u.ke - 1, 0) & ~15;
        const uint32_t in_page = (uint32_t)(1 << a.page_shift) - 1;
        // the first key of the group that load k of a tile takes, moved to the nearest group with a key of the unit
        auto group_key = [&](int tile, int k) -> int {
            const int key = kal + tile * PF_TILE + ((4 * k + wave) * RPL & ~15);
            return min(max(key, g_lo), g_hi);
        };
        auto tile_page = [&](int tile, int k) -> int { return page_of(a, u.seq, group_key(tile, k)); };
        // byte offset of that key's row from Kh
        auto group_at = [&](int page, int key) -> uint64_t {
            const bool there = (uint32_t)page < (uint32_t)a.pages;
            bad |= !there;
            return (uint64_t)(there ? (uint32_t)page : 0u) * page_bytes + (((uint32_t)key & in_page) * (uint32_t)ROWB);
        };
        auto load_group = [&](const char* base, uint64_t at, char* to, uint32_t off) {
            buffer_to_lds(base + at, 16 * ROWB, to, (int)off);
        };
        // V rows of a lane past the unit's keys (and in front of them): the nearest key's
        auto seen_row = [&](int tile, int k, int key) -> uint32_t {
            const int mine = kal + tile * PF_TILE + 4 * k * RPL + drow;
            return (uint32_t)(min(max(mine, u.kb), u.ke - 1) - key);
        };
        auto issue_tile = [&](int tile, int slot) {            // the whole tile, rows one by one
            int page[NLD];
#pragma unroll
            for (int k = 0; k < NLD; ++k) page[k] = tile_page(tile, k);
#pragma unroll
            for (int k = 0; k < NLD; ++k) {
                const int key = group_key(tile, k);
                const uint64_t at = group_at(page[k], key);
                const uint32_t row = seen_row(tile, k, key) * ROWB;
                char* const to = smem + (slot & (NBUF - 1)) * TBYTES + (4 * k + wave) * 1024;
                load_group(Kh, at, to + KREG, row + pieceK);
                load_group(Vh, at, to + VREG, row + pieceV);
            }
        };
        // the loop's loads, one at a time: dma_begin sets up a tile, dma_step issues its loads at fixed places of the two periods (a
        // burst would hold up the wavefront, and with it the SIMD)
        const int t_hi = max(u.ke - 1, 0) & ~(PF_TILE - 1);
        const uint32_t voffK = (uint32_t)(BIG ? drow : grow) * ROWB + pieceK;
        uint32_t voffV[NLD];
#pragma unroll
        for (int k = 0; k < NLD; ++k) voffV[k] = (uint32_t)(BIG ? 4 * k * RPL + drow : grow) * ROWB + pieceV;
        constexpr int LOOKS = BIG ? 1 : NLD;
        int dma_page[LOOKS];                                   // of the tile that dma_begin takes next
        uint64_t dma_at[LOOKS];
        uint32_t dma_dst = 0, dma_dstV = 0, dma_dstep = 0;
        auto look_key = [&](int tile, int k) -> int { return BIG ? min(kal + tile * PF_TILE, t_hi) : group_key(tile, k); };
        auto look_up = [&](int tile) {
#pragma unroll
            for (int k = 0; k < LOOKS; ++k) dma_page[k] = page_of(a, u.seq, look_key(tile, k));
        };
        auto dma_begin = [&](int tile, int slot) {
#pragma unroll
            for (int k = 0; k < LOOKS; ++k) dma_at[k] = group_at(dma_page[k], look_key(tile, k));
            if (kal + (tile + 1) * PF_TILE > u.ke) {           // V rows past the unit's keys
#pragma unroll
                for (int k = 0; k < NLD; ++k) voffV[k] = seen_row(tile, k, look_key(tile, k)) * ROWB + pieceV;
            }
            const bool past = tile >= t1;                      // nobody needs it: the same number of loads, to the scratch area
            dma_dst = past ? (uint32_t)(DUMP + wave * 1024) : (uint32_t)(KREG + (slot & (NBUF - 1)) * TBYTES + wave * 1024);
            dma_dstV = past ? dma_dst : dma_dst + (VREG - KREG);
            dma_dstep = past ? 0u : 4096u;
            look_up(tile + 1);
        };
        auto dma_step = [&](auto I) {                          // i = 0 .. 2 NLD - 1: K (even) or V (odd)
            constexpr int i = decltype(I)::value, k = i >> 1, x = BIG ? 0 : k;
            if constexpr (!(i & 1)) buffer_to_lds(Kh + dma_at[x], (BIG ? PF_TILE : 16) * ROWB, smem + (dma_dst + k * dma_dstep), (int)voffK, BIG ? 4 * k * RPL * ROWB : 0);
            else buffer_to_lds(Vh + dma_at[x], (BIG ? PF_TILE : 16) * ROWB, smem + (dma_dstV + k * dma_dstep), (int)voffV[k]);
        };

        // ---- fragments.  K fragment s of a sub-block: lane (key row l32, half hh) reads piece 2s + hh of its row.  V: lane l of a 16-lane
        // group supplies the address of key row l / 4, 4 columns at 4 (l % 4).  Addresses of the current tile's buffer.
        uint32_t kaddr[NS], vaddr[NB];
        {
            const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)smem;
#pragma unroll
            for (int s = 0; s < NS; ++s) kaddr[s] = base + KREG + l32 * ROWB + Tile<uint16_t, D>::k(l32, 2 * s + hh) * 16;
            const int vrow = 4 * hh + ((lane & 15) >> 2);      // key row inside a group of eight
            const int x2 = (lane >> 4) & 1, q4 = lane & 3;
#pragma unroll
            for (int b = 0; b < NB; ++b)
                vaddr[b] = base + VREG + vrow * ROWB + Tile<uint16_t, D>::v(vrow, 4 * b + 2 * x2 + (q4 >> 1)) * 16 + 8 * (q4 & 1);
        }
        static_assert(D == 64 || D == 128, "swizzles that repeat every eight rows of V");
        auto wait_v = [&]() {                                  // names what the wait covers, so that no product comes ahead of it
            asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vf[0]));
#pragma unroll
            for (int i = 1; i < 2 * NB; ++i) asm volatile("" : "+v"(vf[i]));
        };
        auto rescale = [&](int x, float mx) {                  // rare: the reference of block x moves
            if (__any(mx > m_ref[x] + RESCALE_TAU)) {
                const float m_new = fmaxf(m_ref[x], mx);
                const float mu = (m_new == -__builtin_inff()) ? 0.f : m_new;
                const float alpha = fast_exp2(m_ref[x] - mu);  // m_ref = -inf gives 0
                m_ref[x] = m_new;
                m_use[x] = mu;
                lsum[x] *= alpha;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[x][b][i] *= alpha;
            }
        };
        const f32x16 zero16 = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        // what a raw logit has to exceed for the reference to move: of block A in the lower half-wave, of block B in the upper one
        const float inv_c = 1.0f / a.c;
        float thr_mix = -__builtin_inff();
        // S c - m of the sub-block in its softmax stage; the second half of a period makes weights of it in place, which the first half
        // of the next one adds to the row sums just before it overwrites them
        float tw[2][16];
        float lsa[2] = {0.f, 0.f}, lsb[2] = {0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) tw[x][e] = 0.f;

        // One period, as in attn_mfma64.hip: key0 = first key of sub-block m, which is in its softmax stage; SUB = m & 1.  Before the first
        // sub-block the weights and V fragments are zero, past the last one the K fragments come from a stale buffer and the
        // logits formed from them are never used.
        auto period = [&](int key0, auto sub, auto mask) {
            constexpr int SUB = decltype(sub)::value;
            constexpr int KO = (SUB == 0 ? 1 : 0) * 32 * ROWB; // sub-block m + 1: the other half of the tile that kaddr points at
            constexpr int VO = SUB * 32 * ROWB;
            wait_v();
            float mx[2] = {-__builtin_inff(), -__builtin_inff()};
            auto logit = [&](int x, int e) -> float {
                float sv = S[x][e];
                if constexpr (decltype(mask)::value) {
                    const int key = key0 + 8 * (e / 4) + 4 * hh + (e % 4);
                    if ((uint32_t)(key - lo[x]) > span[x]) sv = -__builtin_inff();
                }
                return sv;
            };
            static_for<0, SLOTS>([&](auto I) {
                constexpr int i = decltype(I)::value;
                constexpr int tt = i / (2 * NB), b = (i >> 1) % NB, x = i & 1;
                o[x][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[NB * tt + b], as_bf16x8(pf[x][tt]), o[x][b], 0, 0, 0);
                if constexpr (i < NS) kf[i] = lds_read_b128<KO>(kaddr[i]);
                constexpr int xs = i / (SLOTS / 2), e0 = PER * (i % (SLOTS / 2));
                static_for<0, PER / 2>([&](auto J) {
                    constexpr int e = e0 + 2 * decltype(J)::value;
                    const float s0 = logit(xs, e), s1 = logit(xs, e + 1);
                    mx[xs] = fmaxf(fmaxf(mx[xs], s0), s1);
                    lsa[xs] += tw[xs][e];                      // weights of sub-block m - 1
                    lsb[xs] += tw[xs][e + 1];
                    tw[xs][e] = __builtin_fmaf(s0, a.c, -m_use[xs]);
                    tw[xs][e + 1] = __builtin_fmaf(s1, a.c, -m_use[xs]);
                });
                if constexpr (i == SLOTS / 4 - 1) dma_step(std::integral_constant<int, NLD * SUB>{});
                if constexpr (NLD == 4 && i == 11) dma_step(std::integral_constant<int, (NLD * SUB + 1) % (2 * NLD)>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            // lower half-wave: block A's row maxima, upper: block B's, each against its own block's threshold
            const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx[0]), __float_as_uint(mx[1]), false, false);
            float mmix;
            asm("v_max_f32 %0, %1, %2" : "=v"(mmix) : "v"(__uint_as_float(sw[0])), "v"(__uint_as_float(sw[1])));
            if (__any(mmix > thr_mix)) {
                const float mx0 = xhalf_max(mx[0]) * a.c, mx1 = xhalf_max(mx[1]) * a.c;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    lsum[x] += lsa[x] + lsb[x];
                    lsa[x] = 0.f; lsb[x] = 0.f;
                    const float old_use = m_use[x];
                    rescale(x, x == 0 ? mx0 : mx1);
                    const float shift = old_use - m_use[x];    // S c - m was formed with the old reference
#pragma unroll
                    for (int e = 0; e < 16; ++e) tw[x][e] += shift;
                }
                thr_mix = ((hh ? m_ref[1] : m_ref[0]) + RESCALE_TAU) * inv_c;
            }
            lds_wait(kf);
            static_for<0, SLOTS>([&](auto I) {
                constexpr int i = decltype(I)::value;
                constexpr int x = i / NS, s = i % NS;
                if constexpr (s == 0) mfma_qk_first(S[x], kf[s], qf[x][s]);
                else mfma_qk(S[x], kf[s], qf[x][s]);
                if constexpr (i < 2 * NB) {
                    // V fragment i = [16-key step][column block]: key rows 0..7 and 8..15 of the step
                    const bf16x4 lower = lds_read_tr16_b64<VO + (i / NB) * 16 * ROWB>(vaddr[i % NB]);
                    const bf16x4 upper = lds_read_tr16_b64<VO + (i / NB) * 16 * ROWB + 8 * ROWB>(vaddr[i % NB]);
                    vf[i] = __builtin_shufflevector(lower, upper, 0, 1, 2, 3, 4, 5, 6, 7);
                }
                constexpr int xw = i / (SLOTS / 2), e0 = PER * (i % (SLOTS / 2));
#pragma unroll
                for (int e = 0; e < PER; ++e) tw[xw][e0 + e] = fast_exp2(tw[xw][e0 + e]);
                // the slot before's weights are packed here: the conversion is not checked by the compiler, and must not directly follow
                // the transcendental that it reads; the product at the head of this slot lies between
                if constexpr (i > 0) {
                    constexpr int xp = (i - 1) / (SLOTS / 2), ep = PER * ((i - 1) % (SLOTS / 2));
                    static_for<0, PER / 2>([&](auto J) {
                        constexpr int e = ep + 2 * decltype(J)::value;
                        pf[xp][e >> 3][(e & 7) >> 1] = pack_bf16(tw[xp][e], tw[xp][e + 1]);
                    });
                }
                if constexpr (i == SLOTS / 4) dma_step(std::integral_constant<int, NLD * SUB + NLD / 2>{});
                if constexpr (NLD == 4 && i == 12) dma_step(std::integral_constant<int, (NLD * SUB + 3) % (2 * NLD)>{});
                __builtin_amdgcn_sched_barrier(0);
            });
            static_for<0, PER / 2>([&](auto J) {
                constexpr int e = 16 - PER + 2 * decltype(J)::value;
                pf[1][e >> 3][(e & 7) >> 1] = pack_bf16_after_nop(tw[1][e], tw[1][e + 1]);
            });
        };

        if (t1 > t0) {
            // ---- prologue: queries and two tiles requested; the queries go through the tile buffers 2 and 3, four or eight whole rows a load
            char* const qlds = smem + (wave < 2 ? KREG : VREG) + 2 * TBYTES + (wave & 1) * TBYTES;
            static_assert(64 * ROWB == TBYTES, "a wavefront's queries fill one tile buffer");
#pragma unroll
            for (int i = 0; i < 64 / RPL; ++i) {
                const int r = i * RPL + lane / LPR;
                const uint16_t* from = query_of<uint16_t, D>(a, u, min(64 * wave + r, rows - 1)) + Tile<uint16_t, D>::k(r, lane % LPR) * 8;
                __builtin_amdgcn_global_load_lds((global_void*)from, (lds_void*)(qlds + i * 1024), 16, 0, 0);
            }
            issue_tile(t0, 0);
            issue_tile(min(t0 + 1, t1 - 1), 1);
            wait_loads<4 * NLD>();                             // the queries have landed
            {
                const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)qlds + l32 * ROWB;
                static_for<0, NS>([&](auto I) {
                    constexpr int s = decltype(I)::value;
                    const uint32_t addr = base + Tile<uint16_t, D>::k(l32, 2 * s + hh) * 16;
                    qf[0][s] = lds_read_b128_acc<0>(addr);
                    qf[1][s] = lds_read_b128_acc<32 * ROWB>(addr);
                });
            }
            asm volatile("s_waitcnt lgkmcnt(0)" : "+a"(qf[0][0]), "+a"(qf[0][1]), "+a"(qf[0][2]), "+a"(qf[0][3]));
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int s = x == 0 ? 4 : 0; s < NS; ++s) asm volatile("" : "+a"(qf[x][s]));
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) pf[x][tt] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 2 * NB; ++i)
#pragma unroll
                for (int p = 0; p < 8; ++p) vf[i][p] = (__bf16)0.f;
            wait_loads<0>();                                   // this wavefront's loads of two tiles have landed
            __builtin_amdgcn_s_barrier();                      // everyone's have, and everyone has its queries
            issue_tile(min(t0 + 2, t1 - 1), 2);
            look_up(t0 + 3);
            static_for<0, NS>([&](auto I) { kf[decltype(I)::value] = lds_read_b128<0>(kaddr[decltype(I)::value]); });
            lds_wait(kf);
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int s = 0; s < NS; ++s)
                    S[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[s], qf[x][s], s == 0 ? zero16 : S[x], 0, 0, 0);
            asm volatile("" : "+v"(S[0]), "+v"(S[1]));

            // ---- one tile (two periods) an iteration.  K fragments come from tile j (second half) and j + 1 (first half), V fragments from
            // tile j; tile j + 3 is requested into the buffer that tile j - 1 has left, and tile j + 2 awaited ahead of the barrier.
            auto tile_iter = [&](int j, auto mask) {
                const int wrap = ((j - t0 + 1) & (NBUF - 1)) == 0 ? TBYTES - NBUF * TBYTES : TBYTES, key0 = kal + j * PF_TILE;
                dma_begin(j + 3, j - t0 + 3);
                period(key0, Flag<false>{}, mask);
#pragma unroll
                for (int s = 0; s < NS; ++s) kaddr[s] += (uint32_t)wrap;
                period(key0 + 32, Flag<true>{}, mask);
#pragma unroll
                for (int b = 0; b < NB; ++b) vaddr[b] += (uint32_t)wrap;
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * NLD) : "memory");
                __builtin_amdgcn_s_barrier();
            };
            int j = t0;
            if (active) {
                for (; j < min(full0, t1); ++j) tile_iter(j, Flag<true>{});
                for (; j < min(full1, t1); ++j) tile_iter(j, Flag<false>{});
                for (; j < t1; ++j) tile_iter(j, Flag<true>{});
            }
            for (; j < t1; ++j) {                              // the wavefront's share of the others' loads
                dma_begin(j + 3, j - t0 + 3);
                static_for<0, 2 * NLD>([&](auto I) { dma_step(I); });
                wait_loads<2 * NLD>();
                __builtin_amdgcn_s_barrier();
            }
            wait_v();
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float tail = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) tail += tw[x][e];
                lsum[x] += lsa[x] + lsb[x] + tail;
            }
            // the last sub-block still owes its O += V^T P^T
#pragma unroll
            for (int tt = 0; tt < 2; ++tt)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        o[x][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[NB * tt + b], as_bf16x8(pf[x][tt]), o[x][b], 0, 0, 0);
        }

        // ---- results: lane (row l32, half hh) holds O[row][32 b + 8 (i / 4) + 4 hh + i % 4] in o[x][b][i]
        int el = (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));   // the lane
        asm volatile("" : "+v"(el));                           // the compiler would keep what the prologue made of it through the loop
        const int e32 = el & 31, eh = el >> 5;
        float ltot[2], z = 0.f;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            ltot[x] = sum_of<PF_TILE>(u, a.window, min(64 * wave + 32 * x + e32, rows - 1), xhalf_sum(lsum[x]));
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[x][b][i], 0.f, z);
        }
        const bool fine = !__any(z != 0.f) && !bad;
        if (el == 0) sh.flag[wave] = fine || !active ? 0 : 1;
        if (bad && el == 0) sh.flag[wave] = 1;
        __syncthreads();                                       // also: the tile buffers are free
        const bool again = __builtin_amdgcn_readfirstlane(sh.flag[0] | sh.flag[1] | sh.flag[2] | sh.flag[3]);
        const int part_off = wave * (VECS * 1024);
        const auto own = slot_rsrc(part, W::slot(u, u.piece), SLOT);
        if (__builtin_expect(again, 0)) {
            // over again, row by row (see plain_row)
#pragma nounroll
            for (int r = wave; r < rows; r += 4) {
                int k0, k1;
                visible<PF_TILE>(u, a.window, r, k0, k1);
                float m, l, po[D / 64];
                plain_row<uint16_t, D>(a, u.seq, u.h, query_of<uint16_t, D>(a, u, r), k0, k1, el, m, l, po);
                if (u.pieces == 1) {
                    const int64_t at = result_of(a, u, r);
                    const float inv = inverse(l);
#pragma unroll
                    for (int e = 0; e < D / 64; ++e) *(__bf16*)(a.out + at * D + 64 * e + el) = (__bf16)(po[e] * inv);
                    if (a.lse && el == 0) a.lse[at] = natural_lse(m, l);
                } else {
                    const int x = (r >> 5) & 1, at = (r >> 6) * (VECS * 1024);
#pragma unroll
                    for (int e = 0; e < D / 64; ++e) {
                        const int d = 64 * e + el;
                        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(po[e]), own,
                                                              at + ((4 * NB * x + d / 8) * 64 + 32 * ((d >> 2) & 1) + (r & 31)) * 16 + (d & 3) * 4, 0, SC1);
                    }
                    if (el < 2) {                              // both halves of the block's lanes keep (m, l)
                        const int to = at + ((VECS - 1) * 64 + 32 * el + (r & 31)) * 16 + 8 * x;
                        __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(l)}, own, to, 0, SC1);
                    }
                }
            }
        }
        bool mine = true;                                      // whether this workgroup stores the unit's results
        if (u.pieces > 1) {
            auto leave = [&]() {
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int q4 = 0; q4 < 4; ++q4)
                            __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(o[x][b][4 * q4]), __float_as_uint(o[x][b][4 * q4 + 1]),
                                                                         __float_as_uint(o[x][b][4 * q4 + 2]), __float_as_uint(o[x][b][4 * q4 + 3])},
                                                                   own, el * 16, part_off + (4 * NB * x + 4 * b + q4) * 1024, SC1);
                __builtin_amdgcn_raw_buffer_store_b128(u32x4{__float_as_uint(m_ref[0]), __float_as_uint(ltot[0]),
                                                             __float_as_uint(m_ref[1]), __float_as_uint(ltot[1])},
                                                       own, el * 16, part_off + (VECS - 1) * 1024, SC1);
            };
            // o, m, l = fa (o, m, l) + fb (those of a slot); products rounded before they are added: the same bits whichever of two pieces does it
            auto add = [&](int slot, bool first) {
#pragma clang fp contract(off)
                const auto src = slot_rsrc(part, slot, SLOT);
                const u32x4 ml = __builtin_amdgcn_raw_buffer_load_b128(src, el * 16, part_off + (VECS - 1) * 1024, SC1);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    u32x4 other[4 * NB];
#pragma unroll
                    for (int v = 0; v < 4 * NB; ++v)
                        other[v] = __builtin_amdgcn_raw_buffer_load_b128(src, el * 16, part_off + (4 * NB * x + v) * 1024, SC1);
                    const float mo = __uint_as_float(ml[2 * x]), lo_ = __uint_as_float(ml[2 * x + 1]);
                    if (first) {
                        m_ref[x] = mo;
                        ltot[x] = lo_;
                    }
                    const float mt = fmaxf(m_ref[x], mo), mz = mt == -__builtin_inff() ? 0.f : mt;
                    const float w = fast_exp2(m_ref[x] - mz), wo = fast_exp2(mo - mz);   // no key seen: m = -inf, weight 0
                    m_ref[x] = mt;
                    if (!first) ltot[x] = w * ltot[x] + wo * lo_;
#pragma unroll
                    for (int v = 0; v < 4 * NB; ++v)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float y = __uint_as_float(other[v][e]);
                            o[x][v >> 2][4 * (v & 3) + e] = first ? y : w * o[x][v >> 2][4 * (v & 3) + e] + wo * y;
                        }
                }
            };
            if (__builtin_expect(again, 0)) {                  // what plain_row left
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                add(W::slot(u, u.piece), true);
            }
            // Pieces are merged pairwise, a binary tree over their numbers: the first of two halves to come to a node leaves its sum in its
            // slot and its name at the node, the second adds that to its own and goes on.  (One workgroup that merged all of them took
            // 3 us a piece: 140 us for 64 tokens of 32 heads on 8 over 30000 keys, in 32 pieces each; so 79.)
#pragma nounroll
            for (int width = 1; width < u.pieces; width *= 2) {
                const int mid = (u.piece & ~(2 * width - 1)) + width;   // the first piece of the node's upper half
                if (mid >= u.pieces) continue;                 // there is none
                int* const node = arrived + u.team0 + mid;  // no other unit has this team for a piece but its first
                __syncthreads();
                if (threadIdx.x == 0) sh.flag[4] = __hip_atomic_load(node, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __syncthreads();
                int other = __builtin_amdgcn_readfirstlane(sh.flag[4]);
                if (other == 0) {
                    leave();
                    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    __syncthreads();
                    if (threadIdx.x == 0) sh.flag[4] = __hip_atomic_exchange(node, team + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    __syncthreads();
                    other = __builtin_amdgcn_readfirstlane(sh.flag[4]);
                    if (other == 0) { mine = false; break; }   // the other half will find it
                }
                if (threadIdx.x == 0) __hip_atomic_store(node, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next launch
                add(W::slot(u, other - 1 - u.team0), false);
            }
        }
        if (mine && active && !(again && u.pieces == 1)) {
            // through LDS, so that a store takes whole rows: piece p (eight columns) of row r lies in slot Tile::k(r, p)
            char* const olds = smem + wave * (64 * ROWB);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const float inv = inverse(ltot[x]);
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        bf16x4 w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(o[x][b][4 * q4 + e] * inv);
                        *(bf16x4*)(olds + (32 * x + e32) * ROWB + Tile<uint16_t, D>::k(e32, 4 * b + q4) * 16 + 8 * eh) = w;
                    }
                const int r = 64 * wave + 32 * x + e32;
                if (a.lse && eh == 0 && r < rows) a.lse[result_of(a, u, r)] = natural_lse(m_ref[x], ltot[x]);
            }
#pragma unroll
            for (int i = 0; i < 64 / RPL; ++i) {
                const int r = i * RPL + el / LPR;
                const u32x4 v = *(const u32x4*)(olds + r * ROWB + Tile<uint16_t, D>::k(r, el % LPR) * 16);
                if (64 * wave + r < rows) *(u32x4*)(a.out + result_of(a, u, 64 * wave + r) * D + (el % LPR) * 8) = v;
            }
        }
        wait_loads<0>();                                       // loads past the last tile: the scratch area is free
        __syncthreads();                                       // ... and so is all of LDS
    }
}

}  // namespace
}  // namespace infmllm
