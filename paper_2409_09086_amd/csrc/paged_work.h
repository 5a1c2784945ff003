// How the attention over pages is shared out (device side).
//
// A unit is (sequence, kv-head, R consecutive query rows); the rows of a kv-head are numbered token * G + head in group, so
// that a group's heads share every key.  Nothing about the sequences is known on the host.  Every team (a workgroup or a
// wavefront) therefore reads the batch's arrays itself, adds up what all units cost and takes its share of the whole, from
// where the shares of the teams before it end: the chip is filled evenly whatever the lengths are, a long sequence is cut over
// many teams, and a team has at most two units that others work on too, its first and its last.  Partial results of those
// (un-normalised output, reference, sum) go through the team's two slots, and are added in an order that does not depend on who does
// it; no team waits for another one.
//
// A unit costs OVERHEAD keys for everything but its keys, ahead of them, and its keys, in whole numbers far below 2^53, held in
// doubles (64-bit divisions in integers take a microsecond).  Shares are equal pieces of that line, but nobody works on little of a unit:
// the team whose share ends at most HEAD into a unit leaves it to the next one, and that whose share ends at most TAIL ahead of
// its end takes the rest along.  What a team's first unit costs beside its keys every team pays, so the unit's runs are dealt out by
// what the shares of its teams leave for them: OVERHEAD less for a team that comes to it from another unit.
#pragma once
#include "paged.h"

namespace infmllm {
namespace {

struct Unit {
    int first;         // token of row 0 of the sequence
    int G, rows;       // rows of the sequence's kv-head
    int pos0;          // position of that token (negative: it and some more have none)
    int seq, h, row0;  // this unit: rows row0 .. row0 + R - 1
    int kb, ke;        // keys that any of its rows sees
    int r0, r1;        // the team's runs of RUN keys of it, counted from align(kb)
    int pieces, piece, team0;   // the teams that share it: team0 + 0 .. pieces - 1; this is number `piece`
    int tok0, rem0;    // row0 = tok0 * G + rem0
    uint32_t inv_g;
    // Token of the unit's row r and its head in the group.  x * inv_g / 2^32 exceeds x / G by less than x / 2^32, so it is exact for
    // x < R + G, G * (R + G) < 2^32.
    __device__ __forceinline__ int token(int r, int& head) const
    {
        const int x = rem0 + r, t = G == 1 ? x : (int)__umulhi((uint32_t)x, inv_g);
        head = x - t * G;
        return tok0 + t;
    }
    __device__ __forceinline__ int token(int r) const { int head; return token(r, head); }
    __device__ __forceinline__ int pos(int r) const { return pos0 + token(r); }
};

// Sequences sq0 .. sq0 + 63 as the batch's arrays describe them, in LDS: a wavefront's own.
struct SeqWindow {
    int sq0;
    int s0[64], s1[64], len[64];
};

// R rows a unit; keys in runs of RUN from a multiple of RUN; a unit costs OVERHEAD keys more than it has.  row_lo, row_hi: the
// sequences with row_lo < rows <= row_hi.  All lanes of a wavefront call everything here.
template <int R, int RUN, int OVERHEAD>
struct Work {
    static constexpr int HEAD = OVERHEAD + 2 * RUN, TAIL = OVERHEAD / 2;
    const int32_t *starts, *lens;
    SeqWindow* win;
    int seqs, tokens, G, Hkv, window, row_lo, row_hi, team, teams;
    uint32_t inv_g;
    int most_keys;             // what a sequence's row of the page table holds
    double chunk, left, off, u0;   // of a share; left of mine; where in the unit I am; where the unit starts
    int seq, h, tile;
    int first, n, pos0, ntile;     // of the sequence
    double base, inc;              // tile i of it costs base + (i + 1) * inc

    // Whatever the arrays hold, 0 <= first, 0 <= n and first + n <= tokens, for differences of entries may not fit an int.
    struct Seq { int first, n, pos0, ntile; double base, inc; };
    __host__ __device__ __forceinline__ Seq describe(int s0, int s1, int len) const
    {
        Seq q;
        len = max(len, 0);
        q.first = min(max(s0, 0), tokens);
        q.n = max(min(s1, tokens), q.first) - q.first;
        const int64_t rows = (int64_t)q.n * G;
        if (rows <= row_lo || rows > row_hi) q.n = 0;
        q.pos0 = q.n > 0 ? len - (s1 - q.first) : 0;
        q.ntile = (int)((q.n * (int64_t)G + R - 1) / R);
        const int ctx = min(max(q.pos0, 0), most_keys), step = max(R / G, 1);
        if (window > 0) { q.base = (double)OVERHEAD + min((double)ctx + q.n, (double)window + step); q.inc = 0.0; }
        else { q.base = (double)OVERHEAD + ctx; q.inc = (double)step; }
        return q;
    }
    // sequences s .. s + 63 come into the window; returns this lane's
    __device__ __forceinline__ Seq fill(int s, int lane)
    {
        const int mine = min(s + lane, seqs - 1);
        const int s0 = starts[mine], s1 = starts[mine + 1], len = lens[mine];
        win->sq0 = s;
        win->s0[lane] = s0; win->s1[lane] = s1; win->len[lane] = len;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        Seq q = describe(s0, s1, len);
        if (s + lane >= seqs) q.n = 0;
        return q;
    }
    __device__ __forceinline__ Seq from_window(int s) const
    {
        const int i = s - win->sq0;
        return describe(__builtin_amdgcn_readfirstlane(win->s0[i]), __builtin_amdgcn_readfirstlane(win->s1[i]),
                        __builtin_amdgcn_readfirstlane(win->len[i]));
    }
    static __host__ __device__ __forceinline__ double before(const Seq& q, int i) { return i * q.base + q.inc * (0.5 * i * (i + 1.0)); }
    __device__ __forceinline__ double of_head(const Seq& q) const { return q.n > 0 ? before(q, q.ntile) : 0.0; }
    __device__ __forceinline__ void take(const Seq& q) { first = q.first; n = q.n; pos0 = q.pos0; ntile = q.ntile; base = q.base; inc = q.inc; }

    static __device__ __forceinline__ double uniform(double x)
    {
        const uint64_t u = __builtin_bit_cast(uint64_t, x);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)u), hi = __builtin_amdgcn_readfirstlane((uint32_t)(u >> 32));
        return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }
    static __device__ __forceinline__ double scan(double mine, int lane)       // over the lanes up to this one
    {
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double x = __shfl_up(mine, d);
            if (lane >= d) mine += x;
        }
        return mine;
    }

    // Cost of a lane's sequences and those of the lanes before it, of its own, and of all.
    struct Sums { double incl, mine, total; };
    template <typename T>
    __device__ __forceinline__ Sums measure(const PagedArgs<T>& a, SeqWindow* win_, int row_lo_, int row_hi_, int lane)
    {
        starts = a.starts; lens = a.lens; win = win_;
        seqs = a.seqs; tokens = a.tokens; G = a.G; Hkv = a.Hkv; window = a.window; row_lo = row_lo_; row_hi = row_hi_; inv_g = a.inv_g;
        most_keys = (int)min((int64_t)a.pages_per_seq << a.page_shift, (int64_t)INT32_MAX - 65536);
        double mine;
        if (seqs <= 64) {
            mine = of_head(fill(0, lane)) * Hkv;
        } else {                                               // a block of consecutive sequences a lane
            const int per = (seqs + 63) / 64;
            mine = 0.0;
            for (int i0 = 0; i0 < per; i0 += 8) {              // loads of eight at a time
                int s0[8], s1[8], len[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int s = min(lane * per + i0 + i, seqs - 1);
                    s0[i] = starts[s]; s1[i] = starts[s + 1]; len[i] = lens[s];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i0 + i < per && lane * per + i0 + i < seqs) mine += of_head(describe(s0[i], s1[i], len[i])) * Hkv;
            }
        }
        const double incl = scan(mine, lane);
        return Sums{incl, mine, uniform(__shfl(incl, 63))};
    }
    // Finds where my share begins.  least: the smallest share, in keys.
    __device__ __forceinline__ void begin(const Sums& sums, int team_, int teams_, int least, int lane)
    {
        team = team_; teams = teams_;
        chunk = fmax(ceil(sums.total / teams), (double)least);
        const double lo = team * chunk;
        left = fmin(chunk, sums.total - lo);
        if (!(left > 0.0)) { left = 0.0; return; }
        const int who = __builtin_ctzll(__ballot(sums.incl > lo));
        double rem = lo - uniform(__shfl(sums.incl - sums.mine, who));
        if (seqs <= 64) {
            seq = who;
        } else {                                               // in that lane's block
            const int per = (seqs + 63) / 64;
            for (int c = 0;; c += 64) {
                const Seq q = fill(who * per + c, lane);
                const double own = c + lane < per ? of_head(q) * Hkv : 0.0, sum = scan(own, lane), all = uniform(__shfl(sum, 63));
                if (rem < all || c + 64 >= per) {
                    const uint64_t past = __ballot(sum > rem);
                    const int w = past ? __builtin_ctzll(past) : 0;
                    rem -= uniform(__shfl(sum - own, w));
                    seq = who * per + c + w;
                    break;
                }
                rem -= all;
            }
            if (seq >= seqs) { left = 0.0; return; }           // costs beyond 2^53 alone, whose sums are rounded
        }
        const Seq now = from_window(seq);
        if (now.n == 0) { left = 0.0; return; }                // likewise
        take(now);
        const Place at = locate(now, Hkv, of_head(now), rem);
        rem = at.rem;
        tile = __builtin_amdgcn_readfirstlane(at.tile);
        h = __builtin_amdgcn_readfirstlane(at.h);
        off = uniform(rem - before(now, tile));
        u0 = lo - off;
        const double cost = base + (tile + 1) * inc;
        if (off > HEAD && cost - off <= TAIL) {                // the team before takes the rest of it along
            left -= cost - off;
            advance(cost, lane);
        }
    }
    // Where rem, counted from a sequence's first unit, lies: its head, the tile (the largest whose predecessors cost no more than what is
    // left) and the rest.  A head and a tile that exist also where rem is off by a rounding, as sums beyond 2^53 are.
    struct Place { int h, tile; double rem; };
    static __host__ __device__ __forceinline__ Place locate(const Seq& q, int heads, double head, double rem)
    {
        Place p;
        p.h = min((int)(rem / head), heads - 1);
        p.rem = rem - p.h * head;
        const double bb = q.base + 0.5 * q.inc;
        p.tile = q.inc > 0.0 ? (int)((sqrt(bb * bb + 2.0 * q.inc * p.rem) - bb) / q.inc) : (int)(p.rem / q.base);
        p.tile = min(max(p.tile, 0), q.ntile - 1);
        while (p.tile > 0 && before(q, p.tile) > p.rem) --p.tile;
        while (p.tile + 1 < q.ntile && before(q, p.tile + 1) <= p.rem) ++p.tile;
        return p;
    }
    // on to the next unit
    __device__ __forceinline__ void advance(double cost, int lane)
    {
        off = 0.0;
        u0 += cost;
        if (left > 0.0 && ++tile == ntile) {
            tile = 0;
            if (++h == Hkv) {
                h = 0;
                do {
                    if (++seq >= seqs) { left = 0.0; break; }
                    if (seq >= win->sq0 + 64) fill(seq, lane);
                    take(from_window(seq));
                } while (n == 0);
            }
        }
    }
    // The next piece of my share; false: there is none.
    __device__ __forceinline__ bool next(Unit& u, int lane)
    {
        if (!(left > 0.0)) return false;
        const double cost = base + (tile + 1) * inc, take_ = fmin(cost - off, left), end = off + take_;
        if (end < cost && end <= HEAD) return false;           // the next team's
        u.first = first; u.G = G; u.rows = n * G; u.pos0 = pos0; u.seq = seq; u.h = h; u.row0 = tile * R;
        u.tok0 = __builtin_amdgcn_readfirstlane(u.row0 / G);
        u.rem0 = __builtin_amdgcn_readfirstlane(u.row0 - u.tok0 * G);
        u.inv_g = inv_g;
        u.ke = min(max(u.pos(min(R, u.rows - u.row0) - 1) + 1, 0), most_keys);
        u.kb = window > 0 ? min(max(u.pos(0) + 1 - window, 0), u.ke) : 0;
        const int runs = (u.ke - (u.kb & ~(RUN - 1)) + RUN - 1) / RUN;
        u.r0 = 0; u.r1 = runs; u.pieces = 1; u.piece = 0; u.team0 = team;
        if (off > HEAD || end < cost - TAIL) {
            u.team0 = min(max((int)((u0 + HEAD) / chunk), 0), team);
            const int last = max(min((int)((u0 + cost - 1.0 - TAIL) / chunk), teams - 1), team);
            u.pieces = last - u.team0 + 1;
            u.piece = team - u.team0;
            const double lo0 = u.team0 * chunk;
            const double w0 = u0 <= lo0 ? chunk : lo0 + chunk - u0 - (u0 - lo0 > TAIL ? OVERHEAD : 0);   // > 0: HEAD exceeds OVERHEAD
            const double all = w0 + (last - u.team0) * chunk - (last > u.team0 ? (last + 1) * chunk - (u0 + cost) : 0.0);
            const double c0 = u.piece == 0 ? 0.0 : w0 + (u.piece - 1) * chunk, c1 = u.piece == 0 ? w0 : c0 + chunk, per = runs / all;
            u.r0 = min((int)(c0 * per), runs);
            if (team < last) u.r1 = min((int)(c1 * per), runs);
        }
        auto scalar = [](int& x) { x = __builtin_amdgcn_readfirstlane(x); };
        scalar(u.first); scalar(u.rows); scalar(u.pos0); scalar(u.seq); scalar(u.h); scalar(u.row0); scalar(u.kb); scalar(u.ke);
        scalar(u.r0); scalar(u.r1); scalar(u.pieces); scalar(u.piece); scalar(u.team0);
        left -= take_;
        advance(cost, lane);
        return true;
    }
    // which of a team's two slots a piece of a shared unit uses: the unit it ends with, or the one it begins with
    static __device__ __forceinline__ int slot(const Unit& u, int piece) { return 2 * (u.team0 + piece) + (piece == 0 ? 1 : 0); }
};

}  // namespace
}  // namespace infmllm
