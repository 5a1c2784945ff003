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
// A team (see paged_work.h) is a workgroup of 8 wavefronts that take a unit's runs in turn and merge in LDS, or, with four units a
// CU and more (two, if they are brief), a single wavefront, which has nobody to wait for.
//
// Measured: 64 tokens over 256..8192 keys of 32 heads on 8, 1.12 GB, 196 us = 5.7 TB/s, where a copy of 1 GB goes at 4.9; 512
// tokens over 10..300 keys 77 to 82 us, by card, = 4.1 to 4.3 TB/s; one token over 1001 keys of 32 heads 10.8 us at the least, 12.1 in the median, of
// which 3 are the way to the first keys, 2 their way, 1 the products, 3 the merges.
#include <algorithm>
#include <climits>
#include <cmath>

#include "paged_rows.h"

namespace infmllm {

namespace {

// TW: wavefronts of a team.
template <typename T, int D, int NRB, int TW>
__global__ void __launch_bounds__(64 * TW, 2)
paged_rows_kernel(PagedArgs<T> a, PagedScratch sc, int least)
{
    typedef RowsWork<T, D, NRB, TW> W;
    __shared__ __attribute__((aligned(1024))) char smem[TW * RowsKernel<T, D, NRB>::STAGE];
    __shared__ RowsShared<W, TW, 16 * NRB> sh;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    {
        W work;
        const auto sums = work.measure(a, &sh.win[wave], 0, INT_MAX, lane);
        // Neighbouring shares may read the same keys: XCD x (workgroups of one residue class mod 8) gets the x-th eighth of them.
        work.begin(sums, (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3), gridDim.x, least, lane);
        sh.place[wave] = work;
    }
    rows_body<T, D, NRB, TW, 1>(a, sc.part, sc.arrived, smem, sh);
}

template <typename T, int D, int NRB, int TW>
hipError_t launch(const PagedArgs<T>& a, const PagedScratch& sc, int teams, int least, hipStream_t st)
{
    hipLaunchKernelGGL((paged_rows_kernel<T, D, NRB, TW>), dim3(teams), dim3(64 * TW), 0, st, a, sc, least);
    return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_d(const PagedArgs<T>& a, const PagedScratch& sc, int max_new, int max_len, hipStream_t st)
{
    constexpr int KEYS = RowsKernel<T, D, 1>::KEYS;
    const int64_t rows = (int64_t)std::max(1, std::min(max_new, a.tokens)) * a.G;
    const int64_t seqs = std::min(a.seqs, a.tokens);
    const int64_t units = a.Hkv * std::min(seqs * ((rows + 15) / 16), (int64_t)a.tokens * a.G / 16 + seqs);   // most there can be
    // The smallest share.  Halving it halves the time that a team takes for its keys (4 D bytes each at some 40 GB/s) and doubles that of
    // the one which merges a unit's pieces (4 D bytes a row and piece at some 80 GB/s): sqrt(keys * rows / 2).
    auto least = [&](int block) { return std::max(4 * KEYS, (int)std::sqrt(0.5 * max_len * (double)std::min<int64_t>(rows, block))); };
    if constexpr (sizeof(T) == 2) {
        if (rows > 16) return launch<T, D, 2, 8>(a, sc, PAGED_CUS, least(32), st);
    }
    // A wavefront a team has nobody to wait for from unit to unit, but is slower with long ones.  us with eight / one, tokens of 32 heads of 128 on 8 over
    // a tenth to all of 100, 300, 700, 1000, 3000 keys: 40 (320 units) 11.0 / 13.1, 15.4 / 17.3, -, 23.0 / 26.5, 55.5 / 62.1; 64 14.4 / 13.1, 17.8 / 18.0, 29.8 /
    // 28.0, 36.2 / 39.0, 84.9 / 90.8; 100 19.5 / 16.2, 24.4 / 21.1, 43.7 / 43.2, 51.4 / 54.6, 125 / 133; 128 22.6 / 15.1, 28.6 / 23.0, -, 59.6 / 61.9, 153 / 157; 100 of 64
    // 16.9 / 12.5, 21.0 / 14.5, -, 35.0 / 32.6, 78.0 / 77.3; 64 in single precision 17.9 / 19.5, 28.2 / 27.0, -, 63.1 / 67.0.  From 1024 units on it is always one: what
    // it can lose is a few percent, and max_len may be a wide bound.  Chunks in single precision: 700 tokens of 16 heads of 64 on 4 (700
    // units) over 1000 keys 52.7 / 50.8, 900 65.8 / 62.0, 300 of 32 heads on 8 beside 31 decoded 87.7 / 76.8, of 128 155 / 150.
    const bool brief = (double)max_len * (2 * D * sizeof(T)) <= 400e3 || (sizeof(T) == 4 && rows > 16);
    if (units >= (brief ? 2 : 4) * PAGED_CUS) return launch<T, D, 1, 1>(a, sc, 8 * PAGED_CUS, 2 * KEYS, st);
    if constexpr (sizeof(T) == 4 && D == 64) {
        // Fewer units are fewer beginnings and merges where teams have more than one.  us with 16 / 32 rows a unit, tokens of 16 heads on 4: 130 (130
        // units of 16) over 100 keys 10.7 / 13.2, over 1000 18.6 / 18.8; 260 15.6 / 15.0, 25.1 / 26.2; 400 20.3 / 19.0, 34.4 / 33.3; five chunks
        // of 33..197 of 8 heads on 2 (300 units) that see 256 keys 16.7 / 14.1.  Heads of 128 have no registers for it.
        if (rows > 16 && units > PAGED_CUS) return launch<T, D, 2, 8>(a, sc, PAGED_CUS, least(32), st);
    }
    return launch<T, D, 1, 8>(a, sc, PAGED_CUS, least(16), st);
}

}  // namespace

template <typename T>
hipError_t launch_paged_rows(const PagedArgs<T>& a, const PagedScratch& sc, int head_dim, int max_new, int max_len, hipStream_t st)
{
    if (head_dim == 128) return launch_d<T, 128>(a, sc, max_new, max_len, st);
    return launch_d<T, 64>(a, sc, max_new, max_len, st);
}
template hipError_t launch_paged_rows<uint16_t>(const PagedArgs<uint16_t>&, const PagedScratch&, int, int, int, hipStream_t);
template hipError_t launch_paged_rows<float>(const PagedArgs<float>&, const PagedScratch&, int, int, int, hipStream_t);

size_t paged_rows_scratch(int head_dim, int elt)
{
    const size_t row = (size_t)(head_dim + 2) * 4;
    return std::max<size_t>((size_t)2 * 8 * PAGED_CUS * 16 * row, elt == 2 ? (size_t)2 * PAGED_CUS * 32 * row : 0);
}

}  // namespace infmllm
