// Attention over pages for batches that hold both chunks and decoded tokens.
//
// Chunks are bound by the matrix cores and leave the memory idle, decoded tokens are bound by the keys that they read and leave the
// matrix cores idle.  One launch gives some compute units of every XCD to the sequences of few rows (rows_body, four wavefronts with
// two buffers each: as many bytes on their way as eight with one) and the others to the chunks (fwd_body).
//
// A compute unit by itself draws MIXED_CU_BYTES a microsecond, all of them together MIXED_BYTES, so that decoding needs no more than
// some 140 units to be as fast as it gets.  It gets as many as make both ends finish together; where the memory is the longer end,
// all that the chunks can do without.  us, two launches one after the other / this: 512 tokens over 4206 keys beside 31 over 512..4096, 32 heads
// on 8, 123 / 88 (78 to 90 by card); 2 x 256 over 1000..2000 beside 100 161 / 128; 1024 over 4500 beside 16 over 100..8000 162 / 131; 100 over 1000..2000 beside 200
// 270 / 222; 2048 on themselves beside 60 of one key 68 / 64.  With 40e3 and 1.7 in the place of 38e3 and 2.1: 88, 153, 129, 223, 80.
#include <algorithm>
#include <climits>

#include "paged_fwd.h"

namespace infmllm {

namespace {

constexpr double MIXED_CU_BYTES = 38e3, MIXED_BYTES = 5.3e6;   // bytes a microsecond: of a compute unit, of all
template <int D> constexpr double MIXED_TILE_US = D == 128 ? 2.1 : 1.25;       // 256 rows by 64 keys on a compute unit
constexpr int MIXED_WAVES = 4;

template <int D, bool BIG>
__global__ void __launch_bounds__(PF_NT) __attribute__((amdgpu_waves_per_eu(1, 1)))
paged_mixed_kernel(PagedArgs<uint16_t> a, PagedScratch sc, float* rows_part, int* rows_arrived, int few)
{
    typedef RowsWork<uint16_t, D, 1, MIXED_WAVES> RW;
    static_assert(MIXED_WAVES * 2 * RowsKernel<uint16_t, D, 1>::STAGE <= PF_LDS<D>, "both ends use the same memory");
    __shared__ __attribute__((aligned(1024))) char smem[PF_LDS<D>];
    __shared__ FwdShared fwd;
    __shared__ RowsShared<RW, MIXED_WAVES, 16> rows;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int xcd = blockIdx.x & 7, li = blockIdx.x >> 3, per_xcd = gridDim.x >> 3;
    RW rw;
    FwdWork fw;
    const auto few_sums = rw.measure(a, &rows.win[wave], 0, few, lane);
    const auto many_sums = fw.measure(a, &fwd.win[wave], few, INT_MAX, lane);
    // compute units of an XCD for the few
    int mine = per_xcd;
    if (many_sums.total > 0.0) {
        const double all = (double)gridDim.x, bytes = few_sums.total * (4.0 * D), chunks = many_sums.total * (MIXED_TILE_US<D> / PF_TILE);   // CU us
        const double tokens = bytes / MIXED_CU_BYTES;          // CU us
        const double even = all * tokens / (tokens + chunks), spare = bytes > 0.0 ? all - chunks * MIXED_BYTES / bytes : 0.0;
        mine = bytes > 0.0 ? min(max((int)(fmax(even, spare) * 0.125 + 0.5), 1), per_xcd - 1) : 0;
        mine = __builtin_amdgcn_readfirstlane(mine);
    }
    if (li < mine) {
        rw.begin(few_sums, xcd * mine + li, 8 * mine, 128, lane);
        rows.place[wave] = rw;
        rows_body<uint16_t, D, 1, MIXED_WAVES, 2>(a, rows_part, rows_arrived, smem, rows);
    } else {
        const int team = xcd * (per_xcd - mine) + li - mine;
        fw.begin(many_sums, team, 8 * (per_xcd - mine), 256, lane);
        fwd.place[wave] = fw;
        fwd_body<D, BIG>(a, sc.part, sc.arrived, smem, fwd, team);
    }
}

}  // namespace

hipError_t launch_paged_mixed(const PagedArgs<uint16_t>& a, const PagedScratch& sc, int head_dim, int few, hipStream_t st)
{
    const bool big = a.page_shift >= 6;
    float* const rows_part = (float*)((char*)sc.part + paged_fwd_scratch(head_dim));
    int* const rows_arrived = sc.arrived + PAGED_TEAMS;
#define INFMLLM_PAGED_MIXED(DD, BB) \
    hipLaunchKernelGGL((paged_mixed_kernel<DD, BB>), dim3(PAGED_CUS), dim3(PF_NT), 0, st, a, sc, rows_part, rows_arrived, few)
    if (head_dim == 128 && big) INFMLLM_PAGED_MIXED(128, true);
    else if (head_dim == 128) INFMLLM_PAGED_MIXED(128, false);
    else if (big) INFMLLM_PAGED_MIXED(64, true);
    else INFMLLM_PAGED_MIXED(64, false);
#undef INFMLLM_PAGED_MIXED
    return hipGetLastError();
}

size_t paged_mixed_scratch(int head_dim) { return paged_fwd_scratch(head_dim) + (size_t)2 * PAGED_CUS * 16 * (head_dim + 2) * 4; }

}  // namespace infmllm
