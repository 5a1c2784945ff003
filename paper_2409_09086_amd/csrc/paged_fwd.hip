// Attention over pages for chunks of new tokens on bf16 MFMA for gfx950: 256 query rows a workgroup.
//
// Bound by the matrix cores.  A wavefront carries 64 query rows as two blocks A and B of 32, so that a K or V fragment read from
// LDS feeds two products, and a SIMD holds one wavefront: whatever that issues is all the SIMD does, and the loop is a
// software pipeline over sub-blocks of 32 keys laid out by hand:
//
//   period m :  MFMA   O += V(m-1)^T P(m-1)^T         (D / 8 products, both blocks)
//               MFMA   S(m+1)^T = K(m+1) Q^T          (D / 8 products, both blocks)
//               VALU   softmax of S(m) -> P(m)        (row maximum, exp2, row sum, bf16)
//               LDS    K fragments of sub-block m+1, V fragments of sub-block m
//               VMEM   loads of the tile three ahead
//
// Tiles of 64 keys rotate through four LDS buffers, filled by loads that go from memory straight into LDS, with one barrier a
// tile.  S^T = K.Q^T leaves a query row in a lane: its statistics stay there, and the weights are the B operand of
// O^T += V^T.P^T as they stand; V is read with the LDS transpose read.  The reference of a row moves only when its maximum outgrew
// it by 2^8, on a side path between the halves of a period.  Weights are rounded to bf16 (half a step, 2^-8, of a weight, and
// the output is rounded as much): as second terms they would double the products that this kernel is bound by.
//
// Pages: the 16 rows of a load's group lie in one page, whose number was read a tile ahead by a scalar load.  With pages
// of 64 rows and more (BIG) a tile has one number.  V rows past the last key that the unit sees are replaced by that key's.
//
// Units are shared out over one workgroup a CU (paged_work.h); the chunk's causal triangle and ragged batches come
// out even that way.
//
// Measured: 2048 tokens over 8192 + 2048 keys of 32 heads 287 to 300 us (by card) = 1.03 to 1.08 PFLOP/s, as long as attn_fwd64 takes over a contiguous cache
// on the same card (297), and 0.90 to 0.94 of a matrix product's rate there (8192: 1.14).  512 tokens over 4206 keys of 32 heads on 8
// 55 us: 64 units in 4 pieces, 7 us to the first product, 31 for 17 tiles, 10 for the merges, 3 for the output.
#include <climits>

#include "paged_fwd.h"

namespace infmllm {

namespace {

template <int D, bool BIG>
__global__ void __launch_bounds__(PF_NT) __attribute__((amdgpu_waves_per_eu(1, 1)))
paged_fwd_kernel(PagedArgs<uint16_t> a, PagedScratch sc)
{
    __shared__ __attribute__((aligned(1024))) char smem[PF_LDS<D>];
    __shared__ FwdShared sh;
    // Neighbouring shares read the same keys: XCD x (workgroups of one residue class mod 8) gets the x-th eighth of them.
    const int team = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    {
        FwdWork work;
        const auto sums = work.measure(a, &sh.win[wave], 0, INT_MAX, lane);
        work.begin(sums, team, gridDim.x, 256, lane);
        sh.place[wave] = work;
    }
    fwd_body<D, BIG>(a, sc.part, sc.arrived, smem, sh, team);
}

}  // namespace

hipError_t launch_paged_fwd(const PagedArgs<uint16_t>& a, const PagedScratch& sc, int head_dim, hipStream_t st)
{
    const bool big = a.page_shift >= 6;
    const dim3 grid(PAGED_CUS), block(PF_NT);
#define INFMLLM_PAGED_FWD(DD, BB) hipLaunchKernelGGL((paged_fwd_kernel<DD, BB>), grid, block, 0, st, a, sc)
    if (head_dim == 128 && big) INFMLLM_PAGED_FWD(128, true);
    else if (head_dim == 128) INFMLLM_PAGED_FWD(128, false);
    else if (big) INFMLLM_PAGED_FWD(64, true);
    else INFMLLM_PAGED_FWD(64, false);
#undef INFMLLM_PAGED_FWD
    return hipGetLastError();
}

size_t paged_fwd_scratch(int head_dim) { return (size_t)2 * PAGED_CUS * (head_dim == 128 ? PF_SLOT<128> : PF_SLOT<64>); }

}  // namespace infmllm
