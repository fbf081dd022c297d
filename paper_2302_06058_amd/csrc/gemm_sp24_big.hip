// 2:4-sparse bf16 GEMM for gfx950, large-problem variant:  C[t][a] = sum_k Bm[t][k] * A[a][k]
// with A given as compressed values + 2-bit indices (the operand of Eq. 3 / Eq. 10 of
// arXiv 2302.06058), for shapes whose matrix work dominates (thousands of weight rows AND
// thousands of tokens: the MLP block of a transformer).
//
// What bounds such a shape on this chip is not the matrix pipe but the bytes every CU pulls from
// its L2 and from LDS per matrix instruction, so the tile is shaped to cut both:
//   * workgroup tile 512 weight rows x 128 tokens on 8 wavefronts; wavefront w owns weight rows
//     [64 w, 64 w + 64) -- two 32-row tiles -- against ALL 128 tokens: 8 accumulator tiles
//     (128 registers), every token fragment read from LDS feeds two matrix instructions, every
//     weight fragment (registers, straight from L2 in the fragment-major layout) feeds four;
//   * per 128-deep stage a workgroup pulls 72 KB of weights + 32 KB of tokens for 2 x 8.4 MFLOP
//     dense-equivalent (52 KB per 8.4 MFLOP; the 256 x 128 tile of the streaming kernel: 68 KB)
//     and reads 256 KB from LDS (streaming kernel: 256 KB for half the work);
//   * the weight fragments of a stage are not double-buffered as a whole: the registers of sub-step
//     s4 are re-loaded with the NEXT stage's fragment as soon as the sub-step's matrix instructions
//     have been issued (one stage of distance at 32 + 8 registers instead of 72);
//   * the token tile of the next stage goes from registers to the other LDS buffer in the middle of
//     the current stage's matrix instructions, so one barrier is all that separates two stages;
//   * token fragments are read three 32-token sub-tiles ahead of the matrix instructions that use them.
// Measured on the MLP block (11008 x 4096 and 4096 x 11008 weights, 8192 tokens): 1.75-2.0 PFLOP/s
// dense-equivalent against 1.5 with 256 x 128 tiles.  The kernel takes the same time with every matrix
// instruction replaced by one ALU operation: what bounds it is each CU's vector-memory path (104 KB per
// stage, every line an L1 miss by construction, ~53 lines in flight per CU at a mean L2 round trip of 250
// clocks: 27 B/clk/CU), and the tile already holds as many accumulators as the register file allows.
// Half tiles (512 x 64, and 256 x 128 inside the persistent loop) for the last, partial round over the
// chip were measured and dropped: the half round they save costs less than their lower efficiency and
// the second copy of the stage code.
#include "gemm_sp24_big_body.hpp"

namespace bimask {
namespace {

__global__ void __launch_bounds__(kBigThreads)
k_gemm_sp24_big(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int64_t Adim, int nk,
                const uint16_t* __restrict__ Bm, int64_t T, int64_t ldb, uint16_t* __restrict__ C, int64_t ldc,
                int tiles_a, int tiles_t, int tpx) {
    gemm_sp24_big_body(A, Ameta, Adim, nk, Bm, T, ldb, C, ldc, tiles_a, tiles_t, tpx, PlainOut{});
}

}  // namespace

// Shapes the large-problem kernel takes: whole stages, a contraction long enough (at least 8 stages) that a
// tile's matrix loop outweighs its prologue and epilogue, and enough tiles that the chip is covered twice over.
bool gemm_sp24_big_shape(int64_t Adim, int64_t K, int64_t T) {
    return K % 128 == 0 && K >= 1024 && Adim >= 1024 && Adim % 8 == 0 &&
           ceil_div(Adim, kBigRows) * ceil_div(T, kBigTokens) >= 512;
}

int launch_gemm_sp24_big(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, const void* Bm, int64_t T,
                         int64_t ldb, void* C, int64_t ldc, hipStream_t s) {
    if (!gemm_sp24_big_shape(Adim, K, T)) return BIMASK_ERR_UNSUPPORTED;
    if (!aligned16(A) || !aligned16(meta) || !aligned16(Bm) || !aligned16(C) || ldb % 8 || ldc % 8) return BIMASK_ERR_UNSUPPORTED;
    const int tiles_a = static_cast<int>(ceil_div(Adim, kBigRows));
    const int64_t tiles_t = ceil_div(T, kBigTokens);
    const int64_t tpx = ceil_div(tiles_t, 8);
    // 32-bit element offsets inside the weight operand and inside the token matrix, 32-bit tile counts
    if (round_up(Adim, 32) * (K / 2) > 0x7FFFFFFFll || T * ldb + K > 0x7FFFFFFFll || tiles_t * tiles_a > 0x0FFFFFFFll)
        return BIMASK_ERR_UNSUPPORTED;
    static DeviceMemo attr_set;
    const int dev = DeviceMemo::device();
    auto kern = k_gemm_sp24_big;
    if (!attr_set.get(dev)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kBigSmem) != hipSuccess)
            return BIMASK_ERR_HIP;
        attr_set.set(dev, 1);
    }
    // 256 persistent workgroups: one per CU (128 KB of LDS and 256 registers per wavefront leave room for one)
    hipLaunchKernelGGL(kern, dim3(256), dim3(kBigThreads), kBigSmem, s,
                       static_cast<const uint16_t*>(A), meta, Adim, static_cast<int>(K / 128),
                       static_cast<const uint16_t*>(Bm), T, ldb, static_cast<uint16_t*>(C), ldc, tiles_a,
                       static_cast<int>(tiles_t), static_cast<int>(tpx));
    return check_launch();
}

}  // namespace bimask
