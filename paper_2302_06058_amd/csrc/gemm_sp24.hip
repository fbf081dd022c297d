// 2:4-sparse bf16 GEMM for gfx950, streaming variant:  C[t][a] = sum_k Bm[t][k] * A[a][k]
// with A given as compressed values + 2-bit indices (the operand of Eq. 3 / Eq. 10 of
// arXiv 2302.06058).
//
// Design (one stage = 128 dense k):
//   * the compressed weights never touch LDS: they are stored fragment-major (see
//     include/bimask.h), i.e. the 16 bytes of values lane l needs for instruction s of a
//     stage sit at [row tile][stage][s][l], so a wavefront fetches each A operand as one
//     fully contiguous 1 KB load (and its indices as one 512-byte load) straight into the
//     operand registers;
//   * the token operand is loaded 256 bytes per row with 16-byte lanes, staged through a
//     double-buffered XOR-swizzled LDS tile and read back as 16-byte fragments;
//   * PF stages of both operands are kept in flight in registers, so a workgroup has
//     PF * (BM*72 + BN*256) bytes outstanding to hide HBM latency;
//   * fp32 accumulators are rounded to bf16, regrouped by a swap between the two lane halves
//     and a pass through LDS, and written as whole row segments with streaming stores.
// Lane/operand mapping of v_smfmac_f32_32x32x32_bf16 (checked on the device): lane l holds
// weight row l%32; with h = l/32, compressed element e of the A register pairs with slot
// 8h + 4((e%4)/2) + idx_e of the B register of token lane half e/4, and idx_e sits in bits
// [2e+1:2e] of the 16-bit index set selected by ABID.
#include "gemm_sp24_body.hpp"

namespace bimask {
namespace {

template <int BM, int BN, int WAVES_M, int WAVES_N, int KG, int PF, bool BGUARD, bool BHALF, bool KTAIL, bool DENSE>
__global__ void __launch_bounds__(64 * WAVES_M * WAVES_N * KG)
k_gemm_sp24(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int64_t Adim, int64_t K,
            const uint16_t* __restrict__ Bm, int64_t T, int64_t ldb, uint16_t* __restrict__ C, int64_t ldc,
            int tiles_a, bool vecC) {
    gemm_sp24_body<BM, BN, WAVES_M, WAVES_N, KG, PF, BGUARD, BHALF, KTAIL, DENSE, BN>(A, Ameta, Adim, K, Bm, T, ldb, C, ldc, tiles_a, vecC, PlainOut{});
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int KG, int PF, bool BGUARD, bool BHALF, bool KTAIL = false, bool DENSE = false>
int run_sp24_t(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, const void* Bm, int64_t T, int64_t ldb,
             void* C, int64_t ldc, hipStream_t s) {
    using S = SpSmem<BN, KG>;
    auto kern = k_gemm_sp24<BM, BN, WAVES_M, WAVES_N, KG, PF, BGUARD, BHALF, KTAIL, DENSE>;
    if (S::kTotal > 48 * 1024) {
        static DeviceMemo attr_set;
        const int dev = DeviceMemo::device();
        if (!attr_set.get(dev)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                    S::kTotal) != hipSuccess) return BIMASK_ERR_HIP;
            attr_set.set(dev, 1);
        }
    }
    const bool vecC = aligned16(C) && (ldc * 2) % 16 == 0;
    const int tiles_a = static_cast<int>(ceil_div(Adim, BM));
    const int64_t tiles_t = ceil_div(T, BN);
    const int64_t grid = ceil_div(tiles_a * tiles_t, 8) * 8;      // whole rounds over the 8 XCDs
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(64 * WAVES_M * WAVES_N * KG), S::kTotal, s,
                       static_cast<const uint16_t*>(A), meta, Adim, K, static_cast<const uint16_t*>(Bm), T, ldb,
                       static_cast<uint16_t*>(C), ldc, tiles_a, vecC);
    return check_launch();
}

template <int BM, int BN, int WAVES_M, int WAVES_N, int PF, bool BHALF = false, int KG = 1>
int run_sp24(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, const void* Bm, int64_t T, int64_t ldb,
             void* C, int64_t ldc, hipStream_t s) {
    const bool rows16 = aligned16(Bm) && (ldb * 2) % 16 == 0;
    if (rows16 && K % SK == 0) return run_sp24_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, BHALF>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
    if (rows16 && K % 8 == 0) return run_sp24_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, BHALF, true>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
    return run_sp24_t<BM, BN, WAVES_M, WAVES_N, KG, 1, true, false>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
}

// dense masked weights: aligned token rows and a contraction that is a multiple of 8 only (the caller
// takes the general dense kernel otherwise)
template <int BM, int BN, int WAVES_M, int WAVES_N, int PF, int KG = 1>
int run_dense_frag(const void* A, int64_t Adim, int64_t K, const void* Bm, int64_t T, int64_t ldb, void* C, int64_t ldc,
                   hipStream_t s) {
    if (K % SK == 0) return run_sp24_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, false, false, true>(A, nullptr, Adim, K, Bm, T, ldb, C, ldc, s);
    return run_sp24_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, false, true, true>(A, nullptr, Adim, K, Bm, T, ldb, C, ldc, s);
}

}  // namespace

// 2:4 GEMM on the fragment-major weight operand.
//   256 x 64, 4 wavefronts, 2 stages prefetched: mid-size problems (the grid covers the chip)
//   128 x 64, 4 wavefronts: weight dimensions that would leave 256-row tiles largely empty, or few tokens
//   256 x 128, 8 wavefronts, 1 stage prefetched: large problems (half the weight traffic per token)
//   64 x 64, 4 wavefronts of 32 x 32: at most 64 weight rows (no matrix work or fragment reads on padding rows)
//   64 x 32, 4 groups of 2 wavefronts / 64 x 64, 2 groups of 4 wavefronts splitting the contraction: few tiles
int launch_gemm_sp24(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, const void* Bm, int64_t T,
                     int64_t ldb, void* C, int64_t ldc, Sp24Tile tile, hipStream_t s) {
    if (!aligned16(A) || !aligned16(meta)) return BIMASK_ERR_ALIGN;
    switch (tile) {
        case Sp24Tile::k256x64: return run_sp24<256, 64, 4, 1, 2, true>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
        case Sp24Tile::k128x64: return run_sp24<128, 64, 4, 1, 2>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
        case Sp24Tile::k256x128: return run_sp24<256, 128, 8, 1, 1>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
        case Sp24Tile::k64x64: return run_sp24<64, 64, 2, 2, 2>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
        case Sp24Tile::k64x32Split: return run_sp24<64, 32, 2, 1, 1, false, 4>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
        case Sp24Tile::k64x64Split: return run_sp24<64, 64, 2, 2, 1, false, 2>(A, meta, Adim, K, Bm, T, ldb, C, ldc, s);
    }
    return BIMASK_ERR_UNSUPPORTED;
}

// The same streaming kernel on the dense masked operand of a ratio with N > 2 (dense 32x32x16 matrix
// instructions).  BIMASK_ERR_UNSUPPORTED when the token rows are not 16-byte aligned or the contraction is no
// multiple of 8: the caller then takes the general dense kernel.
//   128 x 64, 4 wavefronts, 2 stages prefetched; 256 x 128, 8 wavefronts, for large problems; 64 x 64 for at
//   most 64 weight rows.  (256 x 64 with two row tiles per wavefront would need 128 registers of weight
//   fragments per stage in flight.)
int launch_gemm_dense_frag(const void* A, int64_t Adim, int64_t K, const void* Bm, int64_t T, int64_t ldb, void* C,
                           int64_t ldc, hipStream_t s) {
    if (!aligned16(A) || !aligned16(Bm) || (ldb * 2) % 16 != 0 || K % 8 != 0) return BIMASK_ERR_UNSUPPORTED;
    // few tiles: a single stage, or up to two with at most 64 rows, gains nothing from the split (512 x 128 at 256 tokens 4.2 us,
    // split 4.5; 64 x 256 at 784 3.8 / 4.4), longer contractions do (64 x 512 at 784 4.9 -> 4.6, 512 x 264 at 256 5.7 -> 4.6).
    // Beyond 256 tiles only the deepest would (512 x 2304 at 1088 tokens 15.1 us, split 14.7, 512 x 1152 9.3 / 11.0, 512 x 4608
    // 27.5 / 24.2): not worth an instance of the 64 x 64 split.
    if (K > (Adim <= 64 ? 256 : 128) && gemm_few_tiles(Adim, T))
        return run_dense_frag<64, 32, 2, 1, 1, 4>(A, Adim, K, Bm, T, ldb, C, ldc, s);
    if (Adim <= 64) return run_dense_frag<64, 64, 2, 2, 2>(A, Adim, K, Bm, T, ldb, C, ldc, s);
    const bool big = ceil_div(Adim, 256) * ceil_div(T, 128) >= 190;
    // weight dimensions that would leave a fifth or more of the 256-row tiles empty (384 = 1.5 tiles) take 128-row tiles
    const int64_t w256 = round_up(Adim, 256), w128 = round_up(Adim, 128);
    const bool wasteful = (w256 - w128) * 5 >= w256;
    if (big && !wasteful) return run_dense_frag<256, 128, 8, 1, 1>(A, Adim, K, Bm, T, ldb, C, ldc, s);
    return run_dense_frag<128, 64, 4, 1, 2>(A, Adim, K, Bm, T, ldb, C, ldc, s);
}

}  // namespace bimask
