// fp32 N:M GEMM of Bi-Mask (Eq. 3 and Eq. 10 of arXiv 2302.06058) on gfx950:
//     C[t][a] = sum_k Bm[t][perm[k]] * A[a][k]        (perm = null: identity)
// with A in the fragment-major operand format of include/bimask.h, fp32 in, fp32 accumulation, fp32 out.
//
// fp32 layers are small (tens to hundreds of features and tokens), so what counts is the length of the chain of
// dependent memory round trips, not the rate: a workgroup owns one 16 x 16 output tile (four of them side by side in large
// products) and its wavefronts split the CONTRACTION, 32 indices per wavefront and step, so that a layer of 128 inputs is one load round trip, 8 matrix
// instructions per wavefront and one reduction through LDS.  No operand passes through LDS: lane (c, q) = (l % 16,
// l / 16) of v_mfma_f32_16x16x4_f32 wants row c of either operand at contraction index q of four, and which four
// indices one instruction takes is free, so lane quarter q takes the 8 consecutive indices [8 q, 8 q + 8) of the step
// -- half a granule of the operand (16 bytes of slot values, 16 index bits) and 32 contiguous bytes of the token row.
// The column gather of Eq. (10) is in the token loads (4-byte loads through perm), not in a pass of its own.
// Products and sums are fp32 throughout; the wavefronts' partial sums are added in wavefront order.
//
// Measured (forward, W I x J at T tokens, 2:4): 64 x 128 at 32 22 -> 3.0 us (launch floor), 256 x 256 at 256 44 -> 3.2,
// 512 x 512 at 512 82 -> 8.3, 2048 x 2048 at 4096 957 -> 415, 512 x 8 at 401408 436 -> 284, against one 64 x 64 tile of fmaf
// per workgroup that decoded the operand element by element into LDS; the error against float64 fell from
// 1.4e-7 .. 5.7e-7 to 0.8e-7 .. 2.9e-7 (shorter chains of additions).
#include "gemm_f32_body.hpp"

namespace bimask {
namespace {

template <bool SPARSE, bool PERM, int NW, int R>
__global__ void __launch_bounds__(64 * NW)
k_gemm_f32(const float* __restrict__ A, const uint32_t* __restrict__ meta, int64_t Adim, int64_t K,
           const float* __restrict__ Bm, int64_t T, int64_t ldb, const int32_t* __restrict__ perm, float* __restrict__ C,
           int64_t ldc, uint32_t tiles_a, uint32_t tiles) {
    gemm_f32_body<SPARSE, PERM, NW, R>(A, meta, Adim, K, Bm, T, ldb, perm, C, ldc, tiles_a, tiles, PlainOut{});
}

template <bool SPARSE, bool PERM, int NW, int R>
int run_f32_t(const float* A, const uint32_t* meta, int64_t Adim, int64_t K, const float* Bm, int64_t T, int64_t ldb,
              const int32_t* perm, float* C, int64_t ldc, hipStream_t s) {
    const int64_t tiles_a = ceil_div(Adim, kTile * R), tiles = ceil_div(T, kTile) * tiles_a;      // below 2^29: the output fits the card
    if (tiles > 0x7FFFFFFFll) return BIMASK_ERR_SHAPE;
    // A launch counts the work-items of a dimension in 32 bits and cuts off what is beyond, without an error: 2^24 tiles of
    // 256 threads in x alone would be none.  x holds 2^20 tiles (2^30 threads at most), y the rest.
    const uint32_t x = static_cast<uint32_t>(tiles < kTilesX ? tiles : kTilesX);
    const dim3 grid(x, static_cast<uint32_t>(ceil_div(tiles, x)));
    hipLaunchKernelGGL((k_gemm_f32<SPARSE, PERM, NW, R>), grid, dim3(64 * NW), 0, s, A, meta, Adim, K, Bm, T, ldb, perm, C, ldc,
                       static_cast<uint32_t>(tiles_a), static_cast<uint32_t>(tiles));
    return check_launch();
}

template <bool SPARSE, bool PERM>
int run_f32(const float* A, const uint32_t* meta, int64_t Adim, int64_t K, const float* Bm, int64_t T, int64_t ldb,
            const int32_t* perm, float* C, int64_t ldc, hipStream_t s) {
#define BIMASK_GEMM_F32(NW, R) return run_f32_t<SPARSE, PERM, NW, R>(A, meta, Adim, K, Bm, T, ldb, perm, C, ldc, s)
    const int64_t tiles = ceil_div(T, kTile) * ceil_div(Adim, kTile);
    // No wavefront without a step (512 x 8 at 401408 tokens: 812 us with 4 wavefronts of which 3 have nothing to do, 383 with
    // one).  Where 16 x 16 tiles fill the chip several times over, 64 weight rows per workgroup: fewer token loads and whole
    // lines out (the same 284 us; 2048 x 2048 at 4096 565 -> 415; 128 x 512 with 8192 tiles 41 -> 34, with 1024 8.7 / 9.4).
    // Up to 32 rows half of them would be idle (32 x 128 with 8192 tiles 15.1 / 16.0), and a single step gains from 32768
    // tiles on (128 x 16 with 8192 6.5 / 6.9, with 131072 51 -> 47).
    if constexpr (!PERM) {
        if (Adim > 2 * kTile && tiles >= (K <= 32 ? 4 * kManyTiles : kManyTiles)) {
            if (K <= 32) BIMASK_GEMM_F32(1, 4);
            if (K <= 64) BIMASK_GEMM_F32(2, 4);
            BIMASK_GEMM_F32(4, 4);
        }
    }
    if (K <= 32) BIMASK_GEMM_F32(1, 1);
    if (K <= 64) BIMASK_GEMM_F32(2, 1);
    // few tiles: enough wavefronts that each has one or two steps; many tiles fill the chip by themselves
    if (tiles >= 2048 || K <= 128) BIMASK_GEMM_F32(4, 1);
    if (K <= 256) BIMASK_GEMM_F32(8, 1);
    BIMASK_GEMM_F32(16, 1);
#undef BIMASK_GEMM_F32
}

}  // namespace

// The gather in the token loads costs one 4-byte load per token, contraction index and tile of 16 weight rows, the
// separate pass a launch and a read and write of the tokens.  256 x 256 at 256 tokens (64 Ki tile-indices): 4.6 us fused,
// 6.3 with the pass; 512 x 512 at 512 (512 Ki): 19 against 13.
bool gemm_f32_fuses_gather(int64_t T, int64_t Adim, int64_t K) {
    return ceil_div(T, kTile) * ceil_div(Adim, kTile) * K <= (1 << 17);
}

int launch_gemm_f32(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, bool sparse24, const void* Bm, int64_t T,
                    int64_t ldb, const int32_t* perm, void* C, int64_t ldc, hipStream_t s) {
    const float *a = static_cast<const float*>(A), *b = static_cast<const float*>(Bm);
    float* c = static_cast<float*>(C);
    if (sparse24) return perm ? run_f32<true, true>(a, meta, Adim, K, b, T, ldb, perm, c, ldc, s)
                              : run_f32<true, false>(a, meta, Adim, K, b, T, ldb, perm, c, ldc, s);
    return perm ? run_f32<false, true>(a, meta, Adim, K, b, T, ldb, perm, c, ldc, s)
                : run_f32<false, false>(a, meta, Adim, K, b, T, ldb, perm, c, ldc, s);
}

}  // namespace bimask
