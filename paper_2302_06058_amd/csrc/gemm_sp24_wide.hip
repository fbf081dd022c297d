// N:M-sparse bf16 GEMM for wide outputs and contractions up to 512 terms (arXiv 2302.06058, Eq. (3) and Eq. (10)):
//     C[t][a] = sum_k Bsrc[t][perm[k]] * A[a][k]
//
// A workgroup loads its token tile once (64 or 128 whole rows, granules XOR-swizzled as in the streaming kernel; Eq. (10)'s gather
// is a 2-byte scatter on the way in) and its eight wavefronts then work on their own: each takes pairs of weight-row tiles (64
// rows) in turn against ALL tokens of the tile, weights from L2 into registers that are re-loaded as soon as they are used, and
// writes its 64 columns through an LDS strip of its own as whole 128-byte lines.  No barrier after the fill, so one wavefront's
// output overlaps another's products (not its own: its next tile waits for weights requested before its stores).  The weight-row-tile loop of the resident kernel (32 rows per wavefront, a barrier per
// 256) reads every token fragment from LDS for one matrix instruction; here it serves two, and with 128 tokens a weight fragment
// serves four: half the LDS reads and half the weight bytes through the CU.
// Measured, us (resident or streaming -> here; means over four cards, buffers in turn): 384 -> 1536 columns with the gather at 25216
// tokens 45.2 -> 33.1, without 38.4 -> 30.0, 4:8 47.4 -> 37.5; 384 -> 1152 29.3 -> 21.7.  What bounds it (timestamps, 384 -> 1536): 8 us
// until the rows are in LDS, then 5.7 per 64 x 100 tile of a wavefront, half of it its output (4 TB/s over the chip).
#include "gemm_sp24_wide_body.hpp"

namespace bimask {
namespace {

template <int TN, bool DENSE>
__global__ void __launch_bounds__(64 * kWideWaves, 2)
k_gemm_sp24_wide(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int Adim, int K,
                 const uint16_t* __restrict__ Bsrc, int64_t ldb, const int32_t* __restrict__ perm, int64_t T,
                 uint16_t* __restrict__ C, int64_t ldc, int rpt, int wpp, bool stream_out) {
    gemm_sp24_wide_body<TN, DENSE>(A, Ameta, Adim, K, Bsrc, ldb, perm, T, C, ldc, rpt, wpp, stream_out, PlainOut{});
}

template <int TN, bool DENSE>
int run_wide(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, const void* Bsrc, int64_t ldb, const int32_t* perm,
             int64_t T, void* C, int64_t ldc, const WidePlan& p, hipStream_t s) {
    auto kern = k_gemm_sp24_wide<TN, DENSE>;
    static DeviceMemo attr_set;
    const int dev = DeviceMemo::device();
    if (!attr_set.get(dev)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kWideLds) != hipSuccess)
            return BIMASK_ERR_HIP;
        attr_set.set(dev, 1);
    }
    const bool stream_out = streams_out(C, Adim, ldc, false);
    hipLaunchKernelGGL(kern, dim3(p.grid, p.pieces), dim3(64 * kWideWaves), p.lds, s, static_cast<const uint16_t*>(A), meta,
                       static_cast<int>(Adim), static_cast<int>(K), static_cast<const uint16_t*>(Bsrc), ldb, perm, T,
                       static_cast<uint16_t*>(C), ldc, p.rpt, p.wpp, stream_out);
    return check_launch();
}

}  // namespace

// Returns BIMASK_ERR_UNSUPPORTED where shape or alignment are outside this kernel, or another one is the faster.
int launch_gemm_sp24_wide(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, const void* Bsrc, int64_t ldb,
                          const int32_t* perm, int64_t T, void* C, int64_t ldc, hipStream_t s, bool dense) {
    if (K > 512 || K % 8 != 0 || Adim % 8 != 0 || T > 0x7FFFFFFF) return BIMASK_ERR_UNSUPPORTED;
    if (ldc >= (1 << 28)) return BIMASK_ERR_UNSUPPORTED;                // 32-bit offsets over 8 output rows
    if (!aligned16(A) || !aligned16(meta) || !aligned16(Bsrc) || !aligned16(C) || ldb % 8 != 0 || ldc % 8 != 0)
        return BIMASK_ERR_UNSUPPORTED;
    if (!disjoint(Bsrc, T, ldb, K, C, ldc, Adim, 2)) return BIMASK_ERR_UNSUPPORTED;     // pieces of weight rows read the same tokens
    // Where it gains (700 random shapes, us, old -> here).  2-of-4, above one stage of 128 terms and 256 columns: 160 -> 512 at 20591
    // tokens 12.6 -> 9.6, 384 -> 3008 with the gather at 20856 77.6 -> 50.6, 352 -> 1256 at 3617 9.9 -> 8.1; not 128 -> 2944 at 13325
    // 18.5 / 20.9, 480 -> 320 at 34188 21.4 / 23.1 apart, few tokens (184 -> 3936 at 3185 11.1 / 12.1) where the weight stream counts, and
    // many tokens whose columns cannot stream out (192 -> 2320 at 34405 63.0 / 66.6; 4:8 328 -> 728 at 80233 78.7 / 89.4).  Dense,
    // which has no resident kernel: from 256 columns (160 -> 1360 at 12712 23.1 -> 17.7, with the gather 128 -> 800 at 8244 12.9 ->
    // 10.7; not 192 -> 384 with it at 77300 34.7 / 38.3, which un-permutes the weights instead, 464 -> 1480 at 8649 26.6 / 27.7).
    const bool sectors = Adim % 32 == 0 || (T < 16384 && K > (dense ? 160 : 256));
    const bool gains = dense
        ? K >= 64 && K <= 416 && sectors &&
          ((Adim > 512 && T >= 4096) || (Adim > 256 && T >= 5000 && (!perm || K <= 160)) || (Adim > 1024 && T >= 2048))
        : K > 128 && sectors &&
          ((Adim > 512 && T >= 5000) || (Adim > 256 && T >= 16384) || (Adim > 1024 && K > 256 && T >= 3072));
    if (!gains) return BIMASK_ERR_UNSUPPORTED;
    // Two stages, against the resident kernel where that fills one or two rounds of workgroups: it writes rows in pieces of 256
    // columns, this one in pieces of 64, both ends of which lie inside a 128-byte line where the columns are an odd multiple of 32.
    // 1504 shapes and 191 more; resident -> here with the resident kernel's slots more than 70 % (one round) or 80 % full: 8 % slower in
    // the mean (192 -> 3040 with the gather at 32475 tokens 49.8 / 60.4, 160 -> 3232 at 6665 15.3 / 18.6, 224 -> 3680 without at 16316
    // 31.4 / 37.0); with 43 to 62 % 14 % faster, from 33000 tokens 3 %, at 5000 10 %, columns that are multiples of 64 12 %.
    if (!dense && K <= 256 && Adim % 64 != 0 && Adim > (perm ? 768 : 1024) && T > 5400 && T <= 32768 &&
        gemm_sp24_resident_fill(Adim, T) > (T <= 16384 ? 0.7 : 0.8))
        return BIMASK_ERR_UNSUPPORTED;
    // Four stages, where only tiles of 64 tokens fit: not with a second round just begun (448 -> 384 at 16681 tokens 11.7 / 12.9, 480 -> 640
    // at 18165 18.1 / 19.5, 512 -> 576 at 20953 17.6 / 19.2, but 416 -> 544 at 21834 24.0 -> 19.2; 448 -> 480 at 16421, where the streaming
    // kernel's 256-row tiles are not full, 16.9 -> 14.2; 416 -> 1056 at 19755 32.0 -> 25.7; with the gather always).
    if (!dense && !perm && K > 384 && Adim <= 768 && (Adim <= 384 || Adim > 512) && T > 16384 && T < 21760) return BIMASK_ERR_UNSUPPORTED;
    WidePlan p2, p4;
    const double us2 = wide_plan(2, Adim, K, T, perm != nullptr, dense, p2), us4 = wide_plan(4, Adim, K, T, perm != nullptr, dense, p4);
    if (us2 == 0) return BIMASK_ERR_UNSUPPORTED;
    if (us4 != 0 && us4 < us2)
        return dense ? run_wide<4, true>(A, meta, Adim, K, Bsrc, ldb, perm, T, C, ldc, p4, s)
                     : run_wide<4, false>(A, meta, Adim, K, Bsrc, ldb, perm, T, C, ldc, p4, s);
    return dense ? run_wide<2, true>(A, meta, Adim, K, Bsrc, ldb, perm, T, C, ldc, p2, s)
                 : run_wide<2, false>(A, meta, Adim, K, Bsrc, ldb, perm, T, C, ldc, p2, s);
}

}  // namespace bimask
