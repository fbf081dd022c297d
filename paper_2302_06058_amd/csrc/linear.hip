// The linear layer's product with its epilogue:  Z = X (B .* W)^T + bias,  Y = act(Z) + residual  (operand of Eq. (3),
// arXiv 2302.06058), on request with Z's 8-bit checkpoint.  linear_epilogue.hpp holds the epilogue; the main loops are those of
// the plain products (gemm_sp24_body.hpp, gemm_sp24_big_body.hpp, gemm_sp24_wide_body.hpp, gemm_f32_body.hpp).
//
// What bounds it: a few tokens, the weights' bytes (11008 x 4096 at one token 10.5 us for 50.7 MB, 4.8 TB/s; 4096 x 11008 at 13 tokens 12.5);
// the largest products, the plain product's own bound (11008 x 4096 at 8192 tokens with silu and checkpoint 460-530 us by the card's clock,
// the plain product 390-460 beside it); short contractions, the instructions of the epilogue beside the matrix instructions (1536 x 384 at
// 25216 tokens, 4:8 with gelu and checkpoint 74-78 us, with silu 55: the vector units issue 71 % of the time with gelu and the matrix pipe is
// busy 27 %, and two wavefronts per SIMD overlap little of the two; other wavefront priorities change nothing).
#include "gemm_sp24_body.hpp"
#include "gemm_sp24_big_body.hpp"
#include "gemm_sp24_wide_body.hpp"
#include "gemm_f32_body.hpp"
#include "linear_epilogue.hpp"

namespace bimask {
namespace {

template <int BM, int BN, int WAVES_M, int WAVES_N, int KG, int PF, bool BGUARD, bool KTAIL, bool DENSE, int TR>
__global__ void __launch_bounds__(64 * WAVES_M * WAVES_N * KG)
k_linear_sp24(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int64_t Adim, int64_t K,
              const uint16_t* __restrict__ Bm, int64_t T, int64_t ldb, uint16_t* C, int64_t ldc,
              int tiles_a, bool vecC, LinearOut out) {
    gemm_sp24_body<BM, BN, WAVES_M, WAVES_N, KG, PF, BGUARD, false, KTAIL, DENSE, TR>(A, Ameta, Adim, K, Bm, T, ldb, C, ldc, tiles_a, vecC, out);
}

__global__ void __launch_bounds__(kBigThreads)
k_linear_sp24_big(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int64_t Adim, int nk, const uint16_t* __restrict__ Bm,
                  int64_t T, int64_t ldb, uint16_t* C, int64_t ldc, int tiles_a, int tiles_t, int tpx, LinearOut out) {
    gemm_sp24_big_body(A, Ameta, Adim, nk, Bm, T, ldb, C, ldc, tiles_a, tiles_t, tpx, out);
}

template <int TN, bool DENSE>
__global__ void __launch_bounds__(64 * kWideWaves, 2)
k_linear_wide(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int Adim, int K, const uint16_t* __restrict__ Bsrc, int64_t ldb,
              int64_t T, uint16_t* C, int64_t ldc, int rpt, int wpp, bool stream_out, LinearOut out) {
    gemm_sp24_wide_body<TN, DENSE>(A, Ameta, Adim, K, Bsrc, ldb, nullptr, T, C, ldc, rpt, wpp, stream_out, out);
}

template <bool SPARSE, int NW, int R>
__global__ void __launch_bounds__(64 * NW)
k_linear_f32(const float* __restrict__ A, const uint32_t* __restrict__ meta, int64_t Adim, int64_t K, const float* __restrict__ Bm, int64_t T,
             int64_t ldb, float* C, int64_t ldc, uint32_t tiles_a, uint32_t tiles, LinearOutF32 out) {
    gemm_f32_body<SPARSE, false, NW, R>(A, meta, Adim, K, Bm, T, ldb, nullptr, C, ldc, tiles_a, tiles, out);
}

struct Problem {
    const void* A; const uint32_t* meta; int64_t Adim, K; const void* Bm; int64_t T, ldb; void* C; int64_t ldc; hipStream_t s;
};

template <int BM, int BN, int WAVES_M, int WAVES_N, int KG, int PF, bool BGUARD, bool KTAIL, bool DENSE, int TR = BN>
int run_t(const Problem& p, const LinearOut& out) {
    using S = SpSmem<BN, KG>;
    auto kern = k_linear_sp24<BM, BN, WAVES_M, WAVES_N, KG, PF, BGUARD, KTAIL, DENSE, TR>;
    if (S::kTotal > 48 * 1024) {
        static DeviceMemo attr_set;
        const int dev = DeviceMemo::device();
        if (!attr_set.get(dev)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, S::kTotal) != hipSuccess)
                return BIMASK_ERR_HIP;
            attr_set.set(dev, 1);
        }
    }
    const int64_t tiles_a = ceil_div(p.Adim, BM), grid = ceil_div(tiles_a * ceil_div(p.T, BN), 8) * 8;      // whole rounds over the 8 XCDs
    if (grid * (64 * WAVES_M * WAVES_N * KG) > 0xFFFFFFFFll) return BIMASK_ERR_SHAPE;     // a launch counts its work-items in 32 bits
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(64 * WAVES_M * WAVES_N * KG), S::kTotal, p.s,
                       static_cast<const uint16_t*>(p.A), p.meta, p.Adim, p.K, static_cast<const uint16_t*>(p.Bm), p.T, p.ldb,
                       static_cast<uint16_t*>(p.C), p.ldc, static_cast<int>(tiles_a), aligned16(p.C) && p.ldc % 8 == 0, out);
    return check_launch();
}

// (TR: token rows fetched, where the tile has more than there are)
// rows: 0 whole stages of 16-byte token rows, 1 the last stage may end early (K a multiple of 8), 2 any rows (4-byte loads)
template <int BM, int BN, int WAVES_M, int WAVES_N, int PF, int KG, bool DENSE>
int run(const Problem& p, const LinearOut& out, int rows) {
    if (rows == 0) return run_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, false, DENSE>(p, out);
    if (rows == 1) return run_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, true, DENSE>(p, out);
    return run_t<BM, BN, WAVES_M, WAVES_N, KG, 1, true, false, DENSE>(p, out);
}

template <int TN, bool DENSE>
int run_wide(const Problem& p, const LinearOut& out, const WidePlan& w) {
    static DeviceMemo attr_set;
    const int dev = DeviceMemo::device();
    auto kern = k_linear_wide<TN, DENSE>;
    if (!attr_set.get(dev)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kWideLds) != hipSuccess)
            return BIMASK_ERR_HIP;
        attr_set.set(dev, 1);
    }
    hipLaunchKernelGGL(kern, dim3(w.grid, w.pieces), dim3(64 * kWideWaves), w.lds, p.s, static_cast<const uint16_t*>(p.A), p.meta,
                       static_cast<int>(p.Adim), static_cast<int>(p.K), static_cast<const uint16_t*>(p.Bm), p.ldb, p.T,
                       static_cast<uint16_t*>(p.C), p.ldc, w.rpt, w.wpp, streams_out(p.C, p.Adim, p.ldc, false), out);
    return check_launch();
}

// Short contractions and wide outputs: the epilogue is most of the work there, and in this kernel it is each wavefront's own.  Against the
// forms below, us: 1536 x 384 at 25216 tokens, 4:8 with gelu and checkpoint 75 / 92, 2:4 66 / 81, with residual 44 / 54, 4:8 with silu 47 / 68;
// 384 x 384 with gelu and checkpoint 23.0 / 24.2, as 2048 x 512 at 2048 11.2 / 11.6.  Below 2^22 outputs its first rows arrive too late (512 x 512
// at 2048 9.8 / 7.6, 2048 x 512 at 1024 10.5 / 9.0), up to 256 features most of its wavefronts have nothing to do (128 x 512 at 25216 19.0 / 11.3).
template <bool DENSE>
int run_short(const Problem& p, const LinearOut& out) {
    if (p.K > 512 || p.K % 8 || p.Adim % 8 || p.Adim <= 256 || p.T < 2048 || p.Adim < ((1 << 22) + p.T - 1) / p.T || p.T > 0x7FFFFFFF || p.ldc >= (1 << 28)) return BIMASK_ERR_UNSUPPORTED;
    if (!aligned16(p.Bm) || !aligned16(p.C) || p.ldb % 8 || p.ldc % 8 || (out.R && !out.vecR)) return BIMASK_ERR_UNSUPPORTED;
    WidePlan p2, p4;
    const double us2 = wide_plan(2, p.Adim, p.K, p.T, false, DENSE, p2), us4 = wide_plan(4, p.Adim, p.K, p.T, false, DENSE, p4);
    if (us2 == 0) return BIMASK_ERR_UNSUPPORTED;
    return us4 != 0 && us4 < us2 ? run_wide<4, DENSE>(p, out, p4) : run_wide<2, DENSE>(p, out, p2);
}

// the largest problems, on conditions of launch_gemm_sp24_big
int run_big(const Problem& p, const LinearOut& out) {
    if (!gemm_sp24_big_shape(p.Adim, p.K, p.T) || !aligned16(p.Bm) || !aligned16(p.C) || p.ldb % 8 || p.ldc % 8) return BIMASK_ERR_UNSUPPORTED;
    const int64_t tiles_a = ceil_div(p.Adim, kBigRows), tiles_t = ceil_div(p.T, kBigTokens);
    if (round_up(p.Adim, 32) * (p.K / 2) > 0x7FFFFFFFll || p.T * p.ldb + p.K > 0x7FFFFFFFll || tiles_t * tiles_a > 0x0FFFFFFFll)
        return BIMASK_ERR_UNSUPPORTED;
    static DeviceMemo attr_set;
    const int dev = DeviceMemo::device();
    if (!attr_set.get(dev)) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(k_linear_sp24_big), hipFuncAttributeMaxDynamicSharedMemorySize, kBigSmem) != hipSuccess)
            return BIMASK_ERR_HIP;
        attr_set.set(dev, 1);
    }
    hipLaunchKernelGGL(k_linear_sp24_big, dim3(256), dim3(kBigThreads), kBigSmem, p.s, static_cast<const uint16_t*>(p.A), p.meta, p.Adim,
                       static_cast<int>(p.K / 128), static_cast<const uint16_t*>(p.Bm), p.T, p.ldb, static_cast<uint16_t*>(p.C), p.ldc,
                       static_cast<int>(tiles_a), static_cast<int>(tiles_t), static_cast<int>(ceil_div(tiles_t, 8)), out);
    return check_launch();
}

template <bool SPARSE, int NW, int R>
int run_f32_t(const Problem& p, const LinearOutF32& out) {
    const int64_t tiles_a = ceil_div(p.Adim, kTile * R), tiles = ceil_div(p.T, kTile) * tiles_a;
    if (tiles > 0x7FFFFFFFll) return BIMASK_ERR_SHAPE;
    const uint32_t x = static_cast<uint32_t>(tiles < kTilesX ? tiles : kTilesX);
    hipLaunchKernelGGL((k_linear_f32<SPARSE, NW, R>), dim3(x, static_cast<uint32_t>(ceil_div(tiles, x))), dim3(64 * NW), 0, p.s,
                       static_cast<const float*>(p.A), p.meta, p.Adim, p.K, static_cast<const float*>(p.Bm), p.T, p.ldb,
                       static_cast<float*>(p.C), p.ldc, static_cast<uint32_t>(tiles_a), static_cast<uint32_t>(tiles), out);
    return check_launch();
}

// As the plain fp32 product, in tiles of 32 weight rows (a block of the checkpoint) instead of 16.
template <bool SPARSE>
int run_f32(const Problem& p, const LinearOutF32& out) {
    const int64_t tiles = ceil_div(p.T, kTile) * ceil_div(p.Adim, kTile);
    if (p.Adim > 2 * kTile && tiles >= (p.K <= 32 ? 4 * kManyTiles : kManyTiles)) {
        if (p.K <= 32) return run_f32_t<SPARSE, 1, 4>(p, out);
        if (p.K <= 64) return run_f32_t<SPARSE, 2, 4>(p, out);
        return run_f32_t<SPARSE, 4, 4>(p, out);
    }
    if (p.K <= 32) return run_f32_t<SPARSE, 1, 2>(p, out);
    if (p.K <= 64) return run_f32_t<SPARSE, 2, 2>(p, out);
    if (tiles >= 2048 || p.K <= 128) return run_f32_t<SPARSE, 4, 2>(p, out);
    return run_f32_t<SPARSE, 8, 2>(p, out);
}

// Tiles as in the plain products (launch_gemm, launch_gemm_dense_frag state what they measured).
template <bool DENSE>
int run_bf16(const Problem& p, const LinearOut& out) {
    const bool rows16 = aligned16(p.Bm) && p.ldb % 8 == 0 && p.K % 8 == 0;
    const int rows = !rows16 ? 2 : p.K % SK == 0 ? 0 : 1;
    if (const int rc = run_short<DENSE>(p, out); rc != BIMASK_ERR_UNSUPPORTED) return rc;
    if constexpr (!DENSE) {
        const int rc = run_big(p, out);
        if (rc != BIMASK_ERR_UNSUPPORTED) return rc;
    }
    // Long contractions with few tiles: split inside the workgroup.  2-of-4: one 32 x 32 tile on eight wavefronts where such tiles are
    // one per CU at most (serving: the weights are read once, and CUs without a tile read none), with as many stages in flight as the
    // token rows leave registers for (4096 x 4096 at one token 5.7 us, with 64 x 32 tiles 8.6; 4096 x 11008 at 13 12.5 / 17.6).
    const bool deep = p.K > (rows16 ? 256 : 384);
    if constexpr (!DENSE)
        if (p.K > 2048 && ceil_div(p.Adim, 32) * ceil_div(p.T, 32) <= 256) {
            if (rows == 2) return run_t<32, 32, 1, 1, 8, 1, true, false, false>(p, out);
            if (p.T <= 4) return run_t<32, 32, 1, 1, 8, 3, false, true, false, 4>(p, out);
            if (p.T <= 16) return run_t<32, 32, 1, 1, 8, 2, false, true, false, 16>(p, out);
            return run_t<32, 32, 1, 1, 8, 1, false, true, false>(p, out);
        }
    if (deep && gemm_few_tiles(p.Adim, p.T)) {
        if constexpr (!DENSE) return run<64, 32, 2, 1, 1, 4, false>(p, out, rows);
        // (the form for whole stages would not fit the registers)
        else return rows == 2 ? run_t<64, 32, 2, 1, 4, 1, true, false, true>(p, out) : run_t<64, 32, 2, 1, 4, 1, false, true, true>(p, out);
    }
    if constexpr (!DENSE)
        if (deep && p.Adim > 64 && ceil_div(p.Adim, 64) * ceil_div(p.T, 64) <= 256) return run<64, 64, 2, 2, 1, 2, false>(p, out, rows);
    if (p.Adim <= 64) return run<64, 64, 2, 2, 2, 1, DENSE>(p, out, rows);
    const int64_t w256 = round_up(p.Adim, 256), w128 = round_up(p.Adim, 128);
    const bool narrow = (w256 - w128) * 5 >= w256, big = ceil_div(p.Adim, 256) * ceil_div(p.T, 128) >= 190;
    if (!narrow && big) return run<256, 128, 8, 1, 1, 1, DENSE>(p, out, rows);
    return run<128, 64, 4, 1, 2, 1, DENSE>(p, out, rows);
}

}  // namespace

int launch_linear(const void* A, const uint32_t* meta, int64_t Adim, int64_t K, bool sparse24, const void* Bm, int64_t T, int64_t ldb, int dtype,
                  const void* bias, int act, const void* residual, int64_t ldr, void* C, int64_t ldc, uint8_t* ckpt, hipStream_t s) {
    const Problem p{A, meta, Adim, K, Bm, T, ldb, C, ldc, s};
    uint8_t* scales = ckpt ? ckpt + T * ckpt_pitch(Adim) : nullptr;
    if (dtype == BIMASK_F32) {
        const LinearOutF32 out{static_cast<const float*>(bias), static_cast<const float*>(residual), ldr, ckpt, scales, act};
        return sparse24 ? run_f32<true>(p, out) : run_f32<false>(p, out);
    }
    const LinearOut out{static_cast<const uint16_t*>(bias), static_cast<const uint16_t*>(residual), ldr, ckpt, scales, act,
                        aligned16(residual) && ldr % 8 == 0};
    return sparse24 ? run_bf16<false>(p, out) : run_bf16<true>(p, out);
}

}  // namespace bimask
