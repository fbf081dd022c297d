// The linear layer's product with its epilogue:  Z = X (B .* W)^T + bias,  Y = act(Z) + residual  (operand of Eq. (3),
// arXiv 2302.06058), on request with Z's 8-bit checkpoint.  linear_epilogue.hpp holds the epilogue; the main loops are those of
// the plain products (gemm_sp24_body.hpp, gemm_f32_body.hpp) and, for few tokens, the kernel below.
#include "gemm_sp24_body.hpp"
#include "gemm_f32_body.hpp"
#include "linear_epilogue.hpp"

namespace bimask {
namespace {

template <int BM, int BN, int WAVES_M, int WAVES_N, int KG, int PF, bool BGUARD, bool BHALF, bool KTAIL, bool DENSE>
__global__ void __launch_bounds__(64 * WAVES_M * WAVES_N * KG)
k_linear_sp24(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int64_t Adim, int64_t K,
              const uint16_t* __restrict__ Bm, int64_t T, int64_t ldb, uint16_t* C, int64_t ldc,
              int tiles_a, bool vecC, LinearOut out) {
    gemm_sp24_body<BM, BN, WAVES_M, WAVES_N, KG, PF, BGUARD, BHALF, KTAIL, DENSE>(A, Ameta, Adim, K, Bm, T, ldb, C, ldc, tiles_a, vecC, out);
}

// Few tokens (single-token serving and small batches): the weights are read once and nothing else counts, so every workgroup
// takes ONE row tile of 32 against up to 32 tokens and its wavefronts split the contraction, stage by stage, with two stages of
// weight fragments (8.5 KB a wavefront) in flight each.  Token fragments come straight from the rows (L1 and L2 hold them).
// The wavefronts' sums meet in LDS in wavefront order.
constexpr int kFewWaves = 8;

template <bool GUARD, bool DENSE>
__global__ void __launch_bounds__(64 * kFewWaves)
k_linear_few(const uint16_t* __restrict__ A, const uint32_t* __restrict__ Ameta, int64_t Adim, int64_t K, const uint16_t* __restrict__ Bm,
             int64_t T, int64_t ldb, uint16_t* C, int64_t ldc, bool vecC, LinearOut out) {
    constexpr int NW = kFewWaves, NA = DENSE ? 8 : 4, U = DENSE ? 1 : 2;         // stages in flight
    __shared__ f32x4 part[(NW - 1) * 4 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    const int64_t rt = blockIdx.x, t0 = static_cast<int64_t>(blockIdx.y) * 32;
    const int nk = static_cast<int>(ceil_div(K, SK));
    const uint16_t* row = Bm + (t0 + l32 < T ? t0 + l32 : T - 1) * ldb;          // clamped: computed, never stored
    const uint16_t* pa = A + (rt * nk * (NA * 64) + lane) * 8;
    const uint32_t* pm = DENSE ? nullptr : Ameta + (rt * nk * 64 + lane) * 2;
    f32x16 acc[1][1];
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[0][0][q] = 0.f;
    for (int st = wave; st < nk; st += NW * U) {
        u32x4 ra[U][NA];
        u32x2 rm[U];
        BFrag b[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kt = st + u * NW < nk ? st + u * NW : nk - 1;              // clamped: loaded, not used
#pragma unroll
            for (int g = 0; g < NA; ++g) ra[u][g] = *reinterpret_cast<const u32x4*>(pa + (static_cast<int64_t>(kt) * NA + g) * 512);
            if constexpr (!DENSE) rm[u] = *reinterpret_cast<const u32x2*>(pm + static_cast<int64_t>(kt) * 128);
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int64_t k = static_cast<int64_t>(kt) * SK + 64 * c + 16 * s4 + 8 * h;
                    if constexpr (GUARD) {
                        b[u][s4].q[c] = load_guarded(row, k, K);
                    } else {                                                     // K is a multiple of 8: whole granules, or none
                        const u32x4 v = *reinterpret_cast<const u32x4*>(row + (k < K ? k : 0));
                        b[u][s4].q[c] = k < K ? v : (u32x4){0u, 0u, 0u, 0u};
                    }
                }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (st + u * NW < nk) {
#pragma unroll
                for (int s4 = 0; s4 < 4; ++s4) {
                    if constexpr (DENSE) {
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            AFrag af, bh;
                            af.q = ra[u][2 * s4 + x];
                            bh.q = b[u][s4].q[x];
                            acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af.v, bh.v, acc[0][0], 0, 0, 0);
                        }
                    } else {
                        AFrag af;
                        af.q = ra[u][s4];
                        const int idx = static_cast<int>(s4 < 2 ? rm[u].x : rm[u].y);
                        if (s4 & 1) acc[0][0] = __builtin_amdgcn_smfmac_f32_32x32x32_bf16(af.v, b[u][s4].v, acc[0][0], idx, 0, 1);
                        else acc[0][0] = __builtin_amdgcn_smfmac_f32_32x32x32_bf16(af.v, b[u][s4].v, acc[0][0], idx, 0, 0);
                    }
                }
            }
    }
    if (wave > 0)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            part[((wave - 1) * 4 + q) * 64 + lane] = (f32x4){acc[0][0][4 * q], acc[0][0][4 * q + 1], acc[0][0][4 * q + 2], acc[0][0][4 * q + 3]};
    __syncthreads();
    if (wave == 0)
#pragma unroll
        for (int w = 0; w < NW - 1; ++w)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 x = part[(w * 4 + q) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[0][0][4 * q + e] += x[e];
            }
    __syncthreads();
    out.finish<32, 32, 32, 32, 1, 1, 64 * NW>(acc, reinterpret_cast<uint8_t*>(part), wave == 0, 0, 0, lane, rt * 32, t0, Adim, T, C, ldc, vecC);
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

template <int BM, int BN, int WAVES_M, int WAVES_N, int KG, int PF, bool BGUARD, bool BHALF, bool KTAIL, bool DENSE>
int run_t(const Problem& p, const LinearOut& out) {
    using S = SpSmem<BN, KG>;
    auto kern = k_linear_sp24<BM, BN, WAVES_M, WAVES_N, KG, PF, BGUARD, BHALF, KTAIL, DENSE>;
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

// rows: 0 whole stages of 16-byte token rows, 1 the last stage may end early (K a multiple of 8), 2 any rows (4-byte loads)
template <int BM, int BN, int WAVES_M, int WAVES_N, int PF, bool BHALF, int KG, bool DENSE>
int run(const Problem& p, const LinearOut& out, int rows) {
    if (rows == 0) return run_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, BHALF, false, DENSE>(p, out);
    if (rows == 1) return run_t<BM, BN, WAVES_M, WAVES_N, KG, PF, false, BHALF, true, DENSE>(p, out);
    return run_t<BM, BN, WAVES_M, WAVES_N, KG, 1, true, false, false, DENSE>(p, out);
}

template <bool GUARD, bool DENSE>
int run_few(const Problem& p, const LinearOut& out) {
    if (ceil_div(p.Adim, 32) * (64 * kFewWaves) > 0xFFFFFFFFll) return BIMASK_ERR_SHAPE;
    const dim3 grid(static_cast<unsigned>(ceil_div(p.Adim, 32)), static_cast<unsigned>(ceil_div(p.T, 32)));
    hipLaunchKernelGGL((k_linear_few<GUARD, DENSE>), grid, dim3(64 * kFewWaves), 0, p.s, static_cast<const uint16_t*>(p.A), p.meta, p.Adim, p.K,
                       static_cast<const uint16_t*>(p.Bm), p.T, p.ldb, static_cast<uint16_t*>(p.C), p.ldc, aligned16(p.C) && p.ldc % 8 == 0, out);
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
    if (p.T <= 32) return rows == 2 ? run_few<true, DENSE>(p, out) : run_few<false, DENSE>(p, out);
    const bool split32 = p.K > (rows16 ? 256 : 384) && gemm_few_tiles(p.Adim, p.T);
    if (split32) return run<64, 32, 2, 1, 1, false, 4, DENSE>(p, out, rows);
    if (p.Adim <= 64) return run<64, 64, 2, 2, 2, false, 1, DENSE>(p, out, rows);
    const int64_t w256 = round_up(p.Adim, 256), w128 = round_up(p.Adim, 128);
    const bool narrow = (w256 - w128) * 5 >= w256, big = ceil_div(p.Adim, 256) * ceil_div(p.T, 128) >= 190;
    if (!narrow && big) return run<256, 128, 8, 1, 1, false, 1, DENSE>(p, out, rows);
    return run<128, 64, 4, 1, 2, false, 1, DENSE>(p, out, rows);
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
