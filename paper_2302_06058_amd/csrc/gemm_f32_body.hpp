// Tile of the fp32 N:M GEMM for gfx950 (gemm_f32.hip states the design), shared by the plain product and the one with bias,
// activation and residual.
#pragma once
#include "mfma_types.hpp"

namespace bimask {
namespace {

constexpr int kTile = 16;             // output tile: 16 weight rows x 16 tokens
typedef f32x4 f32x4_row __attribute__((aligned(4)));      // 16 bytes of a token row: rows start on 4 bytes at least
constexpr int64_t kManyTiles = 8192;  // 16 x 16 tiles from which a workgroup takes 64 weight rows (one step: 4 times as many)
constexpr int64_t kTilesX = 1 << 20;  // tiles in the x dimension of a launch at most

// one 8-index piece of a weight row: SPARSE: decoded from 4 slot values and 16 index bits
template <bool SPARSE>
struct WeightPiece {
    f32x4 v[SPARSE ? 1 : 2];
    uint32_t bits;
};

template <bool SPARSE>
__device__ __forceinline__ void load_weights(const float* __restrict__ A, const uint32_t* __restrict__ meta, int64_t row,
                                             int64_t k, int64_t ks, WeightPiece<SPARSE>& w) {
    if constexpr (SPARSE) {
        const int64_t g = k >> 2;                            // first of two groups: slots 2g .. 2g+3, nibbles g, g+1
        w.v[0] = *reinterpret_cast<const f32x4*>(A + tiled_val_off(row, 2 * g, ks));
        w.bits = meta[tiled_idx_word(row, g, ks)] >> (4 * (g & 7));
    } else {
        const float* p = A + tiled_dense_off(row, k, ks);
        w.v[0] = *reinterpret_cast<const f32x4*>(p);
        w.v[1] = *reinterpret_cast<const f32x4*>(p + 4);
    }
}

template <bool SPARSE>
__device__ __forceinline__ float weight_at(const WeightPiece<SPARSE>& w, int e) {      // e is compile-time after unrolling
    if constexpr (SPARSE) {
        const uint32_t nib = w.bits >> (4 * (e >> 2));
        const uint32_t p0 = nib & 3u, p1 = (nib >> 2) & 3u, pos = e & 3;
        const float hi = p1 == pos ? w.v[0][2 * (e >> 2) + 1] : 0.f;
        return p0 == pos ? w.v[0][2 * (e >> 2)] : hi;
    } else {
        return w.v[e >> 2][e & 3];
    }
}

// R: row tiles of a workgroup (16 R weight rows x 16 tokens); the token pieces are loaded once for all of them and the output
// leaves in segments of 64 R bytes.  Token rows may start on any 4 bytes: the 16-byte loads need no more (256 x 256 at 50176
// tokens, rows of 1028 bytes, 4:8: 254 us with 4-byte loads, 85).
// OUT: what becomes of the sums (PlainOut: written).
template <bool SPARSE, bool PERM, int NW, int R, class OUT>
__device__ __forceinline__ void
gemm_f32_body(const float* A, const uint32_t* meta, int64_t Adim, int64_t K, const float* Bm, int64_t T, int64_t ldb, const int32_t* perm,
              float* C, int64_t ldc, uint32_t tiles_a, uint32_t tiles, const OUT& out) {
    // partial sums [wave][row tile][register][lane]; strides that spread 64 consecutive outputs over all banks
    constexpr int SQ = 68, SR = 4 * SQ + 1;
    __shared__ float part[NW * R * SR];
    const uint32_t tile = blockIdx.y * gridDim.x + blockIdx.x;
    if (tile >= tiles) return;                               // whole workgroup
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c = lane & 15, q = lane >> 4;
    const uint32_t tt = tile / tiles_a;
    const int64_t a0 = static_cast<int64_t>(tile - tt * tiles_a) * (kTile * R), t0 = static_cast<int64_t>(tt) * kTile;
    const int64_t ks = ceil_div(K, 128);
    const float* brow = Bm + (t0 + c < T ? t0 + c : T - 1) * ldb;      // clamped: computed, never stored

    f32x4 acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int64_t k0 = static_cast<int64_t>(wave) * 32; k0 < K; k0 += 32 * NW) {
        const int64_t k = k0 + 8 * q;                        // this lane's 8 contraction indices (weights zero beyond K)
        WeightPiece<SPARSE> w[R];
#pragma unroll
        for (int r = 0; r < R; ++r)                          // the operand is zero-padded to whole 32-row tiles, not further
            if (r == 0 || a0 + kTile * r < Adim) load_weights<SPARSE>(A, meta, a0 + kTile * r + c, k, ks, w[r]);
        float b[8];
        if constexpr (PERM) {
            int col[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) col[e] = k + e < K ? perm[k + e] : -1;
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = col[e] >= 0 ? brow[col[e]] : 0.f;
        } else {                                             // K is a multiple of 4: whole 16-byte pieces
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                f32x4 x = {0.f, 0.f, 0.f, 0.f};
                if (k + 4 * v < K) x = *reinterpret_cast<const f32x4_row*>(brow + k + 4 * v);
#pragma unroll
                for (int e = 0; e < 4; ++e) b[4 * v + e] = x[e];
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r == 0 || a0 + kTile * r < Adim) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    acc[r] = __builtin_amdgcn_mfma_f32_16x16x4f32(weight_at<SPARSE>(w[r], e), b[e], acc[r], 0, 0, 0);
            }
    }
    // lane (c, q) holds token c, weight rows 4 q .. 4 q + 3 of every row tile
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[(wave * R + r) * SR + e * SQ + lane] = acc[r][e];
    __syncthreads();
    for (int i = tid; i < kTile * kTile * R; i += 64 * NW) {
        const int t = i / (kTile * R), a = i % (kTile * R);
        const float* p = part + (a >> 4) * SR + (a & 3) * SQ + t + 16 * ((a & 15) >> 2);
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) s += p[w * R * SR];
        if constexpr (OUT::kFused) out.finish(s, a0 + a, t0 + t, Adim, T, C, ldc);
        else if (t0 + t < T && a0 + a < Adim) C[(t0 + t) * ldc + a0 + a] = s;
    }
}

}  // namespace
}  // namespace bimask
