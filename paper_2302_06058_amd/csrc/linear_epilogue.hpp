// What the linear layer's product does with its fp32 sums:  Z = sums + bias,  Y = act(Z) + residual, one rounding at the end, and
// on request Z's 8-bit checkpoint (act.hpp).
#pragma once
#include "act.hpp"

namespace bimask {

struct LinearOut {                                       // bf16
    const uint16_t* bias;                                // NULL or Adim entries, 16-byte aligned
    const uint16_t* R;                                   // NULL or the residual; may be the output itself
    int64_t ldr;
    uint8_t* codes;                                      // NULL or the checkpoint
    uint8_t* scales;
    int act;
    bool vecR;                                           // rows of R start on 16 bytes
    static constexpr bool kFused = true;

    // Sums of a workgroup's tile, BM weight rows x BN tokens: a wavefront that is `mine` holds TM x TN accumulators of 32 rows x 32
    // tokens at row WM wm, token WN wn; lane (l32, h) has token l32 and rows 8 q + 4 h + 0..3 in quad q.  A block of the checkpoint is
    // one accumulator's rows of one token: two lanes, so its maximum takes one exchange and no LDS.  Codes, residual and output go
    // through LDS (smem: 2 BM BN bytes at least) and leave or arrive as whole row segments of the tile; the residual waits in the
    // place of the output piece it is added to.
    // Adim is a multiple of 4, so quads are inside or outside; sums beyond it may be NaN and count as 0 in the checkpoint.
    template <int BM, int BN, int WM, int WN, int TM, int TN, int NT, class ACC>
    __device__ __forceinline__ void finish(ACC (&acc)[TM][TN], uint8_t* smem, bool mine, int wm, int wn, int lane, int64_t a0, int64_t t0,
                                           int64_t Adim, int64_t T, uint16_t* C, int64_t ldc, bool vecC) const {
        typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        const int l32 = lane & 31, h = lane >> 5, tid = threadIdx.x;
        const int64_t ar = a0 + wm * WM + 4 * h;         // this lane's first row
        if (bias && mine)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t a = ar + 32 * i + 8 * q;
                    u32x2 b = {0u, 0u};
                    if (a < Adim) b = *reinterpret_cast<const u32x2*>(bias + a);
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[i][j][4 * q + e] += __builtin_bit_cast(float, e & 1 ? b[e >> 1] & 0xFFFF0000u : b[e >> 1] << 16);
                }
        if (codes) {
            constexpr int UPR = BM / 16;                 // 16-byte units of a token's codes in the tile
            uint8_t* sScale = smem + BM * BN;
            if (mine)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        float z[16];
                        uint32_t most = 0;
#pragma unroll
                        for (int q = 0; q < 16; ++q) {
                            z[q] = ar + 32 * i + 8 * (q >> 2) < Adim ? acc[i][j][q] : 0.f;
                            const uint32_t m = __builtin_bit_cast(uint32_t, z[q]) & 0x7FFFFFFFu;
                            most = m > most ? m : most;
                        }
                        const auto both = __builtin_amdgcn_permlane32_swap(most, most, false, false);
                        const int byte = ckpt_scale_byte(both[0] > both[1] ? both[0] : both[1]);
                        const bool bad = byte == kCkptNaN;
                        const float inv = ckpt_inverse(bad ? 127 : byte);
                        uint32_t d[4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) d[q] = ckpt_codes(z + 4 * q, inv, bad);
                        const auto lo = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
                        const auto hi = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
                        const int t = wn * WN + 32 * j + l32, u = (wm * WM + 32 * i) / 16 + h;
                        *reinterpret_cast<u32x4*>(smem + t * BM + ((u ^ (t & (UPR - 1))) << 4)) = (u32x4){lo[0], lo[1], hi[0], hi[1]};
                        if (h == 0) sScale[t * (BM / 32) + wm * (WM / 32) + i] = static_cast<uint8_t>(byte);
                    }
            __syncthreads();
            const int64_t pitch = ckpt_pitch(Adim), blocks = ckpt_blocks(Adim);
            for (int q = tid; q < BN * UPR; q += NT) {
                const int t = q / UPR, u = q % UPR;
                if (t0 + t < T && a0 + 16 * u < pitch)
                    *reinterpret_cast<u32x4*>(codes + (t0 + t) * pitch + a0 + 16 * u) =
                        *reinterpret_cast<const u32x4*>(smem + t * BM + ((u ^ (t & (UPR - 1))) << 4));
            }
            for (int q = tid; q < BN * (BM / 32); q += NT) {
                const int t = q / (BM / 32), b = q % (BM / 32);
                if (t0 + t < T && a0 / 32 + b < blocks) scales[(t0 + t) * blocks + a0 / 32 + b] = sScale[q];
            }
            __syncthreads();
        }
        constexpr int UPR = BM / 8;                      // 16-byte units of a token's outputs in the tile
        if (R) {
            for (int q = tid; q < BN * UPR; q += NT) {
                const int t = q / UPR, u = q % UPR;
                const int64_t a = a0 + 8 * u;
                u32x4 v = {0u, 0u, 0u, 0u};
                if (t0 + t < T && a < Adim) {
                    const uint16_t* src = R + (t0 + t) * ldr + a;
                    if (vecR && a + 8 <= Adim) {
                        v = *reinterpret_cast<const u32x4*>(src);
                    } else {                             // 4-byte pieces (pointer and pitch are 4-byte aligned, Adim even)
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            if (a + 2 * d < Adim) v[d] = *reinterpret_cast<const uint32_t*>(src + 2 * d);
                    }
                }
                *reinterpret_cast<u32x4*>(smem + t * (BM * 2) + ((u ^ ((2 * t) & (UPR - 1))) << 4)) = v;
            }
            __syncthreads();
        }
        if (mine)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    const int t = wn * WN + 32 * j + l32;
                    float y[16];
#pragma unroll
                    for (int q = 0; q < 16; ++q) y[q] = acc[i][j][q];
                    apply_act(y, act);
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const int u = (wm * WM + i * 32 + 16 * p + 8 * h) >> 3;
                        u32x4* unit = reinterpret_cast<u32x4*>(smem + t * (BM * 2) + ((u ^ ((2 * t) & (UPR - 1))) << 4));
                        if (R) {                         // the exchange below, backwards: the pairs that this lane's quads are added to
                            const u32x4 r = *unit;
                            const auto rlo = __builtin_amdgcn_permlane32_swap(r.x, r.z, false, false);
                            const auto rhi = __builtin_amdgcn_permlane32_swap(r.y, r.w, false, false);
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                y[8 * p + 4 * e + 0] += __builtin_bit_cast(float, static_cast<uint32_t>(rlo[e]) << 16);
                                y[8 * p + 4 * e + 1] += __builtin_bit_cast(float, static_cast<uint32_t>(rlo[e]) & 0xFFFF0000u);
                                y[8 * p + 4 * e + 2] += __builtin_bit_cast(float, static_cast<uint32_t>(rhi[e]) << 16);
                                y[8 * p + 4 * e + 3] += __builtin_bit_cast(float, static_cast<uint32_t>(rhi[e]) & 0xFFFF0000u);
                            }
                        }
                        const auto slo = __builtin_amdgcn_permlane32_swap(pack_bf16(y[8 * p + 0], y[8 * p + 1]), pack_bf16(y[8 * p + 4], y[8 * p + 5]), false, false);
                        const auto shi = __builtin_amdgcn_permlane32_swap(pack_bf16(y[8 * p + 2], y[8 * p + 3]), pack_bf16(y[8 * p + 6], y[8 * p + 7]), false, false);
                        *unit = (u32x4){slo[0], shi[0], slo[1], shi[1]};
                    }
                }
        __syncthreads();
        for (int q = tid; q < BN * UPR; q += NT) {
            const int t = q / UPR, u = q % UPR;
            const u32x4 v = *reinterpret_cast<const u32x4*>(smem + t * (BM * 2) + ((u ^ ((2 * t) & (UPR - 1))) << 4));
            const int64_t a = a0 + 8 * u;
            if (t0 + t < T && a < Adim) {
                uint16_t* dst = C + (t0 + t) * ldc + a;
                if (vecC && a + 8 <= Adim) {
                    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(dst));
                } else {
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        if (a + 2 * d < Adim) reinterpret_cast<uint32_t*>(dst)[d] = v[d];
                }
            }
        }
    }
};

struct LinearOutF32 {
    const float* bias;
    const float* R;
    int64_t ldr;
    uint8_t* codes;
    uint8_t* scales;
    int act;
    static constexpr bool kFused = true;

    // One sum per lane, feature a of token t; the 32 lanes of a half wavefront hold a block of the checkpoint and are active together.
    __device__ __forceinline__ void finish(float s, int64_t a, int64_t t, int64_t Adim, int64_t T, float* C, int64_t ldc) const {
        const bool in = a < Adim && t < T;
        float z[1] = {in && bias ? s + bias[a] : s};
        if (codes) {
            const float v = a < Adim ? z[0] : 0.f;
            uint32_t most = __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) {
                const uint32_t o = __shfl_xor(most, x);
                most = o > most ? o : most;
            }
            const int byte = ckpt_scale_byte(most);
            const bool bad = byte == kCkptNaN;
            const float v4[4] = {v, 0.f, 0.f, 0.f};
            const uint32_t code = ckpt_codes(v4, ckpt_inverse(bad ? 127 : byte), bad);
            const int64_t pitch = ckpt_pitch(Adim);
            if (t < T && a < pitch) {
                codes[t * pitch + a] = static_cast<uint8_t>(code);
                if ((a & 31) == 0) scales[t * (pitch / 32) + a / 32] = static_cast<uint8_t>(byte);
            }
        }
        if (in) {
            apply_act(z, act);
            C[t * ldc + a] = R ? z[0] + R[t * ldr + a] : z[0];
        }
    }
};

}  // namespace bimask
