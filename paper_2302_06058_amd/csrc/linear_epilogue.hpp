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

    // Sums of a workgroup's tile, BM weight rows x BN tokens.  Wavefront (wm, wn) holds TM x TN accumulators of 32 rows x 32 tokens from
    // row WM wm, token WN wn on (lane (l32, h): token l32, rows 8 q + 4 h + 0..3 in quad q); with KG > 1 group kg holds a share of every
    // sum.  They go to LDS as fp32 (smem: 4 KG BN BM / PASSES bytes, BM / PASSES rows at a time; 16-byte chunks XOR-swizzled by the token), and
    // every thread then takes 8 consecutive features of a token at a time: residual and output move as whole row segments, a block of
    // the checkpoint is four neighbouring lanes, the groups' shares are added in group order.
    // Adim is a multiple of 4, so a piece's halves are inside or outside; sums beyond it may be NaN and count as 0 in the checkpoint.
    // TIGHT: the state of a persistent loop leaves few registers: nothing is requested ahead, addresses are made when needed.
    template <int BM, int BN, int WM, int WN, int TM, int TN, int NT, int KG, int PASSES, bool TIGHT, class ACC>
    __device__ __forceinline__ void finish(ACC (&acc)[TM][TN], uint8_t* smem, int kg, int wm, int wn, int lane, int64_t a0, int64_t t0,
                                           int64_t Adim, int64_t T, uint16_t* C, int64_t ldc, bool vecC) const {
        typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        constexpr int ROWS = BM / PASSES, UPR = ROWS / 8, STEP = NT / UPR;        // pieces of 8 features; tokens from one piece of a thread to its next
        static_assert(ROWS % WM == 0 && NT % UPR == 0, "a pass takes whole wavefronts, a thread keeps its features");
        int tid = threadIdx.x;
        asm volatile("" : "+v"(lane), "+v"(tid));        // (what depends on them is not kept across the caller's loop)
        f32x4* sums = reinterpret_cast<f32x4*>(smem);
        auto chunk = [](int g, int t, int c) { return (g * BN + t) * (ROWS / 4) + (c ^ (t & (ROWS < 64 ? 7 : 15))); };
        const int64_t pitch = ckpt_pitch(Adim);
        const int n_tok = static_cast<int>(T - t0 < BN ? T - t0 : BN), u = tid % UPR;
#pragma unroll 1
        for (int pass = 0; pass < PASSES; ++pass) {
            const int64_t a = a0 + pass * ROWS + 8 * u;
            const bool in0 = a < Adim, in1 = a + 4 < Adim;
            int t = tid / UPR;
            const uint16_t* src = R + (t0 + t) * ldr + a;
            auto fetch = [&](u32x4& r, const uint16_t* src) {      // the residual of a piece
                if (vecR && in1) {
                    r = *reinterpret_cast<const u32x4*>(src);
                } else if (in0) {                        // 4-byte pieces (pointer and pitch are 4-byte aligned, Adim even)
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        if (d < 2 || in1) r[d] = *reinterpret_cast<const uint32_t*>(src + 2 * d);
                }
            };
            u32x4 ahead = {0u, 0u, 0u, 0u};              // requested before the sums are exchanged, and one piece ahead from then on
            if (!TIGHT && R && t < n_tok) fetch(ahead, src);
            auto fetch_bias = [&]() {
                u32x4 b = {0u, 0u, 0u, 0u};
                if (bias && in0) {
                    const u32x2 x = *reinterpret_cast<const u32x2*>(bias + a);
                    b.x = x.x; b.y = x.y;
                    if (in1) {
                        const u32x2 w = *reinterpret_cast<const u32x2*>(bias + a + 4);
                        b.z = w.x; b.w = w.y;
                    }
                }
                return b;
            };
            const u32x4 b_kept = TIGHT ? (u32x4){0u, 0u, 0u, 0u} : fetch_bias();
            if (pass > 0) __syncthreads();               // the previous pass has been read
            if (PASSES == 1 || wm * WM / ROWS == pass)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            sums[chunk(kg, wn * WN + 32 * j + (lane & 31), (wm * WM % ROWS + 32 * i) / 4 + 2 * q + (lane >> 5))] =
                                (f32x4){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            __syncthreads();
            uint16_t* dst = C + (t0 + t) * ldc + a;
            uint8_t* dst_code = codes + (t0 + t) * pitch + a;
            uint8_t* dst_scale = scales + (t0 + t) * (pitch / 32) + a / 32;
#pragma unroll 1
            for (; t < n_tok; t += STEP) {
                u32x4 r = ahead, b = b_kept;
                if constexpr (TIGHT) {
                    int tt = t;
                    asm volatile("" : "+v"(tt));         // (or the addresses would be kept and stepped)
                    if (R) fetch(r, R + (t0 + tt) * ldr + a);
                    b = fetch_bias();
                    dst = C + (t0 + tt) * ldc + a;
                    dst_code = codes + (t0 + tt) * pitch + a;
                    dst_scale = scales + (t0 + tt) * (pitch / 32) + a / 32;
                } else if (R && t + STEP < n_tok) {
                    src += STEP * ldr;
                    fetch(ahead, src);
                }
                float z[8];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    f32x4 x = sums[chunk(0, t, 2 * u + c)];
#pragma unroll
                    for (int g = 1; g < KG; ++g) x += sums[chunk(g, t, 2 * u + c)];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        z[4 * c + e] = x[e] + __builtin_bit_cast(float, e & 1 ? b[2 * c + (e >> 1)] & 0xFFFF0000u : b[2 * c + (e >> 1)] << 16);
                }
                if (codes) {
                    uint32_t d[2];
                    if (!in1)                            // (nothing of theirs is stored)
#pragma unroll
                        for (int e = 0; e < 8; ++e) z[e] = in0 && e < 4 ? z[e] : 0.f;
                    float most = ckpt_most(z);           // with the other lane of a pair, then the other pair of four
                    most = __builtin_elementwise_maximum(most, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, most), 0xB1, 0xF, 0xF, true)));
                    most = __builtin_elementwise_maximum(most, __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, most), 0x4E, 0xF, 0xF, true)));
                    const int byte = ckpt_scale_byte(most);
                    ckpt_encode(z, byte, d);
                    if (a < pitch) {
                        *reinterpret_cast<u32x2*>(dst_code) = (u32x2){d[0], d[1]};
                        if ((u & 3) == 0) *dst_scale = static_cast<uint8_t>(byte);
                    }
                    dst_code += STEP * pitch;
                    dst_scale += STEP * (pitch / 32);
                }
                apply_act(z, act);
                u32x4 y;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const float lo = __builtin_bit_cast(float, r[d] << 16), hi = __builtin_bit_cast(float, r[d] & 0xFFFF0000u);
                    y[d] = R ? pack_bf16(z[2 * d] + lo, z[2 * d + 1] + hi) : pack_bf16(z[2 * d], z[2 * d + 1]);
                }
                if (vecC && in1) {
                    __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(dst));
                } else if (in0) {
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        if (d < 2 || in1) reinterpret_cast<uint32_t*>(dst)[d] = y[d];
                }
                dst += STEP * ldc;
            }
        }
    }

    // The same within one wavefront, on two accumulators (64 weight rows from a0 x 32 tokens from t0, `rows` of which exist) that began
    // with the bias (start), before they are rounded: checkpoint, activation and residual.  strip: 32 rows of 136 bytes of the wavefront's own.
    // `ahead`: with AHEAD this residual piece, requested before (fetch_residual), replaced by the next one's if there is one.
    typedef unsigned int Piece __attribute__((ext_vector_type(4)));
    __device__ __forceinline__ void fetch_residual(Piece (&ahead)[4], int lane, int a0, int64_t t0, int rows, int Adim) const {
        if (!R) return;
#pragma unroll
        for (int it = 0; it < 4; ++it) {                 // beyond the tile: loaded from its first piece, not used
            const int r = (lane >> 3) + 8 * it, c = 8 * (lane & 7);
            ahead[it] = *reinterpret_cast<const Piece*>(R + (t0 + (r < rows ? r : 0)) * ldr + a0 + (c < Adim - a0 ? c : 0));      // Adim is a multiple of 8
        }
    }
    template <class ACC>
    __device__ __forceinline__ void start(ACC& z, int lane, int a, int Adim) const {
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        const int h = lane >> 5;
        ACC v;                                           // (a new value: elements put into the old one would keep it alive until here)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            u32x2 b = {0u, 0u};
            if (bias && a + 8 * q + 4 * h < Adim) b = *reinterpret_cast<const u32x2*>(bias + a + 8 * q + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = __builtin_bit_cast(float, e & 1 ? b[e >> 1] & 0xFFFF0000u : b[e >> 1] << 16);
        }
        z = v;
    }
    template <bool AHEAD, class ACC>
    __device__ __forceinline__ void before_rounding(ACC& z0, ACC& z1, Piece (&ahead)[4], bool more, uint8_t* strip, int lane, int a0, int64_t t0, int rows,
                                                    int Adim) const {
        typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        asm volatile("" : "+v"(lane));                   // (what depends on it is not kept across the caller's loop)
        const int l32 = lane & 31, h = lane >> 5;
        const int64_t t = t0 + l32;
        if constexpr (!AHEAD) fetch_residual(ahead, lane, a0, t0, rows, Adim);
        if (R) {                                         // as whole row segments into the strip
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                u32x2* d = reinterpret_cast<u32x2*>(strip + ((lane >> 3) + 8 * it) * 136 + 16 * (lane & 7));
                d[0] = (u32x2){ahead[it].x, ahead[it].y};
                d[1] = (u32x2){ahead[it].z, ahead[it].w};
            }
            if (AHEAD && more) fetch_residual(ahead, lane, a0, t0 + 32, rows - 32, Adim);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        int byte[2] = {0, 0};
        auto half = [&](ACC& z, int i) {
            float y[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) y[q] = z[q];
            if (codes && a0 + 32 * i < Adim) {
                uint32_t d[4];
                if (a0 + 32 * i + 32 > Adim)             // uniform, the last tile: features that do not exist count as 0
#pragma unroll
                    for (int q = 0; q < 16; ++q) y[q] = a0 + 32 * i + 8 * (q >> 2) + 4 * h < Adim ? y[q] : 0.f;
                const uint32_t most = __builtin_bit_cast(uint32_t, ckpt_most(y));
                const auto both = __builtin_amdgcn_permlane32_swap(most, most, false, false);
                byte[i] = ckpt_scale_byte(__builtin_elementwise_maximum(__builtin_bit_cast(float, static_cast<uint32_t>(both[0])), __builtin_bit_cast(float, static_cast<uint32_t>(both[1]))));
                ckpt_encode(y, byte[i], d);
                const auto lo = __builtin_amdgcn_permlane32_swap(d[0], d[2], false, false);
                const auto hi = __builtin_amdgcn_permlane32_swap(d[1], d[3], false, false);
                if (l32 < rows)
                    *reinterpret_cast<u32x4*>(codes + t * ckpt_pitch(Adim) + a0 + 32 * i + 16 * h) = (u32x4){lo[0], lo[1], hi[0], hi[1]};
            }
            apply_act(y, act);
            if (R) {
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const u32x2* d = reinterpret_cast<const u32x2*>(strip + l32 * 136 + 2 * (32 * i + 16 * p + 8 * h));
                    const u32x2 r0 = d[0], r1 = d[1];
                    const auto rlo = __builtin_amdgcn_permlane32_swap(r0.x, r1.x, false, false);
                    const auto rhi = __builtin_amdgcn_permlane32_swap(r0.y, r1.y, false, false);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        y[8 * p + 4 * e + 0] += __builtin_bit_cast(float, static_cast<uint32_t>(rlo[e]) << 16);
                        y[8 * p + 4 * e + 1] += __builtin_bit_cast(float, static_cast<uint32_t>(rlo[e]) & 0xFFFF0000u);
                        y[8 * p + 4 * e + 2] += __builtin_bit_cast(float, static_cast<uint32_t>(rhi[e]) << 16);
                        y[8 * p + 4 * e + 3] += __builtin_bit_cast(float, static_cast<uint32_t>(rhi[e]) & 0xFFFF0000u);
                    }
                }
            }
            ACC v;
#pragma unroll
            for (int q = 0; q < 16; ++q) v[q] = y[q];
            z = v;
            __builtin_amdgcn_sched_barrier(0);
        };
        half(z0, 0);
        half(z1, 1);
        if (codes && h == 0 && l32 < rows) {             // both blocks' scale bytes at once
            typedef uint16_t u16_any __attribute__((aligned(1)));
            uint8_t* p = scales + t * ckpt_blocks(Adim) + a0 / 32;
            if (a0 + 32 < Adim) *reinterpret_cast<u16_any*>(p) = static_cast<uint16_t>(byte[0] | byte[1] << 8);
            else *p = static_cast<uint8_t>(byte[0]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
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
            float most = __builtin_fabsf(v);
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) most = __builtin_elementwise_maximum(most, __shfl_xor(most, x));
            const int byte = ckpt_scale_byte(most);
            float v4[4] = {v, 0.f, 0.f, 0.f};
            uint32_t code[1];
            ckpt_encode(v4, byte, code);
            const int64_t pitch = ckpt_pitch(Adim);
            if (t < T && a < pitch) {
                codes[t * pitch + a] = static_cast<uint8_t>(code[0]);
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
