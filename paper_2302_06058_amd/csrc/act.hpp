// Activations, their slopes and the 8-bit checkpoint's block rule (see include/bimask.h), for kernels that apply them to
// fp32 values in registers.
#pragma once
#include "common.hpp"

namespace bimask {

// ---- activations ------------------------------------------------------------------------------------------------
// silu and gelu_tanh are z * sigma(u), u = z and u = z (c1 + c2 z^2), sigma(u) = 1 / (1 + exp(-u)): an exponential that overflows
// makes sigma 0, one that vanishes makes it 1.  Slopes as sigma + z sigma (1 - sigma) u', the product sigma (1 - sigma) first: it is
// exactly 0 at both ends, where the other factors are finite.  gelu is z * Phi(z) with Phi's tail 0.5 erfc(|z| / sqrt 2) =
// exp(-z^2 / 2) R(|z|); R (the Mills ratio over sqrt(2 pi)) as t * polynomial(t), t = 1 / (1 + 0.3 |z|): least squares on the
// relative error, re-weighted to equal peaks, 1.5e-7 over 0 <= |z| <= 14.  The tail itself never comes from 1 - Phi.
// Cost of a value in issue slots (2^x and 1/x take four each): silu 11, gelu_tanh 13, gelu 24; slopes 12, 17, 25.
constexpr float kLog2e = 1.44269504f, kTanhC1 = 1.5957691216f, kTanhC2 = 0.0713548163f;       // 2 sqrt(2/pi), times 0.044715

__device__ __forceinline__ float sigma_of(float minus_u_log2e) {
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(minus_u_log2e));
}

__device__ __forceinline__ float gauss(float z) { return __builtin_amdgcn_exp2f(-0.721347520f * z * z); }       // exp(-z^2 / 2)
__device__ __forceinline__ float phi_cdf(float z, float g) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3f * __builtin_fabsf(z));
    float p = 0.03567478f;
    p = __builtin_fmaf(p, t, -0.1572031f);
    p = __builtin_fmaf(p, t, 0.20635354f);
    p = __builtin_fmaf(p, t, -0.05368367f);
    p = __builtin_fmaf(p, t, 0.12856164f);
    p = __builtin_fmaf(p, t, 0.09991349f);
    p = __builtin_fmaf(p, t, 0.12075396f);
    p = __builtin_fmaf(p, t, 0.1196293f);
    const float tail = g * (t * p);
    return z >= 0.f ? 1.f - tail : tail;
}

// z -> act(z), for n values; act is uniform
template <int n>
__device__ __forceinline__ void apply_act(float (&z)[n], int act) {
    if (act == BIMASK_ACT_NONE) return;
    if (act == BIMASK_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = z[i] <= 0.f ? 0.f : z[i];         // (NaN stays)
    } else if (act == BIMASK_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] *= phi_cdf(z[i], gauss(z[i]));
    } else if (act == BIMASK_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] *= sigma_of(-kLog2e * z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] *= sigma_of(z[i] * __builtin_fmaf(-kLog2e * kTanhC2, z[i] * z[i], -kLog2e * kTanhC1));
    }
}

// z -> act'(z); z is finite or NaN (a checkpoint's values are).  relu: 0 at 0.
template <int n>
__device__ __forceinline__ void apply_slope(float (&z)[n], int act) {
    if (act == BIMASK_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = 1.f;
    } else if (act == BIMASK_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) z[i] = z[i] <= 0.f ? 0.f : z[i] > 0.f ? 1.f : z[i];
    } else if (act == BIMASK_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float g = gauss(z[i]);
            z[i] = __builtin_fmaf(z[i], 0.398942280f * g, phi_cdf(z[i], g));
        }
    } else if (act == BIMASK_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float s = sigma_of(-kLog2e * z[i]);
            z[i] = __builtin_fmaf(z[i], __builtin_fmaf(-s, s, s), s);
        }
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float zz = __builtin_fminf(z[i] * z[i], 1e4f);         // (sigma is 0 or 1 long before; z^2 and u' stay finite)
            const float s = sigma_of(z[i] * __builtin_fmaf(-kLog2e * kTanhC2, zz, -kLog2e * kTanhC1));
            z[i] = __builtin_fmaf(z[i] * __builtin_fmaf(-s, s, s), __builtin_fmaf(3.f * kTanhC2, zz, kTanhC1), s);
        }
    }
}

// ---- 8-bit checkpoints --------------------------------------------------------------------------------------------
// 32 consecutive features of a token share a power of two 2^e, the smallest with rint(max / 2^e) <= 127; every product with
// 2^e or 2^-e is exact, so codes depend on the inputs alone and the values they stand for are exact in bf16 and fp32.
constexpr int kCkptBlock = 32;
__host__ __device__ inline int64_t ckpt_pitch(int64_t cols) { return round_up(cols, kCkptBlock); }      // bytes of codes per token
__host__ __device__ inline int64_t ckpt_blocks(int64_t cols) { return ceil_div(cols, kCkptBlock); }     // scale bytes per token

constexpr int64_t kMaxTokens = int64_t(1) << 38;         // rows of the matrices around the product: sizes in bytes stay in 64 bits
constexpr int kCkptNaN = 255;
// The largest magnitude of n values; a NaN stays one (an instruction takes two values, their signs off on the way).
template <int n>
__device__ __forceinline__ float ckpt_most(const float (&v)[n]) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < n; ++i) most = __builtin_elementwise_maximum(most, __builtin_fabsf(v[i]));
    return most;
}
// The scale byte e + 127 of a block with this largest magnitude.  127.5 is 1.9921875 * 2^6, mantissa bits 0x7F0000: from there on the
// next power.  -126 <= e <= 121 keeps 2^e, 2^-e and 127 * 2^e normal.
__device__ __forceinline__ int ckpt_scale_byte(float largest) {
    const uint32_t most = __builtin_bit_cast(uint32_t, largest) & 0x7FFFFFFFu;
    const int x = static_cast<int>(most >> 23);
    if (x == 255) return kCkptNaN;
    const int b = x - 6 + ((most & 0x7FFFFFu) >= 0x7F0000u ? 1 : 0);
    return b < 1 ? 1 : b > 248 ? 248 : b;
}
__device__ __forceinline__ float ckpt_inverse(int byte) { return __builtin_bit_cast(float, static_cast<uint32_t>(254 - byte) << 23); }
__device__ __forceinline__ float ckpt_scale(int byte) {
    return __builtin_bit_cast(float, byte == kCkptNaN ? 0x7FC00000u : static_cast<uint32_t>(byte) << 23);
}
// n values of a block -> their codes, four a word, first in the low byte.  v * 2^-e is exact, so adding 1.5 * 2^23 rounds it to an
// integer (halves to even) whose two's complement stands in the low byte of the sum.
template <int n>
__device__ __forceinline__ void ckpt_encode(const float (&v)[n], int byte, uint32_t (&out)[n / 4]) {
    const bool bad = byte == kCkptNaN;
    const float inv = ckpt_inverse(bad ? 127 : byte);
    uint32_t q[n];
#pragma unroll
    for (int i = 0; i < n; ++i) q[i] = __builtin_bit_cast(uint32_t, __builtin_fmaf(v[i], inv, 12582912.f));
    if (byte == 248)                                     // e is kept to 121: up to 128 steps
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int k = static_cast<int>(q[i] - 0x4B400000u);
            q[i] = k > 127 ? 127u : k < -127 ? static_cast<uint32_t>(-127) : q[i];
        }
#pragma unroll
    for (int w = 0; w < n / 4; ++w) {
        const uint32_t lo = __builtin_amdgcn_perm(q[4 * w + 1], q[4 * w], 0x0C0C0400u), hi = __builtin_amdgcn_perm(q[4 * w + 3], q[4 * w + 2], 0x0C0C0400u);
        out[w] = bad ? 0u : lo | hi << 16;
    }
}
__device__ __forceinline__ float ckpt_value(uint32_t four, int i, float scale) {      // code i of 4
    return static_cast<float>(static_cast<int8_t>(four >> (8 * i))) * scale;
}

}  // namespace bimask
