// 8-bit activation checkpoints and the gradient through an activation (format and rule: include/bimask.h, act.hpp).
//
//   store     X -> codes + scale bytes        reads esz, writes 33/32 bytes per feature
//   load      codes + scale bytes -> X        the reverse
//   act_bwd   dZ = dY * act'(Z~),  dbias = sum over the tokens of dZ (fp32)
//
// All three are bound by memory: one pass, 16 features (half a block) per thread and step, 16-byte accesses.  8192 x 11008 bf16: store 51 us
// and load 42 (273 MB each: 5.4 and 6.4 TB/s; the codes just written are partly still in the last-level cache), act_bwd with silu 88
// (454 MB, 5.1 TB/s; a plain copy reaches 5.15) and 4 for the strips' sums.  With few rows latency and the activation's slope count: 6347 x 1000
// (32 MB, 6.2 us at the copy's rate) 8.2 with relu and no bias gradient, 11.6 with gelu, 15.4 with both.
#include "act.hpp"

namespace bimask {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));

constexpr int kPiece = 16;                               // features of a thread: half a block of the checkpoint
constexpr int64_t kMaxGroups = 1 << 20;                  // workgroups of a launch; more work runs in a loop (a launch counts its work-items in 32 bits)

template <typename raw>
struct Row16 {                                           // 16 features of a row in registers, as stored
    static constexpr int V = sizeof(raw);                // 16-byte pieces: 2 of bf16, 4 of fp32
    u32x4 v[V];
    __device__ __forceinline__ float get(int i) const {
        if constexpr (sizeof(raw) == 2) {
            const uint32_t w = v[i >> 3][(i >> 1) & 3];
            return __builtin_bit_cast(float, i & 1 ? w & 0xFFFF0000u : w << 16);
        } else {
            return __builtin_bit_cast(float, static_cast<uint32_t>(v[i >> 2][i & 3]));
        }
    }
    __device__ __forceinline__ void put(const float (&f)[kPiece]) {
#pragma unroll
        for (int p = 0; p < V; ++p)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                if constexpr (sizeof(raw) == 2) v[p][d] = pack_bf16(f[8 * p + 2 * d], f[8 * p + 2 * d + 1]);
                else v[p][d] = __builtin_bit_cast(uint32_t, f[4 * p + d]);
            }
    }
    // features c .. c + 15 of a row of `cols`, rows at any element's alignment (the 16-byte accesses need no more); the end of a
    // row in smaller pieces
    __device__ __forceinline__ void load(const raw* row, int64_t c, int64_t cols) {
        constexpr int E = 16 / sizeof(raw);
        row += c;
        const int64_t n = cols - c;
        if (n >= kPiece) {
#pragma unroll
            for (int p = 0; p < V; ++p) v[p] = reinterpret_cast<const u32x4_any*>(row)[p];
            return;
        }
#pragma unroll
        for (int p = 0; p < V; ++p) {
            v[p] = (u32x4){0u, 0u, 0u, 0u};
            if (n >= E * (p + 1)) {
                v[p] = reinterpret_cast<const u32x4_any*>(row)[p];
            } else {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    if constexpr (sizeof(raw) == 4) {
                        if (E * p + d < n) v[p][d] = row[E * p + d];
                    } else {
                        if (E * p + 2 * d + 1 < n) v[p][d] = *reinterpret_cast<const u32_any*>(row + E * p + 2 * d);
                        else if (E * p + 2 * d < n) v[p][d] = row[E * p + 2 * d];
                    }
                }
            }
        }
    }
    __device__ __forceinline__ void store(raw* row, int64_t c, int64_t cols) const {
        constexpr int E = 16 / sizeof(raw);
        row += c;
        const int64_t n = cols - c;
        if (n >= kPiece) {
#pragma unroll
            for (int p = 0; p < V; ++p) reinterpret_cast<u32x4_any*>(row)[p] = v[p];
            return;
        }
#pragma unroll
        for (int p = 0; p < V; ++p) {
            if (n >= E * (p + 1)) {
                reinterpret_cast<u32x4_any*>(row)[p] = v[p];
            } else {
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    if constexpr (sizeof(raw) == 4) {
                        if (E * p + d < n) row[E * p + d] = v[p][d];
                    } else {
                        if (E * p + 2 * d + 1 < n) *reinterpret_cast<u32_any*>(row + E * p + 2 * d) = v[p][d];
                        else if (E * p + 2 * d < n) row[E * p + 2 * d] = static_cast<raw>(v[p][d]);
                    }
                }
            }
        }
    }
};

// The pieces of a matrix in row order, 256 per workgroup and step: token and first feature of this thread's piece.
struct Piece { int64_t t; uint32_t half; };
__device__ __forceinline__ Piece piece_at(int64_t first, uint32_t per_row) {
    const int64_t t0 = first / per_row;                  // uniform
    const uint32_t off = static_cast<uint32_t>(first - t0 * per_row) + threadIdx.x, dt = off / per_row;
    return {t0 + dt, off - dt * per_row};
}

template <typename raw>
__global__ void __launch_bounds__(kThreads)
k_checkpoint_store(const raw* __restrict__ X, int64_t T, int64_t J, int64_t ldx, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                   uint32_t per_row) {
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kThreads; first < T * per_row; first += static_cast<int64_t>(gridDim.x) * kThreads) {
        const Piece p = piece_at(first, per_row);
        if (p.t >= T) return;                            // pieces come in pairs of lanes: a block is never cut
        const int64_t c = static_cast<int64_t>(p.half) * kPiece;
        Row16<raw> x;
        x.load(X + p.t * ldx, c, J);
        float f[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; ++i) f[i] = x.get(i);
        const float most = ckpt_most(f);
        const int byte = ckpt_scale_byte(__builtin_elementwise_maximum(most, __shfl_xor(most, 1)));
        uint32_t four[4];
        ckpt_encode(f, byte, four);
        const u32x4 out = {four[0], four[1], four[2], four[3]};
        *reinterpret_cast<u32x4*>(codes + (p.t * per_row + p.half) * kPiece) = out;
        if (!(p.half & 1)) scales[p.t * (per_row / 2) + p.half / 2] = static_cast<uint8_t>(byte);
    }
}

template <typename raw>
__global__ void __launch_bounds__(kThreads)
k_checkpoint_load(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t T, int64_t J, raw* __restrict__ X,
                  int64_t ldx, uint32_t per_row) {
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * kThreads; first < T * per_row; first += static_cast<int64_t>(gridDim.x) * kThreads) {
        const Piece p = piece_at(first, per_row);
        if (p.t >= T) return;
        const u32x4 q = *reinterpret_cast<const u32x4*>(codes + (p.t * per_row + p.half) * kPiece);
        const float scale = ckpt_scale(scales[p.t * (per_row / 2) + p.half / 2]);
        float f[kPiece];
#pragma unroll
        for (int i = 0; i < kPiece; ++i) f[i] = ckpt_value(q[i >> 2], i & 3, scale);
        Row16<raw> x;
        x.put(f);
        x.store(X + p.t * ldx, static_cast<int64_t>(p.half) * kPiece, J);
    }
}

// A workgroup takes `rows` consecutive tokens of 16 << log2c features: its threads stand 1 << log2c side by side, the others
// below each other, every thread walks down its features with the sums in registers, and the sums meet in LDS in thread order.
// The strips' sums go to the workspace and are added by k_sum_strips in strip order: nothing depends on timing.
template <typename raw>
__global__ void __launch_bounds__(kThreads)
k_act_bwd(const raw* dY, int64_t T, int64_t lddy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, int64_t I, int act,
          raw* dZ, int64_t lddz, float* __restrict__ sums, int64_t ld_sums, int64_t rows, uint32_t per_row, int log2c) {
    __shared__ float part[kThreads][kPiece + 1];
    const uint32_t half = (blockIdx.x << log2c) + (threadIdx.x & ((1u << log2c) - 1));
    const int64_t c = static_cast<int64_t>(half) * kPiece, t0 = static_cast<int64_t>(blockIdx.y) * rows;
    const int64_t t_end = t0 + rows < T ? t0 + rows : T;
    float acc[kPiece];
#pragma unroll
    for (int i = 0; i < kPiece; ++i) acc[i] = 0.f;
    const int64_t step = kThreads >> log2c;
    // U rows are requested before the first is used
    constexpr int U = 2;
    if (c < I)
        for (int64_t tb = t0 + (threadIdx.x >> log2c); tb < t_end; tb += U * step) {
            Row16<raw> x[U];
            u32x4 q[U];
            int byte[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t t = tb + u * step < t_end ? tb + u * step : tb;      // beyond the strip: loaded, not used
                x[u].load(dY + t * lddy, c, I);
                if (codes) {                             // none with act none: the bias gradient alone
                    q[u] = *reinterpret_cast<const u32x4*>(codes + (t * per_row + half) * kPiece);
                    byte[u] = scales[t * (per_row / 2) + half / 2];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t t = tb + u * step;
                if (t >= t_end) break;
                float f[kPiece];
                if (codes) {
                    const float scale = ckpt_scale(byte[u]);
#pragma unroll
                    for (int i = 0; i < kPiece; ++i) f[i] = ckpt_value(q[u][i >> 2], i & 3, scale);
                    apply_slope(f, act);
#pragma unroll
                    for (int i = 0; i < kPiece; ++i) f[i] *= x[u].get(i);
                } else {
#pragma unroll
                    for (int i = 0; i < kPiece; ++i) f[i] = x[u].get(i);
                }
                if (dZ) {
                    x[u].put(f);
                    x[u].store(dZ + t * lddz, c, I);
                }
#pragma unroll
                for (int i = 0; i < kPiece; ++i) acc[i] += f[i];
            }
        }
    if (!sums) return;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) part[threadIdx.x][i] = acc[i];
    __syncthreads();
    const int64_t c0 = (static_cast<int64_t>(blockIdx.x) << log2c) * kPiece;
    for (int k = threadIdx.x; k < kPiece << log2c; k += kThreads) {
        if (c0 + k >= I) break;
        float s = 0.f;
        for (int r = 0; r < kThreads >> log2c; ++r) s += part[(r << log2c) + k / kPiece][k % kPiece];
        sums[static_cast<int64_t>(blockIdx.y) * ld_sums + c0 + k] = s;
    }
}

// 16 features x 16 ranges of strips per workgroup: a chain of additions is strips / 16 long instead of strips (100 strips of 1000
// features 24 us with one thread per feature), and both levels add in a fixed order.
__global__ void __launch_bounds__(kThreads)
k_sum_strips(const float* __restrict__ part, int strips, int64_t ld, int64_t I, float* __restrict__ out) {
    __shared__ float sums[16][17];
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + x;         // (strips are as wide as whole blocks: in bounds)
    float s = 0.f;
    for (int k = y; k < strips; k += 16 * 8) {           // eight requests at once, those beyond the last strip of one that exists
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = part[(k + 16 * u < strips ? k + 16 * u : k) * ld + c];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += k + 16 * u < strips ? v[u] : 0.f;
    }
    sums[y][x] = s;
    __syncthreads();
    if (y == 0 && c < I) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += sums[k][x];
        out[c] = t;
    }
}

unsigned groups(int64_t pieces) {
    const int64_t n = ceil_div(pieces, kThreads);
    return static_cast<unsigned>(n < kMaxGroups ? n : kMaxGroups);
}

}  // namespace

int launch_checkpoint_store(const void* X, int64_t T, int64_t J, int64_t ldx, int dtype, uint8_t* ckpt, hipStream_t s) {
    const uint32_t per_row = static_cast<uint32_t>(ckpt_pitch(J) / kPiece);
    uint8_t* scales = ckpt + T * ckpt_pitch(J);
    const dim3 grid(groups(T * per_row));
    if (dtype == BIMASK_BF16)
        hipLaunchKernelGGL(k_checkpoint_store<uint16_t>, grid, dim3(kThreads), 0, s, static_cast<const uint16_t*>(X), T, J, ldx, ckpt, scales,
                           per_row);
    else
        hipLaunchKernelGGL(k_checkpoint_store<uint32_t>, grid, dim3(kThreads), 0, s, static_cast<const uint32_t*>(X), T, J, ldx, ckpt, scales,
                           per_row);
    return check_launch();
}

int launch_checkpoint_load(const uint8_t* ckpt, int64_t T, int64_t J, int dtype, void* X, int64_t ldx, hipStream_t s) {
    const uint32_t per_row = static_cast<uint32_t>(ckpt_pitch(J) / kPiece);
    const uint8_t* scales = ckpt + T * ckpt_pitch(J);
    const dim3 grid(groups(T * per_row));
    if (dtype == BIMASK_BF16)
        hipLaunchKernelGGL(k_checkpoint_load<uint16_t>, grid, dim3(kThreads), 0, s, ckpt, scales, T, J, static_cast<uint16_t*>(X), ldx, per_row);
    else
        hipLaunchKernelGGL(k_checkpoint_load<uint32_t>, grid, dim3(kThreads), 0, s, ckpt, scales, T, J, static_cast<uint32_t*>(X), ldx, per_row);
    return check_launch();
}

// Feature tiles of up to 256 (16 threads side by side, a row segment of 512 bytes of bf16), and strips of tokens so that about
// 4096 workgroups exist (8192 x 11008 with silu 91.7 us, with 2048 96.8), none with fewer than 4 steps of rows (two requests) where that
// leaves 1024 workgroups (50000 x 400 34.7, with 2 steps 37.4), 2 where it leaves 512 (6347 x 1000 15.4, with 4 15.8), else 1 (512 x 1000
// 6.5, with 2 7.5).
ActBwdPlan plan_act_bwd(int64_t T, int64_t I) {
    ActBwdPlan p;
    const int64_t per_row = ckpt_pitch(I) / kPiece;
    p.log2c = per_row >= 16 ? 4 : ilog2(static_cast<int>(per_row));
    p.tiles = ceil_div(per_row, int64_t(1) << p.log2c);
    const int64_t step = kThreads >> p.log2c;
    const int64_t least = ceil_div(T, 4 * step) * p.tiles >= 1024 ? 4 : ceil_div(T, 2 * step) * p.tiles >= 512 ? 2 : 1, most = ceil_div(T, least * step);
    int64_t strips = ceil_div(4096, p.tiles);
    strips = strips < most ? strips : most;
    p.rows = round_up(ceil_div(T, strips), step);
    p.strips = ceil_div(T, p.rows);
    p.ws_bytes = p.strips > 1 ? static_cast<size_t>(p.strips * ckpt_pitch(I)) * 4 : 0;
    return p;
}

int launch_act_bwd(const void* dY, int64_t T, int64_t lddy, const uint8_t* ckpt, int64_t I, int dtype, int act, void* dZ, int64_t lddz,
                   float* dbias, float* ws, hipStream_t s) {
    const ActBwdPlan p = plan_act_bwd(T, I);
    const int64_t pitch = ckpt_pitch(I);
    const uint32_t per_row = static_cast<uint32_t>(pitch / kPiece);
    const uint8_t* scales = ckpt ? ckpt + T * pitch : nullptr;
    float* sums = !dbias ? nullptr : p.strips > 1 ? ws : dbias;
    if (p.tiles > 0xFFFFFF || p.strips > 0xFFFF) return BIMASK_ERR_SHAPE;
    const dim3 grid(static_cast<unsigned>(p.tiles), static_cast<unsigned>(p.strips));
    if (dtype == BIMASK_BF16)
        hipLaunchKernelGGL(k_act_bwd<uint16_t>, grid, dim3(kThreads), 0, s, static_cast<const uint16_t*>(dY), T, lddy, ckpt, scales, I, act,
                           static_cast<uint16_t*>(dZ), lddz, sums, pitch, p.rows, per_row, p.log2c);
    else
        hipLaunchKernelGGL(k_act_bwd<uint32_t>, grid, dim3(kThreads), 0, s, static_cast<const uint32_t*>(dY), T, lddy, ckpt, scales, I, act,
                           static_cast<uint32_t*>(dZ), lddz, sums, pitch, p.rows, per_row, p.log2c);
    if (int rc = check_launch()) return rc;
    if (dbias && p.strips > 1) {
        hipLaunchKernelGGL(k_sum_strips, dim3(static_cast<unsigned>(ceil_div(I, 16))), dim3(kThreads), 0, s, ws, static_cast<int>(p.strips),
                           pitch, I, dbias);
        return check_launch();
    }
    return BIMASK_OK;
}

}  // namespace bimask
