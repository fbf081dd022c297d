// Dense weight gradient of the straight-through estimator (arXiv 2302.06058, Sec. 3.1) from an 8-bit checkpoint of the layer's input:
//     dW[i][j] = sum_t dY[t][i] * X~[t][j]
//
// Both operands lie with the contraction index t as their slow dimension.  A stage of 64 tokens goes to LDS as it lies in memory
// (the codes put back to bf16 on the way: code * 2^e is exact in bf16), and the transposing LDS read hands every lane the
// consecutive tokens of its row that the matrix instruction wants.  16 lanes of such a read touch four token rows at 32 bytes
// each: the 64-byte chunks of a row are XOR-swizzled by the row so that they fall into different banks.
// Few output tiles and many tokens: workgroups split the tokens, their fp32 sums go to the workspace and are added in order.
#include "act.hpp"

namespace bimask {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kStageT = 64;                              // tokens per stage

union Frag { bf16x8 v; u32x2 d[2]; };

// 4 consecutive tokens of one row per lane, 16 lanes: 4 tokens x 16 rows
__device__ __forceinline__ u32x2 read_turned(const uint8_t* p) {
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
}

enum OutMode { kOutF32 = 0, kOutBF16 = 1, kAddF32 = 2, kAddBF16 = 3 };

__device__ __forceinline__ float bf16_value(uint16_t x) { return __builtin_bit_cast(float, static_cast<uint32_t>(x) << 16); }

template <int MODE>
__device__ __forceinline__ void put(void* out, int64_t at, float v) {
    if constexpr (MODE == kOutF32 || MODE == kAddF32) {
        float* p = static_cast<float*>(out) + at;
        *p = MODE == kAddF32 ? *p + v : v;
    } else {
        uint16_t* p = static_cast<uint16_t*>(out) + at;
        *p = static_cast<uint16_t>(pack_bf16(MODE == kAddBF16 ? bf16_value(*p) + v : v, 0.f));
    }
}
__device__ __forceinline__ void put(int mode, void* out, int64_t at, float v) {
    if (mode == kOutF32) put<kOutF32>(out, at, v);
    else if (mode == kOutBF16) put<kOutBF16>(out, at, v);
    else if (mode == kAddF32) put<kAddF32>(out, at, v);
    else put<kAddBF16>(out, at, v);
}

// BM x BN output tile on WM x WN wavefronts.  WHOLE: rows of dY start on 16 bytes and I is a multiple of 8.
// blockIdx.y: pieces of `rows` tokens; with more than one the sums go to part + blockIdx.y * I * J.
template <int BM, int BN, int WM, int WN, bool WHOLE>
__global__ void __launch_bounds__(64 * WM * WN)
k_weight_grad(const uint16_t* __restrict__ dY, int64_t T, int64_t lddy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
              int64_t I, int64_t J, void* out, int64_t ldo, int mode, float* part, int tiles_j, int tiles, int64_t rows) {
    constexpr int NT = 64 * WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int PA = kStageT * BM / 8 / NT, PB = kStageT * BN / 16 / NT;       // 16-byte pieces per thread and stage
    constexpr int SA = kStageT * BM * 2, SB = kStageT * BN * 2;                  // LDS bytes of a stage
    static_assert(PA >= 1 && PB >= 1, "a piece for every thread");
    extern __shared__ u32x4 smem_u4[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(smem_u4);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WM, wn = wave / WM, l32 = lane & 31, h = lane >> 5;
    // XCD x takes a contiguous run of tiles, so that its L2 serves the token rows of neighbours
    const int per_xcd = (tiles + 7) / 8, n = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((blockIdx.x >> 3) >= static_cast<unsigned>(per_xcd) || n >= tiles) return;
    const int64_t i0 = static_cast<int64_t>(n / tiles_j) * BM, j0 = static_cast<int64_t>(n % tiles_j) * BN;
    const int64_t t_begin = blockIdx.y * rows, t_end = t_begin + rows < T ? t_begin + rows : T;
    const int64_t pitch = ckpt_pitch(J), blocks = ckpt_blocks(J);

    auto swz_a = [](int row) { return BM >= 128 ? row & 3 : (row >> 1) & 1; };
    auto swz_b = [](int row) { return BN >= 128 ? row & 3 : (row >> 1) & 1; };

    u32x4 ra[PA], rb[PB];
    int rs[PB];
    auto load = [&](int64_t t0) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int q = tid + NT * p, row = q / (BM / 8), u = q % (BM / 8);
            const int64_t t = t0 + row, i = i0 + 8 * u;
            if constexpr (WHOLE) {
                const bool in = t < t_end && i < I;
                const u32x4 v = *reinterpret_cast<const u32x4*>(dY + (in ? t * lddy + i : 0));
                ra[p] = in ? v : (u32x4){0u, 0u, 0u, 0u};
            } else {
                ra[p] = (u32x4){0u, 0u, 0u, 0u};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (t < t_end && i + e < I) ra[p][e >> 1] |= static_cast<uint32_t>(dY[t * lddy + i + e]) << (16 * (e & 1));
            }
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int q = tid + NT * p, row = q / (BN / 16), u = q % (BN / 16);
            const int64_t t = t0 + row, j = j0 + 16 * u;
            const bool in = t < t_end && j < pitch;
            const u32x4 v = *reinterpret_cast<const u32x4*>(codes + (in ? t * pitch + j : 0));
            rb[p] = in ? v : (u32x4){0u, 0u, 0u, 0u};
            rs[p] = in ? scales[t * blocks + j / 32] : 0;
        }
    };
    auto stage = [&](uint8_t* s) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int q = tid + NT * p, row = q / (BM / 8), u = q % (BM / 8);
            *reinterpret_cast<u32x4*>(s + row * (BM * 2) + (((u >> 2) ^ swz_a(row)) << 6) + ((u & 3) << 4)) = ra[p];
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int q = tid + NT * p, row = q / (BN / 16), u = q % (BN / 16);
            const float scale = ckpt_scale(rs[p]);
            uint8_t* dst = s + SA + row * (BN * 2) + (((u >> 1) ^ swz_b(row)) << 6) + ((u & 1) << 5);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                u32x4 v;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const uint32_t four = rb[p][2 * x + (d >> 1)];
                    v[d] = pack_bf16(ckpt_value(four, 2 * (d & 1), scale), ckpt_value(four, 2 * (d & 1) + 1, scale));
                }
                *reinterpret_cast<u32x4*>(dst + 16 * x) = v;
            }
        }
    };

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;

    // lane k of a group of 16 reads token row k / 4 of four and 4 (k % 4) .. + 3 of sixteen output rows
    const int krow = 8 * h + ((lane & 15) >> 2), in_chunk = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    int fa[TM], fb[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[i] = krow * (BM * 2) + (((wm * TM + i) ^ swz_a(krow)) << 6) + in_chunk;
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[j] = SA + krow * (BN * 2) + (((wn * TN + j) ^ swz_b(krow)) << 6) + in_chunk;

    const int64_t stages = t_begin < t_end ? ceil_div(t_end - t_begin, kStageT) : 0;
    if (stages > 0) {
        load(t_begin);
        stage(smem);
    }
    __syncthreads();
    for (int64_t st = 0; st < stages; ++st) {
        uint8_t* cur = smem + (st & 1) * (SA + SB);
        const bool more = st + 1 < stages;
        if (more) load(t_begin + (st + 1) * kStageT);
#pragma unroll
        for (int ks = 0; ks < kStageT / 16; ++ks) {
            Frag a[TM], b[TN];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
#pragma unroll
                for (int i = 0; i < TM; ++i) a[i].d[x] = read_turned(cur + fa[i] + (16 * ks + 4 * x) * (BM * 2));
#pragma unroll
                for (int j = 0; j < TN; ++j) b[j].d[x] = read_turned(cur + fb[j] + (16 * ks + 4 * x) * (BN * 2));
            }
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i].v, b[j].v, acc[i][j], 0, 0, 0);
        }
        if (more) stage(smem + ((st + 1) & 1) * (SA + SB));
        __syncthreads();
    }

    const bool split = gridDim.y > 1;
    void* dst = split ? static_cast<void*>(part + static_cast<int64_t>(blockIdx.y) * I * J) : out;
    const int64_t ld = split ? J : ldo;
    const int m = split ? kOutF32 : mode;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t col = j0 + (wn * TN + j) * 32 + l32;
            if (col < J)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    const int64_t row = i0 + (wm * TM + i) * 32 + 8 * (q >> 2) + 4 * h + (q & 3);
                    if (row < I) put(m, dst, row * ld + col, acc[i][j][q]);
                }
        }
}

// fp32: 64 x 64 tiles on four wavefronts, fp32 matrix instructions, whose operands are one element per lane: LDS rows as they lie.
constexpr int kTileF32 = 64, kStageF32 = 32;
__global__ void __launch_bounds__(256)
k_weight_grad_f32(const float* __restrict__ dY, int64_t T, int64_t lddy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                  int64_t I, int64_t J, void* out, int64_t ldo, int mode, float* part, int tiles_j, int tiles, int64_t rows) {
    __shared__ float sA[2][kStageF32][kTileF32 + 1], sB[2][kStageF32][kTileF32 + 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave & 1, wn = wave >> 1, l32 = lane & 31, h = lane >> 5;
    const int n = blockIdx.x;
    if (n >= tiles) return;
    const int64_t i0 = static_cast<int64_t>(n / tiles_j) * kTileF32, j0 = static_cast<int64_t>(n % tiles_j) * kTileF32;
    const int64_t t_begin = blockIdx.y * rows, t_end = t_begin + rows < T ? t_begin + rows : T;
    const int64_t pitch = ckpt_pitch(J), blocks = ckpt_blocks(J);
    float ra[8];
    uint32_t rb[2];
    int rs[2];
    auto load = [&](int64_t t0) {
#pragma unroll
        for (int p = 0; p < 8; ++p) {                    // 4 token rows x 64 features at a time
            const int64_t t = t0 + 4 * p + wave, i = i0 + lane;
            ra[p] = t < t_end && i < I ? dY[t * lddy + i] : 0.f;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p) {                    // 16 token rows x 64 codes at a time
            const int64_t t = t0 + 16 * p + (tid >> 4), j = j0 + 4 * (tid & 15);
            const bool in = t < t_end && j < pitch;
            rb[p] = in ? *reinterpret_cast<const uint32_t*>(codes + t * pitch + j) : 0u;
            rs[p] = in ? scales[t * blocks + j / 32] : 0;
        }
    };
    auto stage = [&](int s) {
#pragma unroll
        for (int p = 0; p < 8; ++p) sA[s][4 * p + wave][lane] = ra[p];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 4; ++e) sB[s][16 * p + (tid >> 4)][4 * (tid & 15) + e] = ckpt_value(rb[p], e, ckpt_scale(rs[p]));
    };
    f32x16 acc;
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[q] = 0.f;
    const int64_t stages = t_begin < t_end ? ceil_div(t_end - t_begin, kStageF32) : 0;
    if (stages > 0) {
        load(t_begin);
        stage(0);
    }
    __syncthreads();
    for (int64_t st = 0; st < stages; ++st) {
        const int s = st & 1;
        const bool more = st + 1 < stages;
        if (more) load(t_begin + (st + 1) * kStageF32);
#pragma unroll
        for (int k = 0; k < kStageF32; k += 2)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(sA[s][k + h][32 * wm + l32], sB[s][k + h][32 * wn + l32], acc, 0, 0, 0);
        if (more) stage(s ^ 1);
        __syncthreads();
    }
    const bool split = gridDim.y > 1;
    void* dst = split ? static_cast<void*>(part + static_cast<int64_t>(blockIdx.y) * I * J) : out;
    const int64_t ld = split ? J : ldo, col = j0 + 32 * wn + l32;
    if (col < J)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int64_t row = i0 + 32 * wm + 8 * (q >> 2) + 4 * h + (q & 3);
            if (row < I) put(split ? kOutF32 : mode, dst, row * ld + col, acc[q]);
        }
}

__global__ void __launch_bounds__(kThreads)
k_sum_pieces(const float* __restrict__ part, int pieces, int64_t I, int64_t J, void* out, int64_t ldo, int mode) {
    const int64_t total = I * J;
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; e < total; e += static_cast<int64_t>(gridDim.x) * kThreads) {
        float s = 0.f;
        for (int k = 0; k < pieces; ++k) s += part[k * total + e];
        const int64_t i = e / J;
        put(mode, out, i * ldo + (e - i * J), s);
    }
}

struct Operands {
    const void* dY; int64_t T, lddy; const uint8_t* codes; const uint8_t* scales; int64_t I, J; void* dW; int64_t lddw; int mode; float* part;
    hipStream_t s;
};

template <int BM, int BN, int WM, int WN, bool WHOLE>
int run_t(const Operands& o, const WeightGradPlan& p) {
    constexpr int lds = 2 * kStageT * (BM + BN) * 2;
    auto kern = k_weight_grad<BM, BN, WM, WN, WHOLE>;
    if (lds > 48 * 1024) {
        static DeviceMemo attr_set;
        const int dev = DeviceMemo::device();
        if (!attr_set.get(dev)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                return BIMASK_ERR_HIP;
            attr_set.set(dev, 1);
        }
    }
    const int64_t tiles = ceil_div(o.I, BM) * ceil_div(o.J, BN), grid = round_up(tiles, 8);
    if (grid * (64 * WM * WN) > 0xFFFFFFFFll) return BIMASK_ERR_SHAPE;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid), static_cast<unsigned>(p.pieces)), dim3(64 * WM * WN), lds, o.s,
                       static_cast<const uint16_t*>(o.dY), o.T, o.lddy, o.codes, o.scales, o.I, o.J, o.dW, o.lddw, o.mode, o.part,
                       static_cast<int>(ceil_div(o.J, BN)), static_cast<int>(tiles), p.rows);
    return check_launch();
}

template <int BM, int BN, int WM, int WN>
int run(const Operands& o, const WeightGradPlan& p) {
    const bool whole = aligned16(o.dY) && o.lddy % 8 == 0 && o.I % 8 == 0;
    return whole ? run_t<BM, BN, WM, WN, true>(o, p) : run_t<BM, BN, WM, WN, false>(o, p);
}

}  // namespace

WeightGradPlan plan_weight_grad(int64_t T, int64_t I, int64_t J, int dtype) {
    WeightGradPlan p;
    const bool f32 = dtype == BIMASK_F32;
    p.big = !f32 && ceil_div(I, 256) * ceil_div(J, 256) >= 192;
    const int64_t bm = f32 ? kTileF32 : p.big ? 256 : 128, stage = f32 ? kStageF32 : kStageT;
    const int64_t tiles = ceil_div(I, bm) * ceil_div(J, bm), stages = ceil_div(T, stage);
    // pieces: about 512 workgroups, none with fewer than 8 stages
    int64_t pieces = p.big || tiles >= 512 ? 1 : ceil_div(512, tiles);
    const int64_t most = stages / 8 > 1 ? stages / 8 : 1;
    pieces = pieces < most ? pieces : most;
    p.rows = ceil_div(stages, pieces) * stage;
    p.pieces = ceil_div(T, p.rows);
    p.ws_bytes = p.pieces > 1 ? static_cast<size_t>(p.pieces) * I * J * 4 : 0;
    return p;
}

int launch_weight_grad(const void* dY, int64_t T, int64_t lddy, const uint8_t* ckpt, int64_t I, int64_t J, int dtype, void* dW, int64_t lddw,
                       int dw_dtype, bool accumulate, float* ws, hipStream_t s) {
    const WeightGradPlan p = plan_weight_grad(T, I, J, dtype);
    const int mode = dw_dtype == BIMASK_BF16 ? (accumulate ? kAddBF16 : kOutBF16) : (accumulate ? kAddF32 : kOutF32);
    const Operands o{dY, T, lddy, ckpt, ckpt + T * ckpt_pitch(J), I, J, dW, lddw, mode, ws, s};
    int rc;
    if (dtype == BIMASK_F32) {
        const int64_t tiles_j = ceil_div(J, kTileF32), tiles = ceil_div(I, kTileF32) * tiles_j;
        if (tiles * 256 > 0xFFFFFFFFll) return BIMASK_ERR_SHAPE;
        hipLaunchKernelGGL(k_weight_grad_f32, dim3(static_cast<unsigned>(tiles), static_cast<unsigned>(p.pieces)), dim3(256), 0, s,
                           static_cast<const float*>(dY), T, lddy, o.codes, o.scales, I, J, dW, lddw, mode, ws, static_cast<int>(tiles_j),
                           static_cast<int>(tiles), p.rows);
        rc = check_launch();
    } else {
        rc = p.big ? run<256, 256, 2, 4>(o, p) : run<128, 128, 2, 2>(o, p);
    }
    if (rc || p.pieces == 1) return rc;
    const int64_t n = ceil_div(I * J, kThreads);
    hipLaunchKernelGGL(k_sum_pieces, dim3(static_cast<unsigned>(n < 4096 ? n : 4096)), dim3(kThreads), 0, s, ws, static_cast<int>(p.pieces), I, J,
                       dW, lddw, mode);
    return check_launch();
}

}  // namespace bimask
