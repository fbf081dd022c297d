// Dense weight gradient of the straight-through estimator (arXiv 2302.06058, Sec. 3.1) from an 8-bit checkpoint of the layer's input:
//     dW[i][j] = sum_t dY[t][i] * X~[t][j]
//
// Both operands lie with the contraction index t as their slow dimension.  A stage of 32 tokens goes to LDS as it lies in memory
// (the codes put back to bf16 on the way: code * 2^e is exact in bf16), and the transposing LDS read hands every lane the
// consecutive tokens of its row that the matrix instruction wants.  16 lanes of such a read touch four token rows at 32 bytes
// each: the 64-byte chunks of a row are XOR-swizzled by the row so that they fall into different banks.
// Few output tiles and many tokens: workgroups split the tokens, their fp32 sums go to the workspace and are added in order.
#include "act.hpp"
#include <type_traits>

namespace bimask {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kStageT = 32;                              // tokens per stage
constexpr int64_t kMaxStages = 1 << 30;                  // of a workgroup, counted (a few beyond the last too) in an int

union Frag { bf16x8 v; u32x2 d[2]; };

// 4 consecutive tokens of one row per lane, 16 lanes: 4 tokens x 16 rows
__device__ __forceinline__ u32x2 read_turned(uint32_t lds, int ofs) {
    typedef __attribute__((address_space(3))) char lds_char;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)((lds_char*)lds + ofs)));
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

// LDS bytes: three stages, later the wavefronts' output strips
template <int BM, int BN, int WM, int WN>
constexpr int kGradLds = 3 * kStageT * (BM + BN) * 2 > WM * WN * 32 * (BN / WN + 4) * 4 ? 3 * kStageT * (BM + BN) * 2 : WM * WN * 32 * (BN / WN + 4) * 4;

// BM x BN output tile on WM x WN wavefronts.  WHOLE: I >= 8 and 32 rows of either operand span less than 2^31 bytes.  Rows of dY
// may start on any element (the 16-byte loads need no more).  Where I is no multiple of 8, the piece that would run over the row's
// end is the row's last 8 features instead: its first `over` rows of the output come twice, the others `over` places late.
// Pieces of `rows` tokens; with more than one the sums go to part + piece * I * J.
//
// Stages of 32 tokens pass through three LDS buffers: while stage s is multiplied, stage s + 2 (requested SETS stages ago, one register
// set each) is put back to bf16 and written, stage s + 2 + SETS is requested, and the first fragments of stage s + 1, complete since the last barrier,
// are read: a stage ends with one barrier and no wait for LDS or memory.  With WHOLE the loads are buffer loads of the piece's rows:
// what lies beyond the last token reads as zero without a comparison, and an address is a scalar base and a constant per thread.
// Columns beyond I or J are multiplied and not stored.
//
// Large tiles are bound by the matrix pipe at the clock that the card's power allows (11008 x 4096 with 8192 tokens 650-720 us, 1.03-1.13
// PFLOP/s, 690-910 launched 25 times in a row under the profiler; 4096 x 4096 238 us; a plain bf16 product of 8192 x 8192 x 8192 reaches
// 1.23); narrow ones by waits (64 x 576 with 200704 tokens 40 us for 145 MB, 3.6 TB/s: some 37 stages a workgroup, each of which ends with a
// barrier, and no pipe is busy above 40 %), plus 6 us for the sums of 170 pieces.
template <int BM, int BN, int WM, int WN, int SETS, bool WHOLE>
__global__ void __launch_bounds__(64 * WM * WN, 2)
k_weight_grad(const uint16_t* __restrict__ dY, int64_t T, int64_t lddy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
              int64_t I, int64_t J, void* out, int64_t ldo, int mode, float* part, uint32_t tiles_j, uint32_t tiles, uint32_t pieces, int64_t rows) {
    constexpr int NT = 64 * WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int PA = kStageT * BM / 8 / NT, PB = (kStageT * BN / 16 + NT - 1) / NT;       // 16-byte pieces per thread and stage
    constexpr int SA = kStageT * BM * 2, SB = kStageT * BN * 2;                  // LDS bytes of a stage
    static_assert(PA >= 1, "a piece for every thread");
    extern __shared__ u32x4 smem_u4[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(smem_u4);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % WM, wn = wave / WM, l32 = lane & 31, h = lane >> 5;
    // XCD x takes a contiguous run of (piece, tile) pairs, tiles fastest, so that its L2 serves the token rows of neighbours
    const uint32_t total = static_cast<uint32_t>(tiles) * static_cast<uint32_t>(pieces), per_xcd = (total + 7) / 8;
    const uint32_t n = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (n >= total) return;
    const uint32_t piece = n / tiles, tile = n - piece * tiles;
    const int64_t i0 = static_cast<int64_t>(tile / tiles_j) * BM, j0 = static_cast<int64_t>(tile % tiles_j) * BN;
    const int64_t t_begin = piece * rows, t_end = t_begin + rows < T ? t_begin + rows : T;
    const int64_t pitch = ckpt_pitch(J), blocks = ckpt_blocks(J);
    const int stages = static_cast<int>(t_begin < t_end ? ceil_div(t_end - t_begin, kStageT) : 0);

    auto has_b = [&](int p) { return kStageT * BN / 16 >= NT * (p + 1) || tid + NT * p < kStageT * BN / 16; };      // 64 and 192 columns: pieces for some of the threads

    auto swz_a = [](int row) { return BM % 128 == 0 ? row & 3 : (row >> 1) & 1; };
    auto swz_b = [](int row) { return BN % 128 == 0 ? row & 3 : (row >> 1) & 1; };

    u32x4 ra[SETS][PA], rb[SETS][PB];
    int rs[SETS][PB];
    uint32_t off_a[PA], off_b[PB], off_s[PB];
    if constexpr (WHOLE) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int q = tid + NT * p, row = q / (BM / 8), u = q % (BM / 8);
            off_a[p] = static_cast<uint32_t>((row * lddy + (i0 + 8 * u + 8 <= I ? i0 + 8 * u : I - 8)) * 2);
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int q = tid + NT * p, row = q / (BN / 16), u = q % (BN / 16);
            const int64_t j = j0 + 16 * u < pitch && has_b(p) ? j0 + 16 * u : 0;
            off_b[p] = static_cast<uint32_t>((has_b(p) ? row : 0) * pitch + j);
            off_s[p] = static_cast<uint32_t>((has_b(p) ? row : 0) * blocks + j / 32);
        }
    }
    // WHOLE: the rows of the next stage to request, as buffers that end with the piece's last row
    const uint16_t* next_a = dY + t_begin * lddy;
    const uint8_t *next_b = codes + t_begin * pitch, *next_s = scales + t_begin * blocks;
    int rows_left = static_cast<int>(t_end - t_begin);
    const int row_a = static_cast<int>(lddy * 2), last_a = static_cast<int>(I * 2), row_b = static_cast<int>(pitch), row_s = static_cast<int>(blocks);
    auto load = [&](int set, int st) {
        if constexpr (WHOLE) {
            const int n = rows_left < kStageT ? rows_left : kStageT, some = n > 0 ? -1 : 0;
            const auto A = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(next_a), 0, ((n - 1) * row_a + last_a) & some, 0x00020000);
            const auto B = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(next_b), 0, (n * row_b) & some, 0x00020000);
            const auto S = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(next_s), 0, (n * row_s) & some, 0x00020000);
            next_a += kStageT * lddy;                    // (past the end they are not read through: their buffers are empty)
            next_b += kStageT * pitch;
            next_s += kStageT * blocks;
            rows_left -= kStageT;
#pragma unroll
            for (int p = 0; p < PA; ++p) ra[set][p] = __builtin_amdgcn_raw_buffer_load_b128(A, off_a[p], 0, 0);
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                rb[set][p] = __builtin_amdgcn_raw_buffer_load_b128(B, off_b[p], 0, 0);
                rs[set][p] = __builtin_amdgcn_raw_buffer_load_b8(S, off_s[p], 0, 0);
            }
        } else {
            const int64_t t0 = t_begin + static_cast<int64_t>(st) * kStageT;
#pragma unroll
            for (int p = 0; p < PA; ++p) {
                const int q = tid + NT * p, row = q / (BM / 8), u = q % (BM / 8);
                const int64_t t = t0 + row, i = i0 + 8 * u;
                ra[set][p] = (u32x4){0u, 0u, 0u, 0u};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (t < t_end && i + e < I) ra[set][p][e >> 1] |= static_cast<uint32_t>(dY[t * lddy + i + e]) << (16 * (e & 1));
            }
#pragma unroll
            for (int p = 0; p < PB; ++p) {
                const int q = tid + NT * p, row = q / (BN / 16), u = q % (BN / 16);
                const int64_t t = t0 + row, j = j0 + 16 * u;
                const bool in = has_b(p) && t < t_end && j < pitch;
                const u32x4 v = *reinterpret_cast<const u32x4*>(codes + (in ? t * pitch + j : 0));
                rb[set][p] = in ? v : (u32x4){0u, 0u, 0u, 0u};
                rs[set][p] = in ? scales[t * blocks + j / 32] : 0;
            }
        }
    };
    auto stage_a = [&](int set, uint8_t* s) {
#pragma unroll
        for (int p = 0; p < PA; ++p) {
            const int q = tid + NT * p, row = q / (BM / 8), u = q % (BM / 8);
            *reinterpret_cast<u32x4*>(s + row * (BM * 2) + (((u >> 2) ^ swz_a(row)) << 6) + ((u & 3) << 4)) = ra[set][p];
        }
    };
    auto stage_b = [&](int set, uint8_t* s, int first, int end) {
#pragma unroll
        for (int p = first; p < end; ++p) {
            const int q = tid + NT * p, row = q / (BN / 16), u = q % (BN / 16);
            const float scale = ckpt_scale(rs[set][p]);
            uint8_t* dst = s + SA + row * (BN * 2) + (((u >> 1) ^ swz_b(row)) << 6) + ((u & 1) << 5);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                u32x4 v;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    const uint32_t four = rb[set][p][2 * x + (d >> 1)];
                    v[d] = pack_bf16(ckpt_value(four, 2 * (d & 1), scale), ckpt_value(four, 2 * (d & 1) + 1, scale));
                }
                if (has_b(p)) *reinterpret_cast<u32x4*>(dst + 16 * x) = v;
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

    Frag a[2][TM], b[2][TN];
    auto read = [&](int slot, uint32_t buf, int ks) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int i = 0; i < TM; ++i) a[slot][i].d[x] = read_turned(buf + fa[i], (16 * ks + 4 * x) * (BM * 2));
#pragma unroll
            for (int j = 0; j < TN; ++j) b[slot][j].d[x] = read_turned(buf + fb[j], (16 * ks + 4 * x) * (BN * 2));
        }
    };
    auto multiply = [&](int slot) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[slot][i].v, b[slot][j].v, acc[i][j], 0, 0, 0);
    };
    // the order in which the compiler is to mix the instructions of a half stage: reads and the rest between matrix instructions
    auto mix = [&]() {
#pragma unroll
        for (int k = 0; k < TM * TN; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                                          // matrix
            __builtin_amdgcn_sched_group_barrier(0x100, (2 * (TM + TN) + TM * TN - 1) / (TM * TN), 0);  // LDS read
            __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);                                          // ALU
            __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);                                          // LDS write
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);                                          // memory read
        }
    };

    if (stages > 0) {
        load(0, 0);
        load(1, 1);
        stage_a(0, smem);
        stage_b(0, smem, 0, PB);
        load(0, 2);
        stage_a(1, smem + (SA + SB));
        stage_b(1, smem + (SA + SB), 0, PB);
#pragma unroll
        for (int k = 1; k < SETS; ++k) load(k, k + 2);
        __syncthreads();
        const uint32_t lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) uint8_t*)smem));
        uint32_t cur = 0, next = SA + SB, after = 2 * (SA + SB);
        read(0, lds + cur, 0);
        auto step = [&](auto set_c, int st) {
            constexpr int set = decltype(set_c)::value;
            read(1, lds + cur, 1);
            multiply(0);
            stage_a(set, smem + after);
            stage_b(set, smem + after, 0, PB > 1 ? PB / 2 : 0);
            mix();
            __builtin_amdgcn_sched_barrier(0);
            read(0, lds + next, 0);
            multiply(1);
            stage_b(set, smem + after, PB > 1 ? PB / 2 : 0, PB);
            load(set, st + 2 + SETS);
            mix();
            __builtin_amdgcn_sched_barrier(0);
            __syncthreads();
            const uint32_t x = cur;
            cur = next;
            next = after;
            after = x;
        };
#pragma unroll 1
        for (int st = 0; st < stages; st += SETS) {      // (a stage beyond the last is one of zeros)
            step(std::integral_constant<int, 0>{}, st);
            step(std::integral_constant<int, 1>{}, st + 1);
            if constexpr (SETS == 4) {
                step(std::integral_constant<int, 2>{}, st + 2);
                step(std::integral_constant<int, 3>{}, st + 3);
            }
        }
    }

    // Output: 32 rows of a wavefront at a time through an LDS strip of its own, so that rows leave as segments of 32 TN columns.
    const bool split = pieces > 1;
    void* dst = split ? static_cast<void*>(part + static_cast<int64_t>(piece) * I * J) : out;
    const int64_t ld = split ? J : ldo;
    constexpr int COLS = 32 * TN, PITCH = COLS + 4;
    static_assert(COLS == BN / WN && WM * WN * 32 * PITCH * 4 <= kGradLds<BM, BN, WM, WN>, "strips fit");
    float* strip = reinterpret_cast<float*>(smem) + wave * (32 * PITCH);
    const int64_t col0 = j0 + wn * COLS + lane;
    __syncthreads();                                     // every wavefront is done with the stage buffers
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row0 = i0 + (wm * TM + i) * 32;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) strip[(8 * (q >> 2) + 4 * h + (q & 3)) * PITCH + 32 * j + l32] = acc[i][j][q];
        const int over = WHOLE ? static_cast<int>(-I & 7) : 0, n_rows = static_cast<int>(I - row0 < 32 ? I - row0 : 32);
        const int late = I - row0 < 32 ? n_rows & ~7 : 32;              // from this row on
        auto write = [&](auto mode_c) {
#pragma unroll 4
            for (int r = 0; r < n_rows; ++r)
#pragma unroll
                for (int c = 0; c < COLS; c += 64)
                    if (col0 + c < J && c + lane < COLS) put<decltype(mode_c)::value>(dst, (row0 + r) * ld + col0 + c, strip[(r + (r >= late ? over : 0)) * PITCH + c + lane]);
        };
        if (split || mode == kOutF32) write(std::integral_constant<int, kOutF32>{});
        else if (mode == kOutBF16) write(std::integral_constant<int, kOutBF16>{});
        else if (mode == kAddF32) write(std::integral_constant<int, kAddF32>{});
        else write(std::integral_constant<int, kAddBF16>{});
    }
}

// fp32: 64 x 64 tiles on 2 x 2 wavefronts, fp32 matrix instructions, whose operands are one element per lane: LDS rows as they lie.
// A load of dY is one token's row for the whole wavefront, a buffer that ends with the row (or is empty beyond the last token); stages
// are requested two ahead.  2048 x 2048 with 4096 tokens 322 us, 107 TFLOP/s; 1000 x 1000 with 4000 99 us (one stage ahead, elements
// compared one by one: 409 and 121).  128 x 128 tiles, which read LDS half as often: 318 and 96, not worth a second form.
constexpr int kStageF32 = 32, kTileF32 = 64;
__global__ void __launch_bounds__(256, 2)
k_weight_grad_f32(const float* __restrict__ dY, int64_t T, int64_t lddy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                  int64_t I, int64_t J, void* out, int64_t ldo, int mode, float* part, int tiles_j, int tiles, int64_t rows) {
    constexpr int B = kTileF32, PA = 8, PB = 2, WPR = B / 4;      // loads per thread and stage; words of codes per token
    __shared__ f32x4 sA4[2][kStageF32 * B / 4], sB4[2][kStageF32 * B / 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    const int l32 = lane & 31, h = lane >> 5, n = blockIdx.x;
    if (n >= tiles) return;
    const int64_t i0 = static_cast<int64_t>(n / tiles_j) * B, j0 = static_cast<int64_t>(n % tiles_j) * B;
    const int64_t t_begin = blockIdx.y * rows, t_end = t_begin + rows < T ? t_begin + rows : T;
    const int64_t pitch = ckpt_pitch(J), blocks = ckpt_blocks(J);
    const int row_bytes = static_cast<int>(I - i0 < B ? I - i0 : B) * 4;
    const int64_t stages = t_begin < t_end ? ceil_div(t_end - t_begin, kStageF32) : 0;
    float ra[2][PA];
    uint32_t rb[2][PB];
    int rs[2][PB];
    auto load = [&](int set, int64_t st) {
        const int64_t t0 = t_begin + st * kStageF32;
#pragma unroll
        for (int p = 0; p < PA; ++p) {                   // wavefront w: rows w, w + 4, ...
            const int64_t t = t0 + 4 * p + wave;
            const auto A = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(dY + t * lddy + i0), 0, t < t_end ? row_bytes : 0, 0x00020000);
            ra[set][p] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(A, 4 * lane, 0, 0));
        }
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const int q = tid + 256 * p, row = q / WPR;
            const int64_t t = t0 + row, j = j0 + 4 * (q % WPR);
            const bool in = t < t_end && j < pitch;
            const uint32_t four = *reinterpret_cast<const uint32_t*>(codes + (in ? t * pitch + j : 0));
            rs[set][p] = in ? scales[t * blocks + j / 32] : 0;
            rb[set][p] = in ? four : 0u;
        }
    };
    auto stage = [&](int set, int buf) {
        float* a = reinterpret_cast<float*>(sA4[buf]);
#pragma unroll
        for (int p = 0; p < PA; ++p) a[(4 * p + wave) * B + lane] = ra[set][p];
#pragma unroll
        for (int p = 0; p < PB; ++p) {
            const float scale = ckpt_scale(rs[set][p]);
            sB4[buf][tid + 256 * p] = (f32x4){ckpt_value(rb[set][p], 0, scale), ckpt_value(rb[set][p], 1, scale), ckpt_value(rb[set][p], 2, scale),
                                              ckpt_value(rb[set][p], 3, scale)};
        }
    };
    f32x16 acc;
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[q] = 0.f;
    auto step = [&](auto set_c, int64_t st) {            // stage st lies in buffer `set`, stage st + 1 is on its way in the other set
        constexpr int set = decltype(set_c)::value;
        load(set, st + 2);
        const float *a = reinterpret_cast<const float*>(sA4[set]) + 32 * wm + l32, *b = reinterpret_cast<const float*>(sB4[set]) + 32 * wn + l32;
#pragma unroll
        for (int k = 0; k < kStageF32; k += 2) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[(k + h) * B], b[(k + h) * B], acc, 0, 0, 0);
        stage(set ^ 1, set ^ 1);
        __syncthreads();
    };
    if (stages > 0) {
        load(0, 0);
        load(1, 1);
        stage(0, 0);
        __syncthreads();
#pragma unroll 1
        for (int64_t st = 0; st < stages; st += 2) {     // (a stage beyond the last is one of zeros)
            step(std::integral_constant<int, 0>{}, st);
            step(std::integral_constant<int, 1>{}, st + 1);
        }
    }
    const bool split = gridDim.y > 1;
    void* dst = split ? static_cast<void*>(part + static_cast<int64_t>(blockIdx.y) * I * J) : out;
    const int64_t ld = split ? J : ldo;
    const int64_t col = j0 + 32 * wn + l32;
    if (col < J)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
            const int64_t row = i0 + 32 * wm + 8 * (q >> 2) + 4 * h + (q & 3);
            if (row < I) put(split ? kOutF32 : mode, dst, row * ld + col, acc[q]);
        }
}

// Sums of the pieces, added in piece order.  Few pieces: four consecutive elements a thread.  Many (a small matrix): 64 elements x 4
// ranges of pieces per workgroup, so that the chain of additions is a quarter as long.
constexpr int kFewPieces = 12;

__global__ void __launch_bounds__(kThreads)
k_sum_few_pieces(const float* __restrict__ part, int pieces, int64_t I, int64_t J, void* out, int64_t ldo, int mode) {
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    const int64_t total = I * J;
    for (int64_t e = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) * 4; e < total; e += static_cast<int64_t>(gridDim.x) * kThreads * 4) {
        const int n = static_cast<int>(total - e < 4 ? total - e : 4);
        const int64_t from = e + 4 <= total ? e : total >= 4 ? total - 4 : 0;        // the last elements: four that exist
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        if (total >= 4) {
#pragma unroll 4
            for (int k = 0; k < pieces; ++k) s += __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(part + k * total + from));
        } else {
            for (int k = 0; k < pieces; ++k)
                for (int x = 0; x < n; ++x) s[x] += part[k * total + x];
        }
        int64_t i = e / J, j = e - i * J;
        const int skip = static_cast<int>(e - from);
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (x < n) {
                const float v = skip + x == 0 ? s[0] : skip + x == 1 ? s[1] : skip + x == 2 ? s[2] : s[3];
                put(mode, out, i * ldo + j, v);
                if (++j == J) { j = 0; ++i; }
            }
    }
}

__global__ void __launch_bounds__(kThreads)
k_sum_pieces(const float* __restrict__ part, int pieces, int64_t I, int64_t J, void* out, int64_t ldo, int mode) {
    __shared__ float sums[4][64];
    const int x = threadIdx.x & 63, y = threadIdx.x >> 6;
    const int64_t total = I * J;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * 64; first < total; first += static_cast<int64_t>(gridDim.x) * 64) {
        const int64_t e = first + x;
        float s = 0.f;
        if (e < total)
            for (int k = y; k < pieces; k += 4 * 12) {   // twelve requests at once, those beyond the last piece of one that exists
                float v[12];
#pragma unroll
                for (int u = 0; u < 12; ++u) v[u] = part[(k + 4 * u < pieces ? k + 4 * u : k) * total + e];
#pragma unroll
                for (int u = 0; u < 12; ++u) s += k + 4 * u < pieces ? v[u] : 0.f;
            }
        sums[y][x] = s;
        __syncthreads();
        if (y == 0 && e < total) {
            const int64_t i = e / J;
            put(mode, out, i * ldo + (e - i * J), ((sums[0][x] + sums[1][x]) + sums[2][x]) + sums[3][x]);
        }
        __syncthreads();
    }
}

struct Operands {
    const void* dY; int64_t T, lddy; const uint8_t* codes; const uint8_t* scales; int64_t I, J; void* dW; int64_t lddw; int mode; float* part;
    hipStream_t s;
};

template <int BM, int BN, int WM, int WN, int SETS, bool WHOLE>
int run(const Operands& o, const WeightGradPlan& p) {
    constexpr int lds = kGradLds<BM, BN, WM, WN>;
    auto kern = k_weight_grad<BM, BN, WM, WN, SETS, WHOLE>;
    if (lds > 48 * 1024) {
        static DeviceMemo attr_set;
        const int dev = DeviceMemo::device();
        if (!attr_set.get(dev)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                return BIMASK_ERR_HIP;
            attr_set.set(dev, 1);
        }
    }
    const int64_t tiles = ceil_div(o.I, BM) * ceil_div(o.J, BN), grid = round_up(tiles * p.pieces, 8);
    if (grid * (64 * WM * WN) > 0xFFFFFFFFll) return BIMASK_ERR_SHAPE;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(grid)), dim3(64 * WM * WN), lds, o.s,
                       static_cast<const uint16_t*>(o.dY), o.T, o.lddy, o.codes, o.scales, o.I, o.J, o.dW, o.lddw, o.mode, o.part,
                       static_cast<uint32_t>(ceil_div(o.J, BN)), static_cast<uint32_t>(tiles), static_cast<uint32_t>(p.pieces), p.rows);
    return check_launch();
}

}  // namespace

// Tile and pieces.  A 256 x 256 tile moves half the LDS bytes of four 128 x 128 ones per product (2048 x 2048 with 4096 tokens 56 us
// in 4 pieces of the 64 tiles, 61 with 256 tiles of 128 x 128; 1024 x 4096 with 8192 81 / 96), as long as tiles and pieces fill the 256
// CUs once without much padding and a piece has the stages that pay for its sums (1024 x 1024 with 4096 34 / 30, 3000 x 1000 with 2000
// 37 / 31).  Narrow matrices: tiles as narrow.  The others: two workgroups per CU are there at once, so at most 512 pieces of tiles, and
// none where the tiles alone fill half of the CUs (3000 x 1000 with 2000 tokens 31 us, in two pieces 35).  A piece's sums cost as much
// as some stages, more of them the larger the matrix: at least 6 stages a piece with up to 16 tiles (200 x 200 with 3000 tokens 12.4 us,
// with 16 stages 16.1), 16 with more (1000 x 1000 with 2000 24.3, with 8 stages 29).  fp32, whose stages take three times as long: pieces also up to
// 256 tiles (1000 x 1000 with 4000 99 us, without 125), of 2 stages up to 64 tiles (100 x 100 with 1000 9.3, with 8 stages 14.7), then 8 (1024 x 512 with 200 11.8 / 15.3).
// More large tiles than CUs: where the last round over the chip would be at most half full, large tiles take the whole rounds and the rows
// behind them a plan of their own, smaller tiles or pieces (4352 x 4096 with 4096 tokens, 272 tiles, 216 us in 128 x 128 tiles, 157 so;
// 4864 x 4096 with 8192, 304, 421 / 308; 6144 x 4096 with 4096, 384, 219 / 211; but 5120 x 5120, 400, 222 / 247).  Over 59 matrices with 768 to 4096
// tokens 0.915 of one plan's time in the geometric mean; 21 of the 354 sizes lose, most at 1536 tokens with a last round above 3/8 (6144 x 4096 94 / 103) or
// up to there behind 240 of 256 CUs (4096 x 5120 with 1024 66 / 68-70), which no simple rule sets apart.
WeightGradPlan plan_weight_grad(int64_t T, int64_t I, int64_t J, int dtype) {
    WeightGradPlan p;
    p.first = 0;
    int64_t bm, bn, stage = kStageT, pieces;
    if (dtype == BIMASK_F32) {
        p.tile = WeightGradPlan::k64x64;
        bm = bn = kTileF32;
        stage = kStageF32;
    } else if (I <= 64 && J > 64) {
        p.tile = round_up(J, 192) < round_up(J, 256) ? WeightGradPlan::k64x192 : WeightGradPlan::k64x256;
        bm = 64;
        bn = p.tile == WeightGradPlan::k64x192 ? 192 : 256;
    } else if (J <= 64 && I > 64) {
        p.tile = WeightGradPlan::k256x64;
        bm = 256;
        bn = 64;
    } else {
        p.tile = WeightGradPlan::k128x128;
        bm = bn = 128;
    }
    const int64_t stages = ceil_div(T, stage), tiles = ceil_div(I, bm) * ceil_div(J, bn), large = ceil_div(I, 256) * ceil_div(J, 256);
    pieces = tiles >= 128 ? 1 : 512 / tiles;
    const int64_t least = dtype == BIMASK_F32 ? (tiles <= 64 ? 2 : 8) : tiles <= 16 ? 6 : 16;
    if (p.tile == WeightGradPlan::k128x128) {
        const int64_t n = large >= 256 ? 1 : 256 / large;
        const double filled = static_cast<double>(I) * static_cast<double>(J) / (static_cast<double>(large) * 65536) *
                              static_cast<double>(large * n) / static_cast<double>(round_up(large * n, 256));
        if (filled >= 0.75 && (n == 1 || stages / n >= 24)) {
            p.tile = WeightGradPlan::k256x256;
            pieces = n;
        }
        const int64_t across = ceil_div(J, 256), whole = large / 256 * 256, bands = whole / across, rest = large - bands * across;
        if (whole > 0 && rest > 0 && rest <= 128 && stages >= 24 && bands * across * 10 >= whole * 9 && J * 8 >= across * 256 * 7) {
            p.first = bands * 256;
            if (I - p.first < 8) p.first -= 256;         // (fewer than 8 rows have no fast form)
            p.tile = WeightGradPlan::k256x256;
            p.pieces = 1;
            p.rows = stages * stage;
            p.ws_bytes = plan_weight_grad(T, I - p.first, J, dtype).ws_bytes;
            return p;
        }
    } else if (dtype == BIMASK_F32 && tiles <= 256) {
        pieces = 512 / tiles;
    }
    int64_t most = stages / least;
    if (most < 1 || (dtype == BIMASK_F32 && stages < 8)) most = 1;
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
    if (p.rows > kMaxStages * kStageT) return BIMASK_ERR_SHAPE;
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
        if (I < 8 || lddy >= (1 << 24) || J >= (1 << 25) || T >= (1ll << 31)) rc = run<128, 128, 2, 2, 2, false>(o, p);
        else if (p.first > 0) {
            Operands f = o;
            f.I = p.first;
            if (int rc1 = run<256, 256, 2, 4, 2, true>(f, p)) return rc1;
            return launch_weight_grad(static_cast<const uint16_t*>(dY) + p.first, T, lddy, ckpt, I - p.first, J, dtype,
                                      static_cast<uint8_t*>(dW) + p.first * lddw * (dw_dtype == BIMASK_BF16 ? 2 : 4), lddw, dw_dtype, accumulate, ws, s);
        }
        else if (p.tile == WeightGradPlan::k256x256) rc = run<256, 256, 2, 4, 2, true>(o, p);
        else if (p.tile == WeightGradPlan::k64x192) rc = run<64, 192, 2, 2, 4, true>(o, p);
        else if (p.tile == WeightGradPlan::k64x256) rc = run<64, 256, 1, 4, 4, true>(o, p);
        else if (p.tile == WeightGradPlan::k256x64) rc = run<256, 64, 4, 1, 4, true>(o, p);
        else rc = run<128, 128, 2, 2, 4, true>(o, p);
    }
    if (rc || p.pieces == 1) return rc;
    const bool few = p.pieces <= kFewPieces;
    const int64_t n = ceil_div(I * J, few ? 4 * kThreads : 64);
    hipLaunchKernelGGL(few ? k_sum_few_pieces : k_sum_pieces, dim3(static_cast<unsigned>(n < (1 << 20) ? n : 1 << 20)), dim3(kThreads), 0, s, ws,
                       static_cast<int>(p.pieces), I, J, dW, lddw, mode);
    return check_launch();
}

}  // namespace bimask
