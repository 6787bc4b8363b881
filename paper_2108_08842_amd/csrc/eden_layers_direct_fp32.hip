// Matrix products of two fp32 operands whose rows are whole 16-byte pieces (eden_linear, eden_linear_input_grad).
//
// out[r][c] = sum_d A(r, d) B(c, d) as products of bf16 terms: x = h + m + l, h the upper 16 bits, m and l the nearest bf16 numbers to what the ones before leave
// (exact), and the six products down to 2^-16 of the first; the others are below 2^-22 together.  The matrix cores do that at 2500 / 6 TFLOP/s at most; their own fp32 products end at 157.
//
// A workgroup has a tile of 128 x 128, two to a CU, a wave 64 x 64.  Operands' tiles are 32 deep (128-byte lines) and go straight into the LDS as fp32; the LDS
// holds five, in turns as in the kernel for two-byte types: the two in use, the next two, the first of the two after that.  A wave reads the
// operands of the next 16 deep and takes them apart in registers while it multiplies those of the last: 5.5 vector instructions an element,
// 176 in the time of 24 products.  Bound by the card's power and the vector unit: 4096 x 8192 x 4096 takes 1380 to 1390 us = 198 TFLOP/s (input gradient 1390 to
// 1400), with the matrix cores busy 65% of the cycles at 1.47 GHz (six launches under a profiler).  Two workgroups fit a CU, but a sum is split over 256 of them only: 3654 x 320, 11904 deep, is 87 tiles in
// two parts and takes 266 us with the matrix cores busy 34% of the cycles.
#include "eden_layers_fetch.h"

namespace eden_layers {
namespace {

constexpr int kThreads = 256, kSide = 128, kDeep = 32, kSlots = 5;
constexpr int kOperand = kSide * kDeep * 4;        // bytes of an operand's tile, a slot of the LDS
constexpr int kLoads = kOperand / 16 / kThreads;   // 16-byte pieces per thread
constexpr int kPieces = kSide * 4 / 16;            // of a row of columns

// Rows of columns: 32 columns at depths 8 apart lie in different banks.
__device__ inline int piece_of_fp32_depth(int depth, int piece) { return depth * (kSide * 4) + ((piece ^ (depth & 8)) << 4); }

// Where a thread's pieces of an operand come from: byte offsets from the tile's first element.
template <bool STRIDED> struct Source {
    const char *base;
    size_t step;               // bytes from one tile to the next
    uint64_t reach;            // bytes from `base` to the end of what may be read
    uint32_t offset[2], stride;   // of piece i: offset[i & 1] + i * stride
    uint32_t depth;            // !STRIDED: depth of this lane's pieces inside a tile
    u32x4 now;                 // of the tile that is being fetched
    uint32_t at[2];

    // rows or columns first .. count - 1 of the operand, depths begin .. end - 1; `whole`: elements of a row of memory
    __device__ Source(const void *p, size_t ld, uint32_t first, uint32_t count, uint32_t begin, uint32_t end, uint32_t whole, int wave, int lane) {
        if constexpr (STRIDED) {
            base = static_cast<const char *>(p) + ((size_t)begin * ld + first) * 4;
            step = (size_t)kDeep * ld * 4;
            reach = ((uint64_t)(end - begin - 1) * ld + (whole - first)) * 4;
            const uint32_t d = wave * 2 + (lane >> 5);             // + 8 i
            offset[0] = (uint32_t)(d * ld * 4) + (lane & 31) * 16;
            offset[1] = (uint32_t)(d * ld * 4) + ((lane & 31) ^ 8) * 16;
            stride = (uint32_t)(8 * ld * 4);
            depth = 0;
        } else {
            const uint32_t rows = min((uint32_t)kSide, count - first);
            base = static_cast<const char *>(p) + ((size_t)first * ld + begin) * 4;
            step = kDeep * 4;
            reach = ((uint64_t)(rows - 1) * ld + (whole - begin)) * 4;
            const uint32_t row = wave * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
            offset[0] = offset[1] = (uint32_t)(row * ld * 4) + piece * 16;
            stride = (uint32_t)(32 * ld * 4);
            depth = piece * 4;
        }
    }
    // The next tile is `left` deep.  What lies beyond is read as zeros.
    __device__ void start(uint32_t left) {
        now = descriptor(base, reach);
        const bool inside = STRIDED ? 0u < left : depth < left;
        at[0] = inside ? offset[0] : kNowhere;                     // (and further on)
        at[1] = inside ? offset[1] : kNowhere;
        base += step;
        reach = reach > step ? reach - step : 0;
    }
    __device__ void fetch(uint32_t slot, int wave, int i) const { load_to_lds(slot + (i * 4 + wave) * 1024, at[i & 1] + i * stride, now); }
};

// Eight neighbouring depths of one row or column
struct Raw { float v[8]; };

// Where a lane reads an operand's tile in the LDS: index base + 32 i + lane % 32, depths 16 s + 8 (lane / 32) .. + 7.
template <bool STRIDED> struct Reader {
    uint32_t at[STRIDED ? 2 : 4];

    __device__ Reader(int base, int lane) {
        const int half = lane >> 5;
        if constexpr (STRIDED) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = base + i * 32 + (lane & 31);
                at[i] = piece_of_fp32_depth(8 * half, col >> 2) + (col & 3) * 4;
            }
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) at[s] = piece_of_row<64>(base + (lane & 31), (s >> 1) * 4 + half * 2 + (s & 1));
        }
    }
    __device__ Raw read(const char *slot, int i, int s) const {
        Raw r;
        if constexpr (STRIDED) {
#pragma unroll
            for (int j = 0; j < 8; ++j) r.v[j] = *reinterpret_cast<const float *>(slot + at[i] + (16 * s + j) * (kSide * 4));
        } else {
            *reinterpret_cast<f32x4 *>(r.v) = *reinterpret_cast<const f32x4 *>(slot + at[2 * s] + i * (32 * kDeep * 4));
            *reinterpret_cast<f32x4 *>(r.v + 4) = *reinterpret_cast<const f32x4 *>(slot + at[2 * s + 1] + i * (32 * kDeep * 4));
        }
        return r;
    }
};

// Elements 2 q and 2 q + 1 as three terms each.
__device__ inline void take_apart(const Raw &r, int q, u32x4 (&terms)[3]) {
    float a = r.v[2 * q], b = r.v[2 * q + 1];
#pragma unroll
    for (int t = 0; t < 3; ++t) terms[t][q] = take_nearest(a, b, t == 0);
}

template <int OP> __global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_direct_fp32(const Product p) {
    constexpr bool kStridedB = OP == kInputGrad;
    constexpr int N = 24;                                          // products 16 deep
    constexpr int kTermA[6] = {2, 1, 0, 1, 0, 0}, kTermB[6] = {0, 1, 2, 0, 1, 0};      // small ones first
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * kOperand];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wave_row = wave >> 1, wave_col = wave & 1;
    const uint32_t row_tiles = tiles_of(p.rows, kSide), col_tiles = tiles_of(p.cols, kSide);
    uint32_t split, row_tile, col_tile;
    place_of(blockIdx.x, gridDim.x, row_tiles, col_tiles, split, row_tile, col_tile);
    const uint32_t row0 = row_tile * kSide, col0 = col_tile * kSide;
    const uint32_t begin = split * p.split_depth, end = min(p.depth, begin + p.split_depth);
    const uint32_t steps = (end - begin + kDeep - 1) / kDeep;      // begin < end: launched for depths above 0 only

    Source<false> a(p.a, p.lda, row0, p.rows, begin, end, p.a_width, wave, lane);
    Source<kStridedB> b(p.b, p.ldb, col0, p.cols, begin, end, p.b_width, wave, lane);
    const Reader<false> reader_a(wave_row * 64, lane);
    const Reader<kStridedB> reader_b(wave_col * 64, lane);

    f32x16 acc[2][2] = {};
    u32x4 ta[2][2][3], tb[2][2][3];                                // [set][tile][term]
    Raw raw[4];                                                    // of A's tiles, of B's

    const uint32_t lds0 = (uint32_t)(size_t)(lds_char *)lds;
    auto depth_left = [&](uint32_t step) { return end - begin > step * kDeep ? end - begin - step * kDeep : 0u; };
    auto read = [&](const char *slot_a, const char *slot_b, int s, int i) {       // raw operand i of four
        raw[i] = i < 2 ? reader_a.read(slot_a, i, s) : reader_b.read(slot_b, i - 2, s);
    };
    auto split_quarter = [&](int set, int n) {                     // elements 2 (n / 4) .. + 1 of raw operand n % 4
        const int i = n % 4, q = n / 4;
        take_apart(raw[i], q, i < 2 ? ta[set][i] : tb[set][i - 2]);
    };
    // Products 16 deep of the half S of a tile, while the next half's operands are read (S = 1: of the next tiles, behind a barrier since when nobody needs the present
    // ones) and taken apart.  S = 0 fetches the first operand's tile after the next, S = 1 the second's.
    auto deep16 = [&](auto half, const char *slot_a, const char *slot_b, uint32_t fetch_to) {
        constexpr int S = decltype(half)::value;
        each<N>([&](auto number) {
            constexpr int j = decltype(number)::value, product = j / 4, i = j % 4 / 2, c = j % 2;
            acc[i][c] = multiply<false>(tb[S][c][kTermB[product]], ta[S][i][kTermA[product]], acc[i][c]);
            if constexpr (S == 1 && j == 0) meet<kLoads>();        // (later: the first operand's tile after the next)
            if constexpr (j < 4) read(slot_a, slot_b, S ^ 1, j);
            constexpr int load = due(j, kLoads, N);
            if constexpr (load >= 0 && S == 0) a.fetch(fetch_to, wave, load);
            if constexpr (load >= 0 && S == 1) b.fetch(fetch_to, wave, load);
            if constexpr (j >= 8) split_quarter(S ^ 1, j - 8);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // Tile number c (first operand of step s: 2 s, second: 2 s + 1) goes to slot c mod 5.
    auto on = [](uint32_t slot, uint32_t tiles) {
        const uint32_t to = slot + tiles * kOperand;
        return to >= (uint32_t)(kSlots * kOperand) ? to - kSlots * kOperand : to;
    };
    auto fetch_tile = [&](auto &source, uint32_t step, uint32_t slot) {
        source.start(depth_left(step));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) source.fetch(lds0 + slot * kOperand, wave, i);
    };
    fetch_tile(a, 0, 0);
    fetch_tile(b, 0, 1);
    fetch_tile(a, 1, 2);
    fetch_tile(b, 1, 3);
    meet<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i) read(lds, lds + kOperand, 0, i);
#pragma unroll
    for (int n = 0; n < 16; ++n) split_quarter(0, n);
    uint32_t slot = 0;                                             // of the first operand of the present step
    for (uint32_t step = 0; step < steps; ++step) {
        const uint32_t slot_b = on(slot, 1), next_a = on(slot, 2), next_b = on(slot, 3), after_a = on(slot, 4);
        a.start(depth_left(step + 2));
        deep16(std::integral_constant<int, 0>(), lds + slot, lds + slot_b, lds0 + after_a);
        b.start(depth_left(step + 2));
        deep16(std::integral_constant<int, 1>(), lds + next_a, lds + next_b, lds0 + slot);
        slot = next_a;
    }

    meet<0>();                                                     // nothing is read or fetched any more: the LDS takes the sums
    finish_wave<OP, EDEN_F32, 2>(p, acc, reinterpret_cast<float *>(lds) + wave * 32 * kRowFloats<2>, row0 + wave_row * 64, col0 + wave_col * 64, 0, lane, split);
}

}  // namespace

hipError_t launch_direct_fp32(Op op, const Product &p, hipStream_t st) {
    const uint32_t grid = tiles_of(p.rows, kSide) * tiles_of(p.cols, kSide) * p.splits;
    if (op == kForward) k_direct_fp32<kForward><<<grid, kThreads, 0, st>>>(p);
    else k_direct_fp32<kInputGrad><<<grid, kThreads, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace eden_layers
