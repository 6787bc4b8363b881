// Matrix products of 4-bit operands, out[r][c] = sum over d of a(r, d) b(c, d), on the matrix cores that take codes and exponents as they are.
//
// A workgroup has a tile of 256 x 256, a wave 128 x 128 of it (256 accumulation registers), or 128 x 128 and 64 x 64, two workgroups to a CU, where the
// result is small.  A product of 32 x 32 x 64 takes 32 cycles and 2 x 1 KB of codes: as many bytes a cycle as a bf16 product of 32 x 32 x 16, at four times the operations.
//   memory -> LDS      a chunk (256 deep, a row's 128 bytes: whole lines) of both operands and their exponents (8 bytes a row, which lie together for neighbouring
//                      rows) straight into the LDS, which holds two such chunks: while one is multiplied the other one arrives
//   LDS -> registers   lane l holds row l % 32 and block 4 (l / 32) + s of the chunk in step s = 0 .. 3: the order of a sum is free as long as both operands have
//                      the same, and this one puts a lane's four exponents into one word, of which a product names the byte
//   barriers           one a chunk, between the last reads of one and the first of the next
// 16-byte pieces of a row are swapped on the way into the LDS, so that neighbouring rows lie in different banks.
//
// The matrix instruction alone, on constant registers, reaches 8650 TFLOP/s here.  8192 x 16384, 4096 deep, bf16: bare 311 to 337 us (3300 to 3530 TFLOP/s), 8192 x 4096, 16384 deep, 231 (4760); the weight gradient
// 4096 x 8192, 8192 deep, 137 (4010, matrix cores busy half of the cycles at 1.9 GHz).  Deep sums are bound by power: that of 4760 reaches 6910 on zeros.  With gelu
// and a checkpoint 425 (30% matrix, 40% vector): the ends, 14 us for each of a CU's eight tiles, have no products beside them.  A large tile's workgroups stay and fetch the next
// tile's first chunk during the end (355 -> 340 us).  Tried and not kept: loads spread over three steps of four, all loads in one step, workgroups of small tiles that stay.
#include "eden_layers_fetch.h"
#include "eden_mx4_kernels.h"

#include <algorithm>

namespace eden_layers {
namespace {

constexpr int kThreads = 256, kSteps = 4;
constexpr uint32_t kResident = 256;                                // CUs
template <int T> struct Tile4 {
    static constexpr int kSide = 64 * T;
    static constexpr int kOperand = kSide * (int)kChunkBytes;      // bytes of an operand's chunk in the LDS
    static constexpr int kLoads = kOperand / 16 / kThreads;        // 16-byte pieces per thread
    static constexpr int kExps = kSide * (int)kChunkBlocks;        // bytes of its exponents
    static constexpr int kStage = 2 * kOperand + 2 * kExps;        // both operands, then both exponents
};

// Where a thread's pieces of an operand's codes come from.
template <int T> struct Codes4 {
    const char *base;
    uint64_t reach;
    uint32_t offset, stride;
    u32x4 now;

    __device__ Codes4(const void *p, uint32_t chunks, uint32_t first, uint32_t count, uint32_t chunk, int wave, int lane) {
        const uint32_t row_bytes = chunks * kChunkBytes, rows = min((uint32_t)Tile4<T>::kSide, count - first), row = wave * 8 + (lane >> 3);
        base = static_cast<const char *>(p) + (size_t)first * row_bytes + (size_t)chunk * kChunkBytes;
        reach = (uint64_t)rows * row_bytes - (uint64_t)chunk * kChunkBytes;
        offset = row * row_bytes + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
        stride = 32 * row_bytes;
    }
    // The next chunk; nothing if there is none
    __device__ void start(bool is) {
        now = descriptor(base, is ? reach : 0);
        base += kChunkBytes;
        reach -= kChunkBytes;
    }
    __device__ void fetch(uint32_t to, int wave, int i) const { load_to_lds(to + (i * 4 + wave) * 1024, offset + i * stride, now); }
};
// The exponents of both: T / 2 waves fetch a kilobyte of either operand's (256 rows: two waves, 128 rows: one).
template <int T> struct Exps4 {
    static constexpr int kWavesEach = T / 2;
    const char *base;
    uint64_t reach, step;
    uint32_t offset, to;
    u32x4 now;

    __device__ Exps4(const Product &p, uint32_t chunks, uint32_t row0, uint32_t col0, uint32_t chunk, int wave, int lane) {
        const bool second = wave >= kWavesEach;
        const uint64_t rows = second ? p.cols : p.rows;
        const uint32_t first = second ? col0 : row0, within = wave - (second ? kWavesEach : 0);
        base = static_cast<const char *>(second ? p.b : p.a) + (size_t)rows * chunks * kChunkBytes + exps_at(rows, first, chunk);
        step = even(rows) * kChunkBlocks;
        reach = step * (chunks - chunk) - (uint64_t)first * kChunkBlocks;          // (behind the last row: the next chunk's, of rows that are not stored)
        offset = wave < 2 * kWavesEach ? within * 1024 + lane * 16 : kNowhere;
        to = 2 * Tile4<T>::kOperand + (second ? Tile4<T>::kExps : 0) + within * 1024;
    }
    __device__ void start(bool is) {
        now = descriptor(base, is ? reach : 0);
        base += step;
        reach = reach > step ? reach - step : 0;
    }
    __device__ void fetch(uint32_t stage) const {
        if (T == 4 || offset != kNowhere) load_to_lds(stage + to, offset, now);       // (a wave that has none would write zeros behind them)
    }
};

__device__ inline i32x8 operand4(u32x4 v) { return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0}; }
template <int S> __device__ inline f32x16 multiply4(u32x4 a, uint32_t exp_a, u32x4 b, uint32_t exp_b, f32x16 c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand4(a), operand4(b), c, 4, 4, S, (int)exp_a, S, (int)exp_b);
}

template <int OP, uint32_t DTYPE, int T> __global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(T == 4 ? 1 : 2, T == 4 ? 1 : 2))) void k_mx4_tiles(const Product p) {
    constexpr int kSide = Tile4<T>::kSide, kOperand = Tile4<T>::kOperand, kLoads = Tile4<T>::kLoads, kStage = Tile4<T>::kStage, N = T * T;
    static_assert(4 * 32 * kRowFloats<T> * 4 <= kStage, "the end's sums");
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStage];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wave_row = wave >> 1, wave_col = wave & 1;
    const uint32_t row_tiles = (p.rows + kSide - 1) / kSide, col_tiles = (p.cols + kSide - 1) / kSide, total = row_tiles * col_tiles * p.splits;
    const uint32_t chunks = chunks_of(p.depth), split_chunks = p.split_depth / kChunk;

    // where a lane reads: step s at piece 4 (lane / 32) + s; tiles of 32 are whole rows apart
    uint32_t at_a[kSteps], at_b[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        at_a[s] = piece_of_row<64>(wave_row * (kSide / 2) + (lane & 31), 4 * (lane >> 5) + s);
        at_b[s] = kOperand + piece_of_row<64>(wave_col * (kSide / 2) + (lane & 31), 4 * (lane >> 5) + s);
    }
    const uint32_t exp_a = 2 * kOperand + (wave_row * (kSide / 2) + (lane & 31)) * kChunkBlocks + 4 * (lane >> 5);
    const uint32_t exp_b = 2 * kOperand + Tile4<T>::kExps + (wave_col * (kSide / 2) + (lane & 31)) * kChunkBlocks + 4 * (lane >> 5);

    // a tile of the result, or a split of one, and where its operands come from
    struct Work {
        uint32_t split, row0, col0, steps;
        Codes4<T> a, b;
        Exps4<T> exps;
    };
    auto work_of = [&](uint32_t id) {
        uint32_t split, row_tile, col_tile;
        place_of(id, total, row_tiles, col_tiles, split, row_tile, col_tile);
        const uint32_t row0 = row_tile * kSide, col0 = col_tile * kSide, first = split * split_chunks;
        return Work{split, row0, col0, min(chunks, first + split_chunks) - first, Codes4<T>(p.a, chunks, row0, p.rows, first, wave, lane), Codes4<T>(p.b, chunks, col0, p.cols, first, wave, lane),
                    Exps4<T>(p, chunks, row0, col0, first, wave, lane)};
    };
    auto start = [](Work &w, uint32_t step) { w.a.start(step < w.steps), w.b.start(step < w.steps), w.exps.start(step < w.steps); };
    const uint32_t lds0 = (uint32_t)(size_t)(lds_char *)lds;
    auto first_chunk = [&](Work &w, uint32_t to) {
        start(w, 0);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) w.a.fetch(lds0 + to, wave, i);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) w.b.fetch(lds0 + to + kOperand, wave, i);
        w.exps.fetch(lds0 + to);
    };

    u32x4 fa[2][T], fb[2][T];
    uint32_t ea[T], eb[T], next_ea[T], next_eb[T];
    auto read = [&](const char *stage, int s, int set, int i) {    // one operand of 2 T
        if (i < T) fb[set][i] = *reinterpret_cast<const u32x4 *>(stage + at_b[s] + i * (32 * (int)kChunkBytes));
        else fa[set][i - T] = *reinterpret_cast<const u32x4 *>(stage + at_a[s] + (i - T) * (32 * (int)kChunkBytes));
    };
    auto read_exps = [&](const char *stage, int i) {
        if (i < T) next_eb[i] = *reinterpret_cast<const uint32_t *>(stage + exp_b + i * (32 * (int)kChunkBlocks));
        else next_ea[i - T] = *reinterpret_cast<const uint32_t *>(stage + exp_a + (i - T) * (32 * (int)kChunkBlocks));
    };
    auto take_exps = [&] {
#pragma unroll
        for (int i = 0; i < T; ++i) ea[i] = next_ea[i], eb[i] = next_eb[i];
    };

    uint32_t now = 0, id = blockIdx.x;
    Work w = work_of(id);
    first_chunk(w, now);
    for (;;) {
        f32x16 acc[T][T] = {};
        // T x T products 64 deep: S = 0 .. 3 of a chunk.  The operands of the following ones are read; S = 3: those of the next chunk, behind a barrier since when nobody needs
        // the present one, into whose place the chunk after the next goes: one operand during S = 3, the other one and the exponents during S = 0.
        auto deep64 = [&](auto step64, const char *stage, uint32_t to) {
            constexpr int S = decltype(step64)::value, set = S & 1, kReads = 2 * T;
            each<N>([&](auto number) {
                constexpr int j = decltype(number)::value, i = j / T;
                acc[i][j % T] = multiply4<S>(fb[set][j % T], eb[j % T], fa[set][i], ea[i], acc[i][j % T]);
                if constexpr (S == 3 && j == 0) meet<0>();
                if constexpr (j % (N / kReads < 1 ? 1 : N / kReads) == 0) {       // (T = 4: reads behind even products, loads behind odd ones)
                    read(stage, (S + 1) & 3, set ^ 1, j * kReads / N);
                    if constexpr (S == 3) read_exps(stage, j * kReads / N);
                }
                constexpr int load = due(j, kLoads, N);
                if constexpr (load >= 0 && S == 3) w.a.fetch(to, wave, load);
                if constexpr (load >= 0 && S == 0) w.b.fetch(to + kOperand, wave, load);
                if constexpr (S == 0 && j == N - 1) w.exps.fetch(to);
                __builtin_amdgcn_sched_barrier(0);
            });
            if constexpr (S == 3) take_exps();
        };
        meet<0>();                                                 // the first chunk has arrived, and the sums of the tile before have left the LDS
        start(w, 1);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) w.a.fetch(lds0 + (kStage - now), wave, i);
#pragma unroll
        for (int i = 0; i < 2 * T; ++i) read(lds + now, 0, 0, i), read_exps(lds + now, i);
        take_exps();
        for (uint32_t step = 0; step < w.steps; ++step) {
            const uint32_t next = kStage - now;
            deep64(std::integral_constant<int, 0>(), lds + now, lds0 + next);
            deep64(std::integral_constant<int, 1>(), lds + now, 0);
            deep64(std::integral_constant<int, 2>(), lds + now, 0);
            start(w, step + 2);
            deep64(std::integral_constant<int, 3>(), lds + next, lds0 + now);
            now = next;
        }
        meet<0>();                                                 // nothing is read or fetched any more: one place takes the next tile's first chunk, the other one the sums, 32 rows of each wave at a time
        const uint32_t split = w.split, row0 = w.row0 + wave_row * (kSide / 2), col0 = w.col0 + wave_col * (kSide / 2);
        if constexpr (T == 4) {                                    // (two workgroups to a CU fill each other's pauses)
            id += gridDim.x;
            if (id < total) {
                w = work_of(id);
                first_chunk(w, now);
            }
        } else {
            id = total;
        }
        finish_wave<OP, DTYPE, T, true>(p, acc, reinterpret_cast<float *>(lds + (kStage - now)) + wave * 32 * kRowFloats<T>, row0, col0, 0, lane, split);
        if (id >= total) break;
    }
}

}  // namespace

hipError_t launch_mx4_tiles(Op op, uint32_t dtype, const Product &p, uint32_t side, hipStream_t st) {
    const uint32_t tiles = ((p.rows + side - 1) / side) * ((p.cols + side - 1) / side) * p.splits, grid = side == 256 ? std::min(tiles, kResident) : tiles;
    auto typed = [&](auto o, auto t) {
        constexpr int OP = decltype(o)::value;
        constexpr uint32_t DTYPE = decltype(t)::value;
        if (side == 256) k_mx4_tiles<OP, DTYPE, 4><<<grid, kThreads, 0, st>>>(p);
        else k_mx4_tiles<OP, DTYPE, 2><<<grid, kThreads, 0, st>>>(p);
    };
    auto with = [&](auto o) {
        if (dtype == EDEN_F32) typed(o, std::integral_constant<uint32_t, EDEN_F32>());
        else if (dtype == EDEN_F16) typed(o, std::integral_constant<uint32_t, EDEN_F16>());
        else typed(o, std::integral_constant<uint32_t, EDEN_BF16>());
    };
    if (op == kForward) with(std::integral_constant<int, kForward>());
    else if (op == kInputGrad) with(std::integral_constant<int, kInputGrad>());
    else typed(std::integral_constant<int, kWeightGrad>(), std::integral_constant<uint32_t, EDEN_BF16>());
    return hipGetLastError();
}

}  // namespace eden_layers
