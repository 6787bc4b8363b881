// Matrix products of the layer operators where the result fills the device and rows are whole 16-byte pieces: fp16 and bf16.
//
// A workgroup has a tile of 256 x 256, a wave 128 x 128 of it: 256 accumulation registers, and of every byte that
// goes from the LDS to the matrix cores 128 products, twice as many as in the general kernel.  A CU holds one such workgroup, a SIMD one wave, so the
// wave itself keeps the matrix core fed.  It takes one product in 32 cycles, the wave issues an instruction in four, and one that its unit does not
// accept at once holds up the products behind it: everything else goes between the products, a little at a time.
//   memory -> LDS      an operand's tile is fetched 64 deep (whole 128-byte lines of its rows), straight into the LDS, which holds five such tiles: the two in
//                      use, the following two, and the first of the two after that.  A tile's eight loads a wave are spread over 32 products.
//   LDS -> registers   the operands of the next 16 deep are read while those of the last are multiplied
//   barriers           one in 64 deep, between the last reads of two tiles and their last products
// 16-byte pieces of a row are swapped on the way into the LDS (each lane fetches the piece that belongs to its place).  A checkpoint's codes cannot go
// straight into the LDS: they are read into registers 64 deep ahead, turned into bf16 numbers and stored while the products run.
//
// Where 256 x 256 would leave CUs idle, tiles of 128 x 128 with waves of 64 x 64, two workgroups to a CU.
//
// The product alone is bound by the card's power: bf16, 8192 x 16384 with 4096 products each takes 820 to 845 us without an end (1300 to 1340 TFLOP/s; a library's product 726 to
// 808), with the matrix cores busy 73% of the cycles at a clock of 1.44 GHz (six launches under a profiler; counters_layers.txt).  Bias, gelu and checkpoint, 0.4 GB to be
// written, make it 960 to 975, a residual 1040: the one workgroup of a CU has nothing to hide its end behind, and the matrix cores are busy 60% of the cycles at 1.6 GHz.
// Input gradient of these sizes with gelu's slope 950 to 970 (59%, 1.67 GHz).  Weight gradient 4096 x 8192 from a checkpoint, 8192 deep, 475 to 495 (1110 to 1160 TFLOP/s): the vector unit, which decodes the
// codes, and the waits for them leave the matrix cores 54% of the cycles at 1.7 to 1.85 GHz.  Tiles of 128: 1021 x 5000, 2048 deep, fp16 33 us (640 TFLOP/s).
// Not faster: nine tiles in the LDS in place of five for tiles of 128 (four steps ahead; a CU's loads bound them, 0.4 to 0.5 us for 64 deep), a second set of
// registers for the codes, tiles of 256 x 128, loads 32 deep (half a line each: twice the requests).
#include "eden_layers_fetch.h"

namespace eden_layers {
namespace {

constexpr int kThreads = 256, kDeep = 64, kSlots = 5;
// T: a wave has T x T products of 32 x 32
template <int T> struct Tile {
    static constexpr int kSide = 64 * T;
    static constexpr int kOperand = kSide * kDeep * 2;             // bytes of an operand's tile, a slot of the LDS
    static constexpr int kLoads = kOperand / 16 / kThreads;        // 16-byte pieces per thread
    static constexpr int kPieces = kSide / 8;                      // of a row of columns
};
// Where a thread's pieces of an operand come from: byte offsets from the tile's first element.
template <int T, bool STRIDED> struct Source {
    static constexpr int kSide = Tile<T>::kSide, kPieces = Tile<T>::kPieces;
    const char *base;
    size_t step;               // bytes from one tile to the next
    uint64_t reach;            // bytes from `base` to the end of what may be read
    uint32_t offset, stride;   // of piece i: offset + i * stride
    uint32_t depth;            // !STRIDED: depth of this lane's pieces inside a tile
    u32x4 now;                 // of the tile that is being fetched: descriptor, this lane's first offset
    uint32_t at;

    // rows or columns first .. count - 1 of the operand, depths begin .. end - 1; `whole`: elements of a row of memory that may be read
    __device__ Source(const void *p, size_t ld, uint32_t first, uint32_t count, uint32_t begin, uint32_t end, uint32_t whole, int wave, int lane) {
        if constexpr (STRIDED) {
            base = static_cast<const char *>(p) + ((size_t)begin * ld + first) * 2;
            step = (size_t)kDeep * ld * 2;
            reach = ((uint64_t)(end - begin - 1) * ld + (whole - first)) * 2;
            const uint32_t d = (wave * 64 + lane) / kPieces, piece = (lane % kPieces) ^ (4 * (d & 3));
            offset = (uint32_t)(d * ld * 2) + piece * 16;
            stride = (uint32_t)(kThreads / kPieces * ld * 2);
            depth = 0;
        } else {
            const uint32_t rows = min((uint32_t)kSide, count - first);
            base = static_cast<const char *>(p) + ((size_t)first * ld + begin) * 2;
            step = kDeep * 2;
            reach = ((uint64_t)(rows - 1) * ld + (whole - begin)) * 2;
            const uint32_t row = wave * 8 + (lane >> 3), piece = (lane & 7) ^ ((row >> 1) & 7);
            offset = (uint32_t)(row * ld * 2) + piece * 16;
            stride = (uint32_t)(32 * ld * 2);
            depth = piece * 8;
        }
    }
    // The next tile is `left` deep.  What lies beyond is read as zeros.
    __device__ void start(uint32_t left) {
        now = descriptor(base, reach);
        at = (STRIDED ? 0u < left : depth < left) ? offset : kNowhere;      // (and further on)
        base += step;
        reach = reach > step ? reach - step : 0;
    }
    // Load i of the tile, into the LDS at `slot`.
    __device__ void fetch(uint32_t slot, int wave, int i) const {
        load_to_lds(slot + (i * 4 + wave) * 1024, at + i * stride, now);
    }
};

// A checkpoint's codes: neighbouring lanes have the pieces of one depth (8 codes each), a thread kLoads depths of a tile.  What lies
// beyond the depths of the split is read as zeros (codes 0, unit 0).
template <int T> struct Codes {
    static constexpr int kSide = Tile<T>::kSide, kLoads = Tile<T>::kLoads, kPieces = Tile<T>::kPieces, kDepths = kThreads / kPieces;
    const uint8_t *codes, *exps;
    uint64_t codes_reach, exps_reach;
    size_t ld;
    uint32_t blocks, at, exp_at;
    rsrc_t codes_now, exps_now;
    u32x2 q[kLoads];
    uint32_t t[kLoads];

    __device__ Codes(const Product &p, uint32_t col0, uint32_t begin, uint32_t end, int tid)
        : codes(static_cast<const uint8_t *>(p.b) + (size_t)begin * p.ldb + col0), exps(p.b_exps + (size_t)begin * p.b_blocks + col0 / kBlock),
          codes_reach((uint64_t)(end - begin) * p.ldb - col0), exps_reach((uint64_t)(end - begin) * p.b_blocks - col0 / kBlock), ld(p.ldb), blocks(p.b_blocks),
          at((tid / kPieces) * (uint32_t)p.ldb + tid % kPieces * 8), exp_at((tid / kPieces) * p.b_blocks + tid % kPieces / 4) {}
    __device__ void start() {
        codes_now = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(codes), 0, (int)(codes_reach < kMostBytes ? (uint32_t)codes_reach : kMostBytes), 0x00020000);
        exps_now = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(exps), 0, (int)(exps_reach < kMostBytes ? (uint32_t)exps_reach : kMostBytes), 0x00020000);
        codes += kDeep * ld;
        exps += (size_t)kDeep * blocks;
        codes_reach = codes_reach > kDeep * ld ? codes_reach - kDeep * ld : 0;
        exps_reach = exps_reach > (uint64_t)kDeep * blocks ? exps_reach - (uint64_t)kDeep * blocks : 0;
    }
    __device__ void load(int i) {
        q[i] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(codes_now, (int)(at + i * kDepths * (uint32_t)ld), 0, 0));
        t[i] = __builtin_amdgcn_raw_buffer_load_b8(exps_now, (int)(exp_at + i * kDepths * blocks), 0, 0);
    }
    // Values 2 h and 2 h + 1 of piece i; the whole piece into the LDS
    __device__ uint32_t two(int i, int h) const {
        const float unit = block_unit(t[i]);
        const uint32_t c = q[i][h >> 1] >> (16 * (h & 1));
        return upper_halves((float)(int8_t)(c & 0xFFu) * unit, (float)(int8_t)((c >> 8) & 0xFFu) * unit);
    }
    __device__ void store(char *tile, int tid, int i, u32x4 words) const {
        *reinterpret_cast<u32x4 *>(tile + piece_of_depth<kSide>(i * kDepths + tid / kPieces, tid % kPieces)) = words;
    }
};

// Where a lane reads an operand's tile in the LDS.  The swaps leave four different places; tiles of 32 (whole rows apart) or steps of 16 deep (whole
// depths apart) are constant distances from them.
template <int T, bool STRIDED> struct Reader {
    static constexpr int kSide = Tile<T>::kSide;
    uint32_t at[STRIDED ? T : 4];

    __device__ Reader(int base, int lane, int swap = 0) {          // STRIDED: tile i is number i ^ swap from `base` on
#pragma unroll
        for (int i = 0; i < (STRIDED ? T : 4); ++i) {
            if constexpr (STRIDED) {                               // of tile i
                const int col = base + (i ^ swap) * 32 + (lane & 16) + (lane & 3) * 4;
                at[i] = piece_of_depth<kSide>((lane >> 5) * 8 + ((lane & 15) >> 2), col >> 3) + (col & 7) * 2;
            } else {                                               // of step i
                at[i] = piece_of_row<kDeep>(base + (lane & 31), 2 * i + (lane >> 5));
            }
        }
    }
    __device__ u32x4 read(const char *slot, int tile, int step) const {
        if constexpr (STRIDED) {
            const char *from = slot + at[tile] + step * (16 * kSide * 2);
            union { s16x4 h[2]; u32x4 w; } r;
            r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)from);
            r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + 4 * kSide * 2));
            return r.w;
        } else {
            return *reinterpret_cast<const u32x4 *>(slot + at[step] + tile * (32 * kDeep * 2));
        }
    }
};

template <int OP, uint32_t DTYPE, int T> __global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(T == 4 ? 1 : 2, T == 4 ? 1 : 2))) void k_direct(const Product p) {
    constexpr int kSide = Tile<T>::kSide, kOperand = Tile<T>::kOperand, kLoads = Tile<T>::kLoads, N = T * T;
    constexpr bool kStridedA = OP == kWeightGrad, kStridedB = OP != kForward, kHalf = DTYPE == EDEN_F16, kCodes = OP == kWeightGrad;
    static_assert(!(kCodes && kHalf), "fp16 next to a checkpoint has two terms");
    __shared__ __attribute__((aligned(1024))) char lds[kSlots * kOperand];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wave_row = wave >> 1, wave_col = wave & 1;
    const uint32_t row_tiles = (p.rows + kSide - 1) / kSide, col_tiles = (p.cols + kSide - 1) / kSide;
    uint32_t split, row_tile, col_tile;
    place_of(blockIdx.x, gridDim.x, row_tiles, col_tiles, split, row_tile, col_tile);
    const uint32_t row0 = row_tile * kSide, col0 = col_tile * kSide;
    const uint32_t begin = split * p.split_depth, end = min(p.depth, begin + p.split_depth);
    const uint32_t steps = (end - begin + kDeep - 1) / kDeep;      // begin < end: launched for depths above 0 only

    Source<T, kStridedA> a(p.a, p.lda, row0, p.rows, begin, end, p.a_width, wave, lane);
    Source<T, kStridedB> b(p.b, kCodes ? 0 : p.ldb, col0, kCodes ? col0 + 1 : p.cols, begin, end, kCodes ? col0 + 1 : p.b_width, wave, lane);
    const int swap = kCodes ? wave_col * (T / 2) : 0;
    const Reader<T, kStridedA> reader_a(wave_row * (kSide / 2), lane, swap);
    const Reader<T, kStridedB> reader_b(wave_col * (kSide / 2), lane);
    Codes<T> codes(p, col0, begin, end, tid);

    f32x16 acc[T][T] = {};
    float sums[T / 2] = {};                                        // row sums of this lane's depths, of the first half of the tiles: the two waves
                                                                   // of a row of waves begin with different halves
    const bool with_sums = kCodes && p.row_sums && col_tile == 0;
    u32x4 fa[2][T], fb[2][T];

    const uint32_t lds0 = (uint32_t)(size_t)(lds_char *)lds;
    auto depth_left = [&](uint32_t step) { return end - begin > step * kDeep ? end - begin - step * kDeep : 0u; };
    auto read = [&](const char *slot_a, const char *slot_b, int s, int set, int i) {              // one operand of 2 T
        if (i < T) fb[set][i] = reader_b.read(slot_b, i, s);
        else fa[set][i - T] = reader_a.read(slot_a, i - T, s);
    };
    // T x T products 16 deep: S = 0 .. 3 of a tile's 64.  The operands of the following ones are read, for S = 3 those of the next tiles, behind a
    // barrier since when nobody needs the present ones.  Into their places go the second operand's tile after the next (S = 3 and the next 0)
    // and the first operand's after that (the next S = 1, 2).
    auto deep16 = [&](auto step16, const char *slot_a, const char *slot_b, uint32_t fetch_to, char *codes_to) {
        constexpr int S = decltype(step16)::value, set = S & 1, kReads = 2 * T, kHalf2 = kLoads / 2;
        u32x4 words;
        each<N>([&](auto number) {
            constexpr int j = decltype(number)::value, i = j / T;
            acc[i][j % T] = multiply<kHalf>(fb[set][j % T], fa[set][i], acc[i][j % T]);
            if constexpr (S == 3 && j == 0) meet<kCodes ? 3 * kLoads : kLoads>();     // (later: the first operand's tile after the next; codes)
            // 2 T reads, kLoads / 2 loads, kLoads / 4 pieces of codes in N = T T products: T = 4: every second, fourth, eighth; T = 2: one each, two, four
            if constexpr ((j + 1) * kReads / N != j * kReads / N) read(slot_a, slot_b, (S + 1) & 3, set ^ 1, j * kReads / N);
            if constexpr (((2 * j + 1) * kHalf2 / N) % 2 == 1 && ((2 * j - 1) * kHalf2 / N) % 2 == 0) {
                constexpr int load = j * kHalf2 / N;
                if constexpr (S == 1 || S == 2) a.fetch(fetch_to, wave, (S - 1) * kHalf2 + load);
                else if constexpr (!kCodes) b.fetch(fetch_to, wave, (S == 3 ? 0 : kHalf2) + load);
            }
            if constexpr (kCodes) {
                constexpr int words_each = kLoads, w = j * words_each / N, piece = ((S + 1) & 3) * (kLoads / 4) + w / 4;         // from S = 3 on
                if constexpr (j == 0 || (j - 1) * words_each / N != w) {
                    words[w % 4] = codes.two(piece, w % 4);
                    if constexpr (w % 4 == 3) {
                        codes.store(codes_to, tid, piece, words);
                        codes.load(piece);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (kCodes)
            if (with_sums) {                                       // row sums: two additions an instruction
                const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
                for (int q = 0; q < T / 2 * 4; ++q) {
                    const uint32_t pair = fa[set][q / 4][q % 4];   // (a cast of the vector's element itself would take its first)
                    sums[q / 4] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), ones, sums[q / 4], false);
                }
            }
    };
    // Tile number c (first operand of step s: 2 s, second: 2 s + 1) goes to slot c mod 5.
    auto on = [](uint32_t slot, uint32_t tiles) {
        const uint32_t to = slot + tiles * kOperand;
        return to >= (uint32_t)(kSlots * kOperand) ? to - kSlots * kOperand : to;
    };
    uint32_t slot = 0;                                             // of the first operand of the present step
    if constexpr (kCodes) {
        codes.start();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) codes.load(i);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) codes.store(lds + kOperand, tid, i, u32x4{codes.two(i, 0), codes.two(i, 1), codes.two(i, 2), codes.two(i, 3)});
        codes.start();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) codes.load(i);
        codes.start();
#pragma unroll
        for (int i = 0; i < kLoads / 4; ++i) {                     // what S = 3 does
            codes.store(lds + 3 * kOperand, tid, i, u32x4{codes.two(i, 0), codes.two(i, 1), codes.two(i, 2), codes.two(i, 3)});
            codes.load(i);
        }
    }
    a.start(depth_left(0));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) a.fetch(lds0, wave, i);
    if constexpr (!kCodes) {
        b.start(depth_left(0));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) b.fetch(lds0 + kOperand, wave, i);
    }
    a.start(depth_left(1));
#pragma unroll
    for (int i = 0; i < kLoads; ++i) a.fetch(lds0 + 2 * kOperand, wave, i);
    if constexpr (!kCodes) {
        b.start(depth_left(1));
#pragma unroll
        for (int i = 0; i < kLoads / 2; ++i) b.fetch(lds0 + 3 * kOperand, wave, i);
    }
    meet<0>();
#pragma unroll
    for (int i = 0; i < 2 * T; ++i) read(lds, lds + kOperand, 0, 0, i);
    for (uint32_t step = 0; step < steps; ++step) {
        const uint32_t slot_b = on(slot, 1), next_a = on(slot, 2), next_b = on(slot, 3), after_a = on(slot, 4);
        deep16(std::integral_constant<int, 0>(), lds + slot, lds + slot_b, lds0 + next_b, lds + next_b);
        a.start(depth_left(step + 2));
        deep16(std::integral_constant<int, 1>(), lds + slot, lds + slot_b, lds0 + after_a, lds + next_b);
        deep16(std::integral_constant<int, 2>(), lds + slot, lds + slot_b, lds0 + after_a, lds + next_b);
        if constexpr (kCodes) codes.start();
        else b.start(depth_left(step + 2));
        deep16(std::integral_constant<int, 3>(), lds + next_a, lds + next_b, lds0 + slot, lds + slot);
        slot = next_a;
    }

    if constexpr (kCodes) {
#pragma unroll
        for (int i = 0; i < T / 2; ++i) {
            sums[i] += __shfl_xor(sums[i], 32);
            if (with_sums && lane < 32) finish_row_sum(p, sums[i], row0 + wave_row * (kSide / 2) + (i ^ swap) * 32 + lane, split);
        }
    }
    meet<0>();                                                     // nothing is read or fetched any more: the LDS takes the sums, 32 rows of each wave at a time
    finish_wave<OP, DTYPE, T>(p, acc, reinterpret_cast<float *>(lds) + wave * 32 * kRowFloats<T>, row0 + wave_row * (kSide / 2), col0 + wave_col * (kSide / 2), swap, lane, split);
}

}  // namespace

hipError_t launch_direct(Op op, uint32_t dtype, const Product &p, uint32_t side, hipStream_t st) {
    const uint32_t grid = ((p.rows + side - 1) / side) * ((p.cols + side - 1) / side) * p.splits;
    auto typed = [&](auto t) {
        constexpr int T = decltype(t)::value;
        if (op == kWeightGrad) k_direct<kWeightGrad, EDEN_BF16, T><<<grid, kThreads, 0, st>>>(p);
        else if (op == kForward && dtype == EDEN_F16) k_direct<kForward, EDEN_F16, T><<<grid, kThreads, 0, st>>>(p);
        else if (op == kForward) k_direct<kForward, EDEN_BF16, T><<<grid, kThreads, 0, st>>>(p);
        else if (dtype == EDEN_F16) k_direct<kInputGrad, EDEN_F16, T><<<grid, kThreads, 0, st>>>(p);
        else k_direct<kInputGrad, EDEN_BF16, T><<<grid, kThreads, 0, st>>>(p);
    };
    if (side == 256) typed(std::integral_constant<int, 4>());
    else typed(std::integral_constant<int, 2>());
    return hipGetLastError();
}

}  // namespace eden_layers
