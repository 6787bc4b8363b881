// Dropout, and the join of a residual block's branches with the norm of the next block: r = x_scale x + scale gate dropout(post(f)), h = pre(r).
//
// Bound by memory: x and f are read once, r and h written once.  LANES threads share a row and keep it in registers, eight neighbouring columns (16 bytes of a
// two-byte type) at a time, so the statistics of both norms take no second pass over memory: a sum over the row is a few lane
// exchanges, for rows of several waves one barrier.  The mean square of a layer norm is taken around the mean, which is known by then: no digits cancel.
//
// bf16: 8192 x 4096 with dropout, gate and both norms rms 44 to 47 us (268 MB at 5.7 to 6.1 TB/s, vector instructions in 68% of the cycles), a norm alone 22 (6.1 TB/s), 4096 x 16384 115 and 42; a single token 3,
// a launch and two trips to memory.  Dropout of 8192 x 8192 45 (6.0 TB/s, vector 59%).  A copy of 1 GiB moves 5.1 TB/s: results of two bytes are stored past the caches, in which they would
// displace operands (8192 x 16384 dropout 128 -> 100 us).  fp32 results are not: a lane's 32 bytes leave in two stores, so each would write part of a line.
// fp32: 8192 x 4096 rms 105 us, layer 111 (537 MB at 4.8 to 5.1 TB/s), a norm alone 41 (6.5 TB/s), dropout of 8192 x 8192 126 (4.3 TB/s; a floor of 105).
#include "eden_blocks_kernels.h"
#include "eden_layers_spread.h"

namespace eden_layers {
namespace {

template <uint32_t DTYPE>
__global__ __launch_bounds__(kSpreadThreads) void k_dropout(const typename Elem<DTYPE>::type *x, size_t ldx, typename Elem<DTYPE>::type *y, size_t ldy, uint32_t rows, uint32_t cols,
                                                            eden_random random, uint32_t shift, uint32_t segments, uint32_t before) {
    const Place at = place(shift, segments, before);
    if (at.row >= rows || at.col >= cols) return;
    const int valid = valid_of(at.col, cols);
    Eight<DTYPE> v;
    v.load(x + (size_t)at.row * ldx, at.col, valid);
    const Bits8 bits = bits_of(key_of(random, eden::kStreamDropout), at.row * words_of(cols) + at.col / 4);
    const float scale = kept_scale(random.threshold);
    float to[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) to[i] = bits.of(i) >= random.threshold ? v[i] * scale : 0.0f;
    store_eight<DTYPE, true>(y + (size_t)at.row * ldy, at.col, to, valid);
}

// Takes the mean (layer) and the size out of a row.  Behind the row's end its values are zeros, and stay so.
template <int LANES, int CHUNKS, class P>
__device__ inline void standardise(float (&v)[CHUNKS][8], const eden_norm &norm, uint32_t cols, const P &place, float *shared, int &turn) {
    const float each = 1.0f / (float)cols;
    if (norm.kind == EDEN_NORM_LAYER) {
        float sum[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v[c][i];
        sum_in_row<LANES>(sum, shared, turn);
        const float mean = sum[0] * each;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[c][i] = place.inside(c, i) ? v[c][i] - mean : 0.0f;
    }
    float sum[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(v[c][i], v[c][i], sum[0]);
    sum_in_row<LANES>(sum, shared, turn);
    const float scale = rho_of<LANES>(sum[0], each, norm.eps, shared, turn, [&](float by) {
        float s = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v[c][i] * by, v[c][i] * by, s);
        return s;
    });
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= scale;
}

// A norm's weights and biases in the lane's columns
template <uint32_t DTYPE, int CHUNKS> struct Weights {
    Eight<DTYPE> weight[CHUNKS], bias[CHUNKS];
    template <class P> __device__ void load(const eden_norm &norm, const P &place) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (norm.weight) place.load(weight[c], norm.weight, c);
            if (norm.bias) place.load(bias[c], norm.bias, c);
        }
    }
    template <class P> __device__ void apply(float (&v)[CHUNKS][8], const eden_norm &norm, const P &place) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if (norm.weight) {
                place.settle(weight[c], c, true);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] *= weight[c][i];
            }
            if (norm.bias) {
                place.settle(bias[c], c, true);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] += bias[c][i];
            }
        }
    }
};

// Waves of a SIMD: rows of up to a wave's eights need few registers, and nothing but other waves hides their loads.  (Two chunks a lane: half as many, or the compiler puts operands into memory.)
template <uint32_t DTYPE> constexpr int waves_of(int lanes, int chunks, bool branch) {
    return lanes == 1024 ? 4 : (DTYPE == EDEN_F32 ? 4 : branch ? 6 : 8) / (chunks == 2 ? 2 : 1);
}

template <uint32_t DTYPE, int LANES, int CHUNKS, bool RAGGED, bool BRANCH>
__global__ __launch_bounds__(LANES > 64 ? LANES : 256) __attribute__((amdgpu_waves_per_eu(waves_of<DTYPE>(LANES, CHUNKS, BRANCH)))) void k_block_join(const eden_join_args a) {
    constexpr int kThreads = LANES > 64 ? LANES : 256, kRows = kThreads / LANES;          // (rows of up to a wave: their waves do not meet)
    __shared__ float shared[kSumFloats<LANES>];
    int turn = 0;
    const uint32_t rows = (uint32_t)a.rows, cols = (uint32_t)a.cols, step = gridDim.x * kRows, sub = row_in_group<LANES>();
    const RowPlace<DTYPE, LANES, CHUNKS, RAGGED> place(cols, threadIdx.x % LANES);
    const uint64_t key = BRANCH && a.random.threshold ? key_of(a.random, eden::kStreamDropout) : 0;
    const uint32_t gate_rows = a.gates > 1 ? rows / (uint32_t)a.gates : rows;
    const float scale = a.scale * kept_scale(a.random.threshold);
    const bool post = a.post.kind != EDEN_NORM_NONE, pre = a.pre.kind != EDEN_NORM_NONE;
    for (uint64_t first = (uint64_t)blockIdx.x * kRows; first < rows; first += step) {
        const bool has = first + sub < rows;
        const uint32_t row = (uint32_t)(has ? first + sub : first);
        float r[CHUNKS][8];
        Eight<DTYPE> x8[CHUNKS], f8[CHUNKS], gate8[CHUNKS];
        Weights<DTYPE, CHUNKS> weights;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            if constexpr (BRANCH) place.load(f8[c], row_of<DTYPE, LANES>(a.f, row, a.ldf), c);
            place.load(x8[c], row_of<DTYPE, LANES>(a.x, row, a.ldx), c);
        }
        if constexpr (!BRANCH) {
            weights.load(a.pre, place);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                place.settle(x8[c], c, has);
#pragma unroll
                for (int i = 0; i < 8; ++i) r[c][i] = x8[c][i];
            }
        } else {
            float f[CHUNKS][8];
            if (post) weights.load(a.post, place);
            if (a.gate) {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) place.load(gate8[c], row_of<DTYPE, LANES>(a.gate, row / gate_rows, a.ld_gate), c);
            }
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                place.settle(f8[c], c, has);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[c][i] = f8[c][i];
            }
            if (post) {
                standardise<LANES, CHUNKS>(f, a.post, cols, place, shared, turn);
                weights.apply(f, a.post, place);
            }
            if (pre) weights.load(a.pre, place);                   // (on their way during what follows)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (a.random.threshold) {
                    const Bits8 bits = bits_of(key, row * words_of(cols) + place.col[c] / 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[c][i] = bits.of(i) >= a.random.threshold ? f[c][i] : 0.0f;
                }
                if (a.gate) {
                    place.settle(gate8[c], c, has);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[c][i] *= gate8[c][i];
                }
                place.settle(x8[c], c, has);
#pragma unroll
                for (int i = 0; i < 8; ++i) r[c][i] = __builtin_fmaf(scale, f[c][i], a.x_scale * x8[c][i]);
                if (a.r && has) place.template store<true>(row_of<DTYPE, LANES>(a.r, row, a.ldr), c, r[c]);
            }
        }
        if (!BRANCH || pre) {
            standardise<LANES, CHUNKS>(r, a.pre, cols, place, shared, turn);
            weights.apply(r, a.pre, place);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
                if (has) place.template store<true>(row_of<DTYPE, LANES>(a.h, row, a.ldh), c, r[c]);
        }
    }
}

}  // namespace

hipError_t launch_dropout(uint32_t dtype, const void *x, size_t ldx, void *y, size_t ldy, uint32_t rows, uint32_t cols, const eden_random &random, hipStream_t st) {
    const Spread s = spread(rows, cols);
    return launches(s, [&](uint32_t before, uint32_t groups) {
        for_type(dtype, [&](auto t) {
            using T = typename Elem<decltype(t)::value>::type;
            k_dropout<decltype(t)::value><<<groups, kSpreadThreads, 0, st>>>(static_cast<const T *>(x), ldx, static_cast<T *>(y), ldy, rows, cols, random, s.shift, s.segments, before);
        });
    });
}

hipError_t launch_block_join(const eden_join_args &args, hipStream_t st) {
    for_type(args.dtype, [&](auto t) {
        JoinShape((uint32_t)args.cols).use((uint32_t)args.cols, [&](auto lanes, auto chunks, auto ragged) {
            constexpr uint32_t DTYPE = decltype(t)::value;
            constexpr int LANES = decltype(lanes)::value, CHUNKS = decltype(chunks)::value, kThreads = LANES > 64 ? LANES : 256, kRows = kThreads / LANES;
            constexpr bool RAGGED = decltype(ragged)::value;
            const uint32_t groups = (uint32_t)std::min<uint64_t>((args.rows + kRows - 1) / kRows, 1u << 16);
            if (args.f) k_block_join<DTYPE, LANES, CHUNKS, RAGGED, true><<<groups, kThreads, 0, st>>>(args);
            else k_block_join<DTYPE, LANES, CHUNKS, RAGGED, false><<<groups, kThreads, 0, st>>>(args);
        });
    });
    return hipGetLastError();
}

}  // namespace eden_layers
