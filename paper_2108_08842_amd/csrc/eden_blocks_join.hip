// Dropout, and the join of a residual block's branches with the norm of the next block: r = x_scale x + scale gate dropout(post(f)), h = pre(r).
//
// Bound by memory: x and f are read once, r and h written once.  LANES threads share a row and keep it in registers, eight neighbouring columns (16 bytes of a
// two-byte type) at a time, so the statistics of both norms take no second pass over memory: a sum over the row is a few lane
// exchanges, for rows of several waves one barrier.  The mean square of a layer norm is taken around the mean, which is known by then: no digits cancel.
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
    store_eight<DTYPE>(y + (size_t)at.row * ldy, at.col, to, valid);
}

// Takes the mean (layer) and the size out of a row.  Behind the row's end its values are zeros, and stay so.
template <int LANES, int CHUNKS>
__device__ inline void standardise(float (&v)[CHUNKS][8], const eden_norm &norm, uint32_t cols, const int (&valid)[CHUNKS], float *shared, int &turn) {
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
            for (int i = 0; i < 8; ++i) v[c][i] = i < valid[c] ? v[c][i] - mean : 0.0f;
    }
    float sum[1] = {0.0f};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[0] = __builtin_fmaf(v[c][i], v[c][i], sum[0]);
    sum_in_row<LANES>(sum, shared, turn);
    const float scale = rsqrtf(sum[0] * each + norm.eps);
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= scale;
}
template <uint32_t DTYPE> __device__ inline void weigh(float (&v)[8], const eden_norm &norm, uint32_t col, int valid) {
    Eight<DTYPE> w;
    if (norm.weight) {
        w.load(norm.weight, col, valid);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    if (norm.bias) {
        w.load(norm.bias, col, valid);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
}

template <uint32_t DTYPE, int LANES, int CHUNKS> __global__ __launch_bounds__(LANES > 256 ? LANES : 256) void k_block_join(const eden_join_args a) {
    constexpr int kThreads = LANES > 64 ? LANES : 256, kRows = kThreads / LANES;          // (rows of up to a wave: their waves do not meet)
    __shared__ float shared[kSumFloats<LANES>];
    int turn = 0;
    const uint32_t rows = (uint32_t)a.rows, cols = (uint32_t)a.cols, lane = threadIdx.x % LANES, step = gridDim.x * kRows;
    const uint64_t key = a.random.threshold ? key_of(a.random, eden::kStreamDropout) : 0;
    const uint32_t gate_rows = a.gates > 1 ? rows / (uint32_t)a.gates : rows;
    for (uint64_t first = (uint64_t)blockIdx.x * kRows; first < rows; first += step) {
        const uint32_t row = (uint32_t)first + threadIdx.x / LANES;
        int valid[CHUNKS];
        float r[CHUNKS][8], f[CHUNKS][8];
        Eight<DTYPE> x8[CHUNKS], f8[CHUNKS];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const uint32_t col = (c * LANES + lane) * 8;
            valid[c] = row < rows && col < cols ? (int)min(8u, cols - col) : 0;
            x8[c].load(row_of<DTYPE>(a.x, row, a.ldx), col, valid[c]);
            if (a.f) f8[c].load(row_of<DTYPE>(a.f, row, a.ldf), col, valid[c]);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) r[c][i] = x8[c][i];
        if (a.f) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[c][i] = f8[c][i];
            if (a.post.kind != EDEN_NORM_NONE) {
                standardise<LANES>(f, a.post, cols, valid, shared, turn);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) weigh<DTYPE>(f[c], a.post, (c * LANES + lane) * 8, valid[c]);
            }
            if (a.gate) {
                const void *gate = row_of<DTYPE>(a.gate, row < rows ? row / gate_rows : 0, a.ld_gate);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    Eight<DTYPE> g;
                    g.load(gate, (c * LANES + lane) * 8, valid[c]);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[c][i] *= g[i];
                }
            }
            const float scale = a.scale * kept_scale(a.random.threshold);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t col = (c * LANES + lane) * 8;
                if (a.random.threshold) {
                    const Bits8 bits = bits_of(key, row * words_of(cols) + col / 4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[c][i] = bits.of(i) >= a.random.threshold ? f[c][i] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) r[c][i] = __builtin_fmaf(scale, f[c][i], a.x_scale * r[c][i]);
                if (a.r && valid[c]) store_eight<DTYPE>(row_of<DTYPE>(a.r, row, a.ldr), col, r[c], valid[c]);
            }
        }
        if (a.pre.kind != EDEN_NORM_NONE) {
            standardise<LANES>(r, a.pre, cols, valid, shared, turn);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t col = (c * LANES + lane) * 8;
                weigh<DTYPE>(r[c], a.pre, col, valid[c]);
                if (valid[c]) store_eight<DTYPE>(row_of<DTYPE>(a.h, row, a.ldh), col, r[c], valid[c]);
            }
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
        for_shape(row_shape((uint32_t)args.cols), [&](auto lanes, auto chunks) {
            constexpr int LANES = decltype(lanes)::value, kThreads = LANES > 64 ? LANES : 256, kRows = kThreads / LANES;
            const uint64_t groups = std::min<uint64_t>((args.rows + kRows - 1) / kRows, 1u << 16);
            k_block_join<decltype(t)::value, LANES, decltype(chunks)::value><<<(uint32_t)groups, kThreads, 0, st>>>(args);
        });
    });
    return hipGetLastError();
}

}  // namespace eden_layers
