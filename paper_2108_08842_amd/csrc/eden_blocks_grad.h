// The gradients of a residual block's join (included by one source for each type).
//
//   d = dr + rho_r (g - [mean g] - n mean(g n)), g = dh w_pre, n = (r - [mean r]) rho_r               brackets: layer norms
//   dx = x_scale d
//   u = w_post n_f + b_post,  v = u 65536 / (65536 - t) where kept, else 0                             gate_grad = sum of scale d v over its rows
//   du = scale gate d 65536 / (65536 - t) where kept, else 0;  df = rho_f (du w_post - [mean] - n_f mean(du w_post n_f))
//   weights' and biases' gradients: sums over the rows of dh n, dh, du n_f, du
//
// Bound by memory: dr, dh, r, f are read once, dx, df written once; statistics are taken again from r and f, which costs a sum over a row that is in
// registers and keeps no memory.  The sums over rows stay in registers of the workgroups, each of which goes through many rows; a second launch adds what they
// have.  No atomics: the same bits every time.
#include "eden_blocks_kernels.h"

namespace eden_layers {
namespace {

constexpr int bit(int sum) { return 1 << sum; }

template <uint32_t DTYPE, int LANES, int CHUNKS, int SUMS>
__global__ __launch_bounds__(LANES > 64 ? LANES : 64) void k_block_grad(const GradArgs args) {
    constexpr int kThreads = LANES > 64 ? LANES : 64, kRows = kThreads / LANES;
    __shared__ float shared[kSumFloats<LANES>];
    int turn = 0;
    const eden_join_grad_args &a = args.a;
    const Share &share = args.share;
    const uint32_t cols = (uint32_t)a.cols, lane = threadIdx.x % LANES, worker = blockIdx.x;
    const uint64_t key = a.random.threshold ? key_of(a.random, eden::kStreamDropout) : 0;
    const float each = 1.0f / (float)cols, kept = kept_scale(a.random.threshold);
    const bool pre = a.dh != nullptr, post = a.post.kind != EDEN_NORM_NONE, pre_layer = a.pre.kind == EDEN_NORM_LAYER, post_layer = a.post.kind == EDEN_NORM_LAYER;

    uint32_t columns[CHUNKS];                                      // valid ones
    Eight<DTYPE> pre_weight[CHUNKS], post_weight[CHUNKS], post_bias[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const uint32_t col = (c * LANES + lane) * 8;
        columns[c] = col < cols ? min(8u, cols - col) : 0;
        if (a.pre.weight) pre_weight[c].load(a.pre.weight, col, columns[c]);
        if (a.post.weight) post_weight[c].load(a.post.weight, col, columns[c]);
        if (a.post.bias) post_bias[c].load(a.post.bias, col, columns[c]);
    }
    float sums[kAllSums][CHUNKS][8] = {};

    // one result's or one part's sums
    auto put = [&](int which, float (&v)[CHUNKS][8], float *to, bool add) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) v[c][i] += __shfl_xor(v[c][i], d);
            }
            if (threadIdx.x < LANES && columns[c]) {
                float *at = to + (c * LANES + lane) * 8;
                Vec<float, 8> out;
                if (add) out = load_some<float, 8>(at, columns[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) out.v[i] = add ? out.v[i] + v[c][i] : v[c][i];
                store_some<float, 8>(at, out, columns[c]);
            }
        }
    };

    const uint32_t first_group = share.splits > 1 ? worker / share.splits : worker * share.groups_each;
    const uint32_t end_group = share.splits > 1 ? first_group + 1 : min(share.gates, first_group + share.groups_each);
    const uint32_t split = share.splits > 1 ? worker % share.splits : 0, split_rows = (share.group_rows + share.splits - 1) / share.splits;
    for (uint32_t group = first_group; group < end_group; ++group) {
        const uint32_t from = min(split * split_rows, share.group_rows), to = min(from + split_rows, share.group_rows);
        const uint64_t group_row = (uint64_t)group * share.group_rows;
        Eight<DTYPE> gate[CHUNKS];
        if (a.gate) {
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) gate[c].load(row_of<DTYPE>(a.gate, group, a.ld_gate), (c * LANES + lane) * 8, columns[c]);
        }
        for (uint32_t at = from; at < to; at += kRows) {
            const bool has = at + threadIdx.x / LANES < to;
            const uint64_t row = group_row + at + (has ? threadIdx.x / LANES : 0);
            Eight<DTYPE> r8[CHUNKS], f8[CHUNKS], dh8[CHUNKS], dr8[CHUNKS];
            int valid[CHUNKS];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t col = (c * LANES + lane) * 8;
                valid[c] = has ? columns[c] : 0;
                if (pre) r8[c].load(row_of<DTYPE>(a.r, row, a.ldr), col, valid[c]);
                if (pre) dh8[c].load(row_of<DTYPE>(a.dh, row, a.lddh), col, valid[c]);
                if (a.dr) dr8[c].load(row_of<DTYPE>(a.dr, row, a.lddr), col, valid[c]);
                if (args.needs_f) f8[c].load(row_of<DTYPE>(a.f, row, a.ldf), col, valid[c]);
            }
            float n[CHUNKS][8], u[CHUNKS][8], d[CHUNKS][8];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[c][i] = pre ? r8[c][i] : 0.0f;
                    u[c][i] = args.needs_f ? f8[c][i] : 0.0f;
                    d[c][i] = a.dr ? dr8[c][i] : 0.0f;
                }
            float two[2];
            if (pre_layer || post_layer) {
                two[0] = two[1] = 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) two[0] += n[c][i], two[1] += u[c][i];
                sum_in_row<LANES>(two, shared, turn);
                const float mean_r = pre_layer ? two[0] * each : 0.0f, mean_f = post_layer ? two[1] * each : 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        n[c][i] = i < valid[c] ? n[c][i] - mean_r : 0.0f;
                        u[c][i] = i < valid[c] ? u[c][i] - mean_f : 0.0f;
                    }
            }
            float rho_r = 0.0f, rho_f = 0.0f;
            if (pre || post) {
                two[0] = two[1] = 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) two[0] = __builtin_fmaf(n[c][i], n[c][i], two[0]), two[1] = __builtin_fmaf(u[c][i], u[c][i], two[1]);
                sum_in_row<LANES>(two, shared, turn);
                if (has) rho_r = rsqrtf(two[0] * each + a.pre.eps), rho_f = rsqrtf(two[1] * each + a.post.eps);       // (of rows that are none, 0 times 0 and not times 1 / 0)
            }
            if (pre) {
                float g[CHUNKS][8];
                two[0] = two[1] = 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float dh = dh8[c][i];
                        n[c][i] *= rho_r;
                        if constexpr (SUMS & bit(kPreWeight)) sums[kPreWeight][c][i] = __builtin_fmaf(dh, n[c][i], sums[kPreWeight][c][i]);
                        if constexpr (SUMS & bit(kPreBias)) sums[kPreBias][c][i] += dh;
                        g[c][i] = a.pre.weight ? dh * pre_weight[c][i] : dh;
                        two[0] += g[c][i], two[1] = __builtin_fmaf(g[c][i], n[c][i], two[1]);
                    }
                sum_in_row<LANES>(two, shared, turn);
                const float c0 = pre_layer ? -rho_r * (two[0] * each) : 0.0f, c1 = -rho_r * (two[1] * each);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[c][i] += __builtin_fmaf(rho_r, g[c][i], __builtin_fmaf(c1, n[c][i], c0));
            }
            if (a.dx) {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    float to8[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) to8[i] = a.x_scale * d[c][i];
                    if (valid[c]) store_eight<DTYPE>(row_of<DTYPE>(a.dx, row, a.lddx), (c * LANES + lane) * 8, to8, valid[c]);
                }
            }
            if (!a.branch) continue;
            const float scale = a.scale * kept;
            two[0] = two[1] = 0.0f;
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const uint32_t col = (c * LANES + lane) * 8;
                Bits8 bits = {};
                if (a.random.threshold) bits = bits_of(key, row * words_of(cols) + col / 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const bool keep = i < valid[c] && bits.of(i) >= a.random.threshold;      // (behind a row's end d is what a layer norm took out)
                    if (post) u[c][i] *= rho_f;
                    d[c][i] = keep ? scale * d[c][i] : 0.0f;
                    if constexpr (SUMS & bit(kGateSum)) {
                        float v = u[c][i];
                        if (a.post.weight) v *= post_weight[c][i];
                        if (a.post.bias) v += post_bias[c][i];
                        sums[kGateSum][c][i] += keep ? d[c][i] * v : 0.0f;       // (what is dropped may be anything)
                    }
                    if (a.gate) d[c][i] = keep ? d[c][i] * gate[c][i] : 0.0f;
                    if constexpr (SUMS & bit(kPostWeight)) sums[kPostWeight][c][i] = __builtin_fmaf(d[c][i], u[c][i], sums[kPostWeight][c][i]);
                    if constexpr (SUMS & bit(kPostBias)) sums[kPostBias][c][i] += d[c][i];
                    if (a.post.weight) d[c][i] *= post_weight[c][i];
                    two[0] += d[c][i], two[1] = __builtin_fmaf(d[c][i], u[c][i], two[1]);
                }
            }
            if (!a.df) continue;
            float c0 = 0.0f, c1 = 0.0f;
            if (post) {
                sum_in_row<LANES>(two, shared, turn);
                c0 = post_layer ? -rho_f * (two[0] * each) : 0.0f, c1 = -rho_f * (two[1] * each);
            }
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if (post) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[c][i] = __builtin_fmaf(rho_f, d[c][i], __builtin_fmaf(c1, u[c][i], c0));
                }
                if (valid[c]) store_eight<DTYPE>(row_of<DTYPE>(a.df, row, a.lddf), (c * LANES + lane) * 8, d[c], valid[c]);
            }
        }
        if constexpr (SUMS & bit(kGateSum))
            if (args.sums[kGateSum] && share.splits == 1) {
                put(kGateSum, sums[kGateSum], args.sums[kGateSum] + group * a.ld_gate_grad, a.accumulate);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sums[kGateSum][c][i] = 0.0f;
            }
    }
    const bool parts = share.workers > 1;
#pragma unroll
    for (int s = 0; s < kAllSums; ++s) {
        if (!(SUMS >> s & 1) || !args.sums[s] || (s == kGateSum && share.splits == 1)) continue;
        put(s, sums[s], args.sums[s] + (parts ? worker * args.ld_sums : 0), !parts && a.accumulate);
    }
}

}  // namespace

template <uint32_t DTYPE> hipError_t launch_block_grad(const GradArgs &args, hipStream_t st) {
    int wanted = 0;
    for (int s = 0; s < kAllSums; ++s) wanted |= args.sums[s] ? bit(s) : 0;
    for_shape(row_shape((uint32_t)args.a.cols), [&](auto lanes, auto chunks) {
        constexpr int LANES = decltype(lanes)::value, CHUNKS = decltype(chunks)::value;
        auto with = [&](auto sums) { k_block_grad<DTYPE, LANES, CHUNKS, decltype(sums)::value><<<args.share.workers, LANES > 64 ? LANES : 64, 0, st>>>(args); };
        constexpr int kPre = bit(kPreWeight), kPreBoth = kPre | bit(kPreBias), kGates = kPre | bit(kGateSum), kRms = kGates | bit(kPostWeight), kAll = bit(kAllSums) - 1;
        if ((wanted & ~kPre) == 0) with(std::integral_constant<int, kPre>());
        else if ((wanted & ~kPreBoth) == 0) with(std::integral_constant<int, kPreBoth>());
        else if ((wanted & ~kGates) == 0) with(std::integral_constant<int, kGates>());
        else if ((wanted & ~kRms) == 0) with(std::integral_constant<int, kRms>());
        else with(std::integral_constant<int, kAll>());
    });
    return hipGetLastError();
}

}  // namespace eden_layers
