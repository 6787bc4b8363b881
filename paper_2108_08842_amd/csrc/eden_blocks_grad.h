// The gradients of a residual block's join (included by one source for each type and kind of norm behind the branch).
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
//
// What counts is registers: sums, operands of this row and of the next (on their way meanwhile, or each row would wait for its loads), weights.  Hence operands stay packed, kinds of norms are compiled in, and the arguments
// are read again for each row.  Dropout, gate, both norms rms / both layer, us with the second launch: bf16 8192 x 4096 77 to 88 / 96 to 103 (403 MB at 4.7 TB/s), 32768 x 1024 80 / 93, 8192 x 8192 172 / 244, 4096 x 16384 320 / 525
// (floor 158), without a branch 8192 x 4096 41 / 49; fp32 8192 x 4096 172 / 190 (floor 158), 8192 x 8192 348 / 378 (316), 4096 x 16384 466 / 715, without a branch 88 / 94 (79).  131072 x 128 bf16 50 / 53, fp32 101 / 108: four rows a
// wave, and a loop that waits.
// What does not fit (the compiler's resource records; a lane's registers that go to memory): above 8192 columns with both norms 33 to 98, with one up to 35; two-byte types: both norms layer up to 2048 columns 2 to 10, rms
// behind the branch and any norm in front from 4097 to 8192 columns 2 to 26; fp32 up to 2048 columns: a norm in front alone 2 to 24, rms behind and layer in front 4 to 7.  Nothing is fetched ahead, and weights are read again for each
// row, where kHeld is false: with a branch above 8192 columns, fp32 above 4096 (without a branch 8192), with a layer norm behind the branch two-byte types above 4096 and fp32 always.
#include "eden_blocks_kernels.h"

namespace eden_layers {
namespace {

// Waves of a SIMD that the registers are shared out to: 512 registers of a lane by the sums and operands of each kind.  wide: operands of four bytes next to a norm in front (512 lanes without a norm behind
// the branch, 8192 x 4096 fp32: two waves, nothing in memory, 175 us rms and 177 layer; four, 8 to 31 registers in memory, 190 and 200)
constexpr int waves_of(int lanes, int chunks, int post, bool wide) { return lanes == 1024 || post < 0 || (post == 0 && chunks == 1 && !(wide && lanes == 512)) ? 4 : lanes == 512 ? 2 : 3; }

// The operands of a row as they lie in memory
template <uint32_t DTYPE, int CHUNKS> struct RowOperands {
    Eight<DTYPE> r[CHUNKS], f[CHUNKS], dh[CHUNKS], dr[CHUNKS];
};

// PRE, POST: kinds of the norms; POST -1: no branch
template <uint32_t DTYPE, int LANES, int CHUNKS, bool RAGGED, int PRE, int POST>
__global__ __launch_bounds__(LANES > 64 ? LANES : 64) __attribute__((amdgpu_waves_per_eu(waves_of(LANES, CHUNKS, POST, DTYPE == EDEN_F32 && PRE != EDEN_NORM_NONE)))) void k_block_grad(const GradArgs args) {
    constexpr int kThreads = LANES > 64 ? LANES : 64, kRows = kThreads / LANES;
    constexpr bool kHeld = (POST < 0 || LANES < 1024) && CHUNKS * sizeof(typename Elem<DTYPE>::type) <= (POST == EDEN_NORM_LAYER ? 2 : 4);       // weights stay in registers, and the next row's operands come while one is worked on
    constexpr bool kPacked = sizeof(typename Elem<DTYPE>::type) == 2 && (waves_of(LANES, CHUNKS, POST, false) == 4 || (CHUNKS == 2 && POST == EDEN_NORM_LAYER));
    constexpr bool kPre = PRE != EDEN_NORM_NONE, kPreLayer = PRE == EDEN_NORM_LAYER, kBranch = POST >= 0, kPost = POST > 0, kPostLayer = POST == EDEN_NORM_LAYER;
    constexpr bool kHas[kAllSums] = {kBranch, kPost, kPostLayer, kPre, kPreLayer};
    __shared__ float shared[kSumFloats<LANES>];
    // Sums of the gate and of the norm's weights behind the branch, of rows so long that the registers have no place for them: in the LDS, each read and written by its own thread only
    constexpr bool kFar = kBranch && LANES == 1024;
    constexpr int kFarSums = kPost ? 2 : 1;
    __shared__ f32x4 far[kFar ? kFarSums * CHUNKS * 2 : 1][kFar ? LANES : 1];
    auto far_at = [] {                                             // (made anew each time: kept, the addresses would take a register for every 64 KB)
        uint32_t at = threadIdx.x;
        asm volatile("" : "+v"(at));
        return at;
    };
    auto far_load = [&](int s, int c, float (&v)[8]) {
        const uint32_t at = far_at();
        const f32x4 low = far[(s * CHUNKS + c) * 2][at], high = far[(s * CHUNKS + c) * 2 + 1][at];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = low[i], v[4 + i] = high[i];
    };
    auto far_store = [&](int s, int c, const float (&v)[8]) {
        const uint32_t at = far_at();
        far[(s * CHUNKS + c) * 2][at] = f32x4{v[0], v[1], v[2], v[3]};
        far[(s * CHUNKS + c) * 2 + 1][at] = f32x4{v[4], v[5], v[6], v[7]};
    };
    auto far_clear = [&](int s) {
        const float zeros[8] = {};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) far_store(s, c, zeros);
    };
    if constexpr (kFar) {
#pragma unroll
        for (int s = 0; s < kFarSums; ++s) far_clear(s);
    }
    int turn = 0;
    const eden_join_grad_args &a = args.a;
    typedef const __attribute__((address_space(4))) GradArgs *Arguments;
    const Share &share = args.share;
    const uint32_t cols = (uint32_t)a.cols, worker = blockIdx.x, sub = row_in_group<LANES>();
    const RowPlace<DTYPE, LANES, CHUNKS, RAGGED> place(cols, threadIdx.x % LANES);
    const uint64_t key = kBranch && a.random.threshold ? key_of(a.random, eden::kStreamDropout) : 0;
    const float each = 1.0f / (float)cols, scale = a.scale * kept_scale(a.random.threshold);

    // The arguments again, from memory: kept, all of them would take more scalar registers than there are
    auto again = [] {
        Arguments k = (Arguments)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(k));
        return k;
    };
    auto weights_of = [&](const void *p, int c, float fill) {
        Eight<DTYPE> w;
        w.fill(fill);
        if (p) place.load(w, p, c), place.settle(w, c, true);
        return w;
    };
    Eight<DTYPE> held_pre[CHUNKS], held_post[CHUNKS], held_post_bias[CHUNKS], held_gate[CHUNKS];
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        if constexpr (kHeld && kPre) held_pre[c] = weights_of(a.pre.weight, c, 1.0f);
        if constexpr (kHeld && kPost) held_post[c] = weights_of(a.post.weight, c, 1.0f);
        if constexpr (kHeld && kPostLayer) held_post_bias[c] = weights_of(a.post.bias, c, 0.0f);
    }
    auto pre_weight = [&](int c) { return kHeld ? held_pre[c] : weights_of(again()->a.pre.weight, c, 1.0f); };
    auto post_weight = [&](int c) { return kHeld ? held_post[c] : weights_of(again()->a.post.weight, c, 1.0f); };
    auto post_bias = [&](int c) { return kHeld ? held_post_bias[c] : weights_of(again()->a.post.bias, c, 0.0f); };
    float sums[kAllSums][CHUNKS][8] = {};

    // one result's or one part's sums
    auto put = [&](int s, float *to, bool add) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            float v[8];
            if (kFar && s < kFarSums) far_load(s, c, v);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = sums[s][c][i];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) v[i] += __shfl_xor(v[i], d);
            }
            if (threadIdx.x < LANES && place.valid[c]) {
                float *at = to + place.col[c];
                Vec<float, 8> out;
                if (add) out = load_some<float, 8>(at, place.valid[c]);
#pragma unroll
                for (int i = 0; i < 8; ++i) out.v[i] = add ? out.v[i] + v[i] : v[i];
                store_some<float, 8>(at, out, place.valid[c]);
            }
        }
    };

    const uint32_t first_group = share.splits > 1 ? worker / share.splits : worker * share.groups_each;
    const uint32_t end_group = share.splits > 1 ? first_group + 1 : min(share.gates, first_group + share.groups_each);
    const uint32_t split = share.splits > 1 ? worker % share.splits : 0, split_rows = (share.group_rows + share.splits - 1) / share.splits;
    const uint32_t from = min(split * split_rows, share.group_rows), to = min(from + split_rows, share.group_rows);
    for (uint32_t group = first_group; group < end_group; ++group) {
        const uint64_t group_row = (uint64_t)group * share.group_rows;
        auto gate_of = [&](int c) { return weights_of(a.gate ? row_of<DTYPE, LANES>(a.gate, group, a.ld_gate) : nullptr, c, 1.0f); };
        auto gate = [&](int c) {
            if constexpr (kHeld) return held_gate[c];
            const Arguments k = again();
            return weights_of(k->a.gate ? row_of<DTYPE, LANES>(k->a.gate, group, k->a.ld_gate) : nullptr, c, 1.0f);
        };
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
            if constexpr (kHeld && kBranch) held_gate[c] = gate_of(c);
        auto row_at = [&](uint32_t at) { return group_row + (kRows == 1 || at + sub < to ? at + sub : from); };
        auto load = [&](RowOperands<DTYPE, CHUNKS> &row8, uint32_t at) {
            const Arguments k = again();
            const uint64_t row = row_at(at);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if constexpr (kPre) {
                    place.load(row8.r[c], row_of<DTYPE, LANES>(k->a.r, row, k->a.ldr), c);
                    place.load(row8.dh[c], row_of<DTYPE, LANES>(k->a.dh, row, k->a.lddh), c);
                }
                if (k->a.dr) place.load(row8.dr[c], row_of<DTYPE, LANES>(k->a.dr, row, k->a.lddr), c);
                if (kBranch && k->needs_f) place.load(row8.f[c], row_of<DTYPE, LANES>(k->a.f, row, k->a.ldf), c);
            }
        };
        RowOperands<DTYPE, CHUNKS> now = {}, next = {};
        if (kHeld && from < to) load(now, from);
        for (uint32_t at = from; at < to; at += kRows) {
            if constexpr (kHeld) {
                if (at + kRows < to) load(next, at + kRows);
            } else {
                now = {};                                          // (what is not there would be carried from row to row)
                load(now, at);
            }
            const bool has = kRows == 1 || at + sub < to;
            const Arguments k = again();
            const uint64_t row = row_at(at);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                if constexpr (kPre) place.settle(now.r[c], c, has), place.settle(now.dh[c], c, has);
                if (k->a.dr) place.settle(now.dr[c], c, has);
                if (kBranch && k->needs_f) place.settle(now.f[c], c, has);
            }
            auto stay_packed = [&] {
                if constexpr (kPacked) {
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) {
                        if constexpr (kPre) now.r[c].stay_packed(), now.dh[c].stay_packed();
                        if constexpr (kBranch) now.f[c].stay_packed();
                        if constexpr (kPre && kHeld) held_pre[c].stay_packed();
                        if constexpr (kPost && kHeld) held_post[c].stay_packed();
                        if constexpr (kPostLayer && kHeld) held_post_bias[c].stay_packed();
                        if constexpr (kBranch && kHeld) held_gate[c].stay_packed();
                    }
                }
            };
            stay_packed();
            auto inside = [&](int c, int i) { return has && place.inside(c, i); };
            // means of layer norms, then sums of squares and of products with r around them
            float three[3], mean_r = 0.0f, mean_f = 0.0f, mean_g = 0.0f;
            if constexpr (kPreLayer || kPostLayer) {
                three[0] = three[1] = three[2] = 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    Eight<DTYPE> w;
                    if constexpr (kPreLayer) w = pre_weight(c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if constexpr (kPreLayer) three[0] += now.r[c][i], three[2] = __builtin_fmaf(now.dh[c][i], w[i], three[2]);
                        if constexpr (kPostLayer) three[1] += now.f[c][i];
                    }
                    if constexpr (kFar) __builtin_amdgcn_sched_barrier(0);
                }
                stay_packed();
                sum_in_row<LANES>(three, shared, turn);
                if constexpr (kPreLayer) mean_r = three[0] * each, mean_g = three[2] * each;
                if constexpr (kPostLayer) mean_f = three[1] * each;
            }
            float rho_r = 0.0f, rho_f = 0.0f, inner = 0.0f;
            if constexpr (kPre || kPost) {
                three[0] = three[1] = three[2] = 0.0f;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    Eight<DTYPE> w;
                    if constexpr (kPre) w = pre_weight(c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if constexpr (kPre) {
                            const float n = kPreLayer && !inside(c, i) ? 0.0f : now.r[c][i] - mean_r;
                            three[0] = __builtin_fmaf(n, n, three[0]);
                            three[2] = __builtin_fmaf(now.dh[c][i] * w[i], n, three[2]);
                        }
                        if constexpr (kPost) {
                            const float u = kPostLayer && !inside(c, i) ? 0.0f : now.f[c][i] - mean_f;
                            three[1] = __builtin_fmaf(u, u, three[1]);
                        }
                    }
                    if constexpr (kFar) __builtin_amdgcn_sched_barrier(0);
                }
                stay_packed();
                sum_in_row<LANES>(three, shared, turn);
                if constexpr (kPre)
                    rho_r = rho_of<LANES>(three[0], each, k->a.pre.eps, shared, turn, [&](float by) {
                        float sum = 0.0f;
#pragma unroll
                        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float n = kPreLayer && !inside(c, i) ? 0.0f : (now.r[c][i] - mean_r) * by;
                                sum = __builtin_fmaf(n, n, sum);
                            }
                        return sum;
                    });
                if constexpr (kPost)
                    rho_f = rho_of<LANES>(three[1], each, k->a.post.eps, shared, turn, [&](float by) {
                        float sum = 0.0f;
#pragma unroll
                        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float u = kPostLayer && !inside(c, i) ? 0.0f : (now.f[c][i] - mean_f) * by;
                                sum = __builtin_fmaf(u, u, sum);
                            }
                        return sum;
                    });
                if (!has) rho_r = rho_f = 0.0f;                    // (of rows that are none, 0 times 0 and not times 1 / 0)
                inner = three[2] * rho_r * each;
            }
            float d[CHUNKS][8];
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[c][i] = now.dr[c][i];
            if constexpr (kPre) {
                // rho (g - mean_g - n rho inner), n = r - mean_r: in this order, for rho^2 may be below the range where rho n is not
                const float c1 = -rho_r * inner;
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    const Eight<DTYPE> w = pre_weight(c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float dh = now.dh[c][i], n = now.r[c][i] - mean_r;
                        sums[kPreWeight][c][i] = __builtin_fmaf(dh, n * rho_r, sums[kPreWeight][c][i]);
                        if constexpr (kPreLayer) sums[kPreBias][c][i] += dh;
                        d[c][i] = __builtin_fmaf(rho_r, __builtin_fmaf(c1, n, kPreLayer ? __builtin_fmaf(dh, w[i], -mean_g) : dh * w[i]), d[c][i]);
                        if (kPacked && i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            if constexpr (kPre && !kPreLayer && kPost) {
                // Behind a row's end d is 0, or NaN where the row's statistics are: the norm behind the branch would add it up.  (Full rows go past it here; as one more
                // condition of `keep` below 8192 x 4096 bf16 takes 76 to 83 us in place of 74 to 77.)
                if (place.partial) {
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[c][i] = place.inside(c, i) ? d[c][i] : 0.0f;
                }
            }
            if (k->a.dx) {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    float to8[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) to8[i] = k->a.x_scale * d[c][i];
                    if (has) place.template store<(LANES >= 64)>(row_of<DTYPE, LANES>(k->a.dx, row, k->a.lddx), c, to8);
                }
            }
            if constexpr (kBranch) {
                float two[2] = {0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    Bits8 bits = {};
                    if (k->a.random.threshold) bits = bits_of(key, row * words_of(cols) + place.col[c] / 4);
                    Eight<DTYPE> w, b;
                    if constexpr (kPost) w = post_weight(c);
                    if constexpr (kPostLayer) b = post_bias(c);
                    const Eight<DTYPE> g = gate(c);
                    float far_gate[8], far_weight[8];
                    if constexpr (kFar) far_load(kGateSum, c, far_gate);
                    if constexpr (kFar && kPost) far_load(kPostWeight, c, far_weight);
                    float(&gate_sum)[8] = kFar ? far_gate : sums[kGateSum][c], (&weight_sum)[8] = kFar ? far_weight : sums[kPostWeight][c];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // behind a row's end d is what a layer norm took out; what is dropped may be anything
                        const bool keep = (!kPreLayer || inside(c, i)) && bits.of(i) >= k->a.random.threshold;
                        const float u = kPost ? (now.f[c][i] - mean_f) * rho_f : now.f[c][i];
                        const float v = kPostLayer ? __builtin_fmaf(u, w[i], b[i]) : kPost ? u * w[i] : u;
                        const float back = keep ? scale * d[c][i] : 0.0f;
                        gate_sum[i] = __builtin_fmaf(back, keep ? v : 0.0f, gate_sum[i]);
                        const float du = keep ? back * g[i] : 0.0f;
                        if constexpr (kPost) {
                            weight_sum[i] = __builtin_fmaf(du, u, weight_sum[i]);
                            if constexpr (kPostLayer) sums[kPostBias][c][i] += du;
                            d[c][i] = du * w[i];
                            if constexpr (kPostLayer) two[0] += d[c][i];
                            two[1] = __builtin_fmaf(d[c][i], u, two[1]);
                        } else {
                            d[c][i] = du;
                        }
                        if (kPacked && i % 2 == 1) __builtin_amdgcn_sched_barrier(0);       // (all eight side by side would take too many registers)
                    }
                    if constexpr (kFar) far_store(kGateSum, c, far_gate);
                    if constexpr (kFar && kPost) far_store(kPostWeight, c, far_weight);
                }
                if (k->a.df) {
                    if constexpr (kPost) {
                        stay_packed();
                        sum_in_row<LANES>(two, shared, turn);
                        const float c0 = -rho_f * (two[0] * each), c1 = -rho_f * (two[1] * each);
#pragma unroll
                        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float u = now.f[c][i] - mean_f;
                                const float v = __builtin_fmaf(c1, u, d[c][i]);
                                d[c][i] = kPostLayer ? __builtin_fmaf(rho_f, v, c0) : rho_f * v;
                            }
                    }
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c)
                        if (has) place.template store<(LANES >= 64)>(row_of<DTYPE, LANES>(k->a.df, row, k->a.lddf), c, d[c]);
                }
            }
            if constexpr (kHeld) now = next;
        }
        if constexpr (kBranch)
            if (args.sums[kGateSum] && share.splits == 1) {
                put(kGateSum, args.sums[kGateSum] + group * a.ld_gate_grad, a.accumulate);
                if constexpr (kFar) far_clear(kGateSum);
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sums[kGateSum][c][i] = 0.0f;
            }
    }
    const bool parts = share.workers > 1;
#pragma unroll
    for (int s = 0; s < kAllSums; ++s) {
        if (!kHas[s] || !args.sums[s] || (s == kGateSum && share.splits == 1)) continue;
        put(s, args.sums[s] + (parts ? worker * args.ld_sums : 0), !parts && a.accumulate);
    }
}

}  // namespace

template <uint32_t DTYPE, int POST> hipError_t launch_block_grad(const GradArgs &args, hipStream_t st) {
    std::conditional_t<(POST >= 0), FullGradShape, GradShape>((uint32_t)args.a.cols).use((uint32_t)args.a.cols, [&](auto lanes, auto chunks, auto ragged) {
        constexpr int LANES = decltype(lanes)::value, CHUNKS = decltype(chunks)::value, kThreads = LANES > 64 ? LANES : 64;
        constexpr bool RAGGED = decltype(ragged)::value;
        if (args.a.dh == nullptr) {
            if constexpr (POST >= 0) k_block_grad<DTYPE, LANES, CHUNKS, RAGGED, EDEN_NORM_NONE, POST><<<args.share.workers, kThreads, 0, st>>>(args);
        } else if (args.a.pre.kind == EDEN_NORM_RMS) {
            k_block_grad<DTYPE, LANES, CHUNKS, RAGGED, EDEN_NORM_RMS, POST><<<args.share.workers, kThreads, 0, st>>>(args);
        } else {
            k_block_grad<DTYPE, LANES, CHUNKS, RAGGED, EDEN_NORM_LAYER, POST><<<args.share.workers, kThreads, 0, st>>>(args);
        }
    });
    return hipGetLastError();
}

}  // namespace eden_layers
