// C ABI of the operators around a residual block (see include/eden_blocks.h for the contract of every call).  Host code only: argument
// checks, how rows are shared out, launches.
#include "eden_blocks_kernels.h"

#include <algorithm>
#include <cmath>

using namespace eden_layers;

namespace {

constexpr uint64_t kMostRows = 1ull << 30;

bool known_type(uint32_t dtype) { return dtype <= EDEN_BF16; }
size_t bytes_of(uint32_t dtype) { return dtype == EDEN_F32 ? 4 : 2; }
int status(hipError_t e) { return e == hipSuccess ? EDEN_OK : EDEN_ERR_HIP; }
bool sizes_ok(uint64_t rows, uint64_t cols) { return rows <= kMostRows && cols <= EDEN_MOST_COLUMNS; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
// A matrix that is read or written: absent only if it has no element; aligned to its elements, rows apart.
bool matrix_ok(const void *p, uint64_t ld, uint64_t rows, uint64_t cols, size_t element) {
    if (rows == 0 || cols == 0) return true;
    return p != nullptr && aligned(p, element) && (rows == 1 || (ld >= cols && ld <= (1ull << 40)));
}
bool optional_ok(const void *p, uint64_t ld, uint64_t rows, uint64_t cols, size_t element) { return p == nullptr || matrix_ok(p, ld, rows, cols, element); }
bool random_ok(const eden_random &r) { return r.threshold <= 65535 && aligned(r.seed_at, 8); }
// scale times what kept values are multiplied by is one factor of the kernels: infinite, it would make NaN of zeros
bool scales_ok(float scale, float x_scale, const eden_random &r) { return std::isfinite(scale * kept_scale(r.threshold)) && std::isfinite(x_scale); }
bool norm_ok(const eden_norm &n, size_t element) {
    if (n.kind > EDEN_NORM_LAYER) return false;
    if (n.kind == EDEN_NORM_NONE) return n.weight == nullptr && n.bias == nullptr;
    return std::isfinite(n.eps) && n.eps >= 0.0f && aligned(n.weight, element) && aligned(n.bias, element) && (n.kind == EDEN_NORM_LAYER || n.bias == nullptr);
}
bool gates_ok(const void *gate, const void *gate_grad, uint64_t gates, uint64_t rows) {
    return (gate == nullptr && gate_grad == nullptr) || (gates >= 1 && gates <= kMostRows && rows % gates == 0);
}

uint64_t sums_distance(uint64_t cols) { return (cols + 7) / 8 * 8; }
// Workgroups that share the rows of a gradient: at most `most`, those that the device holds together, and each with some rows.  full: with a branch, post: and a norm behind it.
// Two rows each at least: with one, 77 x 1000 writes and reads as many sums again as it has operands (16.8 us against 12.1).
Share share_of(uint64_t rows, uint64_t cols, uint64_t gates, bool full, bool post, uint64_t most) {
    const int lanes = full ? FullGradShape((uint32_t)cols).lanes : GradShape((uint32_t)cols).lanes, threads = std::max(64, lanes);
    const uint64_t rows_each = 2 * (uint64_t)(threads / lanes);
    const uint64_t wanted = std::min<uint64_t>(256 * (full && (post || cols > 4096) ? lanes == 512 ? 512 : lanes < 512 ? 768 : 1024 : 1024) / threads, most);
    Share s = {(uint32_t)gates, (uint32_t)(rows / gates), 1, 1, 1};
    if (gates >= wanted || s.group_rows == 0) {
        s.groups_each = (uint32_t)((gates + wanted - 1) / std::max<uint64_t>(wanted, 1));
        s.workers = (uint32_t)((gates + s.groups_each - 1) / s.groups_each);
    } else {
        s.splits = (uint32_t)std::max<uint64_t>(1, std::min(wanted / gates, (s.group_rows + rows_each - 1) / rows_each));
        s.workers = s.gates * s.splits;
    }
    return s;
}

template <uint32_t DTYPE> hipError_t launch_typed(const GradArgs &g, hipStream_t st) {
    if (!g.a.branch) return launch_block_grad<DTYPE, -1>(g, st);
    if (g.a.post.kind == EDEN_NORM_NONE) return launch_block_grad<DTYPE, EDEN_NORM_NONE>(g, st);
    return g.a.post.kind == EDEN_NORM_RMS ? launch_block_grad<DTYPE, EDEN_NORM_RMS>(g, st) : launch_block_grad<DTYPE, EDEN_NORM_LAYER>(g, st);
}
hipError_t launch_grad(const GradArgs &g, hipStream_t st) {
    if (!g.a.branch && g.a.dh == nullptr) return hipSuccess;
    return g.a.dtype == EDEN_F32 ? launch_typed<EDEN_F32>(g, st) : g.a.dtype == EDEN_F16 ? launch_typed<EDEN_F16>(g, st) : launch_typed<EDEN_BF16>(g, st);
}

}  // namespace

extern "C" {

int eden_dropout(const void *x, uint64_t ldx, void *y, uint64_t ldy, uint64_t rows, uint64_t cols, uint32_t dtype, const eden_random *random, void *stream) {
    if (!known_type(dtype) || random == nullptr || !random_ok(*random) || !sizes_ok(rows, cols)) return EDEN_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!matrix_ok(x, ldx, rows, cols, e) || !matrix_ok(y, ldy, rows, cols, e)) return EDEN_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return EDEN_OK;
    return status(launch_dropout(dtype, x, ldx, y, ldy, (uint32_t)rows, (uint32_t)cols, *random, static_cast<hipStream_t>(stream)));
}

int eden_join(const eden_join_args *args, void *stream) {
    if (args == nullptr || !known_type(args->dtype) || !sizes_ok(args->rows, args->cols)) return EDEN_ERR_INVALID_ARG;
    eden_join_args a = *args;
    const size_t e = bytes_of(a.dtype);
    if (!random_ok(a.random) || !norm_ok(a.post, e) || !norm_ok(a.pre, e) || !scales_ok(a.scale, a.x_scale, a.random)) return EDEN_ERR_INVALID_ARG;
    const bool empty = a.rows == 0 || a.cols == 0, normed = a.pre.kind != EDEN_NORM_NONE;
    if (!matrix_ok(a.x, a.ldx, a.rows, a.cols, e) || !optional_ok(a.f, a.ldf, a.rows, a.cols, e) || !optional_ok(a.r, a.ldr, a.rows, a.cols, e) ||
        !optional_ok(a.h, a.ldh, a.rows, a.cols, e) || !gates_ok(a.gate, nullptr, a.gates, a.rows) || !optional_ok(a.gate, a.ld_gate, a.gates, a.cols, e))
        return EDEN_ERR_INVALID_ARG;
    if (a.f == nullptr && !empty && (a.gate || a.r || a.post.kind != EDEN_NORM_NONE || a.random.threshold || !normed)) return EDEN_ERR_INVALID_ARG;
    if (!empty && ((a.h != nullptr) != normed || (a.r == nullptr && a.h == nullptr))) return EDEN_ERR_INVALID_ARG;
    if (empty) return EDEN_OK;
    if (a.gate == nullptr) a.gates = 1;
    return status(launch_block_join(a, static_cast<hipStream_t>(stream)));
}

size_t eden_join_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t gates, uint32_t dtype) {
    if (!known_type(dtype) || !sizes_ok(rows, cols) || rows == 0 || cols == 0) return 0;
    if (gates < 1) gates = 1;
    if (gates > rows || rows % gates) return 0;
    const uint64_t workers = std::max(share_of(rows, cols, gates, false, false, ~0ull).workers, share_of(rows, cols, gates, true, false, ~0ull).workers);
    return workers > 1 ? workers * kAllSums * sums_distance(cols) * sizeof(float) : 0;
}

int eden_join_grad(const eden_join_grad_args *args, void *stream) {
    if (args == nullptr || !known_type(args->dtype) || !sizes_ok(args->rows, args->cols)) return EDEN_ERR_INVALID_ARG;
    GradArgs g = {*args, {}, {}, 0, 0};
    eden_join_grad_args &a = g.a;
    const size_t e = bytes_of(a.dtype);
    const bool normed = a.pre.kind != EDEN_NORM_NONE, post = a.post.kind != EDEN_NORM_NONE;
    if (!random_ok(a.random) || !norm_ok(a.post, e) || !norm_ok(a.pre, e) || !scales_ok(a.scale, a.x_scale, a.random) || !aligned(a.workspace, 16))
        return EDEN_ERR_INVALID_ARG;
    const void *mats[] = {a.dr, a.dh, a.r, a.f, a.dx, a.df};
    const uint64_t lds[] = {a.lddr, a.lddh, a.ldr, a.ldf, a.lddx, a.lddf};
    for (int i = 0; i < 6; ++i)
        if (!optional_ok(mats[i], lds[i], a.rows, a.cols, e)) return EDEN_ERR_INVALID_ARG;
    if (!gates_ok(a.gate, a.gate_grad, a.gates, a.rows) || !optional_ok(a.gate, a.ld_gate, a.gates, a.cols, e) || !optional_ok(a.gate_grad, a.ld_gate_grad, a.gates, a.cols, 4))
        return EDEN_ERR_INVALID_ARG;
    float *sums[kAllSums] = {a.gate_grad, a.post_weight_grad, a.post_bias_grad, a.pre_weight_grad, a.pre_bias_grad};
    uint32_t count = 0;
    for (float *s : sums) {
        if (!aligned(s, 4)) return EDEN_ERR_INVALID_ARG;
        count += s != nullptr;
    }
    // what a norm or a branch that is not there would give
    if ((!normed && (a.dh || a.pre_weight_grad || a.pre_bias_grad)) || (!post && (a.post_weight_grad || a.post_bias_grad))) return EDEN_ERR_INVALID_ARG;
    if ((a.pre_bias_grad && a.pre.kind != EDEN_NORM_LAYER) || (a.post_bias_grad && a.post.kind != EDEN_NORM_LAYER)) return EDEN_ERR_INVALID_ARG;
    if (!a.branch && (a.gate || a.gate_grad || a.df || post || a.random.threshold || (a.dh == nullptr && a.rows && a.cols))) return EDEN_ERR_INVALID_ARG;
    if (a.cols == 0) return EDEN_OK;
    g.needs_f = post || a.gate_grad;
    if (a.rows != 0 && ((g.needs_f && a.f == nullptr) || (a.dh && a.r == nullptr))) return EDEN_ERR_INVALID_ARG;
    if ((a.gate == nullptr && a.gate_grad == nullptr) || a.rows == 0) {
        // (without rows every group's sums are nothing: they are written below)
        if (a.rows != 0 || a.gate_grad == nullptr) a.gates = 1;
    }
    if (!a.dx && !a.df && count == 0) return EDEN_OK;
    const uint64_t ld = sums_distance(a.cols), room = a.workspace ? a.workspace_bytes / (sizeof(float) * ld) : 0;
    g.share = share_of(a.rows, a.cols, a.gates, a.branch, post, count ? std::max<uint64_t>(1, room / count) : ~0ull);
    g.ld_sums = ld;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool parts = g.share.workers > 1;
    SumsArgs add = {};
    add.ld_from = ld, add.cols = (uint32_t)a.cols, add.accumulate = a.accumulate;
    float *space = static_cast<float *>(a.workspace);
    for (int s = 0; s < kAllSums; ++s) {
        g.sums[s] = sums[s];
        if (sums[s] && (s == kPreWeight || s == kPreBias) && a.dh == nullptr) {
            // without dh they are sums over nothing, and the kernel has no place for them
            g.sums[s] = nullptr;
            add.of[add.count] = {space, sums[s]};
            add.rows[add.count] = 1;
            ++add.count;
            continue;
        }
        if (!sums[s] || !parts || (s == kGateSum && g.share.splits == 1)) continue;
        g.sums[s] = space;
        const bool gate = s == kGateSum;
        add.of[add.count] = {space, sums[s]};
        add.parts[add.count] = gate ? g.share.splits : g.share.workers;
        add.rows[add.count] = gate ? (uint32_t)a.gates : 1;
        add.ld_to[add.count] = gate ? (a.gates > 1 ? a.ld_gate_grad : 0) : 0;
        ++add.count;
        space += g.share.workers * ld;
    }
    hipError_t err = launch_grad(g, st);
    if (err == hipSuccess && add.count) err = launch_sums(add, st);
    return status(err);
}

}  // extern "C"
