// C ABI of the 4-bit operands and their products (see include/eden_mx4.h for the contract of every call).  Host code only: argument checks, the choice of a
// kernel, launches.
#include "eden_mx4_kernels.h"

#include <algorithm>

using namespace eden_layers;

namespace {

constexpr uint64_t kMostRows = 1ull << 27, kMostDepth = 1ull << 22, kMostGroups = 0x7FFFFFFFull;

bool known_type(uint32_t dtype) { return dtype <= EDEN_BF16; }
size_t bytes_of(uint32_t dtype) { return dtype == EDEN_F32 ? 4 : 2; }
int status(hipError_t e) { return e == hipSuccess ? EDEN_OK : EDEN_ERR_HIP; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
bool matrix_ok(const void *p, uint64_t ld, uint64_t rows, uint64_t cols, size_t element) {
    if (rows == 0 || cols == 0) return true;
    return p != nullptr && aligned(p, element) && (rows == 1 || (ld >= cols && ld <= (1ull << 40)));
}
bool packed_ok(const void *p, uint64_t rows, uint64_t cols) { return rows == 0 || cols == 0 || (p != nullptr && aligned(p, 16)); }
bool operand_sizes_ok(uint64_t rows, uint64_t cols) { return rows <= kMostRows && cols <= kMostDepth; }
// Workgroups of eight chunks, two rows' at least
bool launchable(uint64_t rows, uint64_t cols) { return (rows / 2 + 1) * (chunks_of(cols) / 4 + 1) <= kMostGroups; }
// Workgroups of 512 threads for 128 rows (of the transpose) and a chunk
bool transposable(uint64_t rows, uint64_t cols) { return ((rows + 127) / 128) * chunks_of(cols) <= most_groups(512); }

uint64_t tile_count(uint64_t rows, uint64_t cols, uint32_t side) { return ((rows + side - 1) / side) * ((cols + side - 1) / side); }
size_t partial_bytes(uint64_t rows, uint64_t cols, uint64_t splits) { return splits * rows * ((cols + 3) / 4 * 4) * sizeof(float); }

struct Shape {
    uint32_t side;
    uint64_t splits;
};
// What an end takes longer than a bare one, us a round of large and of small tiles: the two workgroups of a CU hide some of each other's (8192 x 16384, 4096 deep, in large and in small tiles: bare 312
// and 317 us, gelu 371 and 361, its slope 439 and 375, gelu and checkpoint 414 and 460, residual 399 and 423, fp32 results 331 and 424; 4096 x 16384, 2048 deep: 94 and 95, 135 and 126, 171 and 131, 154 and 135, 117 and 116).
struct End {
    double large, small;
    End(double l, double s) : large(l), small(s) {}
    End(const Finish &f, bool fp32)
        : large((f.codes_in ? 17.0 : f.codes_out ? 14.0 : f.activation ? 8.5 : 0.0) + (f.residual ? 11.0 : 0.0) + (fp32 ? 2.5 : 0.0)),
          small((f.codes_in ? 4.0 : f.codes_out ? 6.0 : f.activation ? 3.3 : 0.0) + (f.residual ? 6.0 : 0.0) + (fp32 ? 6.5 : 0.0)) {}
};
// Tiles of 256 x 256, one to a CU, or of 128 x 128, two to a CU, by what a round of each takes in us.  Measured (bf16): a chunk of 256 deep 1.65 in a full round of the former (8192 x 8192: 250 us at 8192 deep, four
// rounds), 1.2 where CUs are idle (512 x 4096 x 4096: 28); 1.0 in a full round of the latter (2048 x 4096 x 4096: 25, 1500 x 5120 x 8192: 40), 0.55 with one to a CU (512 x 4096 x 4096: 13.6,
// 2048 x 2048 x 2048: 10.6); bare ends 10 and 4 a round.  That puts 4096 x 5120 x 4096 (54 us against 69) and 3000 x 3000 x 1000 (16 against 20) at the latter, 4096 x 4096 x 4096 at the former (38 against 42).
// A sum of small tiles is split over workgroups where that is worth the join, a launch and 8 bytes a result and split at 3 TB/s: 256 x 256, 16384 deep, in 16 parts 11 us against 34; 64 x 4096 x 4096 in
// four 11.2 against 12.2; 1024 x 1024 x 4096 not (two parts: 15.7 against 12.7; four: 20).  (The end is not looked at for that: the workspace is asked for without knowing it.)
Shape shape_of(uint64_t rows, uint64_t cols, uint64_t depth, const End &end) {
    const uint64_t large = tile_count(rows, cols, 256), small = tile_count(rows, cols, 128), chunks = std::max<uint64_t>(1, chunks_of(depth));
    const double cost_large = (double)(large / 256) * (1.65 * (double)chunks + 10.0 + end.large) + (large % 256 ? 1.2 * (double)chunks + 11.0 + end.large : 0.0);
    auto cost_small = [&](uint64_t splits, double more) {
        const uint64_t tiles = small * splits, left = tiles % 512;
        const double deep = (double)((chunks + splits - 1) / splits);
        const double join = splits > 1 ? 4.5 + (double)splits * (double)rows * (double)cols * (8.0 / 3e6) : 0.0;
        return (double)(tiles / 512) * (deep + 4.0 + more) + (left > 256 ? deep + 4.0 + more : left ? 0.55 * deep + 1.5 + more : 0.0) + join;
    };
    Shape best = {128, 1};
    for (uint64_t splits = 2; splits <= 64 && splits <= chunks && small * splits <= 512; ++splits)
        if (cost_small(splits, 0.0) < cost_small(best.splits, 0.0)) best.splits = splits;
    return cost_large < cost_small(best.splits, end.small) ? Shape{256, 1} : best;
}

// Products by few rows.  Above sixteen of them each workgroup reads as much of x as of w and more: those of a short sum and of a result that is no more than one round of workgroups (two to a CU up to
// 32 rows).  Both sides' times stand at the kernel.
bool few(uint64_t rows, uint64_t cols, uint64_t depth) {
    return rows <= kFewRows || (rows * depth <= 1u << 18 && (rows <= 32 ? cols <= 16384 : rows <= kFewMx4 && cols <= 8192));
}

// Launches a product whose operands and end are set.
int run(Op op, uint32_t dtype, Product &p, void *workspace, size_t workspace_bytes, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (workspace == nullptr) workspace_bytes = 0;
    const Shape shape = shape_of(p.rows, p.cols, p.depth, End(p.finish, op == kWeightGrad || dtype == EDEN_F32));
    if (tile_count(p.rows, p.cols, shape.side) * shape.splits > most_groups(256)) return EDEN_ERR_INVALID_ARG;
    uint64_t splits = shape.splits;
    while (splits > 1 && partial_bytes(p.rows, p.cols, splits) > workspace_bytes) --splits;
    const uint64_t chunks = std::max<uint64_t>(1, chunks_of(p.depth)), each = (chunks + splits - 1) / splits;
    p.splits = (uint32_t)((chunks + each - 1) / each);
    p.split_depth = (uint32_t)(each * kChunk);
    p.partial = static_cast<float *>(workspace);
    p.partial_ld = (p.cols + 3) / 4 * 4;
    hipError_t e = launch_mx4_tiles(op, dtype, p, shape.side, st);
    if (e == hipSuccess && p.splits > 1) e = launch_join(op, dtype, p, st);
    return status(e);
}

uint64_t sums_distance(uint64_t cols) { return (cols + 3) / 4 * 4; }
uint64_t sums_parts(uint64_t rows, uint64_t cols) {
    // as many workgroups as the device holds twice over, if every one had one chunk after the other
    const uint64_t chunks = chunks_of(rows), wide = (cols + 127) / 128;
    return std::max<uint64_t>(1, std::min(chunks, (2048 + wide - 1) / std::max<uint64_t>(wide, 1)));
}

}  // namespace

extern "C" {

size_t eden_mx4_bytes(uint64_t rows, uint64_t cols) { return operand_sizes_ok(rows, cols) ? mx4_bytes(rows, cols) : 0; }

size_t eden_mx4_sums_bytes(uint64_t rows, uint64_t cols) {
    if (!operand_sizes_ok(cols, rows) || rows == 0 || cols == 0) return 0;
    const uint64_t parts = sums_parts(rows, cols);
    return parts > 1 ? parts * sums_distance(cols) * sizeof(float) : 0;
}

int eden_mx4_quantize(const void *x, uint64_t ldx, uint64_t rows, uint64_t cols, uint32_t dtype, int transpose, const eden_random *rounding, void *packed, size_t capacity, float *sums,
                      int accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    const uint64_t r = transpose ? cols : rows, c = transpose ? rows : cols;
    if (!known_type(dtype) || !operand_sizes_ok(r, c) || !launchable(r, c) || !matrix_ok(x, ldx, rows, cols, bytes_of(dtype)) || !packed_ok(packed, r, c)) return EDEN_ERR_INVALID_ARG;
    if (transpose && !transposable(r, c)) return EDEN_ERR_INVALID_ARG;
    if ((sums && !transpose) || !aligned(sums, 4) || !aligned(workspace, 16) || (rounding && !aligned(rounding->seed_at, 8))) return EDEN_ERR_INVALID_ARG;
    if (capacity < mx4_bytes(r, c)) return EDEN_ERR_CAPACITY;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Rounding how = {};
    if (rounding) how.random = *rounding, how.stochastic = 1;
    uint8_t *to = static_cast<uint8_t *>(packed);
    if (!transpose) return rows == 0 || cols == 0 ? EDEN_OK : status(launch_mx4_rows(dtype, x, ldx, (uint32_t)rows, (uint32_t)cols, how, to, st));
    if (cols == 0 || (rows == 0 && !sums)) return EDEN_OK;
    const uint64_t ld = sums_distance(cols), room = workspace ? workspace_bytes / (ld * sizeof(float)) : 0;
    uint64_t parts = std::max<uint64_t>(1, std::min(sums_parts(rows, cols), room));
    const uint64_t chunks = chunks_of(rows), each = sums ? std::max<uint64_t>(1, (chunks + parts - 1) / parts) : 1;
    parts = std::max<uint64_t>(1, (chunks + each - 1) / each);
    const bool split = sums && parts > 1;
    hipError_t e = hipSuccess;
    if (rows != 0) {
        e = launch_mx4_columns(dtype, x, ldx, (uint32_t)rows, (uint32_t)cols, how, to, split ? static_cast<float *>(workspace) : sums, ld, !split && accumulate, (uint32_t)each, st);
        if (!split || e != hipSuccess) return status(e);
    }
    SumsArgs add = {};                                             // (of no rows: no parts, zeros)
    add.of[0] = {static_cast<float *>(workspace), sums};
    add.ld_from = ld, add.count = 1, add.cols = (uint32_t)cols, add.parts[0] = rows ? (uint32_t)parts : 0, add.rows[0] = 1, add.accumulate = accumulate != 0;
    return status(launch_sums(add, st));
}

int eden_mx4_restore(const void *packed, uint64_t rows, uint64_t cols, uint32_t dtype, void *x, uint64_t ldx, void *stream) {
    if (!known_type(dtype) || !operand_sizes_ok(rows, cols) || !launchable(rows, cols) || !matrix_ok(x, ldx, rows, cols, bytes_of(dtype)) || !packed_ok(packed, rows, cols)) return EDEN_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return EDEN_OK;
    return status(launch_mx4_restore(dtype, static_cast<const uint8_t *>(packed), (uint32_t)rows, (uint32_t)cols, x, ldx, static_cast<hipStream_t>(stream)));
}

size_t eden_mx4_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t depth, int quantize) {
    if (!operand_sizes_ok(rows, depth) || !operand_sizes_ok(cols, depth) || rows == 0 || cols == 0) return 0;
    const uint64_t splits = shape_of(rows, cols, depth, End(1e9, 0.0)).splits;       // (those of small tiles, if any end takes them)
    return (splits > 1 ? partial_bytes(rows, cols, splits) : 0) + (quantize ? (mx4_bytes(rows, depth) + 15) / 16 * 16 : 0);
}

int eden_mx4_linear(const void *x, uint64_t ldx, const void *x_packed, const void *w_packed, const void *bias, const void *residual, uint64_t ldr, void *y, uint64_t ldy, void *z_checkpoint,
                    size_t z_capacity, uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, uint32_t activation, void *workspace, size_t workspace_bytes, void *stream) {
    if (!known_type(dtype) || activation > EDEN_ACT_SILU || !operand_sizes_ok(m, k) || !operand_sizes_ok(n, k) || !aligned(workspace, 16)) return EDEN_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    const bool own = x != nullptr;
    if (own && x_packed) return EDEN_ERR_INVALID_ARG;
    if (!(own ? matrix_ok(x, ldx, m, k, e) && launchable(m, k) : packed_ok(x_packed, m, k)) || !packed_ok(w_packed, n, k) || !matrix_ok(y, ldy, m, n, e)) return EDEN_ERR_INVALID_ARG;
    if ((bias && !matrix_ok(bias, n, 1, n, e)) || (residual && !matrix_ok(residual, ldr, m, n, e)) || (z_checkpoint && !aligned(z_checkpoint, 16))) return EDEN_ERR_INVALID_ARG;
    if (z_checkpoint && z_capacity < eden_checkpoint_bytes(m, n)) return EDEN_ERR_CAPACITY;
    if (m == 0 || n == 0) return EDEN_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    Product p = {};
    p.a = x_packed, p.b = w_packed;
    p.rows = (uint32_t)m, p.cols = (uint32_t)n, p.depth = (uint32_t)k;
    p.finish.bias = bias, p.finish.residual = residual, p.finish.ld_residual = ldr, p.finish.out = y, p.finish.ld_out = ldy;
    p.finish.activation = activation, p.finish.blocks = (uint32_t)blocks_of(n);
    if (z_checkpoint) {
        p.finish.codes_out = static_cast<uint8_t *>(z_checkpoint);
        p.finish.exps_out = p.finish.codes_out + m * blocks_of(n) * kBlock;
    }
    if (own && m <= EDEN_MX4_ROWS && m * k <= EDEN_MX4_VALUES) return status(launch_mx4_few(dtype, p, x, ldx, st));
    if (own && k) {
        const size_t need = (mx4_bytes(m, k) + 15) / 16 * 16;
        if (workspace == nullptr || workspace_bytes < need) return EDEN_ERR_CAPACITY;
        uint8_t *to = static_cast<uint8_t *>(workspace);
        if (launch_mx4_rows(dtype, x, ldx, (uint32_t)m, (uint32_t)k, {}, to, st) != hipSuccess) return EDEN_ERR_HIP;
        p.a = to;
        workspace = to + need, workspace_bytes -= need;
    }
    if (few(m, n, k)) return status(launch_mx4_few(dtype, p, nullptr, 0, st));
    return run(kForward, dtype, p, workspace, workspace_bytes, stream);
}

int eden_mx4_input_grad(const void *dz_packed, const void *wt_packed, const void *z_checkpoint, uint32_t activation, const void *residual, uint64_t ldr, void *dx, uint64_t ldx, uint64_t m,
                        uint64_t n, uint64_t k, uint32_t dtype, void *workspace, size_t workspace_bytes, void *stream) {
    if (!known_type(dtype) || activation > EDEN_ACT_SILU || !operand_sizes_ok(m, n) || !operand_sizes_ok(k, n) || !aligned(workspace, 16)) return EDEN_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!packed_ok(dz_packed, m, n) || !packed_ok(wt_packed, k, n) || !matrix_ok(dx, ldx, m, k, e) || (residual && !matrix_ok(residual, ldr, m, k, e))) return EDEN_ERR_INVALID_ARG;
    const bool slopes = activation != EDEN_ACT_NONE;
    if (slopes ? m && k && (z_checkpoint == nullptr || !aligned(z_checkpoint, 16)) : z_checkpoint != nullptr) return EDEN_ERR_INVALID_ARG;
    if (m == 0 || k == 0) return EDEN_OK;
    Product p = {};
    p.a = dz_packed, p.b = wt_packed;
    p.rows = (uint32_t)m, p.cols = (uint32_t)k, p.depth = (uint32_t)n;
    p.finish.residual = residual, p.finish.ld_residual = ldr, p.finish.out = dx, p.finish.ld_out = ldx;
    p.finish.activation = activation, p.finish.blocks = (uint32_t)blocks_of(k);
    if (slopes) {
        p.finish.codes_in = static_cast<const uint8_t *>(z_checkpoint);
        p.finish.exps_in = p.finish.codes_in + m * blocks_of(k) * kBlock;
    }
    return run(kInputGrad, dtype, p, workspace, workspace_bytes, stream);
}

int eden_mx4_weight_grad(const void *dyt_packed, const void *xt_packed, float *dw, uint64_t ldw, uint64_t m, uint64_t n, uint64_t k, int accumulate, void *workspace, size_t workspace_bytes,
                         void *stream) {
    if (!operand_sizes_ok(n, m) || !operand_sizes_ok(k, m) || !packed_ok(dyt_packed, n, m) || !packed_ok(xt_packed, k, m) || !matrix_ok(dw, ldw, n, k, 4) || !aligned(workspace, 16))
        return EDEN_ERR_INVALID_ARG;
    if (n == 0 || k == 0) return EDEN_OK;
    Product p = {};
    p.a = dyt_packed, p.b = xt_packed;
    p.rows = (uint32_t)n, p.cols = (uint32_t)k, p.depth = (uint32_t)m;
    p.finish.out = dw, p.finish.ld_out = ldw, p.finish.accumulate = accumulate != 0;
    return run(kWeightGrad, EDEN_BF16, p, workspace, workspace_bytes, stream);
}

}  // extern "C"
