// C ABI of the layer operators (see include/eden_layers.h for the contract of every call).  Host code only: argument checks, the
// choice of a kernel, launches.
#include "eden_layers_kernels.h"

#include <algorithm>

using namespace eden_layers;

namespace {

constexpr uint64_t kMostSize = 1ull << 30;
constexpr uint64_t kMostGroups = 0x7FFFFFFFull;        // workgroups of an element-wise call

bool known_type(uint32_t dtype) { return dtype <= EDEN_BF16; }
size_t bytes_of(uint32_t dtype) { return dtype == EDEN_F32 ? 4 : 2; }
int status(hipError_t e) { return e == hipSuccess ? EDEN_OK : EDEN_ERR_HIP; }

// A matrix that is read or written: absent only if it has no element; aligned to its elements, rows apart.
bool matrix_ok(const void *p, uint64_t ld, uint64_t rows, uint64_t cols, size_t element) {
    if (rows == 0 || cols == 0) return true;
    return p != nullptr && reinterpret_cast<uintptr_t>(p) % element == 0 && (rows == 1 || (ld >= cols && ld <= (1ull << 40)));
}
// The distance between rows of an operand as the kernels take it.  That of a single row may be anything, but loads of whole tiles count on a second row's place, which has to be
// read as zeros, lying behind the first row's end: it becomes the row's length in whole pieces.
uint64_t distance(uint64_t ld, uint64_t rows, uint64_t cols) { return rows > 1 ? ld : (cols + 7) / 8 * 8; }
bool checkpoint_ok(const void *p, uint64_t rows, uint64_t cols) {
    return rows == 0 || cols == 0 || (p != nullptr && reinterpret_cast<uintptr_t>(p) % 16 == 0);
}
size_t codes_bytes(uint64_t rows, uint64_t cols) { return rows * blocks_of(cols) * kBlock; }

// Element-wise launches: at least 1024 values a workgroup but for the ends of rows
bool launchable(uint64_t rows, uint64_t cols) { return rows * (blocks_of(cols) / 64 + 1) <= kMostGroups; }

uint64_t tile_count(uint64_t rows, uint64_t cols, uint32_t side) { return (uint64_t)tiles_of((uint32_t)rows, side) * tiles_of((uint32_t)cols, side); }
size_t partial_bytes(uint64_t rows, uint64_t cols, uint64_t splits) { return splits * rows * ((cols + 3) / 4 * 4 + 1) * sizeof(float); }

// How many workgroups share a tile's sum: `slots` of them fit the device together, and one has at least `least` of the depth.
uint64_t splits_of(uint64_t tiles, uint64_t depth, uint64_t slots, uint64_t least) {
    const uint64_t s = std::min(slots / tiles, depth / least);
    return s < 1 ? 1 : s > 64 ? 64 : s;
}
struct Shape {
    uint32_t side;
    uint64_t splits;
};
// Loads straight into the LDS: tiles of 256 x 256, one to a CU, or of 128 x 128, two to a CU.  Measured (bf16, depth 4096): 64 deep take 1.6 us in a
// full round of the former, 1.2 us where most of the CUs are idle (the clock is higher then), 1.05 us in a full round of the latter and 0.6 us with
// one to a CU; a round's ends 10 and 5 us.  That puts 2048 x 8192 at the former (111 us against 131), 2048 x 4096 at the latter (67 against 87), 4096 x 5120 too
// (a second round of 64 tiles; 92 against 103 at depth 2048).
Shape direct_shape(uint64_t rows, uint64_t cols, uint64_t depth) {
    const uint64_t large = tile_count(rows, cols, 256), small = tile_count(rows, cols, 128), left_large = large % 256, left_small = small % 512;
    const double deep = (double)((depth + 63) / 64);
    const double cost_large = (1.6 * (double)(large / 256) + (left_large > 160 ? 1.6 : left_large ? 1.2 : 0.0)) * deep + 10.0 * (double)((large + 255) / 256);
    const double cost_small = (1.05 * (double)(small / 512) + (left_small > 256 ? 1.05 : left_small ? 0.6 : 0.0)) * deep + 5.0 * (double)((small + 511) / 512);
    if (cost_large < cost_small) return {256, 1};
    // a split is worth its share of the join from 512 deep on (300 x 512 x 1024: 8.5 us against 8.7 with two), from 128 where there is little to join (32 x 1024 x
    // 1024: 9.1 -> 7); up to 128 rows the second operand is streamed once: two workgroups a CU read faster where each has enough of it (64 x 16384 x 4096: 42 -> 33)
    const uint64_t splits = rows * cols <= 40000 ? splits_of(small, depth, 512, 128) : splits_of(small, depth, 256, 512);
    return {128, rows <= 128 ? std::max(splits, splits_of(small, depth, 512, 1024)) : splits};
}
// Through registers: 128 x 128 where those fill the device (fp16 weight gradient 2048 x 4096, 1024 deep: 52 us against 63 with 64 x 64), else 64 x 64, three or more to
// a CU.  `slots`: as many workgroups as split a sum together: 512 (512 x 1001 x 1003 bf16: 13.3 us against 18 with 1024; weight gradients 1001 x 1024, 555 deep, fp32 17.5
// against 19.9; 256 x 256, 8192 deep, 16.3 against 20.8; 568 x 696, 2624 deep, fp16 21.3 against 21.9), between two fp32 operands, with six products of terms, 1024 (2318 x
// 192, 3081 deep: 36 against 39 with 512; 3405 x 128, 1193 deep, 20.5 against 19.6).
Shape tiles_shape(uint64_t rows, uint64_t cols, uint64_t depth, uint64_t slots) {
    if (tile_count(rows, cols, 128) >= 256) return {128, 1};
    return {64, splits_of(tile_count(rows, cols, 64), depth, slots, 96)};
}

// fp32 operands straight into the LDS: 128 x 128, two to a CU.
Shape fp32_shape(uint64_t rows, uint64_t cols, uint64_t depth) { return {128, splits_of(tile_count(rows, cols, 128), depth, 256, 128)}; }

// Rows that start at, and hold, whole 16-byte pieces, and offsets inside a tile that 31 bits hold
bool whole_pieces(const void *p, uint64_t ld, uint64_t inner, uint32_t dtype) {
    const uint64_t piece = dtype == EDEN_F32 ? 4 : 8;
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % piece == 0 && inner % piece == 0 && ld < (1u << 21);
}
// Whether the kernel whose loads go straight into the LDS takes a product: as it is, or with copies of the operands whose rows do not fit.
bool direct_type(Op op, uint32_t dtype, const Product &p) {
    return !(op == kWeightGrad && dtype != EDEN_BF16) && p.depth != 0 && p.cols != 0 && (op != kWeightGrad || p.ldb < (1u << 24));
}
// ... and whether that is the faster one: it has a long way to its first product.  2 bytes: two steps deep and up to 2^20 results the general kernel is (1024 x
// 1024 x 128 bf16 4.1 us against 5.6; 1024 x 1024 x 256 11.8 against 6.4, 2048 x 2048 x 128 7.4 against 6.7).  With a checkpoint below 2^28 products (512 x 512 x 768
// 11.0 against 14.0; 1024 x 1024 x 256 12.5 against 8.6).  fp32 below 1.5 * 2^28 (1024 x 1024 x 256 14.6 against 17.0; 768 x 768 x 768 20.6 against 20.8,
// 2048 x 2048 x 512 35.7 against 31.6).
bool direct_pays(Op op, uint32_t dtype, const Product &p) {
    const double results = (double)p.rows * p.cols, products = results * p.depth;
    if (dtype == EDEN_F32) return products >= 1.5 * (1u << 28);
    if (op == kWeightGrad) return products >= 1u << 28;
    return p.depth > 128 || results > 1u << 20;
}
bool whole_a(Op op, uint32_t dtype, const Product &p) { return whole_pieces(p.a, p.lda, op == kWeightGrad ? p.rows : p.depth, dtype); }
bool whole_b(Op op, uint32_t dtype, const Product &p) { return op == kWeightGrad || whole_pieces(p.b, p.ldb, op == kForward ? p.depth : p.cols, dtype); }
// More than four rows and so many columns that the 128 x 128 tiles' splits fill the device: the few rows' kernel would read x once for every 16 columns (16 x 16384 x
// 4096 bf16: 40 us against 32; 16 x 8192 x 4096 22 against 24).
bool many_columns(uint32_t dtype, const Product &p, uint64_t room) {
    return dtype != EDEN_F32 && p.rows > 4 && p.cols >= 128 * 128 && whole_a(kForward, dtype, p) && whole_b(kForward, dtype, p) &&
           partial_bytes(p.rows, p.cols, direct_shape(p.rows, p.cols, p.depth).splits) <= room;
}

// Copies cost two passes over an operand and are worth it from about 2^30 products on: in 2 bytes 1501 x 1501 x 1501 38 -> 30 us, 1021 x 1001 x 2047 28 -> 26.5, 801 x 1001 x 1335 between
// 20 -> 22 (eden_linear) and 23 -> 20 (input gradient), 831 x 831 x 831 14 -> 18; in fp32 1235 x 7079 x 2681 446 -> 353, 1235 x 1235 x 1235 53 -> 46, 801 x 1001 x 1335 35 -> 37,
// 831 x 831 x 831 22 -> 30, 301 x 2001 x 1001 24 -> 32.  Not for a narrow result (fp32, 2318 x 192 x 3081: 35 -> 47).
uint64_t copy_bytes(uint64_t a, uint64_t b, uint32_t dtype) { return (a + 63) / 64 * 64 * ((b + 63) / 64 * 64) * bytes_of(dtype); }
bool worth_copies(uint64_t rows, uint64_t cols, uint64_t depth) {
    const uint64_t most = 1u << 21, least = 1u << 30;
    return rows >= 256 && cols >= 256 && rows < most && cols < most && depth < most && rows * cols >= least / std::max<uint64_t>(depth, 1);
}
// Replaces an operand by a copy in the workspace.
hipError_t copy_operand(uint32_t dtype, const void *&operand, size_t &ld, uint32_t rows, uint32_t cols, uint8_t *&workspace, size_t &room, hipStream_t st) {
    const uint32_t to_ld = (cols + 63) / 64 * 64;
    const hipError_t e = launch_copy_rows(dtype, operand, ld, rows, cols, workspace, to_ld, st);
    const size_t used = copy_bytes(rows, cols, dtype);
    operand = workspace, ld = to_ld, workspace += used, room -= used;
    return e;
}

// Launches a product whose operands and end are set.
int run(Op op, uint32_t dtype, Product &p, void *workspace, size_t workspace_bytes, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return EDEN_ERR_INVALID_ARG;
    uint8_t *space = static_cast<uint8_t *>(workspace);
    if (workspace == nullptr) workspace_bytes = 0;
    p.a_width = op == kWeightGrad ? p.rows : p.depth;
    p.b_width = op == kForward ? p.depth : p.cols;
    bool direct = direct_type(op, dtype, p) && direct_pays(op, dtype, p);
    if (op == kForward && p.rows <= kFewRows && !(direct && many_columns(dtype, p, workspace_bytes))) return status(launch_rows(dtype, p, st));
    if (direct && !(whole_a(op, dtype, p) && whole_b(op, dtype, p))) {
        // rows along the depth that do not end with a piece need zeros behind it in both operands
        const bool a = !whole_a(op, dtype, p), b = !whole_b(op, dtype, p);
        const uint64_t need = (a ? copy_bytes(p.rows, p.depth, dtype) : 0) + (b ? copy_bytes(p.cols, p.depth, dtype) : 0);
        direct = worth_copies(p.rows, p.cols, p.depth) && need <= workspace_bytes;
        hipError_t e = hipSuccess;
        if (direct && a) {
            e = op == kWeightGrad ? copy_operand(dtype, p.a, p.lda, p.depth, p.rows, space, workspace_bytes, st) : copy_operand(dtype, p.a, p.lda, p.rows, p.depth, space, workspace_bytes, st);
            p.a_width = (uint32_t)p.lda;
        }
        if (direct && b && e == hipSuccess) {
            e = op == kForward ? copy_operand(dtype, p.b, p.ldb, p.cols, p.depth, space, workspace_bytes, st) : copy_operand(dtype, p.b, p.ldb, p.depth, p.cols, space, workspace_bytes, st);
            p.b_width = (uint32_t)p.ldb;
        }
        if (e != hipSuccess) return EDEN_ERR_HIP;
    }
    const Shape shape = !direct ? tiles_shape(p.rows, p.cols, p.depth, op != kWeightGrad && dtype == EDEN_F32 ? 1024 : 512) : dtype == EDEN_F32 ? fp32_shape(p.rows, p.cols, p.depth) : direct_shape(p.rows, p.cols, p.depth);
    if (tile_count(p.rows, p.cols, shape.side) * shape.splits > most_groups(256)) return EDEN_ERR_INVALID_ARG;      // (one launch; such a result has 2^38 places)
    uint64_t splits = p.cols ? shape.splits : 1;                   // (row sums alone have no columns at which a join would find them)
    while (splits > 1 && partial_bytes(p.rows, p.cols, splits) > workspace_bytes) --splits;
    const uint64_t each = ((p.depth + splits - 1) / splits + kSplitUnit - 1) / kSplitUnit * kSplitUnit;
    splits = each ? (p.depth + each - 1) / each : 1;
    p.splits = splits < 1 ? 1 : (uint32_t)splits;
    p.split_depth = (uint32_t)each;
    p.partial = reinterpret_cast<float *>(space);
    p.partial_ld = (p.cols + 3) / 4 * 4;
    hipError_t e = !direct ? launch_tiles(op, dtype, p, shape.side, st) : dtype == EDEN_F32 ? launch_direct_fp32(op, p, st) : launch_direct(op, dtype, p, shape.side, st);
    if (e == hipSuccess && p.splits > 1) e = launch_join(op, dtype, p, st);
    return status(e);
}

}  // namespace

extern "C" {

size_t eden_checkpoint_bytes(uint64_t rows, uint64_t cols) {
    if (rows > kMostSize || cols > kMostSize) return 0;
    return rows * blocks_of(cols) * (kBlock + 1);
}

int eden_checkpoint_save(const void *x, uint64_t ldx, uint64_t rows, uint64_t cols, uint32_t dtype, void *checkpoint, size_t capacity, void *stream) {
    if (!known_type(dtype) || rows > kMostSize || cols > kMostSize || !launchable(rows, cols)) return EDEN_ERR_INVALID_ARG;
    if (!matrix_ok(x, ldx, rows, cols, bytes_of(dtype)) || !checkpoint_ok(checkpoint, rows, cols)) return EDEN_ERR_INVALID_ARG;
    if (capacity < eden_checkpoint_bytes(rows, cols)) return EDEN_ERR_CAPACITY;
    if (rows == 0 || cols == 0) return EDEN_OK;
    uint8_t *codes = static_cast<uint8_t *>(checkpoint);
    return status(launch_save(dtype, x, ldx, (uint32_t)rows, (uint32_t)cols, codes, codes + codes_bytes(rows, cols), static_cast<hipStream_t>(stream)));
}

int eden_checkpoint_restore(const void *checkpoint, uint64_t rows, uint64_t cols, uint32_t dtype, void *x, uint64_t ldx, void *stream) {
    if (!known_type(dtype) || rows > kMostSize || cols > kMostSize || !launchable(rows, cols)) return EDEN_ERR_INVALID_ARG;
    if (!matrix_ok(x, ldx, rows, cols, bytes_of(dtype)) || !checkpoint_ok(checkpoint, rows, cols)) return EDEN_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return EDEN_OK;
    const uint8_t *codes = static_cast<const uint8_t *>(checkpoint);
    return status(launch_restore(dtype, codes, codes + codes_bytes(rows, cols), (uint32_t)rows, (uint32_t)cols, x, ldx, static_cast<hipStream_t>(stream)));
}

size_t eden_layers_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t depth, uint32_t dtype) {
    if (!known_type(dtype) || rows > kMostSize || cols > kMostSize || depth > kMostSize) return 0;
    if (rows == 0 || cols == 0) return 0;
    const uint64_t splits = std::max(dtype == EDEN_F32 ? fp32_shape(rows, cols, depth).splits : direct_shape(rows, cols, depth).splits, tiles_shape(rows, cols, depth, 1024).splits);
    return splits > 1 ? partial_bytes(rows, cols, splits) : 0;
}

size_t eden_layers_copying_bytes(uint64_t rows, uint64_t cols, uint64_t depth, uint32_t dtype) {
    if (!known_type(dtype) || rows > kMostSize || cols > kMostSize || depth > kMostSize) return 0;
    const size_t plain = eden_layers_workspace_bytes(rows, cols, depth, dtype);
    if (!worth_copies(rows, cols, depth)) return plain;
    return plain + copy_bytes(rows, depth, dtype) + copy_bytes(cols, depth, dtype);
}

int eden_linear(const void *x, uint64_t ldx, const void *w, uint64_t ldw, const void *bias, const void *residual, uint64_t ldr, void *y, uint64_t ldy,
                void *z_checkpoint, size_t z_capacity, uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, uint32_t activation, void *workspace,
                size_t workspace_bytes, void *stream) {
    if (!known_type(dtype) || activation > EDEN_ACT_SILU || m > kMostSize || n > kMostSize || k > kMostSize) return EDEN_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!matrix_ok(x, ldx, m, k, e) || !matrix_ok(w, ldw, n, k, e) || !matrix_ok(y, ldy, m, n, e)) return EDEN_ERR_INVALID_ARG;
    if ((bias && !matrix_ok(bias, n, 1, n, e)) || (residual && !matrix_ok(residual, ldr, m, n, e)) || (z_checkpoint && !checkpoint_ok(z_checkpoint, m, n)))
        return EDEN_ERR_INVALID_ARG;
    if (z_checkpoint && z_capacity < eden_checkpoint_bytes(m, n)) return EDEN_ERR_CAPACITY;
    if (m == 0 || n == 0) return EDEN_OK;
    Product p = {};
    p.a = x, p.lda = distance(ldx, m, k), p.b = w, p.ldb = distance(ldw, n, k);
    p.rows = (uint32_t)m, p.cols = (uint32_t)n, p.depth = (uint32_t)k;
    p.finish.bias = bias, p.finish.residual = residual, p.finish.ld_residual = ldr, p.finish.out = y, p.finish.ld_out = ldy;
    p.finish.activation = activation, p.finish.blocks = (uint32_t)blocks_of(n);
    if (z_checkpoint) {
        p.finish.codes_out = static_cast<uint8_t *>(z_checkpoint);
        p.finish.exps_out = p.finish.codes_out + codes_bytes(m, n);
    }
    return run(kForward, dtype, p, workspace, workspace_bytes, stream);
}

int eden_linear_weight_grad(const void *dy, uint64_t ldy, const void *x_checkpoint, float *dw, uint64_t ldw, float *bias_grad, uint64_t m, uint64_t n,
                            uint64_t k, uint32_t dtype, int accumulate, void *workspace, size_t workspace_bytes, void *stream) {
    if (!known_type(dtype) || m > kMostSize || n > kMostSize || k > kMostSize) return EDEN_ERR_INVALID_ARG;
    if (!matrix_ok(dy, ldy, m, n, bytes_of(dtype)) || !checkpoint_ok(x_checkpoint, m, k) || !matrix_ok(dw, ldw, n, k, 4)) return EDEN_ERR_INVALID_ARG;
    if (bias_grad && !matrix_ok(bias_grad, n, 1, n, 4)) return EDEN_ERR_INVALID_ARG;
    if (n == 0 || (k == 0 && !bias_grad)) return EDEN_OK;
    Product p = {};
    p.a = dy, p.lda = distance(ldy, m, n), p.b = x_checkpoint, p.ldb = blocks_of(k) * kBlock;
    p.b_blocks = (uint32_t)blocks_of(k);
    p.b_exps = static_cast<const uint8_t *>(x_checkpoint) + codes_bytes(m, k);
    p.rows = (uint32_t)n, p.cols = (uint32_t)k, p.depth = (uint32_t)m;
    p.finish.out = dw, p.finish.ld_out = ldw, p.finish.accumulate = accumulate != 0;
    p.row_sums = bias_grad;
    return run(kWeightGrad, dtype, p, workspace, workspace_bytes, stream);
}

int eden_linear_input_grad(const void *dz, uint64_t ldz, const void *w, uint64_t ldw, const void *z_checkpoint, uint32_t activation, const void *residual,
                           uint64_t ldr, void *dx, uint64_t ldx, uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, void *workspace,
                           size_t workspace_bytes, void *stream) {
    if (!known_type(dtype) || activation > EDEN_ACT_SILU || m > kMostSize || n > kMostSize || k > kMostSize) return EDEN_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!matrix_ok(dz, ldz, m, n, e) || !matrix_ok(w, ldw, n, k, e) || !matrix_ok(dx, ldx, m, k, e)) return EDEN_ERR_INVALID_ARG;
    if (residual && !matrix_ok(residual, ldr, m, k, e)) return EDEN_ERR_INVALID_ARG;
    const bool slopes = activation != EDEN_ACT_NONE;
    if (slopes ? !checkpoint_ok(z_checkpoint, m, k) : z_checkpoint != nullptr) return EDEN_ERR_INVALID_ARG;
    if (m == 0 || k == 0) return EDEN_OK;
    Product p = {};
    p.a = dz, p.lda = distance(ldz, m, n), p.b = w, p.ldb = distance(ldw, n, k);
    p.rows = (uint32_t)m, p.cols = (uint32_t)k, p.depth = (uint32_t)n;
    p.finish.residual = residual, p.finish.ld_residual = ldr, p.finish.out = dx, p.finish.ld_out = ldx;
    p.finish.activation = activation, p.finish.blocks = (uint32_t)blocks_of(k);
    if (slopes) {
        p.finish.codes_in = static_cast<const uint8_t *>(z_checkpoint);
        p.finish.exps_in = p.finish.codes_in + codes_bytes(m, k);
    }
    return run(kInputGrad, dtype, p, workspace, workspace_bytes, stream);
}

int eden_activation_grad(const void *dy, uint64_t ldy, const void *z_checkpoint, uint32_t activation, void *dz, uint64_t ldz, uint64_t rows,
                         uint64_t cols, uint32_t dtype, void *stream) {
    if (!known_type(dtype) || activation > EDEN_ACT_SILU || rows > kMostSize || cols > kMostSize || !launchable(rows, cols)) return EDEN_ERR_INVALID_ARG;
    const size_t e = bytes_of(dtype);
    if (!matrix_ok(dy, ldy, rows, cols, e) || !matrix_ok(dz, ldz, rows, cols, e) || !checkpoint_ok(z_checkpoint, rows, cols)) return EDEN_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return EDEN_OK;
    const uint8_t *codes = static_cast<const uint8_t *>(z_checkpoint);
    return status(launch_activation_grad(dtype, dy, ldy, codes, codes + codes_bytes(rows, cols), activation, dz, ldz, (uint32_t)rows, (uint32_t)cols,
                                         static_cast<hipStream_t>(stream)));
}

}  // extern "C"
