// nz_mx4_api.hip -- extern "C" boundary of the microscaled 4-bit operators: argument checks and launches.
#include "../../include/nz_mx4.h"
#include "nz_mx4.hpp"

using namespace nz;

namespace {

constexpr uint64_t kMaxSide = 1ull << 31, kMaxElements = 1ull << 38;
constexpr uint64_t kMaxProductSide = 1ull << 30, kMaxRowBytes = 4ull << 20, kMaxOutput = 1ull << 40;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool is_float_type(int t) { return t == NZ_F32 || t == NZ_BF16 || t == NZ_F16; }
bool is_rounding(int r) { return r == NZ_MX4_NEAREST || r == NZ_MX4_STOCHASTIC; }

bool matrix_ok(const nz_mx4_matrix* m, uint64_t rows, uint64_t cols) {
    return m && m->codes && m->scales && aligned16(m->codes) && aligned16(m->scales) && m->pitch % 4 == 0 &&
           m->pitch >= (cols + 31) / 32 && (rows == 1 || m->pitch <= kMaxElements / 32);
}

bool floats_ok(const void* p, int type, uint64_t rows, uint64_t cols, uint64_t ld) {
    return p && aligned16(p) && is_float_type(type) && ld >= cols && (rows == 1 || ld <= kMaxElements);
}

bool shape_ok(uint64_t rows, uint64_t cols) {
    return rows > 0 && cols > 0 && rows < kMaxSide && cols < kMaxSide && rows * cols < kMaxElements;
}

// Division of a block's number b, below 2^29, by nb as a multiplication: with l = ceil(log2 nb) and m = floor(2^(29 + l) / nb) + 1, m nb
// exceeds 2^(29 + l) by at most nb <= 2^l, so that b m / 2^(29 + l) exceeds b / nb by less than 1 / nb and has the same whole part.
MxRows rows_of(uint64_t rows, uint64_t cols) {
    MxRows R;
    R.rows = rows; R.cols = cols;
    R.nb = (uint32_t)((cols + 31) / 32);
    const uint64_t g = ((1ull << 29) - 1) / R.nb;
    R.group = (uint32_t)(g < rows ? g : rows);
    R.nb_shift = 0;
    while ((1ull << R.nb_shift) < R.nb) R.nb_shift++;
    R.nb_mul = (uint32_t)((1ull << (29 + R.nb_shift)) / R.nb + 1);
    return R;
}

// Whole rows of whole blocks without gaps are one long row.
bool one_row(uint64_t rows, uint64_t cols) { return rows > 1 && cols % 128 == 0 && rows * cols < kMaxSide; }

bool operands_ok(const nz_mx4_matrix* in, uint32_t k, const float* d_local, uint64_t ld_local, uint64_t rows, uint64_t cols) {
    if (!shape_ok(rows, cols) || !in || k == 0 || k > kMxMaxOperands) return false;
    for (uint32_t i = 0; i < k; i++)
        if (!matrix_ok(in + i, rows, cols)) return false;
    return !d_local || floats_ok(d_local, NZ_F32, rows, cols, ld_local);
}

// Floats that fill half of the last cache (256 MB) before anyone reads them are written around it: 64 Mi floats there and back in 103 us
// instead of 132, and 144 instead of 156 with a pass that reads them afterwards; 16 Mi floats with such a pass take 38.2 us so and 36.8
// through the caches.
constexpr uint64_t kPastCaches = 128ull << 20;

// What becomes of a sum: floats of `type`, or four bits (type -1).
struct Outcome { int type; void* out; uint64_t ld; uint8_t *codes, *scales; uint64_t pitch; bool stochastic; uint32_t seed; };

template <uint32_t MAX> nz_status sum_to(const nz_mx4_matrix* in, uint32_t k, const float* d_local, uint64_t ld_local, uint64_t rows, uint64_t cols,
                                         const Outcome& O, void* stream) {
    MxSumArgs<MAX> A;
    const uint64_t nb = (cols + 31) / 32;
    bool flat = one_row(rows, cols) && (O.type < 0 ? O.pitch == nb : O.ld == cols) && (!d_local || ld_local == cols);
    for (uint32_t i = 0; i < k; i++) {
        A.in[i] = { reinterpret_cast<const uint8_t*>(in[i].codes), reinterpret_cast<const uint8_t*>(in[i].scales), in[i].pitch };
        flat = flat && in[i].pitch == nb;
    }
    A.R = flat ? rows_of(1, rows * cols) : rows_of(rows, cols);
    A.k = k;
    A.local = d_local; A.ld_local = ld_local;
    A.out = O.out; A.ld = O.ld;
    A.codes = O.codes; A.scales = O.scales; A.pitch = O.pitch; A.seed = O.seed;
    const bool way = O.type < 0 ? O.stochastic : rows * cols * float_bytes(O.type) >= kPastCaches;
    return launch_mx_sum<MAX>(A, O.type, way, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? NZ_OK : NZ_ERR_HIP;
}

nz_status sum_to(const nz_mx4_matrix* in, uint32_t k, const float* d_local, uint64_t ld_local, uint64_t rows, uint64_t cols, const Outcome& O,
                 void* stream) {
    if (k == 1) return sum_to<1>(in, k, d_local, ld_local, rows, cols, O, stream);
    if (k <= kMxSomeOperands) return sum_to<kMxSomeOperands>(in, k, d_local, ld_local, rows, cols, O, stream);
    return sum_to<kMxMaxOperands>(in, k, d_local, ld_local, rows, cols, O, stream);
}

bool product_shape_ok(int kind, uint64_t M, uint64_t N, uint64_t K) {
    return M > 0 && N > 0 && K > 0 && M < kMaxProductSide && N < kMaxProductSide && K < kMaxProductSide && M * N < kMaxOutput &&
           M * K < (kind == NZ_MX4_PRODUCT ? kMaxElements : kMaxOutput) && N * K < kMaxElements;
}

bool product_matrix_ok(const nz_mx4_matrix* m, uint64_t rows, uint64_t cols) {
    return matrix_ok(m, rows, cols) && m->pitch <= kMaxRowBytes / 16;          // (of one row, too)
}

bool product_floats_ok(const void* p, int type, uint64_t cols, uint64_t ld) {
    return floats_ok(p, type, 2, cols, ld) && ld * float_bytes(type) <= kMaxRowBytes;
}

nz_status run_product(MxProductArgs& A, const nz_mx4_matrix* b, int kind, int left, uint64_t M, uint64_t N, uint64_t K, void* d_c, int type,
                      uint64_t ldc, void* d_ws, size_t ws_bytes, void* stream) {
    const size_t need = mx_product_workspace(kind, left, M, N, K);
    if (need && (!d_ws || !aligned16(d_ws) || ws_bytes < need)) return NZ_ERR_INVALID;
    A.b = { reinterpret_cast<const uint8_t*>(b->codes), reinterpret_cast<const uint8_t*>(b->scales), b->pitch };
    A.M = M; A.N = N; A.K = K;
    A.c = d_c; A.ldc = ldc; A.c_type = type;
    A.ws = d_ws;
    return launch_mx_product(A, kind, left, reinterpret_cast<hipStream_t>(stream)) == hipSuccess ? NZ_OK : NZ_ERR_HIP;
}

}  // namespace

extern "C" {

size_t nz_mx4_pitch(size_t cols) { return cols / 128 * 4 + (cols % 128 ? 4 : 0); }

nz_status nz_mx4_quantize(const void* d_in, nz_float_type type, size_t rows, size_t cols, size_t ld, nz_mx4_rounding rounding,
                          uint32_t seed, const nz_mx4_matrix* out, void* stream) {
    if (!shape_ok(rows, cols) || !floats_ok(d_in, type, rows, cols, ld) || !is_rounding(rounding) || !matrix_ok(out, rows, cols))
        return NZ_ERR_INVALID;
    MxConvertArgs A;
    const bool flat = one_row(rows, cols) && ld == cols && out->pitch == cols / 32;
    A.R = flat ? rows_of(1, rows * cols) : rows_of(rows, cols);
    A.in = d_in; A.ld = ld;
    A.codes = reinterpret_cast<uint8_t*>(out->codes); A.scales = reinterpret_cast<uint8_t*>(out->scales); A.pitch = out->pitch;
    A.seed = seed;
    const hipError_t e = launch_mx_quantize(A, type, rounding == NZ_MX4_STOCHASTIC, reinterpret_cast<hipStream_t>(stream));
    return e == hipSuccess ? NZ_OK : NZ_ERR_HIP;
}

nz_status nz_mx4_sum_k(const nz_mx4_matrix* in, uint32_t k, const float* d_local, size_t ld_local, size_t rows, size_t cols,
                       void* d_out, nz_float_type type, size_t ld, void* stream) {
    if (!operands_ok(in, k, d_local, ld_local, rows, cols) || !floats_ok(d_out, type, rows, cols, ld)) return NZ_ERR_INVALID;
    const Outcome O = { type, d_out, ld, nullptr, nullptr, 0, false, 0 };
    return sum_to(in, k, d_local, ld_local, rows, cols, O, stream);
}

nz_status nz_mx4_dequantize(const nz_mx4_matrix* in, size_t rows, size_t cols, void* d_out, nz_float_type type, size_t ld,
                            void* stream) {
    return nz_mx4_sum_k(in, 1, nullptr, 0, rows, cols, d_out, type, ld, stream);
}

nz_status nz_mx4_reduce_k(const nz_mx4_matrix* in, uint32_t k, const float* d_local, size_t ld_local, size_t rows, size_t cols,
                          nz_mx4_rounding rounding, uint32_t seed, const nz_mx4_matrix* out, void* stream) {
    if (!operands_ok(in, k, d_local, ld_local, rows, cols) || !is_rounding(rounding) || !matrix_ok(out, rows, cols)) return NZ_ERR_INVALID;
    const Outcome O = { -1, nullptr, 0, reinterpret_cast<uint8_t*>(out->codes), reinterpret_cast<uint8_t*>(out->scales), out->pitch,
                        rounding == NZ_MX4_STOCHASTIC, seed };
    return sum_to(in, k, d_local, ld_local, rows, cols, O, stream);
}

size_t nz_mx4_workspace_bytes(nz_mx4_kind kind, nz_float_type left, size_t M, size_t N, size_t K) {
    const bool kind_ok = kind == NZ_MX4_PRODUCT || kind == NZ_MX4_LINEAR || kind == NZ_MX4_GRAD;
    if (!kind_ok || (kind != NZ_MX4_PRODUCT && !is_float_type(left)) || !product_shape_ok(kind, M, N, K)) return (size_t)-1;
    return mx_product_workspace(kind, left, M, N, K);
}

nz_status nz_mx4_product(const nz_mx4_matrix* a, const nz_mx4_matrix* b, size_t M, size_t N, size_t K, void* d_c,
                         nz_float_type type, size_t ldc, void* d_ws, size_t ws_bytes, void* stream) {
    if (!product_shape_ok(NZ_MX4_PRODUCT, M, N, K) || !product_matrix_ok(a, M, K) || !product_matrix_ok(b, N, K) || !product_floats_ok(d_c, type, N, ldc))
        return NZ_ERR_INVALID;
    MxProductArgs A = {};
    A.a = { reinterpret_cast<const uint8_t*>(a->codes), reinterpret_cast<const uint8_t*>(a->scales), a->pitch };
    return run_product(A, b, NZ_MX4_PRODUCT, 0, M, N, K, d_c, type, ldc, d_ws, ws_bytes, stream);
}

nz_status nz_mx4_linear(const void* d_x, nz_float_type x_type, size_t ldx, const nz_mx4_matrix* b, size_t M, size_t N, size_t K,
                        void* d_c, nz_float_type type, size_t ldc, void* d_ws, size_t ws_bytes, void* stream) {
    if (!product_shape_ok(NZ_MX4_LINEAR, M, N, K) || !product_floats_ok(d_x, x_type, K, ldx) || !product_matrix_ok(b, N, K) ||
        !product_floats_ok(d_c, type, N, ldc)) return NZ_ERR_INVALID;
    MxProductArgs A = {};
    A.x = d_x; A.ldx = ldx;
    return run_product(A, b, NZ_MX4_LINEAR, x_type, M, N, K, d_c, type, ldc, d_ws, ws_bytes, stream);
}

nz_status nz_mx4_grad(const void* d_g, nz_float_type g_type, size_t ldg, const nz_mx4_matrix* b, size_t M, size_t N, size_t K,
                      void* d_da, nz_float_type type, size_t ldda, void* d_ws, size_t ws_bytes, void* stream) {
    if (!product_shape_ok(NZ_MX4_GRAD, M, N, K) || !product_floats_ok(d_g, g_type, N, ldg) || !product_matrix_ok(b, N, K) ||
        !product_floats_ok(d_da, type, K, ldda)) return NZ_ERR_INVALID;
    MxProductArgs A = {};
    A.x = d_g; A.ldx = ldg;
    return run_product(A, b, NZ_MX4_GRAD, g_type, M, N, K, d_da, type, ldda, d_ws, ws_bytes, stream);
}

}  // extern "C"
