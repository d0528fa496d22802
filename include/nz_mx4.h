/*
 * nz_mx4.h -- C ABI of the microscaled 4-bit operators on MI355X (gfx950).
 *
 * A transport form of fixed rate beside the streams of nz.h: 4.25 bits an element, which the matrix units multiply as it is.
 * It follows the public OCP Microscaling Formats specification (MXFP4: E2M1 elements, one E8M0 scale for 32 of them).
 *
 * A matrix of `rows` x `cols` elements holds each row in blocks of 32 elements along the row:
 *   codes   block i of row r is the 16 bytes at codes + (r * pitch + i) * 16; element j of it lies in byte j / 2, in the low
 *           half for even j.  A code is a sign (bit 3) and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 2..0).
 *   scales  one byte s at scales + r * pitch + i: the block's elements are its codes times 2^(s - 127); s = 255: all are NaN.
 * `pitch` counts blocks, is a multiple of 4 and at least ceil(cols / 32).  Elements of a last block past `cols` have code 0
 * (nz_mx4_quantize and nz_mx4_reduce_k write them so, and the products count on it).  The buffers hold rows * pitch blocks;
 * those past the last one of a row are not written, and their contents do not matter.  A message is a matrix of one row.
 *
 * Conventions are those of nz.h: device pointers 16-byte aligned (codes, scales, floats, workspace), the caller owns every
 * buffer, nothing is allocated, no state is kept, kernels are enqueued on `stream` (of the current device) and never
 * waited for, and two calls may overlap in time only with different workspaces and outputs.  Every call can be recorded into
 * a HIP graph.  Outputs must not overlap inputs, except where it is said.  NZ_ERR_INVALID: a null or misaligned pointer, a
 * size of 0, a pitch or row length that is too small, a value that is not of its enumeration, a workspace that is too small,
 * or a size beyond these limits: rows and cols below 2^31, a matrix of fewer than 2^38 elements; for the products also
 * M, N, K below 2^30 and rows (of codes or floats, by pitch or row length) of at most 4 MiB, M * N and M * K below 2^40.
 * Nothing is launched then.  NZ_ERR_HIP: a launch failed.  Nothing is reported from the device.
 */
#ifndef NZ_MX4_H
#define NZ_MX4_H

#include "nz.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { NZ_F32 = 0, NZ_BF16 = 1, NZ_F16 = 2 } nz_float_type;

typedef enum { NZ_MX4_NEAREST = 0, NZ_MX4_STOCHASTIC = 1 } nz_mx4_rounding;

typedef enum { NZ_MX4_PRODUCT = 0, NZ_MX4_LINEAR = 1, NZ_MX4_GRAD = 2 } nz_mx4_kind;

/* A matrix in device memory; the structure itself is read on the host during the call only. */
typedef struct {
    void*  codes;
    void*  scales;
    size_t pitch;                /* blocks from one row to the next */
} nz_mx4_matrix;

/* Host, pure.  The least pitch of a matrix with `cols` columns: ceil(cols / 32), up to a multiple of 4.  0 for cols = 0. */
size_t nz_mx4_pitch(size_t cols);

/*
 * d_in[r * ld + c] (rows x cols floats of `type`, ld >= cols elements from one row to the next) into four bits.  With p the
 * largest magnitude of a block and E = floor(log2 p) - 2:
 *   NZ_MX4_NEAREST     scale 2^E; each element to the nearest multiple that a code stands for, ties to the even code,
 *                      magnitudes above 6 * 2^E (they are below 8 * 2^E) to 6 * 2^E.
 *   NZ_MX4_STOCHASTIC  scale 2^E, or 2^(E+1) where p > 6 * 2^E, so that no element lies above the largest code; an element
 *                      between two neighbours takes the upper with probability its distance from the lower over theirs, to
 *                      within 2^-17: E[value] = x.  Elements 2i and 2i + 1 of the matrix (rows of whole blocks one after
 *                      another, whatever the pitch) take the low and the high half of fmix32(lo32(i) ^ fmix32(seed +
 *                      0x9E3779B9 * hi32(i))), u, and go up where (u + 1/2) / 2^16 is less than that share.
 * E is held within [-127, 125]: elements below 2^-129 may become 0, and under NZ_MX4_STOCHASTIC those above 6 * 2^125 become
 * that.  A block with an infinity or NaN gets s = 255 and codes 0.  `seed` is not used by NZ_MX4_NEAREST.
 */
nz_status nz_mx4_quantize(const void* d_in, nz_float_type type, size_t rows, size_t cols, size_t ld, nz_mx4_rounding rounding,
                          uint32_t seed, const nz_mx4_matrix* out, void* stream);

/* The floats that a matrix stands for: exact in NZ_F32 and NZ_BF16, rounded once (to nearest even) in NZ_F16.  Magnitudes of 2^128 and more (4 and
 * 6 under s = 253; 2, 3, 4 and 6 under s = 254; no call here writes such a scale) are infinite in all three, and so they are in the sums below. */
nz_status nz_mx4_dequantize(const nz_mx4_matrix* in, size_t rows, size_t cols, void* d_out, nz_float_type type, size_t ld,
                            void* stream);

/*
 * The sum of k matrices (1 <= k <= 64; `in` is a HOST array) and, where d_local is not NULL, of the rank's own float32 data
 * d_local[r * ld_local + c], as nz_reduce_k and nz_reduce_local fold streams: float32, in the order given, d_local last.
 * nz_mx4_reduce_k writes the sum in four bits again, rounded as nz_mx4_quantize would; `out` may be one of the inputs (same
 * codes, scales and pitch).  nz_mx4_sum_k writes it as floats of `type`, rounded once; ld >= cols.  ld_local is not used
 * where d_local is NULL.
 */
nz_status nz_mx4_reduce_k(const nz_mx4_matrix* in, uint32_t k, const float* d_local, size_t ld_local, size_t rows, size_t cols,
                          nz_mx4_rounding rounding, uint32_t seed, const nz_mx4_matrix* out, void* stream);
nz_status nz_mx4_sum_k(const nz_mx4_matrix* in, uint32_t k, const float* d_local, size_t ld_local, size_t rows, size_t cols,
                       void* d_out, nz_float_type type, size_t ld, void* stream);

/* Host, pure.  Workspace bytes of the products below (may be 0: then d_ws may be NULL); `left` is the type of the float
 * operand, not used by NZ_MX4_PRODUCT.  (size_t)-1 for sizes that the products refuse.  Enough for any row length and address: floats of more than
 * 32 rows (NZ_MX4_GRAD: 16) are laid out in it as terms of bfloat16, and bfloat16 counts too, though rows at multiples of 16 bytes whose length
 * is a multiple of 8 elements are read where they lie. */
size_t nz_mx4_workspace_bytes(nz_mx4_kind kind, nz_float_type left, size_t M, size_t N, size_t K);

/*
 * d_c[m * ldc + n] = sum over k of A[m][k] * B[n][k]: M x K and N x K matrices in four bits, C floats of `type`.  Products
 * are exact, sums are float32 (in an order that depends on the sizes alone), C is rounded once.
 */
nz_status nz_mx4_product(const nz_mx4_matrix* a, const nz_mx4_matrix* b, size_t M, size_t N, size_t K, void* d_c,
                         nz_float_type type, size_t ldc, void* d_ws, size_t ws_bytes, void* stream);

/* The same with floats on the left: C = X B^T, X[m][k] = d_x[m * ldx + k] of type x_type.  X is not rounded,
 * but bits of a float32 below 2^-133 are cut off (it is multiplied in terms of bfloat16).  Elements of B of 2^128 and more, which are infinite in
 * nz_mx4_dequantize, have no finite products here and in nz_mx4_grad (infinite, or NaN as those of an infinity and 0); nz_mx4_product
 * multiplies them as they are. */
nz_status nz_mx4_linear(const void* d_x, nz_float_type x_type, size_t ldx, const nz_mx4_matrix* b, size_t M, size_t N, size_t K,
                        void* d_c, nz_float_type type, size_t ldc, void* d_ws, size_t ws_bytes, void* stream);

/*
 * Gradient of both for the left operand: d_da[m * ldda + k] = sum over n of G[m][n] * B[n][k], G[m][n] = d_g[m * ldg + n] the
 * gradient of C.  That of nz_mx4_product for B is the same call with the transpose of G, A for B, and N and M exchanged.
 */
nz_status nz_mx4_grad(const void* d_g, nz_float_type g_type, size_t ldg, const nz_mx4_matrix* b, size_t M, size_t N, size_t K,
                      void* d_da, nz_float_type type, size_t ldda, void* d_ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NZ_MX4_H */
