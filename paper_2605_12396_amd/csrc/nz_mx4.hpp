// nz_mx4.hpp -- arguments and launchers of the microscaled 4-bit kernels, and the device helpers that they share.
#pragma once
#include "nz_common.hpp"

namespace nz {

enum : int { F32 = 0, BF16 = 1, F16 = 2 };
__host__ __device__ constexpr uint32_t float_bytes(int type) { return type == F32 ? 4u : 2u; }

constexpr uint32_t kMxBlock = 32;                 // elements under one scale
constexpr uint32_t kMxMaxOperands = 64, kMxSomeOperands = 8;

struct MxMat { const uint8_t* codes; const uint8_t* scales; uint64_t pitch; };

// What the elementwise kernels walk over: rows of nb blocks.  Row r starts at block r * pitch of a matrix, at element r * ld of
// floats; kernels number the blocks without the pitch, and find the row by a multiplication (nb_mul, nb_shift).
struct MxRows {
    uint64_t rows, cols;
    uint32_t nb;              // blocks of a row
    uint32_t group;           // rows that one value of blockIdx.y covers: group * nb < 2^29
    uint32_t nb_mul, nb_shift;
};

struct MxConvertArgs {
    MxRows R;
    const void* in; uint64_t ld;
    uint8_t* codes; uint8_t* scales; uint64_t pitch;
    uint32_t seed;
};

// MAX: room for operands.  Arguments are copied to the GPU with every launch, so few operands do not carry room for many.
template <uint32_t MAX> struct MxSumArgs {
    MxRows R;
    MxMat in[MAX]; uint32_t k;
    const float* local; uint64_t ld_local;
    void* out; uint64_t ld;                                               // floats
    uint8_t* codes; uint8_t* scales; uint64_t pitch; uint32_t seed;      // or four bits
};

struct MxProductArgs {
    const void* x; uint64_t ldx;      // floats on the left (linear, grad)
    MxMat a, b;                       // four bits on the left (product), and on the right
    uint64_t M, N, K;
    void* c; uint64_t ldc; int c_type;
    void* ws;
};

hipError_t launch_mx_quantize(const MxConvertArgs& A, int type, bool stochastic, hipStream_t st);
// type: of the floats that are written, or -1 for four bits; way: four bits stochastically, floats around the caches
template <uint32_t MAX> hipError_t launch_mx_sum(const MxSumArgs<MAX>& A, int type, bool way, hipStream_t st);

size_t mx_product_workspace(int kind, int left, uint64_t M, uint64_t N, uint64_t K);
hipError_t launch_mx_product(const MxProductArgs& A, int kind, int left, hipStream_t st);

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 2^(s - 127) as the conversion instructions take a scale: they read the exponent bits alone, 0 as 2^-127 and 255 as NaN.
__device__ inline float mx_scale(uint32_t s) { return __uint_as_float(s << 23); }

}  // namespace nz
