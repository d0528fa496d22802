// nz_mx4_product.hip -- products with microscaled 4-bit matrices: both sides in four bits, floats on the left, and the gradient for the left.
//
// C[m][j] = sum over i of left[m][i] * right[j][i]; in the gradient right is B seen by its columns, right[j][i] = B[i][j].
#include "nz_mx4.hpp"

namespace nz {

namespace {

constexpr uint32_t kTile = 64, kDeep = 32;

__device__ inline float held(const MxMat& m, uint64_t row, uint64_t col, bool scaled) {
    const uint64_t at = row * m.pitch + col / 32;
    const uint32_t byte = m.codes[at * 16 + col % 32 / 2];
    const f32x2 v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(byte, scaled ? mx_scale(m.scales[at]) : 1.0f, 0);
    return col & 1 ? v[1] : v[0];
}

template <int T> __device__ inline float float_at(const void* p, uint64_t i) {
    if (T == F32) return reinterpret_cast<const float*>(p)[i];
    if (T == BF16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
    return (float)reinterpret_cast<const _Float16*>(p)[i];
}

// LEFT: type of the floats on the left, or -1 for four bits.
template <int LEFT, bool GRAD>
__global__ __launch_bounds__(256) void k_mx_product(MxProductArgs A) {
    const uint64_t inner = GRAD ? A.N : A.K, outer = GRAD ? A.K : A.N;
    __shared__ float sl[kDeep][kTile + 1], sr[kDeep][kTile + 1];
    const uint32_t across = (uint32_t)((outer + kTile - 1) / kTile);
    const uint64_t m0 = (uint64_t)(blockIdx.x / across) * kTile, j0 = (uint64_t)(blockIdx.x % across) * kTile;
    const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    __shared__ uint32_t scl[kTile], scr[kTile];        // four bits on both sides: the blocks' scales meet before anything can overflow
    for (uint64_t i0 = 0; i0 < inner; i0 += kDeep) {
        for (uint32_t e = threadIdx.x; e < kTile * kDeep; e += 256) {
            const uint32_t i = e % kDeep, m = e / kDeep;
            float v = 0.0f;
            if (m0 + m < A.M && i0 + i < inner) v = LEFT < 0 ? held(A.a, m0 + m, i0 + i, false) : float_at<LEFT < 0 ? 0 : LEFT>(A.x, (m0 + m) * A.ldx + i0 + i);
            sl[i][m] = v;
            const uint32_t gi = GRAD ? e / kTile : i, gj = GRAD ? e % kTile : m;
            v = 0.0f;
            if (j0 + gj < outer && i0 + gi < inner) v = GRAD ? held(A.b, i0 + gi, j0 + gj, true) : held(A.b, j0 + gj, i0 + gi, LEFT >= 0);
            sr[gi][gj] = v;
        }
        if (LEFT < 0 && threadIdx.x < kTile) {
            scl[threadIdx.x] = m0 + threadIdx.x < A.M ? A.a.scales[(m0 + threadIdx.x) * A.a.pitch + i0 / 32] : 127u;
            scr[threadIdx.x] = j0 + threadIdx.x < outer ? A.b.scales[(j0 + threadIdx.x) * A.b.pitch + i0 / 32] : 127u;
        }
        __syncthreads();
        float part[4][4];
        for (int p = 0; p < 4; p++)
            for (int q = 0; q < 4; q++) part[p][q] = LEFT < 0 ? 0.0f : acc[p][q];
        for (uint32_t i = 0; i < kDeep; i++)
            for (int p = 0; p < 4; p++)
                for (int q = 0; q < 4; q++) part[p][q] = fmaf(sl[i][ty * 4 + p], sr[i][tx * 4 + q], part[p][q]);
        for (int p = 0; p < 4; p++)
            for (int q = 0; q < 4; q++) {
                const uint32_t a = scl[ty * 4 + p], b = scr[tx * 4 + q];
                acc[p][q] = LEFT >= 0 ? part[p][q] : acc[p][q] + (a == 255u || b == 255u ? __uint_as_float(0x7FC00000u) : ldexpf(part[p][q], (int)(a + b) - 254));
            }
        __syncthreads();
    }
    for (int p = 0; p < 4; p++)
        for (int q = 0; q < 4; q++) {
            const uint64_t m = m0 + ty * 4 + p, j = j0 + tx * 4 + q;
            if (m >= A.M || j >= outer) continue;
            const uint64_t at = m * A.ldc + j;
            if (A.c_type == F32) reinterpret_cast<float*>(A.c)[at] = acc[p][q];
            else if (A.c_type == BF16) reinterpret_cast<__bf16*>(A.c)[at] = (__bf16)acc[p][q];
            else reinterpret_cast<_Float16*>(A.c)[at] = (_Float16)acc[p][q];
        }
}

}  // namespace

size_t mx_product_workspace(int, int, uint64_t, uint64_t, uint64_t) { return 0; }

hipError_t launch_mx_product(const MxProductArgs& A, int kind, int left, hipStream_t st) {
    const dim3 g((uint32_t)((A.M + kTile - 1) / kTile * (((kind == 2 ? A.K : A.N) + kTile - 1) / kTile)));
    if (kind == 0) hipLaunchKernelGGL((k_mx_product<-1, false>), g, dim3(256), 0, st, A);
    else if (kind == 1 && left == F32) hipLaunchKernelGGL((k_mx_product<F32, false>), g, dim3(256), 0, st, A);
    else if (kind == 1 && left == BF16) hipLaunchKernelGGL((k_mx_product<BF16, false>), g, dim3(256), 0, st, A);
    else if (kind == 1) hipLaunchKernelGGL((k_mx_product<F16, false>), g, dim3(256), 0, st, A);
    else if (left == F32) hipLaunchKernelGGL((k_mx_product<F32, true>), g, dim3(256), 0, st, A);
    else if (left == BF16) hipLaunchKernelGGL((k_mx_product<BF16, true>), g, dim3(256), 0, st, A);
    else hipLaunchKernelGGL((k_mx_product<F16, true>), g, dim3(256), 0, st, A);
    return hipGetLastError();
}

}  // namespace nz
