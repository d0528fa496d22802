// nz_mx4.hip -- conversion of floats into microscaled 4-bit blocks and back, and sums of several such matrices.
//
// A thread holds 8 elements of a block (an octet: 4 bytes of codes), four neighbouring lanes hold the block, and a wave 16 blocks: the
// block's peak takes two exchanges inside groups of four lanes, and codes leave as whole words.  One pass over the data; all of it is bound
// by memory.
#include "nz_mx4.hpp"

namespace nz {

namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kOctets = 2;                       // octets of a thread, kThreads apart (four: 60.4 us instead of 55.8 for 256 MB)

struct Place { uint64_t row; uint32_t blk, q; bool live; };

// Octet number o of a group of rows: which row, which block of it, which quarter of the block.
__device__ inline Place place(const MxRows& R, uint32_t o, uint32_t limit) {
    Place p;
    const uint32_t b = o >> 2;
    p.q = o & 3u;
    p.live = b < limit;
    if (R.rows == 1) { p.row = 0; p.blk = b; return p; }
    const uint32_t r = __umulhi(b << 3, R.nb_mul) >> R.nb_shift;         // b / nb
    p.blk = b - r * R.nb;
    p.row = (uint64_t)blockIdx.y * R.group + r;
    return p;
}

__device__ inline uint32_t blocks_here(const MxRows& R) {
    const uint64_t left = R.rows - (uint64_t)blockIdx.y * R.group;
    return (uint32_t)(left < R.group ? left : R.group) * R.nb;
}

// Octets of the rows before this group's.
__device__ inline uint64_t octets_before(const MxRows& R) { return (uint64_t)blockIdx.y * R.group * R.nb * 4; }

// 16 bytes at any address that suits their elements: rows may start anywhere, and the memory pipeline splits what crosses a line.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 __attribute__((aligned(4))) u32x4_by4;
typedef u32x4 __attribute__((aligned(2))) u32x4_by2;
template <int T> struct Words { typedef u32x4_by2 type; };
template <> struct Words<F32> { typedef u32x4_by4 type; };

template <int T> __device__ inline float as_float(uint32_t v) {
    if (T == BF16) return __uint_as_float(v << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)v);
}

// Eight floats of a row from column c on; those past the row's end are 0.
template <int T> __device__ inline void load8(const void* in, uint64_t row, uint64_t ld, uint64_t c, uint64_t cols, float* x) {
    constexpr uint32_t sz = float_bytes(T);
    const uint8_t* p = reinterpret_cast<const uint8_t*>(in) + (row * ld + c) * sz;
    if (c + 8 <= cols) {
        const typename Words<T>::type* w = reinterpret_cast<const typename Words<T>::type*>(p);
        const u32x4 u = w[0];
        if (T == F32) {
            const u32x4 v = w[1];
#pragma unroll
            for (int i = 0; i < 4; i++) { x[i] = __uint_as_float(u[i]); x[4 + i] = __uint_as_float(v[i]); }
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++) { x[2 * i] = as_float<T>(u[i] & 0xFFFFu); x[2 * i + 1] = as_float<T>(u[i] >> 16); }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (T == F32) x[i] = c + i < cols ? reinterpret_cast<const float*>(p)[i] : 0.0f;
            else x[i] = c + i < cols ? as_float<T>(reinterpret_cast<const uint16_t*>(p)[i]) : 0.0f;
        }
    }
}

template <int T> __device__ inline uint32_t to16(float v) {
    if (T == BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    return __builtin_bit_cast(uint16_t, (_Float16)v);
}

// N floats, packed in w, of a row from column c on; those past the row's end are left alone.  PAST: around the caches.
template <int T, int N, bool PAST> __device__ inline void store_words(void* out, uint64_t row, uint64_t ld, uint64_t c, uint64_t cols, u32x4 w) {
    constexpr uint32_t sz = float_bytes(T);
    static_assert(N * sz == 16, "");
    uint8_t* p = reinterpret_cast<uint8_t*>(out) + (row * ld + c) * sz;
    typename Words<T>::type* const words = reinterpret_cast<typename Words<T>::type*>(p);
    if (c + N <= cols) {
        if (PAST) __builtin_nontemporal_store(w, words);
        else *words = w;
    } else
#pragma unroll
        for (int i = 0; i < N; i++)
            if (c + i < cols) {
                if (T == F32) reinterpret_cast<uint32_t*>(p)[i] = w[i % 4];
                else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)(w[i / 2 % 4] >> (i % 2 * 16));
            }
}

// The largest of four neighbouring lanes' values.
__device__ inline uint32_t max_of_four(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));      // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
}

// One element, stochastically: its code, for a block whose scale has this inverse and a draw of 16 bits.  Its magnitude is scaled so that 1 in
// units of the block becomes 2^-126: then the float's own bits are the grid, with its octaves of two steps each above 1 and, since floats
// below 2^-126 are evenly spaced, the even steps of 1/2 below.  The code is the top of these bits and the share of the distance the 22 bits
// below; adding 2^22 - 33 - 64 u to them carries exactly where (u + 1/2) / 2^16 < share.  What the scaling rounded down (`rest`) counts as
// one more, since the border is a whole number: bits of the magnitude rounded up are above it exactly where the magnitude is.  (Products with
// powers of two: an instruction that adds to the exponent takes four times as long.  The first one is exact but for magnitudes far below any
// border.)
__device__ inline uint32_t stochastic_code(float v, float inverse, uint32_t u) {
    const float a = fabsf(v) * inverse, y = a * 0x1p-126f;
    const uint32_t rest = y * 0x1p126f < a ? 1u : 0u;
    return min((__float_as_uint(y) + (0x3FFFDFu - (u << 6)) + rest) >> 22, 7u);
}

// The keys of a workgroup's draws: octet number `base` + o, 4 pairs of elements an octet; fewer than 2^30 octets lie in a workgroup, so that
// the upper half of a pair's number takes two values at most.
struct Draws {
    uint64_t base;
    uint32_t hi, key0, key1;
    __device__ inline Draws(uint32_t seed, uint64_t first) : base(first), hi((uint32_t)(first >> 30)) {
        key0 = fmix32(seed + 0x9E3779B9u * hi);
        key1 = fmix32(seed + 0x9E3779B9u * (hi + 1u));
    }
    __device__ inline void of(uint32_t o, uint32_t (&h)[4]) const {
        const uint64_t e = base + o;
        const uint32_t key = (uint32_t)(e >> 30) == hi ? key0 : key1, lo = (uint32_t)e * 4u;
#pragma unroll
        for (uint32_t i = 0; i < 4; i++) h[i] = fmix32((lo + i) ^ key);
    }
};

// Eight elements into a word of codes; the block's scale byte comes back in s.  o: the octet's number in the workgroup, for the draws.
template <bool SR> __device__ inline uint32_t encode8(const float* x, const Draws& D, uint32_t o, uint32_t& s) {
    uint32_t peak = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) peak = max(peak, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    peak = max_of_four(peak);
    const uint32_t ex = peak >> 23;
    int b = (int)ex - 2;
    if (SR) b += (peak & 0x7FFFFFu) > 0x400000u ? 1 : 0;
    b = min(max(b, 0), 252);
    const bool bad = ex == 255u;
    uint32_t w = 0;
    if (!SR) {
        const float sc = mx_scale((uint32_t)b);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], sc, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], sc, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], sc, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], sc, 3);
    } else {
        const float inverse = __uint_as_float((uint32_t)(254 - b) << 23);
        uint32_t h[4];
        D.of(o, h);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t c = stochastic_code(x[i], inverse, i % 2 ? h[i / 2] >> 16 : h[i / 2] & 0xFFFFu);
            w |= (c | (__float_as_uint(x[i]) >> 28 & 8u)) << (4 * i);
        }
    }
    s = bad ? 255u : (uint32_t)b;
    return bad ? 0u : w;
}

__device__ inline void decode8(uint32_t w, uint32_t s, float* x) {
    const float sc = mx_scale(s);
    f32x2 v;
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 0); x[0] = v[0]; x[1] = v[1];
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 1); x[2] = v[0]; x[3] = v[1];
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 2); x[4] = v[0]; x[5] = v[1];
    v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, sc, 3); x[6] = v[0]; x[7] = v[1];
}

template <int T, bool SR>
__global__ __launch_bounds__(kThreads) void k_mx_quantize(MxConvertArgs A) {
    const uint32_t limit = blocks_here(A.R);
    const uint32_t first = blockIdx.x * (kThreads * kOctets) + threadIdx.x;
    Place p[kOctets];
    float x[kOctets][8];
    for (uint32_t u = 0; u < kOctets; u++) {
        p[u] = place(A.R, first + u * kThreads, limit);
        if (p[u].live) load8<T>(A.in, p[u].row, A.ld, p[u].blk * 32ull + p[u].q * 8u, A.R.cols, x[u]);
    }
    const Draws D(A.seed, octets_before(A.R) + blockIdx.x * (kThreads * kOctets));
    for (uint32_t u = 0; u < kOctets; u++) {
        if (!p[u].live) continue;                     // (all four lanes of a block)
        uint32_t s;
        const uint32_t w = encode8<SR>(x[u], D, u * kThreads + threadIdx.x, s);
        const uint64_t at = p[u].row * A.pitch + p[u].blk;
        *reinterpret_cast<uint32_t*>(A.codes + at * 16 + p[u].q * 4) = w;
        if (p[u].q == 0) A.scales[at] = (uint8_t)s;
    }
}

// OUT: the floats' type, or -1 for four bits.  WAY: four bits stochastically, floats around the caches.  MAX: the most operands; up to kMxSomeOperands of them are asked for at once.
template <int OUT, bool WAY, uint32_t MAX>
__global__ __launch_bounds__(kThreads) void k_mx_sum(MxSumArgs<MAX> A) {
    const uint32_t limit = blocks_here(A.R);
    constexpr uint32_t U = kOctets;
    constexpr uint32_t G = MAX < kMxSomeOperands ? MAX : kMxSomeOperands;
    const uint32_t first = blockIdx.x * (kThreads * U) + threadIdx.x;
    Place p[U];
    float acc[U][8];
#pragma unroll
    for (uint32_t u = 0; u < U; u++) p[u] = place(A.R, first + u * kThreads, limit);
    for (uint32_t i0 = 0; i0 < A.k; i0 += G) {
        uint32_t w[G][U], s[G][U];
#pragma unroll
        for (uint32_t i = 0; i < G; i++)
            if (i0 + i < A.k)
#pragma unroll
                for (uint32_t u = 0; u < U; u++)
                    if (p[u].live) {
                        const uint64_t at = p[u].row * A.in[i0 + i].pitch + p[u].blk;
                        w[i][u] = *reinterpret_cast<const uint32_t*>(A.in[i0 + i].codes + at * 16 + p[u].q * 4);
                        s[i][u] = A.in[i0 + i].scales[at];
                    }
#pragma unroll
        for (uint32_t i = 0; i < G; i++)
            if (i0 + i < A.k)
#pragma unroll
                for (uint32_t u = 0; u < U; u++) {
                    float x[8];
                    decode8(w[i][u], s[i][u], x);
#pragma unroll
                    for (int j = 0; j < 8; j++) acc[u][j] = i0 + i ? acc[u][j] + x[j] : x[j];
                }
    }
    if (A.local)
#pragma unroll
        for (uint32_t u = 0; u < U; u++)
            if (p[u].live) {
                float x[8];
                load8<F32>(A.local, p[u].row, A.ld_local, p[u].blk * 32ull + p[u].q * 8u, A.R.cols, x);
#pragma unroll
                for (int j = 0; j < 8; j++) acc[u][j] += x[j];
            }
    if constexpr (OUT == F32) {
        // a lane's eight floats are 32 bytes; exchanged through shared memory, a wave's stores are of 16 bytes next to each other
        __shared__ __attribute__((aligned(16))) u32x4 turn[kThreads * 2];
        u32x4* const mine = turn + threadIdx.x / 64 * 128;
        const uint32_t lane = threadIdx.x % 64;
#pragma unroll
        for (uint32_t u = 0; u < U; u++) {
#pragma unroll
            for (uint32_t h = 0; h < 2; h++) {
                u32x4 v;
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = __float_as_uint(acc[u][h * 4 + j]);
                mine[(lane * 2 + h) ^ (lane / 8 & 1)] = v;                 // (so that 16 lanes use all banks)
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (uint32_t h = 0; h < 2; h++) {
                const uint32_t c = h * 64 + lane;                         // quarter c % 2 of the octet of lane c / 2
                const u32x4 v = mine[c ^ (c / 16 & 1)];
                const Place o = place(A.R, first - lane + u * kThreads + c / 2, limit);
                if (o.live) store_words<F32, 4, WAY>(A.out, o.row, A.ld, o.blk * 32ull + o.q * 8u + c % 2 * 4, A.R.cols, v);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    } else {
        const Draws D(A.seed, octets_before(A.R) + blockIdx.x * (kThreads * U));
#pragma unroll
        for (uint32_t u = 0; u < U; u++) {
            if (!p[u].live) continue;
            if constexpr (OUT >= 0) {
                u32x4 v;
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = to16<OUT>(acc[u][2 * j]) | to16<OUT>(acc[u][2 * j + 1]) << 16;
                store_words<OUT, 8, WAY>(A.out, p[u].row, A.ld, p[u].blk * 32ull + p[u].q * 8u, A.R.cols, v);
            } else {
                uint32_t s;
                const uint32_t w = encode8<WAY>(acc[u], D, u * kThreads + threadIdx.x, s);
                const uint64_t at = p[u].row * A.pitch + p[u].blk;
                *reinterpret_cast<uint32_t*>(A.codes + at * 16 + p[u].q * 4) = w;
                if (p[u].q == 0) A.scales[at] = (uint8_t)s;
            }
        }
    }
}

dim3 grid_of(const MxRows& R) {
    const uint64_t rows = R.rows < R.group ? R.rows : R.group;
    return dim3((uint32_t)((rows * R.nb * 4 + kThreads * kOctets - 1) / (kThreads * kOctets)), (uint32_t)((R.rows + R.group - 1) / R.group));
}

template <int T> void quantize_type(const MxConvertArgs& A, bool sr, hipStream_t st) {
    if (sr) hipLaunchKernelGGL((k_mx_quantize<T, true>), grid_of(A.R), dim3(kThreads), 0, st, A);
    else hipLaunchKernelGGL((k_mx_quantize<T, false>), grid_of(A.R), dim3(kThreads), 0, st, A);
}

}  // namespace

hipError_t launch_mx_quantize(const MxConvertArgs& A, int type, bool sr, hipStream_t st) {
    if (type == F32) quantize_type<F32>(A, sr, st);
    else if (type == BF16) quantize_type<BF16>(A, sr, st);
    else quantize_type<F16>(A, sr, st);
    return hipGetLastError();
}

template <int OUT, uint32_t MAX> static void sum_out(const MxSumArgs<MAX>& A, bool way, hipStream_t st) {
    if (way) hipLaunchKernelGGL((k_mx_sum<OUT, true, MAX>), grid_of(A.R), dim3(kThreads), 0, st, A);
    else hipLaunchKernelGGL((k_mx_sum<OUT, false, MAX>), grid_of(A.R), dim3(kThreads), 0, st, A);
}

template <uint32_t MAX> hipError_t launch_mx_sum(const MxSumArgs<MAX>& A, int type, bool way, hipStream_t st) {
    if (type == F32) sum_out<F32, MAX>(A, way, st);
    else if (type == BF16) sum_out<BF16, MAX>(A, way, st);
    else if (type == F16) sum_out<F16, MAX>(A, way, st);
    else sum_out<-1, MAX>(A, way, st);
    return hipGetLastError();
}
template hipError_t launch_mx_sum<1>(const MxSumArgs<1>&, int, bool, hipStream_t);
template hipError_t launch_mx_sum<kMxSomeOperands>(const MxSumArgs<kMxSomeOperands>&, int, bool, hipStream_t);
template hipError_t launch_mx_sum<kMxMaxOperands>(const MxSumArgs<kMxMaxOperands>&, int, bool, hipStream_t);

}  // namespace nz
