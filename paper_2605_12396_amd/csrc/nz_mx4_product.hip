// nz_mx4_product.hip -- products with microscaled 4-bit matrices: both sides in four bits, floats on the left, and the gradient for the left.
//
// All three are C[m][j] = sum over i of left[m][i] * right[j][i]; in the gradient right is B seen by its columns, right[j][i] = B[i][j].
// `inner` is the length of the sum, `outer` the number of columns of C.
#include "nz_mx4.hpp"
#include <type_traits>

namespace nz {

namespace {

enum : int { PRODUCT = 0, LINEAR = 1, GRAD = 2 };

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr uint32_t kNowhere = 0x80000000u;        // an offset behind every buffer: loads from it give 0

// Offsets are below 2^31 (256 rows of at most 8 MiB), so a descriptor of that size checks nothing but kNowhere.
__device__ inline rsrc_t buffer_at(const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7FFFFFFF, 0x00027000); }
__device__ inline i32x4 load16(rsrc_t r, uint32_t off) { return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0)); }

struct TileArgs {
    const uint8_t* left; uint64_t left_pitch;             // bytes of a row
    const uint8_t* left_scales; uint64_t left_spitch;     // product
    const uint8_t* right; uint64_t right_pitch;
    const uint8_t* right_scales; uint64_t right_spitch;
    uint64_t M, outer, inner;
    uint32_t terms;                                       // linear, grad: bf16 terms of a float
    uint32_t steps;                                       // terms counted
    uint32_t tiles_m, tiles_j;
    void* c; uint64_t ldc; int c_type;
};

__device__ inline void store_c(const TileArgs& A, uint64_t at, float v) {
    if (A.c_type == F32) reinterpret_cast<float*>(A.c)[at] = v;
    else if (A.c_type == BF16) reinterpret_cast<__bf16*>(A.c)[at] = (__bf16)v;
    else reinterpret_cast<_Float16*>(A.c)[at] = (_Float16)v;
}

// Which tile: neighbouring workgroups go to the 8 XCDs in turn, so each XCD is given a contiguous run of tiles; in it, bands of 8 tiles of
// m are walked along j, so that the 32 tiles that an XCD works on at a time share a few panels of either side in its L2.
__device__ inline void tile_of(const TileArgs& A, uint32_t& tm, uint32_t& tj) {
    const uint32_t total = A.tiles_m * A.tiles_j, id = blockIdx.x;
    const uint32_t q = total / 8, r = total % 8, x = id % 8;
    const uint32_t t = x * q + min(x, r) + id / 8;
    const uint32_t band = t / (8 * A.tiles_j), first = band * 8;
    const uint32_t height = min(8u, A.tiles_m - first), in = t - band * 8 * A.tiles_j;
    tm = first + in % height;
    tj = in / height;
}

// A tile of BM x BN elements of C by four waves, each a quarter of it in tiles of 32 x 32.  A step covers 128 bytes of every row of the
// left: 256 elements in four bits, 64 in bf16.  While a step is multiplied from one half of the shared memory, the next one is on its way
// to registers, and is written to the other half at the step's end.
// Rows lie in shared memory as 8 chunks of 16 bytes, chunk c of row r at c ^ (r ^ r / 8) % 8, so that 8 lanes that read the same chunk of 8
// rows (and, in the gradient, 8 that write the same chunk of every eighth row) use all banks.
// A lane of group g = lane / 32 takes block 4 g + j of a row (product) or elements 32 g + 8 j .. + 7 (linear, grad) in its j-th matrix
// instruction; which elements meet in one instruction does not matter as long as both sides agree.
template <int OP, int BM, int BN>
__global__ __launch_bounds__(256, 1) void k_mx_tile(TileArgs A) {
    constexpr int TM = BM / 64, TN = BN / 64;
    constexpr int LL = BM / 32;                                        // 16-byte loads of the left by a thread
    constexpr int RL = OP == PRODUCT ? BN / 32 : BN / 128;             // of the right (grad: see below)
    constexpr uint32_t RB = OP == LINEAR ? 32 : 128;                   // bytes of a row of the right in shared memory
    constexpr int GC = BN / 32;                                        // grad: columns of a thread's piece, 8 rows deep
    constexpr uint32_t SB = OP == PRODUCT ? 8 : OP == LINEAR ? 2 : 0;  // scales of a row and step
    __shared__ __attribute__((aligned(16))) uint8_t sl[2][BM * 128];
    __shared__ __attribute__((aligned(16))) uint8_t sr[2][BN * RB];
    __shared__ __attribute__((aligned(16))) uint8_t ssl[2][OP == PRODUCT ? BM * 8 : 16];
    __shared__ __attribute__((aligned(16))) uint8_t ssr[2][SB ? BN * SB : 16];

    uint32_t tm, tj;
    tile_of(A, tm, tj);
    const uint64_t m0 = (uint64_t)tm * BM, j0 = (uint64_t)tj * BN;
    const uint32_t t = threadIdx.x, lane = t % 64, wave = t / 64;
    const uint32_t rows = (uint32_t)min(A.M - m0, (uint64_t)BM), cols = (uint32_t)min(A.outer - j0, (uint64_t)BN);
    const uint32_t nb = (uint32_t)((A.inner + 31) / 32);

    // ---- where a thread's loads come from: rows past the end read the last one, and are not stored ----
    const uint8_t* const left = A.left + m0 * A.left_pitch;
    uint32_t lo[LL];
    for (int i = 0; i < LL; i++) lo[i] = min(t / 8 + 32 * i, rows - 1) * (uint32_t)A.left_pitch + t % 8 * 16;
    const uint8_t* const right = OP == GRAD ? A.right + j0 / 2 : A.right + j0 * A.right_pitch;
    uint32_t ro[RL < 1 ? 1 : RL];
    if (OP == PRODUCT) for (int i = 0; i < RL; i++) ro[i] = min(t / 8 + 32 * i, cols - 1) * (uint32_t)A.right_pitch + t % 8 * 16;
    if (OP == LINEAR) for (int i = 0; i < RL; i++) ro[i] = min(t / 2 + 128 * i, cols - 1) * (uint32_t)A.right_pitch + t % 2 * 16;
    const uint32_t deep = t / 32, across = t % 32;                     // grad: rows 8 deep .. + 7, columns GC across .. + GC - 1
    const bool inside = OP != GRAD || across * GC < (uint32_t)((A.outer + 31) / 32 * 32 - j0);

    i32x4 lv[LL], rv[RL < 1 ? 1 : RL];
    uint32_t gw[8], gs[8];
    uint64_t slv = 0, srv = 0;

    auto fetch = [&](uint32_t s) {
        const uint32_t rs = OP == PRODUCT ? s : s / A.terms;           // step of the right
        const rsrc_t bl = buffer_at(left + (uint64_t)s * 128);
        const bool l_in = OP == PRODUCT ? s * 8 + t % 8 < nb : A.terms > 1 || (uint64_t)rs * 64 + t % 8 * 8 < A.inner;
        for (int i = 0; i < LL; i++) lv[i] = load16(bl, l_in ? lo[i] : kNowhere);
        if (OP == PRODUCT) {
            const rsrc_t br = buffer_at(right + (uint64_t)s * 128);
            for (int i = 0; i < RL; i++) rv[i] = load16(br, l_in ? ro[i] : kNowhere);
            // scales: a thread's row of either side, 8 blocks; those past the row's end become 0 (the codes there are 0)
            const rsrc_t sl_ = buffer_at(A.left_scales + m0 * A.left_spitch + (uint64_t)s * 8);
            const rsrc_t sr_ = buffer_at(A.right_scales + j0 * A.right_spitch + (uint64_t)s * 8);
            const uint32_t left_here = nb - s * 8;
            const uint32_t a = min(t % BM, rows - 1) * (uint32_t)A.left_spitch, b = min(t % BN, cols - 1) * (uint32_t)A.right_spitch;
            const uint32_t hi_in = left_here > 4 ? 4u : kNowhere;
            const uint32_t a0 = __builtin_amdgcn_raw_buffer_load_b32(sl_, a, 0, 0), a1 = __builtin_amdgcn_raw_buffer_load_b32(sl_, hi_in == 4u ? a + 4 : kNowhere, 0, 0);
            const uint32_t b0 = __builtin_amdgcn_raw_buffer_load_b32(sr_, b, 0, 0), b1 = __builtin_amdgcn_raw_buffer_load_b32(sr_, hi_in == 4u ? b + 4 : kNowhere, 0, 0);
            const uint64_t keep = left_here >= 8 ? ~0ull : (1ull << (8 * left_here)) - 1;
            slv = ((uint64_t)a1 << 32 | a0) & keep;
            srv = ((uint64_t)b1 << 32 | b0) & keep;
        } else if (OP == LINEAR) {
            const rsrc_t br = buffer_at(right + (uint64_t)rs * 32);
            const bool r_in = rs * 2 + t % 2 < nb;
            for (int i = 0; i < RL; i++) rv[i] = load16(br, r_in ? ro[i] : kNowhere);
            const rsrc_t sr_ = buffer_at(A.right_scales + j0 * A.right_spitch + (uint64_t)rs * 2);
            const uint32_t b = __builtin_amdgcn_raw_buffer_load_b16(sr_, min(t % BN, cols - 1) * (uint32_t)A.right_spitch, 0, 0);
            srv = rs * 2 + 1 < nb ? b : b & 0xFFu;
        } else {
            const rsrc_t br = buffer_at(right + (uint64_t)rs * 64 * A.right_pitch);
            const rsrc_t sr_ = buffer_at(A.right_scales + j0 / 32 + (uint64_t)rs * 64 * A.right_spitch);
            for (int r = 0; r < 8; r++) {
                const uint32_t row = deep * 8 + r;
                const bool in = inside && (uint64_t)rs * 64 + row < A.inner;
                const uint32_t off = in ? row * (uint32_t)A.right_pitch + across * (GC / 2) : kNowhere;
                gw[r] = GC == 8 ? __builtin_amdgcn_raw_buffer_load_b32(br, off, 0, 0) : (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(br, off, 0, 0);
                gs[r] = __builtin_amdgcn_raw_buffer_load_b8(sr_, in ? row * (uint32_t)A.right_spitch + across * GC / 32 : kNowhere, 0, 0);
            }
        }
    };

    auto swz = [](uint32_t row, uint32_t chunk) { return row * 128 + (chunk ^ ((row ^ row >> 3) & 7)) * 16; };

    auto put = [&](int h) {
        for (int i = 0; i < LL; i++) *reinterpret_cast<i32x4*>(&sl[h][swz(t / 8 + 32 * i, t % 8)]) = lv[i];
        if (OP == PRODUCT) {
            for (int i = 0; i < RL; i++) *reinterpret_cast<i32x4*>(&sr[h][swz(t / 8 + 32 * i, t % 8)]) = rv[i];
            if (t < BM) *reinterpret_cast<uint64_t*>(&ssl[h][t * 8]) = slv;
            if (t < BN) *reinterpret_cast<uint64_t*>(&ssr[h][t * 8]) = srv;
        } else if (OP == LINEAR) {
            for (int i = 0; i < RL; i++) *reinterpret_cast<i32x4*>(&sr[h][(t / 2 + 128 * i) * 32 + t % 2 * 16]) = rv[i];
            if (t < BN) *reinterpret_cast<uint16_t*>(&ssr[h][t * 2]) = (uint16_t)srv;
        } else {
            // 8 rows x GC columns of codes become GC rows x 8 of bf16
            uint32_t p[8][GC / 2];
            for (int r = 0; r < 8; r++) {
                const float sc = mx_scale(gs[r]);
                p[r][0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(gw[r], sc, 0));
                p[r][1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(gw[r], sc, 1));
                if constexpr (GC == 8) {
                    p[r][2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(gw[r], sc, 2));
                    p[r][3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(gw[r], sc, 3));
                }
            }
            for (int c = 0; c < GC; c++) {
                i32x4 v;
                for (int d = 0; d < 4; d++)
                    v[d] = c & 1 ? __builtin_amdgcn_perm(p[2 * d + 1][c / 2], p[2 * d][c / 2], 0x07060302u)
                                 : __builtin_amdgcn_perm(p[2 * d + 1][c / 2], p[2 * d][c / 2], 0x05040100u);
                *reinterpret_cast<i32x4*>(&sr[h][swz(across * GC + c, deep)]) = v;
            }
        }
    };

    f32x16 acc[TM][TN];
#pragma unroll
    for (int a = 0; a < TM; a++)
#pragma unroll
        for (int b = 0; b < TN; b++) acc[a][b] = f32x16{};
    const uint32_t g = lane / 32, l32 = lane % 32;
    const uint32_t wm = wave / 2 * (BM / 2), wj = wave % 2 * (BN / 2);

    auto multiply = [&](int h) {
        if constexpr (OP == PRODUCT) {
            int sa[TM], sb[TN];
            for (int a = 0; a < TM; a++) sa[a] = *reinterpret_cast<const int*>(&ssl[h][(wm + a * 32 + l32) * 8 + g * 4]);
            for (int b = 0; b < TN; b++) sb[b] = *reinterpret_cast<const int*>(&ssr[h][(wj + b * 32 + l32) * 8 + g * 4]);
            auto block = [&](auto J) {
                constexpr int j = decltype(J)::value;
                i32x4 x[TM], y[TN];
                for (int a = 0; a < TM; a++) x[a] = *reinterpret_cast<const i32x4*>(&sl[h][swz(wm + a * 32 + l32, g * 4 + j)]);
                for (int b = 0; b < TN; b++) y[b] = *reinterpret_cast<const i32x4*>(&sr[h][swz(wj + b * 32 + l32, g * 4 + j)]);
                for (int a = 0; a < TM; a++)
                    for (int b = 0; b < TN; b++) {
                        const i32x8 xa = { x[a][0], x[a][1], x[a][2], x[a][3], 0, 0, 0, 0 }, yb = { y[b][0], y[b][1], y[b][2], y[b][3], 0, 0, 0, 0 };
                        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(xa, yb, acc[a][b], 4, 4, j, sa[a], j, sb[b]);
                    }
            };
            block(std::integral_constant<int, 0>{}); block(std::integral_constant<int, 1>{});
            block(std::integral_constant<int, 2>{}); block(std::integral_constant<int, 3>{});
        } else {
            i32x4 w[TN];
            float sc[TN];
            if (OP == LINEAR)
                for (int b = 0; b < TN; b++) {
                    w[b] = *reinterpret_cast<const i32x4*>(&sr[h][(wj + b * 32 + l32) * 32 + g * 16]);
                    sc[b] = mx_scale(ssr[h][(wj + b * 32 + l32) * 2 + g]);
                }
            for (int j = 0; j < 4; j++) {
                bf16x8 x[TM], y[TN];
                for (int a = 0; a < TM; a++) x[a] = *reinterpret_cast<const bf16x8*>(&sl[h][swz(wm + a * 32 + l32, g * 4 + j)]);
                for (int b = 0; b < TN; b++) {
                    if (OP == GRAD) {
                        y[b] = *reinterpret_cast<const bf16x8*>(&sr[h][swz(wj + b * 32 + l32, g * 4 + j)]);
                    } else {
                        i32x4 v;
                        v[0] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[b][j], sc[b], 0));
                        v[1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[b][j], sc[b], 1));
                        v[2] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[b][j], sc[b], 2));
                        v[3] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[b][j], sc[b], 3));
                        y[b] = __builtin_bit_cast(bf16x8, v);
                    }
                }
                for (int a = 0; a < TM; a++)
                    for (int b = 0; b < TN; b++) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[a], y[b], acc[a][b], 0, 0, 0);
            }
        }
    };

    fetch(0);
    put(0);
    for (uint32_t s = 0; s < A.steps; s++) {
        __syncthreads();
        if (s + 1 < A.steps) fetch(s + 1);
        multiply(s & 1);
        if (s + 1 < A.steps) put((s + 1) & 1);
    }

#pragma unroll
    for (int a = 0; a < TM; a++)
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const uint32_t m = wm + a * 32 + i / 4 * 8 + g * 4 + i % 4;
#pragma unroll
            for (int b = 0; b < TN; b++) {
                const uint32_t j = wj + b * 32 + l32;
                if (m < rows && j < cols) store_c(A, (m0 + m) * A.ldc + j0 + j, acc[a][b][i]);
            }
        }
}

// Floats of the left as bf16 terms that add up to them: one for bf16, two for fp16 (11 bits), three for float32 (24 bits).  Each term
// takes the top of what is left, cut off (not rounded, which could carry past the largest float32), so every difference is exact; an
// infinity or NaN is its first term alone.  Rows become whole steps of 64 elements, term after term in a step, zeros behind the end.
template <int T>
__global__ __launch_bounds__(256) void k_mx_terms(const void* x, uint64_t ldx, uint64_t M, uint64_t inner, uint32_t chunks, uint16_t* out) {
    constexpr int terms = T == F32 ? 3 : T == F16 ? 2 : 1;
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;               // 8 elements
    const uint64_t per_row = (uint64_t)chunks * 8;
    const uint64_t m = id / per_row;
    if (m >= M) return;
    const uint64_t o = id % per_row, i0 = o * 8;
    uint32_t w[terms][4];
    for (int i = 0; i < 8; i++) {
        float v = 0.0f;
        if (i0 + i < inner) {
            const uint64_t at = m * ldx + i0 + i;
            if (T == F32) v = reinterpret_cast<const float*>(x)[at];
            else if (T == F16) v = (float)reinterpret_cast<const _Float16*>(x)[at];
            else v = __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(x)[at] << 16);
        }
        const bool plain = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
        for (int q = 0; q < terms; q++) {
            uint32_t top = __float_as_uint(v) & 0xFFFF0000u;
            if (q == 0 && v != v) top |= 0x00400000u;
            if (q > 0 && !plain) top = 0;
            v -= __uint_as_float(top);
            if (i % 2 == 0) w[q][i / 2] = top >> 16; else w[q][i / 2] |= top;
        }
    }
    uint16_t* const at = out + m * chunks * 64 * terms + (o / 8) * 64 * terms + o % 8 * 8;
    for (int q = 0; q < terms; q++) *reinterpret_cast<uint4*>(at + q * 64) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
}

template <int OP> hipError_t launch_tiles(TileArgs& T, hipStream_t st) {
    auto count = [&](uint32_t bm, uint32_t bn) {
        T.tiles_m = (uint32_t)((T.M + bm - 1) / bm); T.tiles_j = (uint32_t)((T.outer + bn - 1) / bn);
        return T.tiles_m * T.tiles_j;
    };
    if (count(256, 256) >= 192) hipLaunchKernelGGL((k_mx_tile<OP, 256, 256>), dim3(count(256, 256)), dim3(256), 0, st, T);
    else hipLaunchKernelGGL((k_mx_tile<OP, 128, 128>), dim3(count(128, 128)), dim3(256), 0, st, T);
    return hipGetLastError();
}

// Whether the matrix instructions can be fed from the caller's rows: bf16, rows and their ends at multiples of 16 bytes.
bool fed_directly(const MxProductArgs& A, uint64_t inner, int left) { return left == BF16 && A.ldx % 8 == 0 && inner % 8 == 0; }

}  // namespace

size_t mx_product_workspace(int kind, int left, uint64_t M, uint64_t N, uint64_t K) {
    if (kind == PRODUCT) return 0;
    const uint64_t inner = kind == GRAD ? N : K;
    return (inner + 63) / 64 * 128 * M * (left == F32 ? 3 : left == F16 ? 2 : 1);
}

hipError_t launch_mx_product(const MxProductArgs& A, int kind, int left, hipStream_t st) {
    TileArgs T = {};
    T.M = A.M; T.outer = kind == GRAD ? A.K : A.N; T.inner = kind == GRAD ? A.N : A.K;
    T.c = A.c; T.ldc = A.ldc; T.c_type = A.c_type;
    T.right = A.b.codes; T.right_pitch = A.b.pitch * 16; T.right_scales = A.b.scales; T.right_spitch = A.b.pitch;
    T.terms = 1;
    if (kind == PRODUCT) {
        T.left = A.a.codes; T.left_pitch = A.a.pitch * 16; T.left_scales = A.a.scales; T.left_spitch = A.a.pitch;
        T.steps = (uint32_t)((T.inner + 255) / 256);
        return launch_tiles<PRODUCT>(T, st);
    }
    const uint32_t chunks = (uint32_t)((T.inner + 63) / 64);
    if (fed_directly(A, T.inner, left)) {
        T.left = reinterpret_cast<const uint8_t*>(A.x); T.left_pitch = A.ldx * 2;
    } else {
        T.terms = left == F32 ? 3 : left == F16 ? 2 : 1;
        const uint32_t grid = (uint32_t)((A.M * chunks * 8 + 255) / 256);
        uint16_t* const ws = reinterpret_cast<uint16_t*>(A.ws);
        if (left == F32) hipLaunchKernelGGL((k_mx_terms<F32>), dim3(grid), dim3(256), 0, st, A.x, A.ldx, A.M, T.inner, chunks, ws);
        else if (left == F16) hipLaunchKernelGGL((k_mx_terms<F16>), dim3(grid), dim3(256), 0, st, A.x, A.ldx, A.M, T.inner, chunks, ws);
        else hipLaunchKernelGGL((k_mx_terms<BF16>), dim3(grid), dim3(256), 0, st, A.x, A.ldx, A.M, T.inner, chunks, ws);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        T.left = reinterpret_cast<const uint8_t*>(ws); T.left_pitch = (uint64_t)chunks * 128 * T.terms;
    }
    T.steps = chunks * T.terms;
    return kind == LINEAR ? launch_tiles<LINEAR>(T, st) : launch_tiles<GRAD>(T, st);
}

}  // namespace nz
