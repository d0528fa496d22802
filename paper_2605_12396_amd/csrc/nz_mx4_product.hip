// nz_mx4_product.hip -- products with microscaled 4-bit matrices: both sides in four bits, floats on the left, and the gradient for the left.
//
// All three are C[m][j] = sum over i of left[m][i] * right[j][i]; in the gradient right is B seen by its columns, right[j][i] = B[i][j].
// `inner` is the length of the sum, `outer` the number of columns of C.
#include "nz_mx4.hpp"
#include <algorithm>
#include <type_traits>

namespace nz {

namespace {

enum : int { PRODUCT = 0, LINEAR = 1, GRAD = 2 };

// Steps that are not parted: linear's right lies two steps to a load's line, each of them as many steps as a float has terms.
__host__ __device__ constexpr uint32_t unit_of(int op, uint32_t terms) { return op == LINEAR ? 2 * terms : 1; }

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

constexpr uint32_t kNowhere = 0x80000000u;        // an offset behind every buffer: loads from it give 0

// Offsets are below 2^31 (256 rows of at most 8 MiB), so a descriptor of that size checks nothing but kNowhere.
__device__ inline rsrc_t buffer_at(const void* p) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, 0x7FFFFFFF, 0x00027000); }
__device__ inline i32x4 load16(rsrc_t r, uint32_t off) { return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0)); }

template <int BYTES> __device__ inline void load_lds(rsrc_t r, uint8_t* to, uint32_t off) {       // to: of the wave's first lane
    typedef __attribute__((address_space(3))) void* lds_t;
    if constexpr (BYTES == 16) __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t)to, 16, off, 0, 0, 0);
    else __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t)to, 4, off, 0, 0, 0);
}

template <typename F> __device__ __forceinline__ void unroll4(F f) {
    f(std::integral_constant<int, 0>{}); f(std::integral_constant<int, 1>{}); f(std::integral_constant<int, 2>{}); f(std::integral_constant<int, 3>{});
}

struct TileArgs {
    const uint8_t* left; uint64_t left_pitch;             // bytes of a row
    const uint8_t* left_scales; uint64_t left_spitch;     // product
    const uint8_t* right; uint64_t right_pitch;
    const uint8_t* right_scales; uint64_t right_spitch;
    uint64_t M, outer, inner;
    uint32_t terms, per_term;                             // linear, grad: bf16 terms of a float; 2^31 over that, upwards
    uint32_t steps;                                       // terms counted
    uint32_t tiles_m, tiles_j;
    uint32_t parts;                                       // of the length, each a workgroup's; more than one: sums go to `sums`, M rows of
    float* sums; uint64_t sum_pitch;                      // sum_pitch floats for each part
    void* c; uint64_t ldc; int c_type;
};

// Which tile: neighbouring workgroups go to the 8 XCDs in turn, so each XCD is given a contiguous run of tiles; in it, bands of 8 tiles of
// m are walked along j, so that the 32 tiles that an XCD works on at a time share a few panels of either side in its L2.
__device__ inline void tile_of(const TileArgs& A, uint32_t& tm, uint32_t& tj) {
    const uint32_t total = A.tiles_m * A.tiles_j, id = blockIdx.x % total;
    const uint32_t q = total / 8, r = total % 8, x = id % 8;
    const uint32_t t = x * q + min(x, r) + id / 8;
    const uint32_t band = t / (8 * A.tiles_j), first = band * 8;
    const uint32_t height = min(8u, A.tiles_m - first), in = t - band * 8 * A.tiles_j;
    tm = first + in % height;
    tj = in / height;
}

// A tile of BM x BN elements of C by WM x WN waves, each in tiles of 32 x 32.  A step covers 128 bytes of every row of the left: 256
// elements in four bits, 64 in bf16.  While a step is multiplied from one half of the shared memory, the next one is on its way to the other.
// Rows lie in shared memory as 8 chunks of 16 bytes, chunk c of row r at c ^ r / 2 % 8, so that 16 lanes that read the same chunk of 16 rows
// use all 64 banks; chunks are exchanged where they are loaded from, since a wave's direct loads fill shared memory in the order of its lanes.
// A lane of group g = lane / 32 takes block 4 g + j of a row (product) or elements 32 g + 8 j .. + 7 (linear, grad) in its j-th matrix
// instruction; which elements meet in one instruction does not matter as long as both sides agree.
template <int OP, int BM, int BN, int WM, int WN> struct Tile {
    static constexpr uint32_t NT = 64 * WM * WN;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    static constexpr int LL = BM * 8 / NT, RL = OP == PRODUCT ? BN * 8 / NT : 0;           // 16-byte loads of a thread
    static constexpr int SL = OP == PRODUCT ? BM * 4 / NT : 0, SR = OP == PRODUCT ? BN * 4 / NT : 0;       // 4-byte loads of a pair's scales
    static constexpr uint32_t PW = BN * 32 / NT;                       // grad: columns of a thread's piece, two rows deep

    struct Half {
        uint8_t l[BM * 128];
        uint8_t r[OP == LINEAR ? BN * 32 : BN * 128];                   // (linear: room for results)
    };
    // What is loaded for several steps at a time, since a request to the L2 costs the same for 8 bytes of a row as for 128.  product: the scales
    // of the left and of the right for a pair of steps; linear: the right's scales and codes for four steps of it, which are 128 bytes of a row.
    // (8192^3 in four bits 281 us instead of 303; 4096 rows of bf16 through 4096 x 8192 202 instead of 214, 512 through 8192 x 8192 81 instead of 98.)
    struct Group {
        uint8_t s[OP == PRODUCT ? BM * 16 : OP == LINEAR ? BN * 8 : 16], r[OP == PRODUCT ? BN * 16 : OP == LINEAR ? BN * 128 : 16];
    };
    static_assert(OP != LINEAR || NT == BN * 2, "");

    // Results leave through a half's memory: 32 rows of as many columns as it has room for from every wave.  Bytes of such a row, with 16
    // more that spread the rows over the banks; columns in tiles of 32.
    static constexpr uint32_t out_bytes(int tiles, uint32_t size) { return tiles * 32 * size + 16; }
    static constexpr int out_tiles(uint32_t size) {
        int n = TN;
        while (32 * out_bytes(n, size) * WM * WN > sizeof(Half)) n /= 2;
        return n;
    }

    // What stays the same from step to step.  Rows past the end read the last one, and are not stored.
    const TileArgs& A;
    uint32_t t, lane, wave, g, l32, wm, wj, rows, cols, nb;
    uint64_t m0, j0;
    const uint8_t *left, *right, *left_s, *right_s;
    uint32_t part, first, steps;                                       // this workgroup's steps: from `first` to below `steps`
    uint32_t right0;                                                   // linear: the right's first step, an even number
    uint32_t lo[LL], ro[RL ? RL : 1], slo[SL ? SL : 1], sro[SR ? SR : 1];
    uint32_t lchunk, sword;                                            // the chunk, and the word of a pair's scales, that this thread's loads take
    uint32_t gd, gq;                                                   // grad: rows 2 gd, 2 gd + 1 and columns PW gq .. of a piece

    __device__ __forceinline__ explicit Tile(const TileArgs& args) : A(args) {
        uint32_t tm, tj;
        tile_of(A, tm, tj);
        tm = __builtin_amdgcn_readfirstlane(tm); tj = __builtin_amdgcn_readfirstlane(tj);      // (the same in all lanes anyway)
        m0 = (uint64_t)tm * BM; j0 = (uint64_t)tj * BN;
        part = __builtin_amdgcn_readfirstlane(blockIdx.x / (A.tiles_m * A.tiles_j));
        const uint32_t unit = unit_of(OP, A.terms), units = (A.steps + unit - 1) / unit;
        first = min((uint32_t)((uint64_t)units * part / A.parts) * unit, A.steps);
        steps = min((uint32_t)((uint64_t)units * (part + 1) / A.parts) * unit, A.steps);
        first = __builtin_amdgcn_readfirstlane(first); steps = __builtin_amdgcn_readfirstlane(steps);
        right0 = __builtin_amdgcn_readfirstlane(right_step(first));
        t = threadIdx.x; lane = t % 64; wave = __builtin_amdgcn_readfirstlane(t / 64);
        g = lane / 32; l32 = lane % 32;
        wm = wave / WN * (BM / WM); wj = wave % WN * (BN / WN);
        rows = (uint32_t)min(A.M - m0, (uint64_t)BM); cols = (uint32_t)min(A.outer - j0, (uint64_t)BN);
        nb = (uint32_t)((A.inner + 31) / 32);
        left = A.left + m0 * A.left_pitch;
        right = OP == GRAD ? A.right + j0 / 2 : A.right + j0 * A.right_pitch;
        left_s = A.left_scales + m0 * A.left_spitch;
        right_s = OP == GRAD ? A.right_scales + j0 / 32 : A.right_scales + j0 * A.right_spitch;
        lchunk = t % 8 ^ t / 16 % 8;
        sword = t % 4 ^ wave % 2 * 2;
#pragma unroll
        for (int i = 0; i < LL; i++) lo[i] = min(t / 8 + NT / 8 * i, rows - 1) * (uint32_t)A.left_pitch + lchunk * 16;
#pragma unroll
        for (int i = 0; i < RL; i++) ro[i] = min(t / 8 + NT / 8 * i, cols - 1) * (uint32_t)A.right_pitch + lchunk * 16;
#pragma unroll
        for (int i = 0; i < SL; i++) slo[i] = min(t / 4 + NT / 4 * i, rows - 1) * (uint32_t)A.left_spitch + sword * 4;
#pragma unroll
        for (int i = 0; i < SR; i++) sro[i] = min(t / 4 + NT / 4 * i, cols - 1) * (uint32_t)A.right_spitch + sword * 4;
        gd = t % 32; gq = t / 32;
    }

    // Step s of the left belongs to this step of the right.
    __device__ __forceinline__ uint32_t right_step(uint32_t s) const {
        return OP == PRODUCT ? s : __umulhi(2 * s, A.per_term);
    }

    // Sends for step s: the left (grad: all), and the rest.  What lies past the end of a row comes as zeros, and all of a step past the last.
    __device__ __forceinline__ void fetch(uint32_t s, Half* h) {
        const uint32_t rs = right_step(s);
        const rsrc_t bl = buffer_at(left + (uint64_t)s * 128);
        const bool on = s < steps;
        const bool in = OP == PRODUCT ? on & (s * 8 + lchunk < nb) : on & ((A.terms > 1) | ((uint64_t)rs * 64 + lchunk * 8 < A.inner));
#pragma unroll
        for (int i = 0; i < LL; i++) load_lds<16>(bl, h->l + (i * NT + wave * 64) * 16, in ? lo[i] : kNowhere);
    }

    // grad: a piece of the right for step s, to registers (a piece of 32 columns is one block; one of 16 half of one).
    struct Piece { uint32_t w[2][PW / 8], s[2]; };
    __device__ __forceinline__ void fetch_piece(uint32_t s, Piece& P) {
        if constexpr (OP == GRAD) {
            const uint32_t rs = right_step(s);
            const rsrc_t br = buffer_at(right + (uint64_t)rs * 64 * A.right_pitch), bs = buffer_at(right_s + (uint64_t)rs * 64 * A.right_spitch);
            const bool c_in = (s < steps) & (gq * PW < (uint32_t)((A.outer + 31) / 32 * 32 - j0));
#pragma unroll
            for (int r = 0; r < 2; r++) {
                const uint32_t row = gd * 2 + r;
                const bool in = c_in & ((uint64_t)rs * 64 + row < A.inner);
                const uint32_t off = in ? row * (uint32_t)A.right_pitch + gq * (PW / 2) : kNowhere;
                if constexpr (PW == 32) {
                    const i32x4 v = load16(br, off);
#pragma unroll
                    for (int i = 0; i < 4; i++) P.w[r][i] = v[i];
                } else {
                    const auto v = __builtin_amdgcn_raw_buffer_load_b64(br, off, 0, 0);
                    P.w[r][0] = v[0]; P.w[r][1] = v[1];
                }
                P.s[r] = __builtin_amdgcn_raw_buffer_load_b8(bs, in ? row * (uint32_t)A.right_spitch + gq * PW / 32 : kNowhere, 0, 0);
            }
        }
    }

    // product: the right for step s.
    __device__ __forceinline__ void fetch_right(uint32_t s, Half* h) {
        if constexpr (OP == PRODUCT) {
            const rsrc_t br = buffer_at(right + (uint64_t)s * 128);
            const bool in = (s < steps) & (s * 8 + lchunk < nb);
#pragma unroll
            for (int i = 0; i < RL; i++) load_lds<16>(br, h->r + (i * NT + wave * 64) * 16, in ? ro[i] : kNowhere);
        }
    }

    // The group that step s belongs to, counted from the first.
    __device__ __forceinline__ uint32_t group_of(uint32_t s) const {
        return OP == PRODUCT ? (s - first) / 2 : OP == LINEAR ? (right_step(s) - right0) / 4 : 0;
    }

    // A share of a group.  product: the scales of one side for steps s and s + 1.  linear: quarter q of the rows, from step rs of the right on.
    template <bool RIGHT> __device__ __forceinline__ void fetch_scales(uint32_t s, Group* to) {
        const rsrc_t b = buffer_at((RIGHT ? right_s : left_s) + (uint64_t)s * 8);
        const bool in = (s < steps) & (s * 8 + sword * 4 < nb);
#pragma unroll
        for (int i = 0; i < (RIGHT ? SR : SL); i++)
            load_lds<4>(b, (RIGHT ? to->r : to->s) + (i * NT + wave * 64) * 4, in ? (RIGHT ? sro : slo)[i] : kNowhere);
    }
    __device__ __forceinline__ void fetch_quarter(uint32_t rs, uint32_t q, Group* to) {
        const rsrc_t br = buffer_at(right + (uint64_t)rs * 32), bs = buffer_at(right_s + (uint64_t)rs * 2);
        const uint32_t row = min(t / 8 + NT / 8 * q, cols - 1);
        load_lds<16>(br, to->r + (q * NT + wave * 64) * 16, rs * 2 + lchunk < nb ? row * (uint32_t)A.right_pitch + lchunk * 16 : kNowhere);
        if (wave % 4 == q)
            load_lds<4>(bs, to->s + wave * 256, rs * 2 + t % 2 * 4 < nb ? min(t / 2, cols - 1) * (uint32_t)A.right_spitch + t % 2 * 4 : kNowhere);
    }

    // The first group, and in step s (of a pair its second: SECOND) a share of the group after the one that s belongs to.
    __device__ __forceinline__ void fetch_first(Group* to) {
        if constexpr (OP == PRODUCT) { fetch_scales<false>(first, to); fetch_scales<true>(first, to); }
        if constexpr (OP == LINEAR)
            for (uint32_t q = 0; q < 4; q++) fetch_quarter(right0, q, to);
    }
    template <bool SECOND> __device__ __forceinline__ void fetch_share(uint32_t s, Group* to) {
        if constexpr (OP == PRODUCT) fetch_scales<SECOND>(SECOND ? s + 1 : s + 2, to);
        if constexpr (OP == LINEAR) {                                  // (the same share again for a float's other terms)
            const uint32_t r = right_step(s) - right0;
            fetch_quarter(right0 + (r / 4 + 1) * 4, r % 4, to);
        }
    }

    // grad: two rows of codes become columns of bf16, two rows to a word.
    __device__ __forceinline__ void turn(const Piece& P, Half* h) {
        if constexpr (OP == GRAD) {
            const float s0 = mx_scale(P.s[0]), s1 = mx_scale(P.s[1]);
#pragma unroll
            for (uint32_t w = 0; w < PW / 8; w++)
                unroll4([&](auto B) {
                    const uint32_t p = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(P.w[0][w], s0, B.value));
                    const uint32_t q = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(P.w[1][w], s1, B.value));
                    const uint32_t col = gq * PW + w * 8 + B.value * 2;
                    *reinterpret_cast<uint32_t*>(h->r + col * 128 + ((gd / 4 ^ col / 2 % 8) * 16) + gd % 4 * 4) = __builtin_amdgcn_perm(q, p, 0x05040100u);
                    *reinterpret_cast<uint32_t*>(h->r + (col + 1) * 128 + ((gd / 4 ^ col / 2 % 8) * 16) + gd % 4 * 4) =
                        __builtin_amdgcn_perm(q, p, 0x07060302u);
                });
        }
    }

    // What a lane multiplies: a fragment of either side for one of a step's four matrix instructions, and what serves all four.
    struct Frag { i32x4 x[TM], y[TN]; };
    struct Side { int sl[TM], sr[TN]; i32x4 w[TN]; };

    // SECOND: s is the second step of its pair
    template <bool SECOND> __device__ __forceinline__ void load_side(uint32_t s, const Group* from, Side& S) {
        if constexpr (OP == PRODUCT) {
            const uint32_t in = nb - min(s * 8 + g * 4, nb);           // blocks of this lane's four that there are
            const int keep = in >= 4 ? -1 : (1 << 8 * in) - 1;
            const uint32_t at = (SECOND ^ l32 / 16) * 8 + g * 4;       // (the pair's two steps change places every 16 rows, so that all banks are used)
#pragma unroll
            for (int a = 0; a < TM; a++) S.sl[a] = *reinterpret_cast<const int*>(from->s + (wm + a * 32 + l32) * 16 + at) & keep;
#pragma unroll
            for (int b = 0; b < TN; b++) S.sr[b] = *reinterpret_cast<const int*>(from->r + (wj + b * 32 + l32) * 16 + at) & keep;
        }
        if constexpr (OP == LINEAR) {
            const uint32_t rs = right_step(s), blk = rs * 2 + g;
            const uint32_t at = (rs - right0) % 4 * 2 + g;
#pragma unroll
            for (int b = 0; b < TN; b++) {
                S.w[b] = *reinterpret_cast<const i32x4*>(from->r + (wj + b * 32 + l32) * 128 + (at ^ l32 / 2 % 8) * 16);
                const uint32_t sb = from->s[(wj + b * 32 + l32) * 8 + at];
                S.sr[b] = blk < nb ? sb : 0;
            }
        }
    }

    __device__ __forceinline__ void load_frag(int j, const Half* h, Frag& F) {
        const uint32_t c = ((g * 4 + j) ^ l32 / 2 % 8) * 16;
#pragma unroll
        for (int a = 0; a < TM; a++) F.x[a] = *reinterpret_cast<const i32x4*>(h->l + (wm + a * 32 + l32) * 128 + c);
        if constexpr (OP != LINEAR)
#pragma unroll
            for (int b = 0; b < TN; b++) F.y[b] = *reinterpret_cast<const i32x4*>(h->r + (wj + b * 32 + l32) * 128 + c);
    }

    // linear: the right's part of a fragment, from four bits.
    template <int j> __device__ __forceinline__ void widen(const Side& S, Frag& F) {
        if constexpr (OP == LINEAR)
#pragma unroll
            for (int b = 0; b < TN; b++)
                unroll4([&](auto B) {
                    F.y[b][B.value] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(S.w[b][j], mx_scale(S.sr[b]), B.value));
                });
    }

    template <int j> __device__ __forceinline__ void multiply(const Frag& F, const Side& S, f32x16 (&acc)[TM][TN]) {
#pragma unroll
        for (int a = 0; a < TM; a++)
#pragma unroll
            for (int b = 0; b < TN; b++)
                if constexpr (OP == PRODUCT) {
                    const i32x8 x = { F.x[a][0], F.x[a][1], F.x[a][2], F.x[a][3], 0, 0, 0, 0 }, y = { F.y[b][0], F.y[b][1], F.y[b][2], F.y[b][3], 0, 0, 0, 0 };
                    acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y, x, acc[a][b], 4, 4, j, S.sr[b], j, S.sl[a]);
                } else {
                    acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, F.y[b]), __builtin_bit_cast(bf16x8, F.x[a]), acc[a][b], 0, 0, 0);
                }
    }

    static __device__ __forceinline__ void pin() { __builtin_amdgcn_sched_barrier(0); }

    // This wave's loads have arrived, its reads and writes of shared memory are done, and so are everyone's.  The fences keep the compiler from
    // moving reads and writes across; they reach shared memory through any pointer, since none here is declared to be the only one to its memory
    // (what a direct load brings is read through another, and `from` and `to` of a step may be one).
    static __device__ __forceinline__ void meet() {
        pin();
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");          // (before the wait, so that no load can be sent behind it)
        __builtin_amdgcn_s_waitcnt(0x0070);                            // vmcnt(0), lgkmcnt(0): direct loads too
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        pin();
    }

    // The order of a quarter of a step: `gap` matrix instructions, then a read of shared memory and `loads` loads, and so on; the rest between.
    static constexpr int kGap = TM * TN / (TM + (OP == LINEAR ? 0 : TN));
    template <int gap, int loads, bool turning = false, int reads = 1> static __device__ __forceinline__ void order() {
#pragma unroll
        for (int i = 0; i < TM * TN / gap; i++) {
            __builtin_amdgcn_sched_group_barrier(0x8, gap, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
            if (loads) __builtin_amdgcn_sched_group_barrier(0x10, loads ? loads : 1, 0);
            if (OP == LINEAR) __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
            if (OP == GRAD && turning)
#pragma unroll
                for (int k = 0; k < (int)PW / (TM * TN / gap); k++) {
                    __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
                    __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                }
        }
        pin();
    }

    // Step s, whose first fragments are in registers already.  The workgroup meets while the last of its four multiplications is still to
    // come: from then on `cur` is free for step s + 2, and the first fragments of step s + 1 can be read from `next`.  (grad: P holds step s + 1
    // of the right, and then gets step s + 3.  `from` is the group of step s + 1, `to` the one after the group of s: they are the same where s is
    // its group's last step.)
    template <bool SECOND> __device__ __forceinline__ void step(uint32_t s, Half* cur, Half* next, const Group* from,
                                                                Group* to, Piece& P, Frag& F, Side& S, f32x16 (&acc)[TM][TN]) {
        Frag F1, F2, F3;
        load_frag(1, cur, F1);
        widen<1>(S, F1);
        fetch_right(s + 1, next);
        fetch_share<SECOND>(s, to);
        multiply<0>(F, S, acc);
        order<kGap, 2>();
        load_frag(2, cur, F2);
        widen<2>(S, F2);
        multiply<1>(F1, S, acc);
        order<kGap, 0>();
        load_frag(3, cur, F3);
        widen<3>(S, F3);
        turn(P, next);
        multiply<2>(F2, S, acc);
        order<kGap, 0, true>();
        meet();
        fetch_piece(s + 3, P);
        fetch(s + 2, cur);
        Side S1;
        load_side<!SECOND>(s + 1, from, S1);
        load_frag(0, next, F);
        widen<0>(S1, F);
        multiply<3>(F3, S, acc);
        order<1, 1, false, (2 * (TM + TN) + TM * TN - 1) / (TM * TN)>();
        S = S1;
    }

    // The wave's part of C, 32 rows at a time, through a part of a half's memory: a lane holds 4 neighbouring columns of a row (the right is
    // the matrix instructions' first operand), and leaves with 16 bytes of a row next to those of its neighbours.
    template <typename T> __device__ __forceinline__ void store(void* to, uint64_t ld, uint8_t* scratch, const f32x16 (&acc)[TM][TN]) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        constexpr int B = out_tiles(sizeof(T));
        static_assert(B >= 1 && TN % B == 0, "");
        constexpr uint32_t W = B * 32, E = 16 / sizeof(T);             // columns of a pass; elements of 16 bytes
        constexpr uint32_t P = out_bytes(B, sizeof(T));
        uint8_t* const mine = scratch + wave * 32 * P;
        const rsrc_t rc = buffer_at(reinterpret_cast<T*>(to) + m0 * ld + j0);
        const uint32_t pitch = (uint32_t)ld * (uint32_t)sizeof(T);
        const bool wide = pitch % 16 == 0;
#pragma unroll
        for (int a = 0; a < TM; a++)
#pragma unroll
            for (int b0 = 0; b0 < TN; b0 += B) {
#pragma unroll
                for (int b = 0; b < B; b++)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f32x16& c = acc[a][b0 + b];
                        const t4 v = { (T)c[i], (T)c[i + 1], (T)c[i + 2], (T)c[i + 3] };
                        *reinterpret_cast<t4*>(mine + l32 * P + (b * 32 + i * 2 + g * 4) * sizeof(T)) = v;
                    }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                const uint32_t m1 = wm + a * 32, j1 = wj + b0 * 32;
                if (wide) {
#pragma unroll
                    for (uint32_t r = 0; r < 32; r += 64 * E / W) {
                        const uint32_t row = r + lane / (W / E), col = lane % (W / E) * E, m = m1 + row, j = j1 + col;
                        const i32x4 v = *reinterpret_cast<const i32x4*>(mine + row * P + col * sizeof(T));
                        const uint32_t off = m * pitch + j * (uint32_t)sizeof(T);
                        __builtin_amdgcn_raw_buffer_store_b128(v, rc, m < rows && j + E <= cols ? off : kNowhere, 0, 0);
                        if (m < rows && j < cols && j + E > cols)
                            for (uint32_t e = 0; j + e < cols; e++)
                                put(rc, reinterpret_cast<const T*>(mine + row * P)[col + e], off + e * (uint32_t)sizeof(T));
                    }
                } else {
                    for (uint32_t e = lane; e < 32 * W; e += 64) {
                        const uint32_t row = e / W, col = e % W, m = m1 + row, j = j1 + col;
                        put(rc, reinterpret_cast<const T*>(mine + row * P)[col], m < rows && j < cols ? m * pitch + j * (uint32_t)sizeof(T) : kNowhere);
                    }
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            }
    }

    template <typename T> static __device__ __forceinline__ void put(rsrc_t r, T v, uint32_t off) {
        if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), r, off, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, v), r, off, 0, 0);
    }
};

template <int OP, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 1) void k_mx_tile(TileArgs A) {
    typedef Tile<OP, BM, BN, WM, WN> Tl;
    __shared__ __attribute__((aligned(16))) typename Tl::Half h0, h1;
    __shared__ __attribute__((aligned(16))) typename Tl::Group groups[2];
    Tl T(A);
    f32x16 acc[Tl::TM][Tl::TN];
#pragma unroll
    for (int a = 0; a < Tl::TM; a++)
#pragma unroll
        for (int b = 0; b < Tl::TN; b++) acc[a][b] = f32x16{};
    uint32_t s = T.first;
    typename Tl::Piece P0, P1;                                         // of even and odd steps from the first, two steps ahead of their use
    T.fetch_piece(s, P0);
    T.fetch_piece(s + 1, P1);
    T.fetch(s, &h0);
    T.fetch_right(s, &h0);
    T.fetch_first(groups);
    T.fetch(s + 1, &h1);
    T.turn(P0, &h0);
    T.fetch_piece(s + 2, P0);
    T.meet();
    typename Tl::Frag F;
    typename Tl::Side S;
    T.template load_side<false>(s, groups, S);
    T.load_frag(0, &h0, F);
    T.template widen<0>(S, F);
    const auto group = [&](uint32_t number) { return groups + number % 2; };
    for (; s + 1 < T.steps; s += 2) {
        T.template step<false>(s, &h0, &h1, group(T.group_of(s + 1)), group(T.group_of(s) + 1), P1, F, S, acc);
        T.template step<true>(s + 1, &h1, &h0, group(T.group_of(s + 2)), group(T.group_of(s + 1) + 1), P0, F, S, acc);
    }
    if (s < T.steps) T.template step<false>(s, &h0, &h1, group(T.group_of(s + 1)), group(T.group_of(s) + 1), P1, F, S, acc);
    Tl::meet();                                                        // (nor may a load reach shared memory after the workgroup's end)
    uint8_t* const scratch = reinterpret_cast<uint8_t*>(&h0);
    if (A.parts > 1) T.template store<float>(A.sums + T.part * A.M * A.sum_pitch, A.sum_pitch, scratch, acc);
    else if (A.c_type == F32) T.template store<float>(A.c, A.ldc, scratch, acc);
    else if (A.c_type == BF16) T.template store<__bf16>(A.c, A.ldc, scratch, acc);
    else T.template store<_Float16>(A.c, A.ldc, scratch, acc);
}

// A float as bf16 terms that add up to it: one for bf16, two for fp16 (11 bits), three for float32 (24 bits).  Each term takes the top of
// what is left, cut off (not rounded, which could carry past the largest float32), so every difference is exact; an infinity or NaN is its
// first term alone.  top: the terms' bits in the upper half of a word.
__host__ __device__ constexpr int terms_of(int type) { return type == F32 ? 3 : type == F16 ? 2 : 1; }

template <int T> __device__ __forceinline__ void cut(float v, uint32_t (&top)[terms_of(T)]) {
    const bool plain = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
#pragma unroll
    for (int q = 0; q < terms_of(T); q++) {
        top[q] = __float_as_uint(v) & 0xFFFF0000u;
        if (q == 0 && v != v) top[q] |= 0x00400000u;
        if (q > 0 && !plain) top[q] = 0;
        v -= __uint_as_float(top[q]);
    }
}

// Eight floats as they lie in memory: loaded in 16-byte words, or one by one with zeros for those past the end; then cut into terms.
template <int T> struct Eight {
    i32x4 w[float_bytes(T) / 2];

    // off: of the first in bytes, or kNowhere
    __device__ __forceinline__ void load_words(rsrc_t r, uint32_t off) {
#pragma unroll
        for (uint32_t i = 0; i < float_bytes(T) / 2; i++) w[i] = load16(r, off == kNowhere ? off : off + i * 16);
    }

    __device__ __forceinline__ void load_each(rsrc_t r, uint32_t off, uint32_t n) {
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) {
            const uint32_t at = i < n ? off + i * float_bytes(T) : kNowhere;
            if (T == F32) w[i / 4][i % 4] = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
            else {
                const uint32_t v = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
                w[0][i / 2] = i % 2 ? (int)((uint32_t)w[0][i / 2] | v << 16) : (int)v;
            }
        }
    }

    __device__ __forceinline__ float value(int i) const {
        if (T == F32) return __int_as_float(w[i / 4][i % 4]);
        const uint16_t h = (uint16_t)((uint32_t)w[0][i / 2] >> (i % 2 * 16));
        return T == F16 ? (float)__builtin_bit_cast(_Float16, h) : __uint_as_float((uint32_t)h << 16);
    }

    __device__ __forceinline__ void terms(i32x4 (&out)[terms_of(T)]) const {
        if constexpr (T == BF16) { out[0] = w[0]; return; }
#pragma unroll
        for (int i = 0; i < 4; i++) {
            uint32_t a[terms_of(T)], b[terms_of(T)];
            cut<T>(value(2 * i), a);
            cut<T>(value(2 * i + 1), b);
#pragma unroll
            for (int q = 0; q < terms_of(T); q++) out[q][i] = (int)(a[q] >> 16 | b[q]);
        }
    }
};

// The left for the tiles: rows of whole steps of 64 elements, term after term in a step, zeros behind the end.
template <int T>
__global__ __launch_bounds__(256) void k_mx_terms(const uint8_t* x, uint64_t ldx, bool wide, uint64_t M, uint64_t inner, uint32_t chunks,
                                                  uint16_t* out) {
    constexpr int terms = terms_of(T);
    const uint64_t id = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;       // 8 elements
    const uint64_t per_row = (uint64_t)chunks * 8;
    const uint64_t m = id / per_row;
    if (m >= M) return;
    const uint64_t o = id % per_row, i0 = o * 8;
    const uint32_t n = i0 >= inner ? 0 : (uint32_t)min(inner - i0, (uint64_t)8);
    i32x4 w[terms];
    Eight<T> e;
    const rsrc_t r = buffer_at(x + m * ldx * float_bytes(T));
    if (wide && n == 8) e.load_words(r, (uint32_t)i0 * float_bytes(T)); else e.load_each(r, (uint32_t)i0 * float_bytes(T), n);
    e.terms(w);
    uint16_t* const at = out + m * chunks * 64 * terms + (o / 8) * 64 * terms + o % 8 * 8;
    for (int q = 0; q < terms; q++) *reinterpret_cast<i32x4*>(at + q * 64) = w[q];
}

// The left for k_mx_rows: a thread copies 16 bytes, zeros behind the end of a row.
template <int SIZE>
__global__ __launch_bounds__(256) void k_mx_lay(const uint8_t* x, uint64_t pitch, uint32_t M, uint64_t inner, uint8_t* out) {
    constexpr uint32_t E = 16 / SIZE;
    const uint64_t per_row = (inner + 7) / 8 * 8 / E, id = (uint64_t)blockIdx.x * 256 + threadIdx.x, m = id / per_row, i0 = id % per_row * E;
    if (m >= M) return;
    i32x4 w = {};
#pragma unroll
    for (uint32_t i = 0; i < E; i++)
        if (i0 + i < inner) {
            if (SIZE == 4) w[i % 4] = reinterpret_cast<const int*>(x + m * pitch)[i0 + i];
            else w[i / 2 % 4] |= (int)((uint32_t)reinterpret_cast<const uint16_t*>(x + m * pitch)[i0 + i] << (i % 2 * 16));
        }
    reinterpret_cast<i32x4*>(out)[id] = w;
}

struct RowArgs {
    const uint8_t* left; uint64_t left_pitch;             // codes or floats, and bytes of a row
    const uint8_t* left_scales; uint64_t left_spitch;
    const uint8_t* right; uint64_t right_pitch; const uint8_t* right_scales; uint64_t right_spitch;
    uint32_t M; uint64_t outer, inner;
    void* c; uint64_t ldc; int c_type;
};

__device__ __forceinline__ void store_one(void* c, int type, uint64_t at, float v) {
    if (type == F32) reinterpret_cast<float*>(c)[at] = v;
    else if (type == BF16) reinterpret_cast<__bf16*>(c)[at] = (__bf16)v;
    else reinterpret_cast<_Float16*>(c)[at] = (_Float16)v;
}

// Few rows on the left: bound by the codes of the right, which pass once from memory through registers to the matrix units.
// A workgroup of 8 waves makes 16 NJ columns of up to 16 MF rows; each wave sums over an eighth of the length, and the eighths are added in
// their order at the end.  A wave takes S units of 128 elements at a time: it asks for all of the right's codes of these units, for their
// scales, which it spreads through shared memory of its own (a load for every unit would read four bytes of a row at a time), and for the
// left, which serves all NJ tiles of 16 columns.  LEFT: type of the floats (then a unit is four matrix instructions a term, lane group
// g = lane / 16 taking elements 32 g + 8 j .. + 7 in the j-th; rows start at multiples of 16 bytes and have a multiple of 8 elements), or -1
// for four bits (one instruction, group g taking block g).
// The matrix instructions take 16 rows whether there are as many or not.  FEW: as many rows as few_rows says, which also come through shared
// memory, each byte loaded and cut into terms once; else every lane loads the fragments that it multiplies, and the next units' codes are on
// their way meanwhile (FEW has room for two workgroups on a compute unit instead, where there are more than 256).  FEW saves the cutting: one
// row against 8192 x 8192, codes from memory, float32 14.8 us instead of 21.4, fp16 14.5 / 18.8; against 4096 x 4096 7.8 / 10.1 and 7.5 / 9.1.
// What is not cut gains less or loses: four bits 11.9 / 11.6, four rows 11.9 / 12.5 (codes in the caches 7.6 / 7.8 and 7.7 / 8.8), bf16 14.2 / 13.0
// (9.6 / 9.4, four rows 10.1 / 10.7); against 4096 x 4096 5.4 / 4.8 and 6.4 / 5.4.
__host__ __device__ constexpr uint32_t few_rows(int left) { return left < 0 ? 4 : left == F32 ? 1 : left == F16 ? 2 : 4; }

template <int LEFT, int MF, int NJ, bool FEW>
__global__ __launch_bounds__(512, FEW ? 4 : 2) void k_mx_rows(RowArgs A) {
    constexpr int T = LEFT < 0 ? BF16 : LEFT;
    constexpr int terms = terms_of(T);
    constexpr int S = FEW ? 8 : LEFT < 0 ? 4 : MF * terms >= 6 ? 1 : MF * terms >= 2 ? 2 : 4;
    constexpr uint32_t LB = LEFT < 0 ? S * 64 : S * 128 * float_bytes(T);                     // bytes of a row of the left and S units
    constexpr uint32_t kScaleWords = 16 * NJ * S, FR = few_rows(LEFT);
    constexpr uint32_t RowB = LEFT < 0 ? LB : S * 256;                                        // of a row and term in shared memory
    struct Own { uint8_t left[FEW ? FR * terms * RowB : 16]; uint32_t scales[kScaleWords]; uint32_t left_scales[FEW && LEFT < 0 ? FR * S : 4]; };
    union Shared { Own own[8]; float part[8][MF * NJ][256]; };
    __shared__ __attribute__((aligned(16))) Shared sh;
    const uint32_t t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64), r16 = lane % 16, g = lane / 16;
    const uint64_t j0 = (uint64_t)blockIdx.x * (16 * NJ);
    const uint32_t cols = (uint32_t)min(A.outer - j0, (uint64_t)(16 * NJ));
    const uint32_t nb = (uint32_t)((A.inner + 31) / 32), units = (nb + 3) / 4;
    const uint32_t u0 = (uint32_t)((uint64_t)units * wave / 8), u1 = (uint32_t)((uint64_t)units * (wave + 1) / 8);
    Own& own = sh.own[wave];

    f32x4 acc[MF][NJ];
#pragma unroll
    for (int a = 0; a < MF; a++)
#pragma unroll
        for (int b = 0; b < NJ; b++) acc[a][b] = f32x4{};
    uint32_t ro[NJ], lo[MF], lso[MF];
#pragma unroll
    for (int b = 0; b < NJ; b++) ro[b] = min(b * 16 + r16, cols - 1) * (uint32_t)A.right_pitch + g * 16;
#pragma unroll
    for (int a = 0; a < MF; a++) {
        const uint32_t m = min(a * 16 + r16, A.M - 1);
        lo[a] = m * (uint32_t)A.left_pitch + (LEFT < 0 ? g * 16 : 0);
        lso[a] = m * (uint32_t)A.left_spitch;
    }

    constexpr uint32_t SW = (kScaleWords + 63) / 64;
    i32x4 w[S][NJ];
    uint32_t sw[SW];
    auto ask = [&](uint32_t u) {                                        // the right's codes, and its scales, a word a unit
        const rsrc_t br = buffer_at(A.right + j0 * A.right_pitch + (uint64_t)u * 64), bs = buffer_at(A.right_scales + j0 * A.right_spitch + (uint64_t)u * 4);
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int b = 0; b < NJ; b++) w[s][b] = load16(br, ((u + s < u1) & ((u + s) * 4 + g < nb)) ? ro[b] + s * 64 : kNowhere);
#pragma unroll
        for (uint32_t i = 0; i < SW; i++) {
            const uint32_t e = i * 64 + lane, row = e / S, un = e % S;
            sw[i] = __builtin_amdgcn_raw_buffer_load_b32(bs, u + un < u1 ? min(row, cols - 1) * (uint32_t)A.right_spitch + un * 4 : kNowhere, 0, 0);
        }
    };
    if (!FEW) ask(u0);
    for (uint32_t u = u0; u < u1; u += S) {
        const rsrc_t bl = buffer_at(A.left + (uint64_t)u * LB / S), bls = buffer_at(A.left_scales + (uint64_t)u * 4);
        if (FEW) ask(u);
        // the left
        i32x4 x[FEW ? 1 : S][MF][FEW ? 1 : LEFT < 0 ? 1 : 4 * terms];
        uint32_t xs[S][MF];
        if constexpr (FEW) {
            constexpr uint32_t E = LEFT < 0 ? 16 : 8 * float_bytes(T);  // bytes of a lane's piece: a block, or eight floats
            constexpr uint32_t LN = FR * LB / E / 64;
            const uint64_t end = LEFT < 0 ? (uint64_t)nb * 16 : A.inner * float_bytes(T);               // bytes of a row
            Eight<T> lv[LN];
            uint32_t ls = 0;
#pragma unroll
            for (uint32_t i = 0; i < LN; i++) {
                const uint32_t e = (i * 64 + lane) * E, row = e / LB, at = e % LB;
                const bool in = (row < A.M) & (u + at / (LB / S) < u1) & ((uint64_t)u * (LB / S) + at < end);
                lv[i].load_words(bl, in ? row * (uint32_t)A.left_pitch + at : kNowhere);
            }
            if constexpr (LEFT < 0) {
                const uint32_t row = lane / S, un = lane % S;
                ls = __builtin_amdgcn_raw_buffer_load_b32(bls, ((row < A.M) & (u + un < u1)) ? row * (uint32_t)A.left_spitch + un * 4 : kNowhere, 0, 0);
            }
#pragma unroll
            for (uint32_t i = 0; i < SW; i++) own.scales[i * 64 + lane] = sw[i];
#pragma unroll
            for (uint32_t i = 0; i < LN; i++) {
                const uint32_t e = (i * 64 + lane) * 16, row = e / RowB, at = e % RowB;
                i32x4 v[terms];
                lv[i].terms(v);
#pragma unroll
                for (int q = 0; q < terms; q++) *reinterpret_cast<i32x4*>(&own.left[(row * terms + q) * RowB + at]) = v[q];
            }
            if (LEFT < 0 && lane < FR * S) own.left_scales[lane] = ls;
        } else {
#pragma unroll
            for (int s = 0; s < S; s++)
#pragma unroll
                for (int a = 0; a < MF; a++) {
                    if constexpr (LEFT < 0) {
                        const bool in = (u + s < u1) & ((u + s) * 4 + g < nb);
                        x[s][a][0] = load16(bl, in ? lo[a] + s * 64 : kNowhere);
                        xs[s][a] = __builtin_amdgcn_raw_buffer_load_b32(bls, in ? lso[a] + s * 4 : kNowhere, 0, 0);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            const uint32_t i = s * 128 + g * 32 + j * 8;
                            const bool in = (u + s < u1) & ((uint64_t)u * 128 + i < A.inner);
                            Eight<T> e;
                            e.load_words(bl, in ? lo[a] + i * float_bytes(T) : kNowhere);
                            i32x4 v[terms];
                            e.terms(v);
#pragma unroll
                            for (int q = 0; q < terms; q++) x[s][a][j * terms + q] = v[q];
                        }
                    }
                }
#pragma unroll
            for (uint32_t i = 0; i < SW; i++) if (kScaleWords % 64 == 0 || i * 64 + lane < kScaleWords) own.scales[i * 64 + lane] = sw[i];
        }
        i32x4 now[S][NJ];
#pragma unroll
        for (int s = 0; s < S; s++)
#pragma unroll
            for (int b = 0; b < NJ; b++) now[s][b] = w[s][b];
        if (!FEW) ask(u + S);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");

        const uint32_t few = FEW ? min(r16, A.M - 1) : 0;               // this lane's row of the left
#pragma unroll
        for (int s = 0; s < S; s++) {
            uint32_t sb[NJ];
#pragma unroll
            for (int b = 0; b < NJ; b++) {
                const uint32_t v = reinterpret_cast<const uint8_t*>(own.scales)[((b * 16 + r16) * S + s) * 4 + g];
                sb[b] = (u + s) * 4 + g < nb ? v : 0;                   // (a word holds more blocks than the last unit has)
            }
            if constexpr (LEFT < 0) {
#pragma unroll
                for (int a = 0; a < MF; a++) {
                    const uint32_t v = FEW ? (uint32_t)reinterpret_cast<const uint8_t*>(own.left_scales)[(few * S + s) * 4 + g] : __builtin_amdgcn_ubfe(xs[s][a], 8 * g, 8);
                    const uint32_t sa = (u + s) * 4 + g < nb ? v : 0;
                    const i32x4 p = FEW ? *reinterpret_cast<const i32x4*>(&own.left[few * RowB + s * 64 + g * 16]) : x[FEW ? 0 : s][a][0];
#pragma unroll
                    for (int b = 0; b < NJ; b++) {
                        const i32x4 q = now[s][b];
                        const i32x8 p8 = { p[0], p[1], p[2], p[3], 0, 0, 0, 0 }, q8 = { q[0], q[1], q[2], q[3], 0, 0, 0, 0 };
                        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p8, q8, acc[a][b], 4, 4, 0, sa, 0, sb[b]);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    i32x4 v[terms];
                    if constexpr (FEW)
#pragma unroll
                        for (int q = 0; q < terms; q++)
                            v[q] = *reinterpret_cast<const i32x4*>(&own.left[(few * terms + q) * RowB + s * 256 + g * 64 + j * 16]);
#pragma unroll
                    for (int b = 0; b < NJ; b++) {
                        i32x4 y;
                        unroll4([&](auto B) { y[B.value] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(now[s][b][j], mx_scale(sb[b]), B.value)); });
#pragma unroll
                        for (int a = 0; a < MF; a++)
#pragma unroll
                            for (int q = 0; q < terms; q++)
                                acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, FEW ? v[q] : x[FEW ? 0 : s][a][FEW ? 0 : j * terms + q]),
                                                                                    __builtin_bit_cast(bf16x8, y), acc[a][b], 0, 0, 0);
                    }
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }

    __syncthreads();                                                    // (the sums take the place of what the waves kept)
#pragma unroll
    for (int a = 0; a < MF; a++)
#pragma unroll
        for (int b = 0; b < NJ; b++)
#pragma unroll
            for (int i = 0; i < 4; i++) sh.part[wave][a * NJ + b][(g * 4 + i) * 16 + r16] = acc[a][b][i];
    __syncthreads();
    const uint32_t outs = min(A.M, 16u * MF) * 16 * NJ;
    for (uint32_t e = t; e < outs; e += 512) {
        const uint32_t m = e / (16 * NJ), j = e % (16 * NJ);
        if (j >= cols) continue;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; k++) v += sh.part[k][m / 16 * NJ + j / 16][m % 16 * 16 + j % 16];
        store_one(A.c, A.c_type, m * A.ldc + j0 + j, v);
    }
}

// Two tiles of 16 columns a workgroup from 512 tiles on, so that half as many workgroups read the left: 16 rows of bf16 through 8192 x 4096
// 9.8 us, by one tile each 13.9, through 16384 x 4096 18.6 and 26.2, one row there 14.5 and 14.7.  Fewer tiles keep a workgroup each, which fills
// the chip: 4096 columns 8.0 us, by two 9.1.  Not best for every count of rows near the border: one row of bf16 through 8192 x 4096 takes 9.1, by
// one tile each 8.2, and 16 rows through 6144 x 4096 13.2, by two 9.4.
template <int LEFT, int MF, bool FEW> void launch_rows(const RowArgs& R, hipStream_t st) {
    const uint64_t tiles = (R.outer + 15) / 16;
    if (tiles >= 512) hipLaunchKernelGGL((k_mx_rows<LEFT, MF, 2, FEW>), dim3((uint32_t)((tiles + 1) / 2)), dim3(512), 0, st, R);
    else hipLaunchKernelGGL((k_mx_rows<LEFT, MF, 1, FEW>), dim3((uint32_t)tiles), dim3(512), 0, st, R);
}

template <int LEFT> hipError_t launch_rows(const RowArgs& R, hipStream_t st) {
    if (R.M <= few_rows(LEFT)) launch_rows<LEFT, 1, true>(R, st);
    else if (R.M <= 16) launch_rows<LEFT, 1, false>(R, st);
    else launch_rows<LEFT, 2, false>(R, st);
    return hipGetLastError();
}

// The gradient for few rows: bound by the codes as well.  A workgroup of 8 waves takes 256 columns of B over a part of its rows; a wave takes
// 32 rows at a time, a lane 8 of them (group g = lane / 16) in 16 columns (lane % 16), turns its 8 x 16 codes into 16 fragments of 8 rows in
// registers, and multiplies them with the same 8 elements of up to 16 rows of the left: the j-th instruction makes the columns 16 i + j.
// Columns need as many fragments as there are, so that nothing is exchanged between lanes.  The next 32 rows are on their way meanwhile.
// Waves are added in their order through shared memory, parts by k_mx_join.  LEFT: as for k_mx_rows, floats.
template <int LEFT>
__global__ __launch_bounds__(512, 2) void k_mx_grad_rows(RowArgs A, uint32_t parts, float* sums, uint64_t sum_pitch) {
    constexpr int terms = terms_of(LEFT);
    struct Own { uint32_t scales[64]; };
    union Shared { Own own[8]; float part[8][16][256]; };
    __shared__ __attribute__((aligned(16))) Shared sh;
    const uint32_t t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64), c16 = lane % 16, g = lane / 16;
    const uint32_t strips = gridDim.x / parts, strip = blockIdx.x % strips, part = blockIdx.x / strips;
    const uint64_t j0 = (uint64_t)strip * 256;
    const uint32_t cols = (uint32_t)min(A.outer - j0, (uint64_t)256), blocks = (cols + 31) / 32;
    const uint32_t units = (uint32_t)((A.inner + 31) / 32), slices = parts * 8, slice = part * 8 + wave;
    const uint32_t u0 = (uint32_t)((uint64_t)units * slice / slices), u1 = (uint32_t)((uint64_t)units * (slice + 1) / slices);
    const uint32_t lo = min(c16, A.M - 1) * (uint32_t)A.left_pitch;
    Own& own = sh.own[wave];

    f32x4 acc[16];
#pragma unroll
    for (int i = 0; i < 16; i++) acc[i] = f32x4{};
    uint2 w[8];
    uint32_t sw;
    Eight<LEFT> e;
    auto ask = [&](uint32_t u) {
        const uint64_t n0 = (uint64_t)u * 32;
        const rsrc_t br = buffer_at(A.right + n0 * A.right_pitch + j0 / 2), bs = buffer_at(A.right_scales + n0 * A.right_spitch + j0 / 32);
        const uint32_t here = u < u1 ? (uint32_t)min(A.inner - n0, (uint64_t)32) : 0;
#pragma unroll
        for (uint32_t r = 0; r < 8; r++) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b64(br, ((g * 8 + r < here) & (c16 / 2 < blocks)) ? (g * 8 + r) * (uint32_t)A.right_pitch + c16 * 8 : kNowhere, 0, 0);
            w[r] = make_uint2(v[0], v[1]);
        }
        // (a word holds the scales of four blocks of a row; those past the last block belong to columns that are not stored)
        const uint32_t row = lane / 2;
        sw = __builtin_amdgcn_raw_buffer_load_b32(bs, ((row < here) & (lane % 2 * 4 < blocks)) ? row * (uint32_t)A.right_spitch + lane % 2 * 4 : kNowhere, 0, 0);
        e.load_words(buffer_at(A.left + n0 * float_bytes(LEFT)), g * 8 < here ? lo + g * 8 * float_bytes(LEFT) : kNowhere);
    };
    ask(u0);
    for (uint32_t u = u0; u < u1; u++) {
        own.scales[lane] = sw;
        i32x4 x[terms];
        e.terms(x);
        uint2 now[8];
#pragma unroll
        for (int r = 0; r < 8; r++) now[r] = w[r];
        ask(u + 1);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        float sc[8];
#pragma unroll
        for (uint32_t r = 0; r < 8; r++) sc[r] = mx_scale(reinterpret_cast<const uint8_t*>(own.scales)[(g * 8 + r) * 8 + c16 / 2]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int h = 0; h < 2; h++)
            unroll4([&](auto B) {
                uint32_t p[8];
#pragma unroll
                for (int r = 0; r < 8; r++) p[r] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(h ? now[r].y : now[r].x, sc[r], B.value));
                i32x4 even, odd;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    even[i] = (int)__builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], 0x05040100u);
                    odd[i] = (int)__builtin_amdgcn_perm(p[2 * i + 1], p[2 * i], 0x07060302u);
                }
                constexpr int j = B.value * 2;
#pragma unroll
                for (int q = 0; q < terms; q++) {
                    acc[h * 8 + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[q]), __builtin_bit_cast(bf16x8, even), acc[h * 8 + j], 0, 0, 0);
                    acc[h * 8 + j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x[q]), __builtin_bit_cast(bf16x8, odd), acc[h * 8 + j + 1], 0, 0, 0);
                }
            });
    }
    __syncthreads();                                                    // (the sums take the place of the scales)
#pragma unroll
    for (int j = 0; j < 16; j += 4)
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (g * 4 + i < A.M) {
                const f32x4 v = { acc[j][i], acc[j + 1][i], acc[j + 2][i], acc[j + 3][i] };
                *reinterpret_cast<f32x4*>(&sh.part[wave][g * 4 + i][c16 * 16 + j]) = v;
            }
    __syncthreads();
    for (uint32_t o = t; o < A.M * 256; o += 512) {
        const uint32_t m = o / 256, j = o % 256;
        if (j >= cols) continue;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; k++) v += sh.part[k][m][j];
        if (parts > 1) sums[((uint64_t)part * A.M + m) * sum_pitch + j0 + j] = v;
        else store_one(A.c, A.c_type, m * A.ldc + j0 + j, v);
    }
}

// Rows up to which k_mx_rows is taken.  Against 4096 x 4096 in four bits and with bf16, in microseconds: 32 rows 8.0 and 11.7, by tiles 11.5
// and 14.8; 64 rows (with room for them in its registers) 11.8 and 19.1, by tiles 12.6 and 17.3, against 8192 x 8192 24.9 and 39.1, by
// tiles 20.0 and 30.0.
constexpr uint64_t kFewRows = 32;
// And k_mx_grad_rows, which has registers for no more.  bf16, 16 rows through 4096 x 4096 12.0 us, by tiles 17.5; through 8192 x 8192 20.2 and 33.4;
// one row 9.2 and 16.3, 16.5 and 32.7.
constexpr uint64_t kFewGradRows = 16;

// Sums of the parts of a length, in their order, into C: a thread makes four neighbouring columns.
__global__ __launch_bounds__(64) void k_mx_join(const float* sums, uint32_t parts, uint64_t M, uint64_t outer, uint64_t pitch, void* c, uint64_t ldc, int type) {
    const uint64_t id = (uint64_t)blockIdx.x * 64 + threadIdx.x, per_row = pitch / 4, m = id / per_row, j = id % per_row * 4;
    if (m >= M) return;
    f32x4 v = {};
    for (uint32_t p = 0; p < parts; p += 8) {                           // (eight on their way at once)
        f32x4 w[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) w[i] = p + i < parts ? *reinterpret_cast<const f32x4*>(sums + ((p + i) * M + m) * pitch + j) : f32x4{};
#pragma unroll
        for (uint32_t i = 0; i < 8; i++)
            if (p + i < parts) v += w[i];
    }
    for (uint32_t i = 0; i < 4; i++)
        if (j + i < outer) store_one(c, type, m * ldc + j + i, v[i]);
}

// How a product is laid over the chip: tiles of 256 x 256, one workgroup to a compute unit, or of 128 x 128, two; and the length in parts,
// whose sums a second kernel joins, where there are fewer tiles than compute units.  The least of these estimates in microseconds is taken:
// a step of a tile takes `alone` where few of them run, and `share` more where each compute unit has one (two of 128 x 128: twice
// that), since all draw on the same caches and the same power.  Against the best of all tiles and parts on 66 shapes (40 to 4096 rows, sides
// of 1024 to 8192, operands in the caches) the choice costs 1.3 % on average, and 8 % at most but for few tiles in four bits (512 rows through
// 1024 x 4096: in four parts 14.6 us, in one 12.2; with operands from memory 15.5 and 15.8).  For instance bf16 on the left, 256 rows through
// 4096 x 4096: tiles of 128 37.6 us and in four parts 24.9, tiles of 256 73.9; 2048 rows through 8192 x 8192: 231.0, of 256 194.0.
struct Plan { uint32_t tile, parts; };
struct StepCost { float alone128, share128, alone256, share256; };
constexpr StepCost kStepCost[3] = { { 0.60f, 0.30f, 1.40f, 0.75f }, { 0.42f, 0.30f, 1.15f, 0.45f }, { 0.80f, 0.25f, 1.45f, 0.28f } };

Plan plan_tiles(int op, uint64_t M, uint64_t outer, uint32_t steps, uint32_t unit) {
    Plan best = { 256, 1 };
    float least = 0.0f;
    // A part has a whole number of units, and one at least: of more parts some would have no steps, and write and join sums of zeros.  The estimate
    // counts single steps all the same, which chooses better (float32, 52 rows through 1213 x 197: two units in two parts 13.4 us, in one 15.8).
    const uint32_t units = (steps + unit - 1) / unit;
    for (uint32_t tile = 128; tile <= 256; tile *= 2) {
        const float alone = tile == 128 ? kStepCost[op].alone128 : kStepCost[op].alone256;
        const float share = tile == 128 ? kStepCost[op].share128 : kStepCost[op].share256;
        const float resident = tile == 128 ? 512.0f : 256.0f;
        const uint64_t tiles = ((M + tile - 1) / tile) * ((outer + tile - 1) / tile);
        for (uint32_t parts = 1; parts <= 16 && (parts == 1 || (parts <= steps / 2 && tiles * parts <= 512)); parts++) {
            const float groups = (float)(tiles * parts), rounds = (float)(uint64_t)((groups + resident - 1.0f) / resident);
            const float step = alone + share * (groups < resident ? groups : resident) / 256.0f;
            float us = 6.0f + rounds * (5.0f + step * (float)((steps + parts - 1) / parts));
            if (parts > 1) us += 3.0f + (float)(parts * M * outer) * 8.0f / 4e6f;      // the joining kernel; its sums written and read
            if ((tile == 128 && parts == 1) || us < least) { best = { tile, std::min(parts, units) }; least = us; }
        }
    }
    return best;
}

uint64_t sum_pitch(uint64_t outer) { return (outer + 3) / 4 * 4; }

void launch_join(const float* sums, uint32_t parts, uint64_t M, uint64_t outer, void* c, uint64_t ldc, int type, hipStream_t st) {
    const uint64_t pitch = sum_pitch(outer);
    hipLaunchKernelGGL(k_mx_join, dim3((uint32_t)((M * (pitch / 4) + 63) / 64)), dim3(64), 0, st, sums, parts, M, outer, pitch, c, ldc, type);
}

size_t sums_bytes(const Plan& p, uint64_t M, uint64_t outer) { return p.parts > 1 ? (size_t)p.parts * M * sum_pitch(outer) * 4 : 0; }

template <int OP> hipError_t launch_tiles(TileArgs& T, const Plan& p, float* sums, hipStream_t st) {
    T.tiles_m = (uint32_t)((T.M + p.tile - 1) / p.tile); T.tiles_j = (uint32_t)((T.outer + p.tile - 1) / p.tile);
    T.parts = p.parts; T.sums = sums; T.sum_pitch = sum_pitch(T.outer);
    const dim3 grid(T.tiles_m * T.tiles_j * p.parts);
    // (Eight waves where the right is read as it lies: two on a SIMD fill each other's gaps, 41.3 us instead of 46.8 for 4096^3 in four bits.
    // The gradient's turning of the right is cheaper in pieces of whole blocks, four waves': 243 us instead of 255 for 4096 x 8192 x 4096.)
    if (p.tile == 256) hipLaunchKernelGGL((k_mx_tile<OP, 256, 256, 2, OP == GRAD ? 2 : 4>), grid, dim3(OP == GRAD ? 256 : 512), 0, st, T);
    else hipLaunchKernelGGL((k_mx_tile<OP, 128, 128, 2, 2>), grid, dim3(256), 0, st, T);
    if (p.parts > 1) launch_join(sums, p.parts, T.M, T.outer, T.c, T.ldc, T.c_type, st);
    return hipGetLastError();
}

// Whether the matrix instructions can be fed from the caller's rows: bf16, rows and their ends at multiples of 16 bytes.
bool fed_directly(const MxProductArgs& A, uint64_t inner, int left) { return left == BF16 && A.ldx % 8 == 0 && inner % 8 == 0; }

uint32_t steps_of(int kind, int left, uint64_t inner) {
    return kind == PRODUCT ? (uint32_t)((inner + 255) / 256) : (uint32_t)((inner + 63) / 64) * terms_of(left);
}

size_t terms_bytes(int kind, int left, uint64_t M, uint64_t inner) { return kind == PRODUCT ? 0 : (inner + 63) / 64 * 128 * M * terms_of(left); }

template <int T> void launch_terms(const MxProductArgs& A, uint64_t inner, uint32_t chunks, hipStream_t st) {
    const uint64_t groups = (A.M * chunks * 8 + 255) / 256, x = std::min<uint64_t>(groups, 1u << 22);       // (a launch has fewer than 2^32 threads along x)
    hipLaunchKernelGGL((k_mx_terms<T>), dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x)), dim3(256), 0, st, reinterpret_cast<const uint8_t*>(A.x), A.ldx,
                       A.ldx * float_bytes(T) % 16 == 0, A.M, inner, chunks, reinterpret_cast<uint16_t*>(A.ws));
}

size_t laid_bytes(int left, uint64_t M, uint64_t inner) { return (M * ((inner + 7) / 8 * 8) * float_bytes(left) + 255) / 256 * 256; }

// Parts of the rows of B in k_mx_grad_rows: a workgroup for every compute unit, 32 rows at least for every wave; not more than one kernel
// joins quickly: one row through 16384 x 512 10.6 us, in up to 16 parts 11.1, in up to 64 12.3; through 65536 x 1024 19.3, 25.2 and 18.5; through
// 8192 x 1024 9.8, 9.2 and 9.8.
uint32_t grad_parts(uint64_t outer, uint64_t inner) {
    const uint64_t strips = (outer + 255) / 256, most = (inner + 255) / 256;
    const uint64_t parts = strips >= 256 ? 1 : 256 / strips;
    return (uint32_t)std::min<uint64_t>(std::min(parts, most), 32);
}

// The left's floats for few rows: laid out anew where they cannot be read in 16-byte words.
hipError_t lay_left(const MxProductArgs& A, int left, RowArgs& R, hipStream_t st) {
    R.left = reinterpret_cast<const uint8_t*>(A.x); R.left_pitch = A.ldx * float_bytes(left);
    if ((R.M == 1 || R.left_pitch % 16 == 0) && R.inner % 8 == 0) return hipSuccess;
    const uint64_t row = (R.inner + 7) / 8 * 8 * float_bytes(left);
    uint8_t* const ws = reinterpret_cast<uint8_t*>(A.ws);
    const dim3 grid((uint32_t)((R.M * row / 16 + 255) / 256));
    if (left == F32) hipLaunchKernelGGL((k_mx_lay<4>), grid, dim3(256), 0, st, R.left, R.left_pitch, R.M, R.inner, ws);
    else hipLaunchKernelGGL((k_mx_lay<2>), grid, dim3(256), 0, st, R.left, R.left_pitch, R.M, R.inner, ws);
    R.left = ws; R.left_pitch = row;
    return hipGetLastError();
}

hipError_t launch_few(const MxProductArgs& A, int kind, int left, hipStream_t st) {
    RowArgs R = {};
    R.right = A.b.codes; R.right_pitch = A.b.pitch * 16; R.right_scales = A.b.scales; R.right_spitch = A.b.pitch;
    R.M = (uint32_t)A.M; R.outer = kind == GRAD ? A.K : A.N; R.inner = kind == GRAD ? A.N : A.K;
    R.c = A.c; R.ldc = A.ldc; R.c_type = A.c_type;
    if (kind == PRODUCT) {
        R.left = A.a.codes; R.left_pitch = A.a.pitch * 16; R.left_scales = A.a.scales; R.left_spitch = A.a.pitch;
        return launch_rows<-1>(R, st);
    }
    const hipError_t e = lay_left(A, left, R, st);
    if (e != hipSuccess) return e;
    if (kind == LINEAR) {
        R.inner = (R.inner + 7) / 8 * 8;                                // (laid out or not: the codes behind the end are 0)
        return left == F32 ? launch_rows<F32>(R, st) : left == F16 ? launch_rows<F16>(R, st) : launch_rows<BF16>(R, st);
    }
    const uint32_t parts = grad_parts(R.outer, R.inner);
    float* const sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(A.ws) + laid_bytes(left, A.M, R.inner));
    const uint64_t pitch = sum_pitch(R.outer);
    const dim3 grid((uint32_t)((R.outer + 255) / 256) * parts);
    if (left == F32) hipLaunchKernelGGL((k_mx_grad_rows<F32>), grid, dim3(512), 0, st, R, parts, sums, pitch);
    else if (left == F16) hipLaunchKernelGGL((k_mx_grad_rows<F16>), grid, dim3(512), 0, st, R, parts, sums, pitch);
    else hipLaunchKernelGGL((k_mx_grad_rows<BF16>), grid, dim3(512), 0, st, R, parts, sums, pitch);
    if (parts > 1) launch_join(sums, parts, R.M, R.outer, R.c, R.ldc, R.c_type, st);
    return hipGetLastError();
}

}  // namespace

size_t mx_product_workspace(int kind, int left, uint64_t M, uint64_t N, uint64_t K) {
    const uint64_t inner = kind == GRAD ? N : K, outer = kind == GRAD ? K : N;
    if (kind != GRAD && M <= kFewRows) return kind == PRODUCT ? 0 : laid_bytes(left, M, inner);
    if (kind == GRAD && M <= kFewGradRows) {
        const uint32_t parts = grad_parts(outer, inner);
        return laid_bytes(left, M, inner) + (parts > 1 ? parts * M * sum_pitch(outer) * 4 : 0);
    }
    // (bf16 may need no terms, but then it has the plan of one term)
    const Plan p = plan_tiles(kind, M, outer, steps_of(kind, left, inner), unit_of(kind, terms_of(left)));
    return terms_bytes(kind, left, M, inner) + sums_bytes(p, M, outer);
}

hipError_t launch_mx_product(const MxProductArgs& A, int kind, int left, hipStream_t st) {
    if (A.M <= (kind == GRAD ? kFewGradRows : kFewRows)) return launch_few(A, kind, left, st);
    TileArgs T = {};
    T.M = A.M; T.outer = kind == GRAD ? A.K : A.N; T.inner = kind == GRAD ? A.N : A.K;
    T.c = A.c; T.ldc = A.ldc; T.c_type = A.c_type;
    T.right = A.b.codes; T.right_pitch = A.b.pitch * 16; T.right_scales = A.b.scales; T.right_spitch = A.b.pitch;
    T.terms = 1;
    T.steps = steps_of(kind, left, T.inner);
    const Plan p = plan_tiles(kind, T.M, T.outer, T.steps, unit_of(kind, terms_of(left)));
    float* const sums = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(A.ws) + terms_bytes(kind, left, T.M, T.inner));
    if (kind == PRODUCT) {
        T.left = A.a.codes; T.left_pitch = A.a.pitch * 16; T.left_scales = A.a.scales; T.left_spitch = A.a.pitch;
        return launch_tiles<PRODUCT>(T, p, sums, st);
    }
    const uint32_t chunks = (uint32_t)((T.inner + 63) / 64);
    if (fed_directly(A, T.inner, left)) {
        T.left = reinterpret_cast<const uint8_t*>(A.x); T.left_pitch = A.ldx * 2;
    } else {
        T.terms = terms_of(left);
        if (left == F32) launch_terms<F32>(A, T.inner, chunks, st);
        else if (left == F16) launch_terms<F16>(A, T.inner, chunks, st);
        else launch_terms<BF16>(A, T.inner, chunks, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        T.left = reinterpret_cast<const uint8_t*>(A.ws); T.left_pitch = (uint64_t)chunks * 128 * T.terms;
    }
    T.per_term = (0x80000000u + T.terms - 1) / T.terms;
    return kind == LINEAR ? launch_tiles<LINEAR>(T, p, sums, st) : launch_tiles<GRAD>(T, p, sums, st);
}

}  // namespace nz
