// Products of two matrices on the matrix cores, tile by tile: the core of the head's operators (head_kernels.h).
//
//   C[m, n] = sum over k of A(m, k) B(n, k)
//
// A workgroup of WAVES_M x WAVES_N waves makes a BM x BN tile of C; a wave holds its (BM / WAVES_M) x (BN / WAVES_N) part as
// 16 x 16 fragments in registers.  K goes by in steps of 128 bytes (64 16-bit values or 128 8-bit ones) that are copied from memory
// straight into LDS (global_load_lds_dwordx4, no registers on the way), STAGES deep, with one barrier per step, which both
// publishes a step and frees the buffer of the one before.
//
// An operand comes in one of two layouts:
//   KC  k contiguous (rows of m or n): the LDS tile is [rows][128 bytes]; a fragment is read with ds_read_b128.  16-byte chunk c of
//       row r lies at chunk c ^ (r / 2 % 8), so that the 16 rows of a fragment, of which two span the 64 banks, meet no bank twice.
//   KS  k strided (rows of k): the LDS tile is [k][columns].  A fragment of 16-bit values is read with ds_read_b64_tr_b16, which
//       gives lane i of 16 the column i of a 4 x 16 block; the four rows of a block would lie in the same banks, so chunk c of
//       row k lies at chunk c ^ (2 (k % 4) + 8 (k / 8 % 2)).  fp32 values are read one by one, 16 columns of rows k, k + 4, k + 8 and k + 12
//       at a time: chunk c ^ 4 (k / 4 % 4).
// The copy into LDS writes lane after lane, so the permutation is made by which chunk a lane asks for.
//
// Rows past the end of an operand are read as its last row (their results are not stored); positions past the end of K are read
// from a line of zeros in both operands, so that nothing outside the operands is ever multiplied.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace svip {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int STEP_BYTES = 128;                   // of K per step

// Zeros that lanes past the end of K read (the largest read is 16 bytes a lane).
__device__ __attribute__((aligned(256))) static const unsigned zero_line[64] = {};

enum { KC = 0, KS = 1 };

struct Operand {
    const char *base;          // element (0, 0) of the tile's operand
    long long stride;          // bytes between its rows (of m or n: KC, of k: KS)
    long long plane;           // bytes between its planes (see TERMS)
};

// Copies 16 bytes a lane into LDS at `lds` (wave-uniform) + 16 * lane.  Written as assembly so that the compiler does not wait for
// the copy before every LDS read that might alias it; wait_copies_and_meet() is the wait.  A copy may not follow the write of M0, its LDS address, at
// once: one wait state lies between them, which nobody but this code puts into assembly.  (It costs nothing: loss of 8192 x 151936 x 2048 in bf16 3.75 to
// 3.79 ms, where 3.78 was measured without it.)
__device__ __forceinline__ void copy_to_lds(const char *base, unsigned voff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy_to_lds(const char *lane_address, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(lane_address) : "memory", "m0");
}
// All but the last `LEFT` copies of this wave have landed and its LDS reads have returned; then the barrier.
template <int LEFT>
__device__ __forceinline__ void wait_copies_and_meet()
{
    static_assert(LEFT < 64, "the counter has six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// One operand's part of a workgroup's tile: ROWS rows (KC) or columns (KS).
template <int LAYOUT, int ROWS, int THREADS, int ESIZE>
struct Stager {
    static constexpr int CHUNKS = ROWS * STEP_BYTES / 16;
    static constexpr int ROUNDS = CHUNKS > THREADS ? CHUNKS / THREADS : 1;      // (fewer chunks than threads: some are copied twice)
    static constexpr int BYTES = ROWS * STEP_BYTES;
    static constexpr int STEP = STEP_BYTES / ESIZE, PER_CHUNK = 16 / ESIZE;   // elements
    static constexpr int PER_ROW = ROWS / PER_CHUNK;                           // KS: chunks in a row
    static_assert(CHUNKS % 64 == 0 && (CHUNKS >= THREADS ? CHUNKS % THREADS == 0 : THREADS % CHUNKS == 0), "whole waves copy");

    Operand op;
    unsigned voff[ROUNDS];
    unsigned lds[ROUNDS];      // wave-uniform

    // rows: of the operand from the tile's first on, at least 1 (KS: columns, whole chunks)
    __device__ void init(const Operand &o, int rows)
    {
        op = o;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int c = (r * THREADS + (int)threadIdx.x) % CHUNKS;
            lds[r] = (unsigned)__builtin_amdgcn_readfirstlane(c & ~63) * 16u;
            if (LAYOUT == KC) {
                const int row = c >> 3, chunk = (c & 7) ^ ((row >> 1) & 7);
                voff[r] = (unsigned)(row < rows ? row : rows - 1) * (unsigned)op.stride + (unsigned)chunk * 16u;
            } else {
                const int k = c / PER_ROW, chunk = (c % PER_ROW) ^ twist(k);
                voff[r] = (unsigned)k * (unsigned)op.stride + (unsigned)(chunk < rows / PER_CHUNK ? chunk : 0) * 16u;
            }
        }
    }
    __device__ static int twist(int k) { return (ESIZE == 4 ? k & 12 : ((k & 3) << 1) | (k & 8)) & (PER_ROW - 1); }

    __device__ __forceinline__ const char *step_base(int k, int plane) const
    {
        return op.base + plane * op.plane + (LAYOUT == KC ? (long long)k * ESIZE : k * op.stride);
    }
    // Round r of the copy of the step at `k` (element index, a multiple of the step), whose base is `base`, into the buffer at `at`; k_end:
    // elements of K.
    __device__ __forceinline__ void copy_round(int r, const char *base, unsigned at, int k, int k_end) const
    {
        if (k + STEP <= k_end) {
            copy_to_lds(base, voff[r], at + lds[r]);
        } else {
            const int c = (r * THREADS + (int)threadIdx.x) % CHUNKS;
            const int mine = LAYOUT == KC ? k + ((c & 7) ^ ((c >> 4) & 7)) * PER_CHUNK : k + c / PER_ROW;
            copy_to_lds(mine < k_end ? base + voff[r] : reinterpret_cast<const char *>(zero_line), at + lds[r]);
        }
    }
    __device__ __forceinline__ void copy_whole_round(int r, const char *base, unsigned at) const { copy_to_lds(base, voff[r], at + lds[r]); }
    __device__ __forceinline__ void copy(unsigned at, int k, int k_end, int plane) const
    {
        const char *base = step_base(k, plane);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) copy_round(r, base, at, k, k_end);
    }
};

// Reads fragments of an operand's LDS tile: 16 rows of m or n from `row0` (a multiple of 16) and half a step, or a whole step of 8-bit values.
// Lane l has row l % 16; of K it has, for 16 bits, the 8 values from 8 (l / 16) on in half h, for fp32 the 4 from 4 (l / 16) on.
template <int LAYOUT, int ROWS, int ESIZE>
struct Reader {
    unsigned at[2];
    __device__ void init(int lane)
    {
        const int row = lane & 15, g = lane >> 4;
        if (LAYOUT == KC) {
            at[0] = (unsigned)(row * STEP_BYTES + (((g) ^ (row >> 1)) & 7) * 16);
            at[1] = (unsigned)(row * STEP_BYTES + (((4 + g) ^ (row >> 1)) & 7) * 16);
        } else if (ESIZE == 2) {
            const int k = 8 * g + (row >> 2);
            at[0] = (unsigned)(k * ROWS * 2 + (row & 1) * 8);
            at[1] = (unsigned)((((row & 3) >> 1)) ^ Stager<KS, ROWS, 64, 2>::twist(k));
        } else {
            at[0] = (unsigned)(4 * g * ROWS * 4 + (row & 3) * 4);
            at[1] = (unsigned)((row >> 2) ^ Stager<KS, ROWS, 64, 4>::twist(4 * g));
        }
    }
    __device__ __forceinline__ void half(const char *tile, int row0, int h, s16x8 &f) const
    {
        if (LAYOUT == KC) {
            f = *reinterpret_cast<const s16x8 *>(tile + at[h] + row0 * STEP_BYTES);
        } else {
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const unsigned a = at[0] + (((unsigned)(row0 / 8)) ^ at[1]) * 16u;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + a + (32 * h) * ROWS * 2));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + a + (32 * h + 4) * ROWS * 2));
            f = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    __device__ __forceinline__ void half(const char *tile, int row0, int h, f32x4 &f) const
    {
        if (LAYOUT == KC) {
            f = *reinterpret_cast<const f32x4 *>(tile + at[h] + row0 * STEP_BYTES);
        } else {
            const char *p = tile + at[0] + (((unsigned)(row0 / 4)) ^ at[1]) * 16u;
#pragma unroll
            for (int q = 0; q < 4; ++q) f[q] = *reinterpret_cast<const float *>(p + (16 * h + q) * ROWS * 4);
        }
    }
    __device__ __forceinline__ i32x8 whole(const char *tile, int row0) const
    {
        const i32x4 lo = *reinterpret_cast<const i32x4 *>(tile + at[0] + row0 * STEP_BYTES);
        const i32x4 hi = *reinterpret_cast<const i32x4 *>(tile + at[1] + row0 * STEP_BYTES);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// What the products are made of.
struct Bf16 {
    using Frag = s16x8;
    static constexpr int SIZE = 2;
    __device__ static __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
struct F16 {
    using Frag = s16x8;
    static constexpr int SIZE = 2;
    __device__ static __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};
struct F32 {
    using Frag = f32x4;
    static constexpr int SIZE = 4;
    __device__ static __forceinline__ f32x4 mfma(f32x4 a, f32x4 b, f32x4 c)
    {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[q], b[q], c, 0, 0, 0);
        return c;
    }
};

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, int STAGES_>
struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, STAGES = STAGES_;
    static constexpr int THREADS = 64 * WAVES_M * WAVES_N;
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, FM = WM / 16, FN = WN / 16;
    static constexpr int STAGE_BYTES = (BM + BN) * STEP_BYTES;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES;
    static constexpr int WAVES_PER_EU = FM * FN > 32 ? 1 : 2;          // (registers for one wave, or two)
    static_assert(WM % 16 == 0 && WN % 16 == 0, "whole fragments");
};

// The loop over K.  TERMS = 1: one plane each.  TERMS = 2: two planes (high and low part) of B, and the products with low and with high.
// TERMS = 3: two planes each, and the products low x high, high x low and high x high, the small ones first.
template <typename T, typename S, int LA, int LB, int TERMS>
__device__ __forceinline__ void multiply(const Operand &a, int a_rows, const Operand &b, int b_rows, int k0, int k_end, char *smem,
                                         f32x4 (&acc)[S::FM][S::FN])
{
    Stager<LA, S::BM, S::THREADS, T::SIZE> sa;
    Stager<LB, S::BN, S::THREADS, T::SIZE> sb;
    sa.init(a, a_rows);
    sb.init(b, b_rows);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN;
    Reader<LA, S::BM, T::SIZE> ra;
    Reader<LB, S::BN, T::SIZE> rb;
    ra.init(lane);
    rb.init(lane);
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    constexpr int STEP = STEP_BYTES / T::SIZE, COPIES = decltype(sa)::ROUNDS + decltype(sb)::ROUNDS;
    const int per_term = (k_end - k0 + STEP - 1) / STEP, steps = TERMS * per_term;
    const unsigned lds0 = (unsigned)(uintptr_t)smem;
    // The copy of a step in COPIES parts.
    struct {
        const char *a, *b;
        unsigned at;
        int k;
    } next = {};
    auto aim = [&](int s, int buffer) {
        const int term = TERMS == 1 ? 0 : s / per_term;
        next.k = k0 + (s - term * per_term) * STEP;
        next.at = lds0 + (unsigned)buffer * S::STAGE_BYTES;
        next.a = sa.step_base(next.k, TERMS == 3 && term == 0);       // plane 0: high, 1: low
        next.b = sb.step_base(next.k, TERMS != 1 && term == TERMS - 2);
    };
    auto copy_part = [&](int p, auto whole) {
        constexpr int A = decltype(sa)::ROUNDS;
        if constexpr (decltype(whole)::value) {
            if (p < A)
                sa.copy_whole_round(p, next.a, next.at);
            else
                sb.copy_whole_round(p - A, next.b, next.at + S::BM * STEP_BYTES);
        } else {
            if (p < A)
                sa.copy_round(p, next.a, next.at, next.k, k_end);
            else
                sb.copy_round(p - A, next.b, next.at + S::BM * STEP_BYTES, next.k, k_end);
        }
    };
    auto copy = [&](int s, int buffer) {
        aim(s, buffer);
#pragma unroll
        for (int p = 0; p < COPIES; ++p) copy_part(p, std::false_type{});
    };
    // Step s is multiplied in two halves of K.  Its second half is read into registers while the first is multiplied, the next step's first
    // half while the second is: a row's fragment of A is replaced as soon as the row's products are under way.  Between the two, when every
    // wave has all of step s in registers, one barrier: the next step has landed, and the buffer of this one is copied over.  The
    // barrier comes LAG rows into the second half, which cover the last reads of it.  The copy that it allows is issued in parts, one or two
    // to a row: all at once they would fill the queue of the address unit (16 cycles each) and hold up the wave's products.
    constexpr int LAG = S::FM / 4;
    typename T::Frag fa[S::FM], fb[2][S::FN];
    const char *tile = smem;
    auto read_a = [&](int i, int h) { ra.half(tile, wm + 16 * i, h, fa[i]); };
    auto read_b = [&](int h) {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) rb.half(tile + S::BM * STEP_BYTES, wn + 16 * j, h, fb[h][j]);
    };
    auto row = [&](int i, int h) {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = T::mfma(fa[i], fb[h][j], acc[i][j]);
    };
#pragma unroll
    for (int s = 0; s < S::STAGES; ++s)
        if (s < steps) copy(s, s);
    if (steps >= S::STAGES)
        wait_copies_and_meet<(S::STAGES - 1) * COPIES>();
    else
        wait_copies_and_meet<0>();
    read_b(0);
#pragma unroll
    for (int i = 0; i < S::FM; ++i) read_a(i, 0);
    int buffer = 0;
    constexpr int PER_ROW = (COPIES + S::FM - 1) / S::FM, FIRST_ROWS = S::FM - LAG;
    bool more = false;
    int s = 0;
    // MAIN: a step behind which a whole one is copied; what its first rows carry is the rest of the copy begun in the step before it, also whole.
    auto step = [&](auto main) __attribute__((always_inline)) {
        constexpr bool MAIN = decltype(main)::value;
        read_b(1);
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            row(i, 0);
            read_a(i, 1);
#pragma unroll
            for (int p = (FIRST_ROWS + i) * PER_ROW; p < (FIRST_ROWS + i + 1) * PER_ROW; ++p)
                if (p < COPIES && (MAIN || more)) copy_part(p, main);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < LAG; ++i) row(i, 1);
        __builtin_amdgcn_sched_barrier(0);
        if (MAIN || s + S::STAGES <= steps)
            wait_copies_and_meet<(S::STAGES - 2) * COPIES>();
        else
            wait_copies_and_meet<0>();
        more = MAIN || s + S::STAGES < steps;
        if (more) aim(s + S::STAGES, buffer);
        buffer = buffer + 1 == S::STAGES ? 0 : buffer + 1;
        tile = smem + buffer * S::STAGE_BYTES;
        read_b(0);                         // (after the last step: of what the buffer held before, and not used)
#pragma unroll
        for (int i = LAG; i < S::FM; ++i) {
            row(i, 1);
            read_a(i - LAG, 0);
#pragma unroll
            for (int p = (i - LAG) * PER_ROW; p < (i - LAG + 1) * PER_ROW; ++p)
                if (p < COPIES && (MAIN || more)) copy_part(p, main);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = S::FM - LAG; i < S::FM; ++i) read_a(i, 0);
    };
    if (steps > 0) step(std::false_type{}), ++s;
    if (TERMS == 1 || (k_end - k0) % STEP == 0) {
        const int last = k0 + (steps - 1) * STEP + STEP <= k_end || TERMS != 1 ? steps : steps - 1;      // whole steps end here
        for (; s + S::STAGES < last; ++s) step(std::true_type{});
    }
    for (; s < steps; ++s) step(std::false_type{});
}

}  // namespace svip
