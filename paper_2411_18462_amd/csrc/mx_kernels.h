// Kernels of the head in 4 bits: quantisation, rows read back by token, and the product with the hidden states.
//
// A value is a code of e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, two to a byte, the even column's in the low half) times its block's
// scale, a power of two as e8m0, for 32 neighbours of a row.  The matrix cores multiply such codes and take a scale for each 32 values along K
// themselves (16x16x128: lane l holds 32 values of row l % 16, those of block l / 16).  All products of two codes of a block lie within 2^8 of one another,
// so nothing is lost ahead of the sums in fp32.
#pragma once
#include "../../include/svip.h"
#include "head_store.h"

namespace svip {

constexpr int MX_BLOCK = 32, MX_RUN = 128;             // values to a scale; rows are filled up to whole runs
constexpr int E8M0_NAN = 255;

// ---- quantisation ------------------------------------------------------------------------------------------------------------------------
//
// The scale is 2^e with the least e >= -127 that brings the block's largest magnitude to 6, the largest e2m1 number, or below (no value is
// cut off); dividing by it is exact, so a code is x / 2^e rounded once.  e2m1 has no NaN: a block that holds a value that is not finite has the
// scale 255, the NaN of e8m0, and codes of zero.

__device__ __forceinline__ int mx_scale_code(unsigned amax)         // of the bits of the largest magnitude, e + 127; 127 for a block of zeros
{
    if (amax >= 0x7f800000u) return E8M0_NAN;
    if (amax == 0u) return 127;
    const int e = (int)(amax >> 23) - 2 + ((amax & 0x7fffffu) > 0x400000u);        // 6 = 1.5 * 2^2
    return e < 0 ? 0 : e;
}
// 2^(127 - code): at most 253 for finite values
__device__ __forceinline__ float mx_inverse(int code) { return code == E8M0_NAN ? 0.f : __uint_as_float((unsigned)(254 - code) << 23); }
// 2^(code - 127)
__device__ __forceinline__ float mx_scale(int code)
{
    return code == E8M0_NAN ? NAN : __uint_as_float(code == 0 ? 0x00400000u : (unsigned)code << 23);
}

struct MxQuantizeArgs {
    const void *x;
    long long row_stride;      // elements
    int rows, cols, runs;      // runs: of 128 columns in a row
    unsigned char *q;
    long long q_stride;
    unsigned char *scale;
    long long scale_stride;
};

constexpr int MX_WG = 256;
// 16 lanes (fp32: 32) a run, one load and one store a lane.  HBM: 128256 x 4096 in bf16 252 us, 5.3 TB/s (a copy: 5.1); 64 x 4096 2.4 us, a launch.
template <int DT>
__global__ __launch_bounds__(MX_WG) void k_mx_quantize(MxQuantizeArgs a)
{
    constexpr int VEC = Stored<DT>::VEC, LANES = MX_RUN / VEC, PER_BLOCK = MX_BLOCK / VEC;
    using X = typename Stored<DT>::type;
    const unsigned run = blockIdx.x * (MX_WG / LANES) + threadIdx.x / LANES;
    if (run >= (unsigned)a.rows * (unsigned)a.runs) return;
    const unsigned r = run / (unsigned)a.runs, c = (run - r * (unsigned)a.runs) * MX_RUN + threadIdx.x % LANES * VEC;
    const X *p = static_cast<const X *>(a.x) + (long long)r * a.row_stride + c;
    float v[VEC];
    if ((int)c + VEC <= a.cols) {              // (the memory takes a load of 16 bytes at any address)
        typedef X vec __attribute__((ext_vector_type(VEC), aligned(sizeof(X))));
        const vec w = *reinterpret_cast<const vec *>(p);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (float)w[i];
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (int)c + i < a.cols ? (float)p[i] : 0.f;
    }
    unsigned m = 0u;
#pragma unroll
    for (int i = 0; i < VEC; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = PER_BLOCK / 2; o; o /= 2) m = max(m, (unsigned)__shfl_xor((int)m, o));
    const int code = mx_scale_code(m);
    const float inv = mx_inverse(code);
    unsigned q = 0u;
    if (code != E8M0_NAN) {
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0] * inv, v[1] * inv, 1.f, 0);
        q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2] * inv, v[3] * inv, 1.f, 1);
        if constexpr (VEC == 8) {
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4] * inv, v[5] * inv, 1.f, 2);
            q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6] * inv, v[7] * inv, 1.f, 3);
        }
    }
    unsigned char *to = a.q + (long long)r * a.q_stride + c / 2;
    if constexpr (VEC == 8)
        *reinterpret_cast<unsigned *>(to) = q;
    else
        *reinterpret_cast<unsigned short *>(to) = (unsigned short)q;
    if (threadIdx.x % PER_BLOCK == 0) a.scale[(long long)r * a.scale_stride + c / MX_BLOCK] = (unsigned char)code;
}

// ---- rows read back ------------------------------------------------------------------------------------------------------------------------

struct MxRowsArgs {
    const unsigned char *q;
    long long q_stride;
    const unsigned char *scale;
    long long scale_stride;
    int rows, cols, chunks;    // chunks: of 8 columns in a row of the result
    const int *ids;            // [n], or null: rows 0 .. n - 1
    int n;
    void *out;
    long long out_stride;      // elements
};

// 8 values a lane: 4 bytes of codes, 16 or 32 bytes of values.  HBM: 128256 x 4096 to bf16 242 us, 5.5 TB/s; 8192 rows of 4096 by their ids 21 us, 4.0 TB/s; 64 rows
// of 2048 2.6 us, a launch.
template <int DT>
__global__ __launch_bounds__(MX_WG) void k_mx_rows(MxRowsArgs a)
{
    using X = typename Stored<DT>::type;
    const unsigned i = blockIdx.x * MX_WG + threadIdx.x, row = i / (unsigned)a.chunks;
    if (row >= (unsigned)a.n) return;
    const int c = (int)(i - row * (unsigned)a.chunks) * 8;
    const int id = a.ids ? a.ids[row] : (int)row;
    float v[8];
    if (id >= 0 && id < a.rows) {
        const unsigned q = *reinterpret_cast<const unsigned *>(a.q + id * a.q_stride + c / 2);
        const float s = mx_scale(a.scale[id * a.scale_stride + c / MX_BLOCK]);
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 w[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 1),
                         __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.f, 3)};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = w[e / 2][e % 2] * s;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = id < 0 ? 0.f : NAN;
    }
    X *to = static_cast<X *>(a.out) + (long long)row * a.out_stride + c;
    if (c + 8 <= a.cols) {
        typedef X vec __attribute__((ext_vector_type(8), aligned(sizeof(X))));
        vec w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = (X)v[e];
        *reinterpret_cast<vec *>(to) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < a.cols) to[e] = (X)v[e];
    }
}

// ---- logits --------------------------------------------------------------------------------------------------------------------------------
//
// Tiles of the product as in head_tile.h, copied into LDS step by step of K, two buffers deep or more.  A step is 128 bytes of a row: 256 values of 4-bit
// hidden states, multiplied in two halves, and 128 values of 8-bit ones, with 64 bytes of the weight.
//
// Few rows wait for the weight's bytes (64 x 128256 x 2048, 8-bit hidden states: 40 us, 3.9 TB/s; 1 row: 28 us, 5.0).  Large tiles wait for what feeds the products.
// A copy takes a compute unit about 7 cycles for each cache line that it touches, whether 128 bytes of it or 4:
// - The scales of a row and a step are 8 bytes, and copied step by step they would be as many lines as the codes.  They come in groups of GROUP steps.
// - 4 bits: steps of whole lines, 256 x 256 tiles.  1088 x 128256 x 4096: 385-413 us, 2.8-3.0 PFLOP/s (the library's largest 4-bit products reach 2.3 here,
//   its 8-bit ones 2.9; in fp32 450 us, 558 MB of logits), products under way in 40 % of the cycles at 1.9 GHz.  Leaving out one thing at a time of 434 us then: the copies 371, the reads of the scales 381 (bank
//   conflicts, now gone), the stores 388.  16 waves of 64 x 64 take 440, 8 of 128 x 64 453, 8 that replace each fragment as soon as its products are under way
//   512 (they spill), 4 of 128 x 128 488, two workgroups with 128 x 128 479, two with 256 x 128 in steps of 128 values 513.
// - 8 bits: the products take twice as long, and what counts is a second workgroup that multiplies while one waits: 256 x 128 tiles twice a unit leave room
//   for steps of 128 values only.  The same sizes: 529-540 us (without copies 353), in steps of 256 values with one workgroup 606-637, 256 x 256 tiles 583-605.

template <int BITS> constexpr int MX_STEP = BITS == 4 ? 2 * MX_RUN : MX_RUN;       // values of K to a step; BITS: of the hidden states

struct MxLogitsArgs {
    Operand weight, hidden;    // codes, in bytes; m = vocabulary, n = rows
    Operand weight_scale, hidden_scale;
    int N, V, K;               // K: values
    Tiles tiles;
    void *out;
    long long out_stride;      // elements
    int per_split;             // of K, a multiple of the step
    float *part;               // [splits][N][part_stride] where there are several, null: one
    long long part_stride;
};

// Copies 4 bytes a lane into LDS at `lds` (wave-uniform) + 4 * lane; see copy_to_lds.
__device__ __forceinline__ void copy4_to_lds(const char *base, unsigned voff, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds), "v"(voff), "s"(base) : "memory", "m0");
}

constexpr int MX_HALF = MX_RUN / 2;                    // bytes of a run

// A tile of codes in 4 bits in LDS with steps of 128 values: lines of 128 bytes hold two rows of 64.  The 16 bytes q (0 .. 3) of row r are chunk
// (4 (r % 2) + q) ^ (r / 4) % 4 of line r / 2, so that the same bytes of 16 neighbour rows, which 16 lanes read at a time, lie in different banks.
__device__ __forceinline__ unsigned mx_place(int row, int q) { return (unsigned)((row >> 1) * 128 + (((row & 1) * 4 + q) ^ (row >> 2 & 3)) * 16); }
template <int ROWS, int THREADS>
struct CodeStager {
    static constexpr int CHUNKS = ROWS * 4, ROUNDS = CHUNKS > THREADS ? CHUNKS / THREADS : 1, BYTES = ROWS * MX_HALF;
    static_assert(CHUNKS % 64 == 0 && (CHUNKS >= THREADS ? CHUNKS % THREADS == 0 : THREADS % CHUNKS == 0), "whole waves copy");
    const char *base;
    unsigned voff[ROUNDS], lds[ROUNDS];                // lds: wave-uniform
    __device__ void init(const Operand &o, int rows)
    {
        base = o.base;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int c = (r * THREADS + (int)threadIdx.x) % CHUNKS, x = (c & 7) ^ (c >> 4 & 3), row = (c >> 3) * 2 + (x >> 2);
            lds[r] = (unsigned)__builtin_amdgcn_readfirstlane(c & ~63) * 16u;
            voff[r] = (unsigned)min(row, rows - 1) * (unsigned)o.stride + (unsigned)(x & 3) * 16u;
        }
    }
    __device__ __forceinline__ void copy(unsigned at, long long byte, long long, int) const
    {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) copy_to_lds(base + byte, voff[r], at + lds[r]);
    }
};

// The scales of RUNS runs of 128 values of ROWS rows in 4 bits: [ROWS][4 RUNS] in LDS.  Rows past the end are read as the last one.
// Rows of 32 bytes: in rows 8 to 15 of 16 neighbours the words are swapped in pairs, so that the same ones of all 16 lie in different banks.
template <int ROWS, int THREADS, int RUNS>
struct ScaleStager {
    static constexpr int PITCH = 4 * RUNS, BYTES = ROWS * PITCH, ROUNDS = ROWS * RUNS / THREADS;
    static_assert(ROWS * RUNS % THREADS == 0 && THREADS / RUNS % 16 == 0 && RUNS <= 8, "whole rounds, and a thread's rows swap alike");
    __device__ static __forceinline__ unsigned place(int row, int byte) { return (unsigned)(row * PITCH + (RUNS == 8 ? byte ^ (row & 8) : byte)); }
    const char *base;
    unsigned stride;
    int last;
    __device__ void init(const Operand &o, int rows)
    {
        base = o.base;
        stride = (unsigned)o.stride;
        last = rows - 1;
    }
    // the runs from value k on, 4 bytes a lane; past k_end, a multiple of 128, the last one of the row again.  Addresses are made here each time and not kept in
    // registers.
    __device__ __forceinline__ void copy(unsigned at, int k, int k_end) const
    {
        unsigned tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        const unsigned run = RUNS == 8 ? tid % RUNS ^ (tid / RUNS & 8u) / 4u : tid % RUNS;
        const unsigned off = (unsigned)min(k + (int)run * MX_RUN, k_end - MX_RUN) / MX_BLOCK;
        at += (unsigned)__builtin_amdgcn_readfirstlane(tid & ~63u) * 4u;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            copy4_to_lds(base, (unsigned)min((int)(tid / RUNS) + r * (THREADS / RUNS), last) * stride + off, at + r * THREADS * 4);
    }
};

// Scales of hidden states in 8 bits, one for 128 values: those of HELD runs in LDS at a time.
constexpr int HELD = 32, HELD_PITCH = HELD + 4;

__device__ __forceinline__ i32x8 wide(i32x4 v) { return __builtin_shufflevector(v, v, 0, 1, 2, 3, -1, -1, -1, -1); }

// Of a row's 8 scales of a step of two halves those of the blocks that lane group g multiplies, g of either half: bytes 0 and 1.
__device__ __forceinline__ int scales_of(const char *row, unsigned pick)
{
    const uint2 v = *reinterpret_cast<const uint2 *>(row);
    return (int)__builtin_amdgcn_perm(v.y, v.x, pick);
}

// Logits of a tile.  BITS: of the hidden states.
template <typename S, int BITS, int DT>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::THREADS > 512 ? 4 : S::WAVES_PER_EU))) void k_mx_logits(MxLogitsArgs a)
{
    constexpr int STEP = MX_STEP<BITS>, HALVES = STEP / MX_RUN;
    constexpr int CODES_A = S::BM * STEP / 2, STAGE = CODES_A + S::BN * STEP_BYTES, SCALED = S::BM + (BITS == 4 ? S::BN : 0);
    constexpr int ROOM = S::STAGES * STAGE > 81920 ? 163840 : 81920;           // of LDS: all of a CU's, or half
    // steps to a group: 4 if there is room, 2 or 8 where the threads take so many
    constexpr int GROUP = S::BM * HALVES * 4 < S::THREADS || S::BN * HALVES * 4 < S::THREADS ? 8
                          : S::STAGES * STAGE + 2 * SCALED * HALVES * 16 + (BITS == 8 ? S::BN * HELD_PITCH : 0) <= ROOM ? 4 : 2;
    static_assert(S::STAGES - 2 < GROUP, "the wait for a group's first step covers the group's scales");
    static_assert(S::STAGES * STAGE >= S::BM * S::BN * 2, "store_rows lays the tile out where the codes were");
    using ScaleA = ScaleStager<S::BM, S::THREADS, GROUP * HALVES>;
    using ScaleB = ScaleStager<S::BN, S::THREADS, GROUP * HALVES>;
    constexpr int SCALES = SCALED * ScaleA::PITCH;
    struct Lds {
        char codes[S::STAGES][STAGE], scales[2][SCALES];
        unsigned char held[BITS == 8 ? S::BN * HELD_PITCH : 0];
    };
    __shared__ __attribute__((aligned(1024))) Lds lds;
    char *const smem = lds.codes[0];
    const unsigned tiles = (unsigned)a.tiles.m * (unsigned)a.tiles.n, split = blockIdx.x / tiles;
    int tm, tn;
    tile_of(blockIdx.x - split * tiles, a.tiles, 4, tm, tn);
    const int v0 = tm * S::BM, n0 = tn * S::BN, k0 = (int)split * a.per_split, k_end = min(a.K, k0 + a.per_split);
    const auto from = [](Operand o, int row) {
        o.base += (long long)row * o.stride;
        return o;
    };
    std::conditional_t<BITS == 4, Stager<KC, S::BM, S::THREADS, 1>, CodeStager<S::BM, S::THREADS>> sa;
    Stager<KC, S::BN, S::THREADS, 1> sb;
    ScaleA sw;
    ScaleB sh;
    sa.init(from(a.weight, v0), a.V - v0);
    sb.init(from(a.hidden, n0), a.N - n0);
    sw.init(from(a.weight_scale, v0), a.V - v0);
    if (BITS == 4) sh.init(from(a.hidden_scale, n0), a.N - n0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN, g = lane >> 4, l16 = lane & 15;
    const unsigned pick = 0x0c0c0400u + 0x0101u * (unsigned)g, place = mx_place(l16, g);
    Reader<KC, S::BM, 1> ra;
    Reader<KC, S::BN, 1> rb;
    ra.init(lane);
    rb.init(lane);
    f32x4 acc[S::FM][S::FN];
#pragma unroll
    for (int i = 0; i < S::FM; ++i)
#pragma unroll
        for (int j = 0; j < S::FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    constexpr int COPIES = decltype(sa)::ROUNDS + decltype(sb)::ROUNDS;
    const int steps = (k_end - k0 + STEP - 1) / STEP, groups = (steps + GROUP - 1) / GROUP;
    const unsigned lds0 = (unsigned)(uintptr_t)smem;
    // The last step of an odd K has one of two halves.  The other is zeros, with the last scales of its row again: a NaN among them stands in the first half too.
    auto copy = [&](int s, unsigned buffer) {
        const int k = k0 + s * STEP;
        sa.copy(lds0 + buffer, k / 2, k_end / 2, 0);
        if (BITS == 4)
            sb.copy(lds0 + buffer + CODES_A, k / 2, k_end / 2, 0);
        else
            sb.copy(lds0 + buffer + CODES_A, k, k_end, 0);
    };
    auto copy_scales = [&](int group) {
        const unsigned at = (unsigned)(uintptr_t)lds.scales[group & 1];
        sw.copy(at, k0 + group * GROUP * STEP, k_end);
        if (BITS == 4) sh.copy(at + ScaleA::BYTES, k0 + group * GROUP * STEP, k_end);
    };
    // (8 bits) the scales of the steps from s0 on; nobody reads those of the steps before any more
    auto hold = [&](int s0) {
        const int count = min(HELD, steps - s0);
        for (int i = threadIdx.x; i < S::BN * HELD / 4; i += S::THREADS) {
            const int r = i / (HELD / 4), q = i % (HELD / 4) * 4, n = min(n0 + r, a.N - 1);
            const char *p = a.hidden_scale.base + n * a.hidden_scale.stride + k0 / MX_RUN + s0 + q;
            unsigned word = 0u;
            if (q + 4 <= count)
                __builtin_memcpy(&word, p, 4);
            else
                for (int e = 0; e < count - q; ++e) word |= (unsigned)(unsigned char)p[e] << (8 * e);
            *reinterpret_cast<unsigned *>(lds.held + r * HELD_PITCH + q) = word;
        }
    };
    copy_scales(0);
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s)
        if (s < steps) copy(s, s * STAGE);
    unsigned buffer = 0, next = (S::STAGES - 1) * STAGE;       // of this step, and of the one that is copied
    for (int s = 0; s < steps; ++s) {
        if (BITS == 8 && s % HELD == 0) {
            if (s) __syncthreads();
            hold(s);                       // (the barrier below publishes them)
        }
        if (s + S::STAGES - 2 < steps)
            wait_copies_and_meet<(S::STAGES - 2) * COPIES>();
        else
            wait_copies_and_meet<0>();
        if (s + S::STAGES - 1 < steps) copy(s + S::STAGES - 1, next);
        if (s % GROUP == 0 && s / GROUP + 1 < groups) copy_scales(s / GROUP + 1);
        const char *ta = smem + buffer, *tb = ta + CODES_A, *scale = lds.scales[s / GROUP & 1] + ScaleA::place(l16, s % GROUP * (4 * HALVES));
        int sca[S::FM], scb[S::FN];
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const char *p = scale + (wm + 16 * i) * ScaleA::PITCH;
            sca[i] = BITS == 4 ? scales_of(p, pick) : *reinterpret_cast<const unsigned char *>(p + g);
        }
#pragma unroll
        for (int j = 0; j < S::FN; ++j)
            scb[j] = BITS == 4 ? scales_of(scale + (S::BM + wn + 16 * j) * ScaleA::PITCH, pick) : lds.held[(wn + 16 * j + l16) * HELD_PITCH + s % HELD];
        const auto half = [&](auto which) {
            constexpr int H = decltype(which)::value;
            i32x8 fa[S::FM], fb[S::FN];
            s16x8 v;
#pragma unroll
            for (int j = 0; j < S::FN; ++j) {
                if constexpr (BITS == 4) {
                    rb.half(tb, wn + 16 * j, H, v);
                    fb[j] = wide(__builtin_bit_cast(i32x4, v));
                } else {
                    fb[j] = rb.whole(tb, wn + 16 * j);
                }
            }
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                if constexpr (BITS == 4)
                    ra.half(ta, wm + 16 * i, H, v);
                else
                    v = *reinterpret_cast<const s16x8 *>(ta + (wm + 16 * i) * MX_HALF + place);
                fa[i] = wide(__builtin_bit_cast(i32x4, v));
            }
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], acc[i][j], 4, BITS == 4 ? 4 : 0, H, sca[i], H, scb[j]);
        };
        half(std::integral_constant<int, 0>{});
        if constexpr (HALVES == 2) half(std::integral_constant<int, 1>{});
        buffer = buffer + STAGE == S::STAGES * STAGE ? 0 : buffer + STAGE;
        next = next + STAGE == S::STAGES * STAGE ? 0 : next + STAGE;
    }
    using X = typename Stored<DT>::type;
    if (a.part) {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int n = n0 + wn + 16 * j + l16;
            if (n >= a.N) continue;
            float *row = a.part + ((long long)split * a.N + n) * a.part_stride;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int v = v0 + wm + 16 * i + 4 * g;
                if (v < a.part_stride) *reinterpret_cast<f32x4 *>(row + v) = acc[i][j];       // (V filled up to fours)
            }
        }
    } else if constexpr (DT != SVIP_F32) {
        store_rows<S, X>(smem, a.N - n0, a.V - v0, static_cast<X *>(a.out) + n0 * a.out_stride + v0, a.out_stride, [&](int i, int j) { return acc[i][j]; });
    } else {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int n = n0 + wn + 16 * j + l16;
            if (n >= a.N) continue;
            X *row = static_cast<X *>(a.out) + n * a.out_stride;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int v = v0 + wm + 16 * i + 4 * g;
                if (v < a.V) put_up_to_4<DT>(row + v, acc[i][j], a.V - v);
            }
        }
    }
}

struct MxJoinArgs {
    const float *part;
    long long part_stride;
    int splits, N, V;
    void *out;
    long long out_stride;
};
// The sums of the splits of K, four logits a thread.
template <int DT>
__global__ __launch_bounds__(256) void k_mx_join(MxJoinArgs a)
{
    const int groups = (int)((a.part_stride + 1023) / 1024), n = blockIdx.x / groups;
    const int v = ((blockIdx.x - n * groups) * 256 + (int)threadIdx.x) * 4;
    if (v >= a.V) return;
    const float *p = a.part + n * a.part_stride + v;
    f32x4 s = *reinterpret_cast<const f32x4 *>(p);
    for (int k = 1; k < a.splits; ++k) s += *reinterpret_cast<const f32x4 *>(p + (long long)k * a.N * a.part_stride);
    put_up_to_4<DT>(static_cast<typename Stored<DT>::type *>(a.out) + n * a.out_stride + v, s, a.V - v);
}

}  // namespace svip
