// Kernels of the head's operators: the matrix that turns hidden states into logits, in 8 bits for serving, and the cross entropy over
// its logits with the gradient for training.  The products are those of head_tile.h with m = vocabulary (or hidden channel) and
// n = rows of hidden states (or vocabulary), so that a lane's four results are neighbours in memory.
#pragma once
#include "../../include/svip.h"
#include "head_store.h"
#include "wave_ops.h"

namespace svip {

constexpr float HEAD_LOG2E = 1.4426950408889634f;
constexpr double HEAD_LN2 = 0.69314718055994530942;

// ---- 8 bits with a scale for each block ------------------------------------------------------------------------------------------------
//
// The scale is 2^e with the least e >= -127 that brings the block's largest finite magnitude to 448, the largest e4m3 number, or below: the
// matrix cores multiply by such scales themselves, and dividing by one is exact, so a code is x / 2^e rounded once.  (With a scale of
// amax / 448 a block's largest value would be a code without error; e4m3 keeps three mantissa bits at any magnitude, so all that a power
// of two costs is up to one bit at the small end of 2^15 : 1.)  Values that are not finite do not count for e and become the code of NaN.

constexpr int QBLOCK = 128;

__device__ __forceinline__ int scale_code(unsigned amax)            // e + 127; 127 for a block of zeros
{
    if (amax == 0u) return 127;
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u);        // 448 = 1.75 * 2^8
    return e < 0 ? 0 : e;
}
__device__ __forceinline__ float inverse_scale(int code) { return __uint_as_float((unsigned)(254 - code) << 23); }
__device__ __forceinline__ unsigned codes4(float a, float b, float c, float d, float inv)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inv, b * inv, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c * inv, d * inv, r, true);
    unsigned u = (unsigned)r;
    const float x[4] = {a, b, c, d};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if ((__float_as_uint(x[i]) & 0x7f800000u) == 0x7f800000u) u = (u & ~(0xffu << (8 * i))) | (0x7fu << (8 * i));
    return u;
}

struct QuantizeArgs {
    const void *x;
    long long row_stride;      // elements
    int rows, cols, kb;        // kb: blocks of 128 columns
    unsigned char *q;
    long long q_stride;
    unsigned char *scale;
    long long scale_stride;
};

// 16 bytes of x from column c of row r on, as floats, zeros past the last column.  Rows begin wherever their type may: the memory takes a load of
// 16 bytes at any address.
template <int DT>
__device__ __forceinline__ void load_chunk(const QuantizeArgs &a, long long r, int c, float (&v)[Stored<DT>::VEC])
{
    constexpr int VEC = Stored<DT>::VEC;
    using X = typename Stored<DT>::type;
    const X *p = static_cast<const X *>(a.x) + r * a.row_stride + c;
    if (c + VEC <= a.cols) {
        typedef X vec __attribute__((ext_vector_type(VEC), aligned(sizeof(X))));
        const vec w = *reinterpret_cast<const vec *>(p);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = (float)w[i];
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = c + i < a.cols ? (float)p[i] : 0.f;
    }
}
template <int DT>
__device__ __forceinline__ void store_codes(unsigned char *p, const float (&v)[Stored<DT>::VEC], float inv)
{
    if constexpr (Stored<DT>::VEC == 8) {
        uint2 u;
        u.x = codes4(v[0], v[1], v[2], v[3], inv);
        u.y = codes4(v[4], v[5], v[6], v[7], inv);
        *reinterpret_cast<uint2 *>(p) = u;
    } else {
        *reinterpret_cast<unsigned *>(p) = codes4(v[0], v[1], v[2], v[3], inv);
    }
}

// Blocks of 1 x 128: 16 lanes (fp32: 32) a block, one load and one store a lane.  64 rows of 4096 bf16: 2.8 us, a launch; 100000 x 5000: 310 us, 4.8 TB/s.
constexpr int QUANT_WG = 256;
template <int DT>
__global__ __launch_bounds__(QUANT_WG) void k_quantize_rows(QuantizeArgs a)
{
    constexpr int VEC = Stored<DT>::VEC, LANES = QBLOCK / VEC, PER_WG = QUANT_WG / LANES;
    const long long block = (long long)blockIdx.x * PER_WG + threadIdx.x / LANES;
    if (block >= (long long)a.rows * a.kb) return;
    const long long r = block / a.kb;
    const int kb = (int)(block - r * a.kb), lane = threadIdx.x % LANES;
    float v[VEC];
    load_chunk<DT>(a, r, kb * QBLOCK + lane * VEC, v);
    unsigned m = 0u;
#pragma unroll
    for (int i = 0; i < VEC; ++i) m = max(m, finite_magnitude(v[i]));
#pragma unroll
    for (int o = LANES / 2; o; o /= 2) m = max(m, (unsigned)__shfl_xor((int)m, o));
    const int code = scale_code(m);
    store_codes<DT>(a.q + r * a.q_stride + kb * QBLOCK + lane * VEC, v, inverse_scale(code));
    if (lane == 0) a.scale[r * a.scale_stride + kb] = (unsigned char)code;
}

// Blocks of 128 x 128: a workgroup each, the block in registers between its two uses, so that it is read once.  128256 x 4096 bf16: 291 us, 5.4 TB/s (a
// copy of 1 GiB: 5.2).
template <int DT>
__global__ __launch_bounds__(QUANT_WG) void k_quantize_blocks(QuantizeArgs a)
{
    constexpr int VEC = Stored<DT>::VEC, LANES = QBLOCK / VEC, ROWS = QUANT_WG / LANES, ROUNDS = QBLOCK / ROWS;
    const int kb = blockIdx.x % (unsigned)a.kb, rb = blockIdx.x / (unsigned)a.kb;
    const int c = kb * QBLOCK + (threadIdx.x % LANES) * VEC, r0 = rb * QBLOCK + threadIdx.x / LANES;
    float v[ROUNDS][VEC];
    unsigned m = 0u;
    if ((kb + 1) * QBLOCK <= a.cols) {         // whole columns: rows behind the last are read as the last, all loads under way at once
        using X = typename Stored<DT>::type;
        typedef X vec __attribute__((ext_vector_type(VEC), aligned(sizeof(X))));
        vec w[ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int r = r0 + i * ROWS < a.rows ? r0 + i * ROWS : a.rows - 1;
            w[i] = *reinterpret_cast<const vec *>(static_cast<const X *>(a.x) + r * a.row_stride + c);
        }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = (float)w[i][j];
    } else {
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) load_chunk<DT>(a, r0 + i * ROWS < a.rows ? r0 + i * ROWS : a.rows - 1, c, v[i]);
    }
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) m = max(m, finite_magnitude(v[i][j]));
#pragma unroll
    for (int o = 32; o; o /= 2) m = max(m, (unsigned)__shfl_xor((int)m, o));
    __shared__ unsigned top[QUANT_WG / 64];
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = m;
    __syncthreads();
    m = max(max(top[0], top[1]), max(top[2], top[3]));
    const int code = scale_code(m);
    const float inv = inverse_scale(code);
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
        if (r0 + i * ROWS < a.rows) store_codes<DT>(a.q + (long long)(r0 + i * ROWS) * a.q_stride + c, v[i], inv);
    if (threadIdx.x == 0) a.scale[rb * a.scale_stride + kb] = (unsigned char)code;
}

// ---- logits from 8-bit matrices ------------------------------------------------------------------------------------------------------------

struct HeadLogitsArgs {
    Operand weight, hidden;    // codes; m = vocabulary, n = rows
    const unsigned char *weight_scale, *hidden_scale;
    long long weight_scale_stride, hidden_scale_stride;
    int N, V, K;
    Tiles tiles;
    void *out;
    long long out_stride;      // elements
    int per_split;             // of K, a multiple of the step
    float *part;               // [splits][N][part_stride] where there are several, null: one
    long long part_stride;
};

constexpr int SCALE_STEPS = 64;                        // steps whose scales are in LDS at a time
constexpr int SCALE_PITCH = SCALE_STEPS + 4, SCALE_WORDS = SCALE_STEPS / 4;

// Logits of a tile.  1088 rows x 128256 x 4096: 600-609 us, 1.9 PFLOP/s, in large tiles of 8 us and 1.65 us a step, products under way in 51 % of the cycles
// at 2.07 GHz (1088 rows are 1280 in such tiles; the first launches, before the card has settled its clock, take up to 720 us); 64 rows x
// 128256 x 2048: 56 us, the weight's bytes at 4.9 TB/s.  A step is 128 values of K: one block of each operand.
// For 16-bit logits the matrix cores multiply the codes, and take the scales as they are (16x16x128, one scale per 32 values; here all
// of a step's are the same).  Their sums are not quite fp32: of 8 products next to one another along K, what lies below 2^-13 of the
// largest is dropped (found with single products; random codes are off by 5e-5 of a sum's rms), which is nothing beside the
// rounding of the result to 8 or 11 bits.  For fp32 logits the codes become bf16, which holds them exactly, at half the rate: a call
// of few rows, which waits for the weight's bytes, loses nothing by it.
__device__ __forceinline__ s16x8 codes_to_bf16(int lo, int hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, 1.f, true)};
    return __builtin_bit_cast(s16x8, v);
}
template <typename S, int DT>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::WAVES_PER_EU))) void k_head_logits(HeadLogitsArgs a)
{
    constexpr int WEIGHT_BLOCKS = (S::BM + QBLOCK - 1) / QBLOCK;
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    __shared__ __attribute__((aligned(4))) unsigned char scale_bytes[(S::BN + WEIGHT_BLOCKS) * SCALE_PITCH];
    unsigned char *const hs = scale_bytes, *const ws = scale_bytes + S::BN * SCALE_PITCH;
    const unsigned tiles = (unsigned)a.tiles.m * (unsigned)a.tiles.n, split = blockIdx.x / tiles;
    int tm, tn;
    tile_of(blockIdx.x - split * tiles, a.tiles, 4, tm, tn);
    const int v0 = tm * S::BM, n0 = tn * S::BN, k0 = (int)split * a.per_split, k_end = min(a.K, k0 + a.per_split);
    Operand w = a.weight, h = a.hidden;
    w.base += (long long)v0 * w.stride;
    h.base += (long long)n0 * h.stride;
    Stager<KC, S::BM, S::THREADS, 1> sa;
    Stager<KC, S::BN, S::THREADS, 1> sb;
    sa.init(w, a.V - v0);
    sb.init(h, a.N - n0);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN;
    static_assert(QBLOCK % S::WM == 0, "a wave's rows of the weight share a scale");
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
    const int steps = (k_end - k0) / QBLOCK;
    const unsigned lds0 = (unsigned)(uintptr_t)smem;
    auto copy = [&](int s) {
        const unsigned at = lds0 + (unsigned)(s % S::STAGES) * S::STAGE_BYTES;
        sa.copy(at, k0 + s * QBLOCK, k_end, 0);
        sb.copy(at + S::BM * STEP_BYTES, k0 + s * QBLOCK, k_end, 0);
    };
    // The scales of SCALE_STEPS steps into LDS, read four at a time, all under way before the first is needed.
    constexpr int ROWS = S::BN + WEIGHT_BLOCKS, ROUNDS = (ROWS * SCALE_WORDS + S::THREADS - 1) / S::THREADS;
    static_assert(ROUNDS <= 32, "a bit of `nan` each");
    static_assert(SCALE_WORDS == 16 && S::THREADS % 64 == 0, "a row's words are read by 16 lanes side by side");
    // (fp32: behind a row's scales whether it has held the byte 255, the NaN of e8m0, up to now)
    auto scales = [&](int s0) {
        const int count = steps - s0 < SCALE_STEPS ? steps - s0 : SCALE_STEPS;
        unsigned word[ROUNDS];
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            const int i = k * S::THREADS + (int)threadIdx.x, r = i / SCALE_WORDS, q = i % SCALE_WORDS;
            const int n = n0 + r < a.N ? n0 + r : a.N - 1, block = v0 / QBLOCK + r - S::BN, last = (a.V - 1) / QBLOCK;
            const unsigned char *p = (r < S::BN ? a.hidden_scale + n * a.hidden_scale_stride
                                                : a.weight_scale + (block < last ? block : last) * a.weight_scale_stride) + k0 / QBLOCK;
            word[k] = 0u;
            if (4 * q + 4 <= count)
                __builtin_memcpy(&word[k], p + s0 + 4 * q, 4);
            else
                for (int e = 4 * q; e < count; ++e) word[k] |= (unsigned)p[s0 + e] << (8 * (e & 3));
        }
#pragma unroll
        for (int k = 0; k < ROUNDS; ++k) {
            const int i = k * S::THREADS + (int)threadIdx.x, r = i / SCALE_WORDS, q = i % SCALE_WORDS;
            if (r < ROWS) *reinterpret_cast<unsigned *>(scale_bytes + r * SCALE_PITCH + 4 * q) = word[k];
            if constexpr (DT == SVIP_F32) {
                const bool nan = (__ballot((~word[k] - 0x01010101u) & word[k] & 0x80808080u) >> (lane & 48) & 0xffffu) != 0;
                unsigned char *const held = scale_bytes + r * SCALE_PITCH + SCALE_STEPS;
                if (r < ROWS && q == 0 && (nan || s0 == 0)) *held = nan;
            }
        }
    };
    const int w_row = (v0 % QBLOCK + wm) / QBLOCK;
#pragma unroll
    for (int s = 0; s < S::STAGES - 1; ++s)
        if (s < steps) copy(s);
    for (int s = 0; s < steps; ++s) {
        if (s % SCALE_STEPS == 0) {
            if (s) __syncthreads();
            scales(s);                     // (the barrier below publishes them)
        }
        if (s + S::STAGES - 2 < steps)
            wait_copies_and_meet<(S::STAGES - 2) * COPIES>();
        else
            wait_copies_and_meet<0>();
        if (s + S::STAGES - 1 < steps) copy(s + S::STAGES - 1);
        const char *ta = smem + (s % S::STAGES) * S::STAGE_BYTES, *tb = ta + S::BM * STEP_BYTES;
        const int at = s % SCALE_STEPS;
        const int sca = ws[w_row * SCALE_PITCH + at];
        int scb[S::FN];
        i32x8 fa[S::FM], fb[S::FN];
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            scb[j] = hs[(wn + 16 * j + (lane & 15)) * SCALE_PITCH + at];
            fb[j] = rb.whole(tb, wn + 16 * j);
        }
#pragma unroll
        for (int i = 0; i < S::FM; ++i) fa[i] = ra.whole(ta, wm + 16 * i);
        if constexpr (DT != SVIP_F32) {
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int j = 0; j < S::FN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[i], fb[j], acc[i][j], 0, 0, 0, sca, 0, scb[j]);
        } else {
#pragma unroll
            for (int j = 0; j < S::FN; ++j) {
                s16x8 b[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) b[q] = codes_to_bf16(fb[j][2 * q], fb[j][2 * q + 1]);
#pragma unroll
                for (int i = 0; i < S::FM; ++i) {
                    f32x4 block = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 0; q < 4; ++q) block = Bf16::mfma(codes_to_bf16(fa[i][2 * q], fa[i][2 * q + 1]), b[q], block);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] += __builtin_amdgcn_ldexpf(block[e], sca + scb[j] - 254);
                }
            }
        }
    }
    // For the 8-bit instruction a scale of 255 is NaN, for the sum of exponents above 2^128: its row's or tokens' logits become NaN here.  (As a choice in
    // each step 2 to 3 % of a call.)
    if constexpr (DT == SVIP_F32)
#pragma unroll
        for (int j = 0; j < S::FN; ++j)
            if (hs[(wn + 16 * j + (lane & 15)) * SCALE_PITCH + SCALE_STEPS] | ws[w_row * SCALE_PITCH + SCALE_STEPS])
#pragma unroll
                for (int i = 0; i < S::FM; ++i) acc[i][j] = f32x4{NAN, NAN, NAN, NAN};
    using X = typename Stored<DT>::type;
    if (a.part) {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int n = n0 + wn + 16 * j + (lane & 15);
            if (n >= a.N) continue;
            float *row = a.part + ((long long)split * a.N + n) * a.part_stride;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int v = v0 + wm + 16 * i + 4 * (lane >> 4);
                if (v < a.part_stride) *reinterpret_cast<f32x4 *>(row + v) = acc[i][j];       // (V filled up to fours)
            }
        }
    } else if constexpr (DT != SVIP_F32) {
        store_rows<S, X>(smem, a.N - n0, a.V - v0, static_cast<X *>(a.out) + n0 * a.out_stride + v0, a.out_stride, [&](int i, int j) { return acc[i][j]; });
    } else {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int n = n0 + wn + 16 * j + (lane & 15);
            if (n >= a.N) continue;
            X *row = static_cast<X *>(a.out) + n * a.out_stride;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int v = v0 + wm + 16 * i + 4 * (lane >> 4);
                if (v < a.V) put_up_to_4<DT>(row + v, acc[i][j], a.V - v);
            }
        }
    }
}

struct HeadLogitsJoinArgs {
    const float *part;
    long long part_stride;
    int splits, N, V;
    void *out;
    long long out_stride;
};
// The sums of the splits of K, four logits a thread.
template <int DT>
__global__ __launch_bounds__(256) void k_head_logits_join(HeadLogitsJoinArgs a)
{
    const int groups = (int)((a.part_stride + 1023) / 1024), n = blockIdx.x / groups;
    const int v = ((blockIdx.x - n * groups) * 256 + (int)threadIdx.x) * 4;
    if (v >= a.V) return;
    const float *p = a.part + n * a.part_stride + v;
    f32x4 s = *reinterpret_cast<const f32x4 *>(p);
    for (int k = 1; k < a.splits; ++k) s += *reinterpret_cast<const f32x4 *>(p + (long long)k * a.N * a.part_stride);
    put_up_to_4<DT>(static_cast<typename Stored<DT>::type *>(a.out) + n * a.out_stride + v, s, a.V - v);
}

// ---- cross entropy -------------------------------------------------------------------------------------------------------------------------

// What the calls of a loss and its gradient compute once for all tiles, in the workspace.
struct HeadScalars {
    float to_log2;             // accumulated products -> logits / T in units of log 2
    float grad_top;            // largest finite |grad_loss| of a row that counts
    float hidden_mult;         // accumulated G' W -> gradient of the hidden states per grad_loss
    float weight_mult;         // accumulated G'^T (weighted H) -> gradient of the weight
    float weight_parts;        // fp32: what the parts of the weight are multiplied by
    int weighted_shift;        // of the weighted hidden states: k_head_pack
};

// A row's weight in the loss, grad_loss, as m 2^e with 1/2 < |m| <= 1.
constexpr int NO_EXPONENT = -(1 << 20);                // of zero and of what is not finite: below all others
__device__ __forceinline__ bool is_finite(float g) { return (__float_as_uint(g) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ int weight_exponent(float g)
{
    if (g == 0.f || !is_finite(g)) return NO_EXPONENT;
    const int e = __builtin_amdgcn_frexp_expf(g) - (fabsf(__builtin_amdgcn_frexp_mantf(g)) == 0.5f);
    return e < 127 ? e : 127;                          // (|m| < 2 where 2^128 would be no fp32 number)
}
__device__ __forceinline__ float weight_mantissa(float g)
{
    const int e = weight_exponent(g);
    return e == NO_EXPONENT ? (g == 0.f ? 0.f : 1.f) : __builtin_amdgcn_ldexpf(g, -e);
}

struct HeadArgs {
    Operand weight, hidden;    // of the tile kernels: m = vocabulary of the piece, n = rows
    int N, V, D;               // V: rows of the weight in this piece; D: elements of K
    int v0;                    // the piece's first token
    Tiles tiles;
    const HeadScalars *sc;
    float to_log2;             // where the products are of the values themselves: logits_scale()
    const float *row_inv;      // fp32 [N]: one over what a row's parts are multiplied by
    const int *targets;
    float2 *part;              // [tiles of the vocabulary][N] (largest, sum of exp2 relative to it), base 2
    float *target_logit;       // [N] logits / T of the targets, base 2
    const float *lse;          // [N]
    const float *grad_loss;    // [N]
    char *grad;                // [planes][N][grad_stride]: softmax - one-hot of the piece; null: not wanted
    char *weighted;            // up to 64 rows in 16 bits: [2][N][grad_stride], the same times m of the rows' weights in two parts; null: not wanted
    long long grad_stride;     // elements
    long long grad_plane;      // bytes
    int low_plane;             // whether `grad` has a second plane, of low parts
    int vocab;                 // tokens in all
    unsigned *flags;
};

__device__ __forceinline__ bool counts(int target, int vocab) { return target >= 0 && target < vocab; }

// Accumulated products -> logits / T in units of log 2 (parts: of a row's own scale besides).
template <int TERMS>
__device__ __forceinline__ float logits_scale(const HeadArgs &a)
{
    return TERMS == 3 ? a.sc->to_log2 : a.to_log2;
}
// The four 16-lane rows of a wave, lane by lane.
template <typename Op>
__device__ __forceinline__ float across_rows(float v, Op op)
{
    const auto h = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(h[0]), __uint_as_float(h[1]));
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Statistics of a tile of logits: per row the largest and the sum of exponentials over the tile's tokens, one record a row and tile, so that the
// tiles need not wait for one another.  The products bound it: 8192 rows x 151936 x 2048 in bf16 take 3.66 to 3.78 ms (1.35 to 1.39 PFLOP/s, products under way
// in 69 % of the cycles at the 1.9 GHz the card keeps under them), of which the exponentials are 3 of the 52 us of a tile.
template <typename T, typename S, int TERMS>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::WAVES_PER_EU))) void k_head_stats(HeadArgs a)
{
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    int tm, tn;
    tile_of(blockIdx.x, a.tiles, 4, tm, tn);
    const int v0 = tm * S::BM, n0 = tn * S::BN;
    Operand w = a.weight, h = a.hidden;
    w.base += (long long)v0 * w.stride;
    h.base += (long long)n0 * h.stride;
    f32x4 acc[S::FM][S::FN];
    multiply<T, S, KC, KC, TERMS>(w, a.V - v0, h, a.N - n0, 0, a.D, smem, acc);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN, first = v0 + wm + 4 * (lane >> 4);
    const float to_log2 = logits_scale<TERMS>(a);
    float c[S::FN], top[S::FN], sum[S::FN];
    int t[S::FN];                          // where a row's target is among this lane's tokens: 16 i + e
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = n0 + wn + 16 * j + (lane & 15), m = n < a.N ? n : a.N - 1;
        t[j] = n < a.N ? a.targets[m] - a.v0 - first : -1;
        c[j] = TERMS == 3 ? to_log2 * a.row_inv[m] : to_log2;
    }
    if (v0 + S::BM > a.V) {                // the last tile: nothing behind the vocabulary
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (first + 16 * i + e >= a.V)
#pragma unroll
                    for (int j = 0; j < S::FN; ++j) acc[i][j][e] = -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        top[j] = acc[0][j][0];
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top[j] = fmaxf(top[j], acc[i][j][e]);
        if ((unsigned)t[j] < (unsigned)S::WM && (t[j] & 12) == 0) {
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < S::FM; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) z = t[j] == 16 * i + e ? acc[i][j][e] : z;
            if (first + t[j] < a.V) a.target_logit[n0 + wn + 16 * j + (lane & 15)] = z * c[j];
        }
    }
    // (c is positive: the largest product is the largest logit)
#pragma unroll
    for (int j = 0; j < S::FN; ++j) top[j] = across_rows(top[j], OpMax{}) * c[j];
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const float base = top[j] == -INFINITY ? 0.f : top[j];
        sum[j] = 0.f;
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[j] += __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], c[j], -base));
    }
    __syncthreads();
    float2 *red = reinterpret_cast<float2 *>(smem);        // [WAVES_M][BN]
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        sum[j] = across_rows(sum[j], OpSum{});
        if (lane < 16) red[(wave % S::WAVES_M) * S::BN + wn + 16 * j + lane] = make_float2(top[j], sum[j]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < S::BN && n0 + i < a.N; i += S::THREADS) {
        float2 r = red[i];
#pragma unroll
        for (int k = 1; k < S::WAVES_M; ++k) {
            const float2 o = red[k * S::BN + i];
            const float m = fmaxf(r.x, o.x), base = m == -INFINITY ? 0.f : m;
            r = make_float2(m, r.y * __builtin_amdgcn_exp2f(r.x - base) + o.y * __builtin_amdgcn_exp2f(o.x - base));
        }
        a.part[(long long)(a.v0 / S::BM + tm) * a.N + n0 + i] = r;
    }
}

struct HeadFinishArgs {
    const float2 *part;
    int records, N, vocab;
    const float *target_logit;
    const int *targets;
    float *loss, *lse;
    unsigned *flags;
};
// A row's records joined in 64 bits: 16 rows a workgroup, 16 threads a row, eight records of each at a time, so that a thread waits for memory four times where
// one by one it did 32 times.  4096 rows of 501 records: 7.5 us (20 one by one).
constexpr int FINISH_ROWS = 16, FINISH_WG = 256, FINISH_BATCH = 8;
__global__ __launch_bounds__(FINISH_WG) static void k_head_finish(HeadFinishArgs a)
{
    __shared__ float tops[FINISH_WG];
    __shared__ double sums[FINISH_WG];
    const int r = threadIdx.x % FINISH_ROWS, k = threadIdx.x / FINISH_ROWS, row = blockIdx.x * FINISH_ROWS + r;
    const int n = row < a.N ? row : a.N - 1;
    constexpr int SLICES = FINISH_WG / FINISH_ROWS;
    float top = -INFINITY;
    double sum = 0.0;
    for (int i = k; i < a.records; i += SLICES * FINISH_BATCH) {
        float2 p[FINISH_BATCH];
#pragma unroll
        for (int q = 0; q < FINISH_BATCH; ++q) {
            const int at = i + q * SLICES;
            p[q] = a.part[(long long)(at < a.records ? at : k) * a.N + n];
            if (at >= a.records) p[q] = make_float2(-INFINITY, 0.f);
        }
        float m = top;
#pragma unroll
        for (int q = 0; q < FINISH_BATCH; ++q) m = fmaxf(m, p[q].x);
        const float base = m == -INFINITY ? 0.f : m;
        sum *= (double)__builtin_amdgcn_exp2f(top - base);
#pragma unroll
        for (int q = 0; q < FINISH_BATCH; ++q) sum += (double)(p[q].y * __builtin_amdgcn_exp2f(p[q].x - base));
        top = m;
    }
    tops[threadIdx.x] = top;
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (k != 0 || row >= a.N) return;
    for (int i = 1; i < SLICES; ++i) top = fmaxf(top, tops[i * FINISH_ROWS + r]);
    const float base = top == -INFINITY ? 0.f : top;
    sum = 0.0;
    for (int i = 0; i < SLICES; ++i) sum += sums[i * FINISH_ROWS + r] * (double)__builtin_amdgcn_exp2f(tops[i * FINISH_ROWS + r] - base);
    const double lse2 = (double)top + log2(sum);
    const int t = a.targets[n];
    const bool use = counts(t, a.vocab);
    if (t >= a.vocab) atomicOr(a.flags, (unsigned)SVIP_FLAG_BAD_TOKEN);
    a.lse[n] = (float)(lse2 * HEAD_LN2);
    a.loss[n] = use ? (float)((lse2 - (double)a.target_logit[n]) * HEAD_LN2) : 0.f;
}

// ---- its gradient ------------------------------------------------------------------------------------------------------------------------

// G' = softmax - one-hot of a tile of recomputed logits, rows without a target zero, in the products' type.  Its entries reach from 1 down to
// nothing: fp16 (and the two parts of an fp32 value) carry them times 2^15, which keeps 11 bits down to 2^-29.  bf16 keeps its 8 bits
// at any magnitude: its rounding, at most 2^-8 of a value, is of the size of the rounding of the gradients themselves.  In a sum over many rows these roundings
// even out; the weight's gradient of few rows takes a 16-bit G' in two parts, high and low: of 1 to 8 rows it was up to 1.8 times as far off with one part
// (17 rows x 128256 x 2048 in bf16: 494 us with one, 509 with two, 514 with the plane for the other gradient).  These parts are of m G', m 2^e the rows' weights, and the hidden states are multiplied by 2^e
// alone, which rounds nothing, so that the gradient is off by its own rounding, whatever the weights (with the weights in the hidden
// states it was up to 1.43 times as far off).  The gradient of the hidden states, and many rows' of the weight, read G' as it is: its -1 at the target is
// exact, and m would make it a number that is rounded (1000 rows of one weight: 1.60 times as far off as an fp32 result rounded once, now 1.03).
constexpr float GRAD_SCALE_F16 = 32768.f;

template <typename T> struct GradOf;
template <> struct GradOf<Bf16> {
    using type = __bf16;
    static constexpr float SCALE = 1.f;
};
template <> struct GradOf<F16> {
    using type = _Float16;
    static constexpr float SCALE = GRAD_SCALE_F16;
};
template <> struct GradOf<F32> {
    using type = float;
    static constexpr float SCALE = 1.f;
};

// The logits are computed again (their sums took the whole vocabulary): 4096 rows x 32256 tokens x 4096 in bf16, 0.82 ms, 1.31 PFLOP/s.
template <typename T, typename S, int TERMS>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::WAVES_PER_EU))) void k_head_softmax(HeadArgs a)
{
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    int tm, tn;
    tile_of(blockIdx.x, a.tiles, 4, tm, tn);
    const int v0 = tm * S::BM, n0 = tn * S::BN;
    Operand w = a.weight, h = a.hidden;
    w.base += (long long)v0 * w.stride;
    h.base += (long long)n0 * h.stride;
    f32x4 acc[S::FM][S::FN];
    multiply<T, S, KC, KC, TERMS>(w, a.V - v0, h, a.N - n0, 0, a.D, smem, acc);

    using X = typename GradOf<T>::type;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN, first = v0 + wm + 4 * (lane >> 4);
    const int cols = (int)a.grad_stride - v0;              // (columns behind the vocabulary are zeros)
    float c[S::FN], base[S::FN], scale[S::FN];
    int t[S::FN];                          // where a row's target is among this lane's tokens: 16 i + e
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = n0 + wn + 16 * j + (lane & 15), m = n < a.N ? n : a.N - 1, target = a.targets[m];
        c[j] = TERMS == 3 ? logits_scale<TERMS>(a) * a.row_inv[m] : logits_scale<TERMS>(a);
        t[j] = target - a.v0 - first;
        base[j] = a.lse[m] * HEAD_LOG2E;
        scale[j] = counts(target, a.vocab) ? GradOf<T>::SCALE : 0.f;
    }
#pragma unroll
    for (int j = 0; j < S::FN; ++j)
#pragma unroll
        for (int i = 0; i < S::FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float p = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][e], c[j], -base[j]));
                if (t[j] == 16 * i + e) p -= 1.f;
                acc[i][j][e] = scale[j] != 0.f && first + 16 * i + e < a.V ? p * scale[j] : 0.f;
            }
    X *out = reinterpret_cast<X *>(a.grad) + n0 * a.grad_stride + v0;
    if constexpr (sizeof(X) == 2) {
        const auto high = [&](int i, int j) { return acc[i][j]; };
        const auto low = [&](int i, int j) {
            typedef X x4 __attribute__((ext_vector_type(4)));
            return acc[i][j] - __builtin_convertvector(__builtin_convertvector(acc[i][j], x4), f32x4);
        };
        if (a.grad) store_rows<S, X>(smem, a.N - n0, cols, out, a.grad_stride, high);
        if (a.low_plane) store_rows<S, X>(smem, a.N - n0, cols, out + a.grad_plane / 2, a.grad_stride, low);
        if constexpr (TERMS == 1 && S::BN <= 64)
            if (a.weighted) {
#pragma unroll
                for (int j = 0; j < S::FN; ++j) {
                    const int n = n0 + wn + 16 * j + (lane & 15);
                    const float m = weight_mantissa(a.grad_loss[n < a.N ? n : a.N - 1]);
#pragma unroll
                    for (int i = 0; i < S::FM; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = scale[j] != 0.f ? acc[i][j][e] * m : 0.f;
                }
                out = reinterpret_cast<X *>(a.weighted) + n0 * a.grad_stride + v0;
                store_rows<S, X>(smem, a.N - n0, cols, out, a.grad_stride, high);
                store_rows<S, X>(smem, a.N - n0, cols, out + a.grad_plane / 2, a.grad_stride, low);
            }
    } else {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int n = wn + 16 * j + (lane & 15);
            if (n0 + n >= a.N) continue;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int m = wm + 16 * i + 4 * (lane >> 4);
                if (m < cols) *reinterpret_cast<f32x4 *>(out + n * a.grad_stride + m) = acc[i][j];
            }
        }
    }
}

struct HeadHiddenArgs {
    Operand weight, grad;      // m = hidden channels (k strided), n = rows (k contiguous); k = tokens of the piece
    int N, D, V;
    Tiles tiles;
    int splits, per_split;     // tokens of a split, a multiple of the step
    int first;                 // the first piece: nothing to add to
    float *sum;                // [splits][N][D]
};
// Gradient of the hidden states: G' W over the tokens of a piece, added to what the pieces before it gave.  The weight is read as it lies, k strided.  4096
// rows x 32256 tokens x 4096 in bf16: 0.76 ms, 1.42 PFLOP/s; its 256 tiles are one round of the CUs.
template <typename T, typename S, int TERMS>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::WAVES_PER_EU))) void k_head_grad_hidden(HeadHiddenArgs a)
{
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    const unsigned tiles = (unsigned)a.tiles.m * (unsigned)a.tiles.n, split = blockIdx.x / tiles;
    int tm, tn;
    tile_of(blockIdx.x - split * tiles, a.tiles, 4, tm, tn);
    const int d0 = tm * S::BM, n0 = tn * S::BN, k0 = (int)split * a.per_split, k_end = min(a.V, k0 + a.per_split);
    Operand w = a.weight, g = a.grad;
    w.base += T::SIZE * d0;
    g.base += (long long)n0 * g.stride;
    f32x4 acc[S::FM][S::FN];
    multiply<T, S, KS, KC, TERMS>(w, a.D - d0, g, a.N - n0, k0, k_end, smem, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN;
    float *sum = a.sum + (long long)split * a.N * a.D;
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = n0 + wn + 16 * j + (lane & 15);
        if (n >= a.N) continue;
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const int d = d0 + wm + 16 * i + 4 * (lane >> 4);
            if (d >= a.D) continue;
            f32x4 *p = reinterpret_cast<f32x4 *>(sum + (long long)n * a.D + d);
            *p = a.first ? acc[i][j] : *p + acc[i][j];
        }
    }
}

struct HeadHiddenFinishArgs {
    const float *sum;
    int splits, slices;        // slices: JOIN_SLICES or 1
    int N, D, Dp;              // D of the output, Dp of the sums (both multiples of 4)
    const HeadScalars *sc;
    const int *targets;
    const float *grad_loss;
    int vocab;
    void *out;
    long long out_stride;
};
// A workgroup takes 64 columns of four: of one row with four slices of its splits side by side, or, where there are few splits, of four rows.
constexpr int JOIN_COLUMNS = 64, JOIN_SLICES = 4, JOIN_BATCH = 8;
template <int DT>
__global__ __launch_bounds__(JOIN_COLUMNS * JOIN_SLICES) void k_head_hidden_finish(HeadHiddenFinishArgs a)
{
    __shared__ f32x4 sums[JOIN_SLICES][JOIN_COLUMNS];
    const int groups = (a.D + 4 * JOIN_COLUMNS - 1) / (4 * JOIN_COLUMNS), group = blockIdx.x / groups;
    const int column = threadIdx.x % JOIN_COLUMNS, part = threadIdx.x / JOIN_COLUMNS, slice = a.slices == 1 ? 0 : part;
    const int n = a.slices == 1 ? group * JOIN_SLICES + part : group;
    const int d = ((blockIdx.x - group * groups) * JOIN_COLUMNS + column) * 4;
    const bool use = n < a.N && counts(a.targets[n], a.vocab);
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (use && d < a.D) {
        const float *p = a.sum + (long long)n * a.Dp + d;
        const long long next = (long long)a.N * a.Dp;
        for (int k = slice; k < a.splits; k += a.slices * JOIN_BATCH) {
            f32x4 v[JOIN_BATCH];
#pragma unroll
            for (int q = 0; q < JOIN_BATCH; ++q) {
                const int at = k + q * a.slices;
                if (at < a.splits) v[q] = *reinterpret_cast<const f32x4 *>(p + at * next);
            }
#pragma unroll
            for (int q = 0; q < JOIN_BATCH; ++q)
                if (k + q * a.slices < a.splits) s += v[q];
        }
    }
    if (a.slices > 1) {
        sums[slice][column] = s;
        __syncthreads();
    }
    if (slice || n >= a.N || d >= a.D) return;
    if (a.slices > 1)
        for (int k = 1; k < JOIN_SLICES; ++k) s += sums[k][column];
    const float m = use ? a.grad_loss[n] * a.sc->hidden_mult : 0.f;
    Stored<DT>::put4(static_cast<typename Stored<DT>::type *>(a.out) + n * a.out_stride + d, s * m);
}

struct HeadWeightArgs {
    Operand hidden, grad;      // m = hidden channels, n = tokens of the piece, both k strided; k = rows
    int N, D, V, Dp;           // D: channels of the output, Dp: of the operand
    Tiles tiles;
    const HeadScalars *sc;
    void *out;                 // row 0: the piece's first token
    long long out_stride;
};
// Gradient of the weight: G'^T (weighted H), both operands k strided: twice the LDS reads of 16 bytes a row, as the transposing read gives 8.
// 4096 rows x 32256 tokens x 4096 in bf16: 0.82 ms, 1.32 PFLOP/s.
template <typename T, typename S, int TERMS, int DT>
__global__ __launch_bounds__(S::THREADS) __attribute__((amdgpu_waves_per_eu(S::WAVES_PER_EU))) void k_head_grad_weight(HeadWeightArgs a)
{
    __shared__ __attribute__((aligned(1024))) char smem[S::LDS_BYTES];
    int tm, tn;
    tile_of(blockIdx.x, a.tiles, 4, tm, tn);
    const int d0 = tm * S::BM, v0 = tn * S::BN;
    Operand h = a.hidden, g = a.grad;
    h.base += T::SIZE * d0;
    g.base += T::SIZE * v0;
    f32x4 acc[S::FM][S::FN];
    multiply<T, S, KS, KS, TERMS>(h, a.Dp - d0, g, (int)(g.stride / T::SIZE) - v0, 0, a.N, smem, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN;
    const float mult = a.sc->weight_mult;
    using X = typename Stored<DT>::type;
    X *out = static_cast<X *>(a.out) + v0 * a.out_stride + d0;
    if constexpr (sizeof(X) == 2) {
        store_rows<S, X>(smem, a.V - v0, a.D - d0, out, a.out_stride, [&](int i, int j) { return acc[i][j] * mult; });
    } else {
#pragma unroll
        for (int j = 0; j < S::FN; ++j) {
            const int v = wn + 16 * j + (lane & 15);
            if (v0 + v >= a.V) continue;
#pragma unroll
            for (int i = 0; i < S::FM; ++i) {
                const int d = wm + 16 * i + 4 * (lane >> 4);
                if (d0 + d < a.D) *reinterpret_cast<f32x4 *>(out + v * a.out_stride + d) = acc[i][j] * mult;
            }
        }
    }
}

// ---- what goes before the products -----------------------------------------------------------------------------------------------------------

// fp32 values as two fp16 parts: x 2^s = high + low, with 2^s bringing the largest magnitude of the row (hidden states in the logits) or of the matrix
// (the weight) to [2^14, 2^15), of the weighted hidden states, which are summed over, to [2^13, 2^15).  Together they keep 22 bits of a value down to 2^-17 of that largest one, and 2^-40 of it
// below; of a product all but low x low is taken.  Products of three bf16 parts would need no scale, but six products for 24 bits.
__device__ __forceinline__ float part_scale(int exponent)
{
    if (exponent == NO_EXPONENT) return 1.f;
    return __uint_as_float((unsigned)min(max(127 + 14 - exponent, 1), 253) << 23);
}
__device__ __forceinline__ void store_parts(char *out, long long plane, const float (&v)[8], float s)
{
    f16x8 high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        high[e] = (_Float16)(v[e] * s);
        low[e] = (_Float16)(v[e] * s - (float)high[e]);
    }
    *reinterpret_cast<f16x8 *>(out) = high;
    *reinterpret_cast<f16x8 *>(out + plane) = low;
}

struct HeadMaxArgs {
    const void *x;
    long long stride;          // elements
    int rows, cols;            // cols: whole 16 bytes
    const int *targets;        // null, or hidden states: rows without a target do not count, the others are multiplied by their weight
    const float *grad_loss;
    int vocab;
    int *out;                  // [workgroups]: exponents of the largest magnitudes (2^e <= x < 2^(e + 1)), NO_EXPONENT: all zeros
};
// Exponent of the largest finite magnitude of a matrix, one for each workgroup, so that nothing has to be cleared or joined in memory.  A wave takes rows.
constexpr int MAX_GROUPS = 2048;
template <int DT>
__global__ __launch_bounds__(256) void k_head_max(HeadMaxArgs a)
{
    constexpr int VEC = Stored<DT>::VEC;
    using X = typename Stored<DT>::type;
    typedef X vec __attribute__((ext_vector_type(VEC)));
    __shared__ int tops[4];
    const int lane = threadIdx.x & 63;
    int top = NO_EXPONENT;
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += gridDim.x * 4) {
        int e = 0;
        float m = 1.f;
        if (a.targets) {
            if (!counts(a.targets[r], a.vocab)) continue;
            const float g = a.grad_loss[r];
            e = weight_exponent(g);
            m = fabsf(weight_mantissa(g));
            if (e == NO_EXPONENT) continue;
        }
        const X *x = static_cast<const X *>(a.x) + r * a.stride;
        unsigned most = 0u;
#pragma unroll 4
        for (int c = lane * VEC; c < a.cols; c += 64 * VEC) {
            const vec v = *reinterpret_cast<const vec *>(x + c);
#pragma unroll
            for (int q = 0; q < VEC; ++q) most = max(most, finite_magnitude((float)v[q]));
        }
        if (most) {
            const float in_1_2 = most < 0x800000u ? 1.f : __uint_as_float((most & 0x7fffffu) | 0x3f800000u);       // (below 2^-126: as that)
            top = max(top, e + max((int)(most >> 23), 1) - 127 - (in_1_2 * m < 1.f) + (in_1_2 * m >= 2.f));
        }
    }
#pragma unroll
    for (int o = 32; o; o /= 2) top = max(top, __shfl_xor(top, o));
    if (lane == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) a.out[blockIdx.x] = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
}

struct HeadScalarsArgs {
    HeadScalars *sc;
    const int *weight_max, *hidden_max;    // null, or what k_head_max wrote
    int weight_groups, hidden_groups;
    int fine;                  // the weights' mantissas are in G'
    int N, vocab;
    float temperature;
    const int *targets;
    const float *grad_loss;    // null: a loss alone
    float grad_scale;          // of G'
    unsigned *flags;
};
constexpr int SCALARS_WG = 1024;
__global__ __launch_bounds__(SCALARS_WG) static void k_head_scalars(HeadScalarsArgs a)
{
    __shared__ float tops[SCALARS_WG / 64];
    __shared__ int most[2][SCALARS_WG / 64];
    float top = 0.f;
    int m[2] = {NO_EXPONENT, NO_EXPONENT};                 // of the weight, of the weighted hidden states
    bool bad = false;
    for (int i = threadIdx.x; i < a.weight_groups; i += SCALARS_WG) m[0] = max(m[0], a.weight_max[i]);
    for (int i = threadIdx.x; i < a.hidden_groups; i += SCALARS_WG) m[1] = max(m[1], a.hidden_max[i]);
    if (a.grad_loss)
        for (int n = threadIdx.x; n < a.N; n += SCALARS_WG) {
            const int t = a.targets[n];
            const float g = a.grad_loss[n];
            bad |= t >= a.vocab;
            if (counts(t, a.vocab) && is_finite(g)) top = fmaxf(top, fabsf(g));
        }
    top = wave_reduce(top, OpMax{});
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int o = 32; o; o /= 2) m[q] = max(m[q], __shfl_xor(m[q], o));
    if ((threadIdx.x & 63) == 0) {
        tops[threadIdx.x >> 6] = top;
        most[0][threadIdx.x >> 6] = m[0];
        most[1][threadIdx.x >> 6] = m[1];
    }
    if (bad) atomicOr(a.flags, (unsigned)SVIP_FLAG_BAD_TOKEN);
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < SCALARS_WG / 64; ++i) {
        top = fmaxf(top, tops[i]);
        m[0] = max(m[0], most[0][i]);
        m[1] = max(m[1], most[1][i]);
    }
    // The weighted hidden states are H (grad_loss / grad_top) 2^(shift + e), e of grad_top, or H 2^(shift + e), e of the row's own weight where its mantissa
    // is in G'.  fp16 and parts: the largest |H grad_loss| is at least 2^m1, so that either is below 2^15 and the largest above 2^13.  Other
    // types hold any that is no larger than the hidden states.  (No further up than leaves the result's multiplier a normal number.)
    const int e = top > 0.f ? weight_exponent(top) : 0;
    const int shift = min(!a.hidden_max ? -e : m[1] == NO_EXPONENT ? 0 : 13 - m[1], 111);
    const float ws = a.weight_max ? part_scale(m[0]) : 1.f;
    const double t = 1.0 / (double)a.temperature;
    a.sc->weight_parts = ws;
    a.sc->to_log2 = (float)(1.4426950408889634 * t / (double)ws);
    a.sc->grad_top = top;
    a.sc->hidden_mult = (float)(t / ((double)a.grad_scale * (double)ws));
    a.sc->weight_mult = (float)(t / (double)a.grad_scale * ldexp(a.fine ? 1.0 : (double)top, a.fine ? -shift : -shift - e));
    a.sc->weighted_shift = a.fine ? shift : shift + e;
}

struct HeadPackArgs {
    const void *x;
    long long stride;          // elements
    int rows, cols, cols_p;    // cols_p: of the packed rows, a multiple of 8
    char *out;                 // [planes][rows][cols_p] 16-bit
    long long plane;           // bytes
    const HeadScalars *sc;
    const int *targets;        // hidden states for the gradient of the weight: weighted rows (k_head_scalars), 0 where they do not count
    const float *grad_loss;
    int fine;
    int vocab;
    float *row_inv;            // hidden states for the logits: parts of their own scale for each row
    int whole;                 // fp32 as it is, no parts
    int row_threads;           // of a workgroup, side by side in a row: a power of two
};
template <int DT>
__device__ __forceinline__ void load_columns(const HeadPackArgs &a, long long r, int c, float (&v)[8])
{
    using X = typename Stored<DT>::type;
    constexpr int VEC = Stored<DT>::VEC;                   // 16 bytes
    typedef X vec __attribute__((ext_vector_type(VEC)));
    const X *x = static_cast<const X *>(a.x) + r * a.stride + c;
    if (c + 8 <= a.cols) {
#pragma unroll
        for (int q = 0; q < 8; q += VEC) {
            const vec w = *reinterpret_cast<const vec *>(x + q);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[q + e] = (float)w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? (float)x[e] : 0.f;
    }
}
// Eight columns a thread: a weight (fp32), or hidden states weighted for the gradient of the weight.
template <int DT>
__global__ __launch_bounds__(256) void k_head_pack(HeadPackArgs a)
{
    const unsigned blocks = (unsigned)(a.cols_p + 8 * a.row_threads - 1) / (unsigned)(8 * a.row_threads), group = blockIdx.x / blocks;
    const unsigned in_row = threadIdx.x & (unsigned)(a.row_threads - 1);
    const long long r = (long long)group * (256 / a.row_threads) + threadIdx.x / (unsigned)a.row_threads;
    const int c = (int)((blockIdx.x - group * blocks) * (unsigned)a.row_threads + in_row) * 8;
    if (r >= a.rows || c >= a.cols_p) return;
    float v[8];
    load_columns<DT>(a, r, c, v);
    if (a.targets) {
        const bool use = counts(a.targets[r], a.vocab);
        const float g = a.grad_loss[r], top = a.sc->grad_top;
        const float w = !is_finite(g) ? NAN : a.fine ? 1.f : top > 0.f ? g / top : 0.f;
        const int shift = a.sc->weighted_shift + (a.fine && is_finite(g) ? weight_exponent(g) : 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = use ? __builtin_amdgcn_ldexpf(v[e] * w, shift) : 0.f;
    }
    char *out = a.out + (r * a.cols_p + c) * 2;
    if (DT == SVIP_F32 && a.whole) {
        float *p = reinterpret_cast<float *>(a.out) + r * a.cols_p + c;
        *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else if constexpr (DT == SVIP_F32) {
        store_parts(out, a.plane, v, a.targets ? 1.f : a.sc->weight_parts);
    } else {
        using X = typename Stored<DT>::type;
        typedef X x8 __attribute__((ext_vector_type(8)));
        x8 y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (X)v[e];
        *reinterpret_cast<x8 *>(out) = y;
    }
}
// fp32 hidden states for the logits, a wave each row: one that does not count may hold anything and costs the others nothing.
__global__ __launch_bounds__(256) static void k_head_pack_rows(HeadPackArgs a)
{
    const int r = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (r >= a.rows) return;
    unsigned m = 0u;
    float v[8];
    for (int c = lane * 8; c < a.cols_p; c += 512) {
        load_columns<SVIP_F32>(a, r, c, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, finite_magnitude(v[e]));
    }
#pragma unroll
    for (int o = 32; o; o /= 2) m = max(m, (unsigned)__shfl_xor((int)m, o));
    const float s = part_scale(m ? (int)(m >> 23) - 127 : NO_EXPONENT);
    for (int c = lane * 8; c < a.cols_p; c += 512) {
        load_columns<SVIP_F32>(a, r, c, v);
        store_parts(a.out + ((long long)r * a.cols_p + c) * 2, a.plane, v, s);
    }
    if (lane == 0) a.row_inv[r] = 1.f / s;
}

}  // namespace svip
