// Kernels of svip_sample: a token for each row of logits, every row with its own temperature, top-k, top-p and min-p (not in the paper).
//
// Weights are w = exp2((z - m) c) with c = log2(e) / T and m the row's largest logit, in 64 bits: which token a uniform falls on, and which
// value the nucleus ends at, are borders between sums of up to V weights, and a rounding of 2^-24 in each weight moves such a border by more than
// the narrowest cells are wide.  A weight costs about 17 instructions of 5.3 cycles (measured; in fp32 7 of 2.7).  Sums that decide are integers in
// units of 2^-S (S = 62 - ceil(log2 V), at most 51) of 2^R, a power of two within 2^1/2 of the largest weight, so that no order of additions changes a result and
// atomics may be used.  Where single logits are summed, each is rounded to units.  A tile's mass is rounded to them as a whole: it comes from a sum in fp64 in a
// fixed order (rows without filter) or of integers in units of 2^-50 of the tile's own 2^R, 53 bits of which count (steps); and the draw inside a tile goes by
// its share of that mass, in the tile's own units.
//
// Two launches, three or four where a call has top_p or min_p.  k_sample_tiles reads the rows once: a wave has a tile of 4096 logits in registers, in chunks
// of 64 neighbours.  k_sample_rows, a workgroup each row, does what the row's settings need beside that.  What a wave leaves for the row:
//   T = 0         the tile's maximum
//   no filter     and its mass; the draw finds the tile by the masses and goes through that tile alone again
//   top-k         and the maximum of every chunk.  The k-th largest of those is no larger than the k-th largest logit, so chunks below it hold no
//                 candidate: the others are read again, what is at or above it goes into a list in LDS, and all settings are decided on the list.  Where there
//                 are fewer chunks than that (or more than 1024 are asked for) the row's own keys tell what goes into the list
//   top-p, min-p  and the mass of the tile's logits from the top down to each of 512 equal steps of log2 w, which reach as far as the border can be.  From the
//                 tiles' masses follows the step that holds the border, exactly; k_sample_border reads such rows again, without exponentials, counts what
//                 lies above that step and marks what lies in it, tile by tile; a list of those decides what of them stays, and the draw goes by the tiles'
//                 masses and through one tile.
// Rows that do not fit these (a list of more than 4096, +inf, logits of more than 2^18 octaves) are swept as often as a radix select over their keys
// needs (row_by_sweeps: 44 rows of 32000 with mixed settings took 79 us when those with a top_k of 1000 came here, and 38 by lists).
//
// What bounds them (us, launches of k_sample_tiles + _border + _rows; bf16):
//   1088 x 128256   T = 0: 50 + 5 + 5 + 15, the memory (279 MB at 5.6 TB/s); no filter: 110 + 5 + 5 + 24, fp64 instructions (83 us at the rate they reach alone,
//                   2.3 GHz); top-k 50, top-p 0.9: 57 + 5 + 9 + 30; top-p 0.9: 138 + 14 + 67 + 50.  (A border launch that has nothing to do takes 5, and is left
//                   out where no top_p and min_p are given.)  Of the 149 that the tiles of top-p 0.9 take launched alone, 142 are left without the stores of
//                   their steps' masses (144 MB), 92 without the weights, 94 without the weights and the LDS additions, 50 for the reading: the weights first,
//                   then the steps' numbers and sums
//   64 x 128256     top-k 50, top-p 0.9: 5 + 2 + 12; top-p 0.9: 15 + 12 + 18; mixed settings: 13 + 10 + 21.  A row is one workgroup's in the last
//                   launch: latencies, one after the other
//   1 x 32000 fp32  top-k 50, top-p 0.9: 4 + 1.5 + 10
#pragma once
#include "../../include/svip.h"
#include "warp_kernels.h"

namespace svip {

struct SampleArgs {
    const void *logits;
    long long row_stride;
    int V;
    const float *temperature;  // [N] each, or null: 1, off, off, off
    const int *top_k;
    const float *top_p, *min_p;
    const float *u;
    int *token;
    float *prob;               // or null
    int *kept;                 // or null
    unsigned *flags;
    int unit_bits;             // S
    int tiles, groups;         // of a row; groups: workgroups of k_sample_tiles
    char *data;                // [N] RowData, [tiles] TileData
};

constexpr int TILES_WG = 256, TILES_WAVES = TILES_WG / 64;             // k_sample_tiles
constexpr int SAMPLE_WG = 512, SAMPLE_WAVES = SAMPLE_WG / 64;          // k_sample_rows
constexpr int SAMPLE_CHUNK = 64, SAMPLE_TILE = 64 * SAMPLE_CHUNK;       // logits of a chunk and of a wave, which has as many as lanes
constexpr int SAMPLE_STEPS = 512;                      // of log2 w
constexpr int TILE_UNIT_BITS = 50;                     // masses of a tile, relative to its own R: 2^12 weights of up to 2^1/2 fit 64 bits
constexpr int SAMPLE_BINS = 1024;
constexpr int SAMPLE_LIST = 4096;
constexpr int SMALL_LIST = 128;
constexpr int SAMPLE_TOP_K = 1024;
constexpr int SAMPLE_MAX_TILES = (1 << 22) / SAMPLE_TILE;

// What a wave leaves of its tile.
struct TileData {
    float top;                             // the largest logit
    int count;                             // logits above -inf
    double mass;                           // relative to 2^R of its own (rows without filter)
    unsigned long long down_to[SAMPLE_STEPS];      // mass from the top down to the end of each step, in units of 2^-50 of that
    float chunk_top[64];
    unsigned long long above;              // k_sample_border: mass above the row's border step, in the row's units
    int kept, undecided;                   // logits above it and in it
    unsigned long long in_step[64];        // which those are: value e of a lane's vector u is that lane's bit of word u N + e
};
// Of a row, in front of its tiles: what k_sample_border found, and k_sample_rows goes by.
struct RowData {
    int found;                             // 0: for the sweeps
    int by_mass;                           // top_p's border is in the step (or min_p alone decides)
    float upper, lower;                    // logits from upper on are above the step, from lower on in it (and not below min_p)
    unsigned long long target;             // top_p: the mass that what stays has to reach
    int step;                              // counted from that of the largest logit, downwards
    float top;
    unsigned long long pad[4];
};
__host__ __device__ inline size_t row_bytes(int tiles) { return sizeof(RowData) + (size_t)tiles * sizeof(TileData); }
__device__ __forceinline__ RowData *row_data(char *data, int n, int tiles) { return reinterpret_cast<RowData *>(data + n * row_bytes(tiles)); }
__device__ __forceinline__ TileData *tiles_of(RowData *row) { return reinterpret_cast<TileData *>(row + 1); }

// 2^f for |f| <= 1/2, by the Chebyshev series of exp(f ln 2) up to f^9: off by at most 1.9e-14 of the result.  The coefficients are kept in scalar
// registers: as constants each of them would be moved into a vector register pair for every weight, two more instructions to each of ten.
constexpr double ROUND_64 = 6755399441055744.0;        // 1.5 * 2^52: added to a number below 2^51 it leaves it, rounded to a whole one, in the low bits
struct Exp2Series {
    double c[10];
    __device__ __forceinline__ Exp2Series()
        : c{1.0000000000000135, 0.69314718055995, 0.240226506956403, 0.05550410866444782, 0.009618129193942278, 0.0013333558230151053, 0.0001540343374614693,
            1.5252657267483816e-05, 1.3259646267083092e-06, 1.0208689005253291e-07}
    {
#pragma unroll
        for (int i = 0; i < 10; ++i) asm("" : "+s"(c[i]));
    }
    // 2^(n + f - from), n in the low bits of `rounded`, n - from >= -1000
    __device__ __forceinline__ double operator()(double rounded, double f, int from) const
    {
        double r = c[9];
#pragma unroll
        for (int i = 8; i >= 0; --i) r = fma(r, f, c[i]);
        return __hiloint2double(__double2hiint(r) + ((__double2loint(rounded) - from) << 20), __double2loint(r));
    }
};
// 2^(52 - bits), bits <= 51: added to a weight below 2 it leaves the weight in units of 2^-bits, rounded, in the low bits of the sum
__device__ __forceinline__ double unit_of(int bits) { return __longlong_as_double((long long)(1023 + 52 - bits) << 52); }
__device__ __forceinline__ unsigned long long units_of(double w, double unit)
{
    return (unsigned long long)__double_as_longlong(w + unit) - (unsigned long long)__double_as_longlong(unit);
}

// Weights relative to 2^R, R = m c rounded to a whole number: that of the largest logit is between 2^-1/2 and 2^1/2, and weights relative to different
// R differ by a power of two.
struct SampleWeights {
    double m, c;               // the largest logit; log2(e) / T
    double least;              // the logit whose weight is 2^-1000; smaller ones, and NaN, are taken for it (which is nothing in any unit here)
    double part;               // m c - R
    double unit;
    int R;
    bool near;                 // |m c| < 2^30: of_tile may be used
    Exp2Series exp2;
    __device__ __forceinline__ SampleWeights(float top, double c_, int unit_bits) : c(c_) { set(top, unit_bits); }
    __device__ __forceinline__ void set(float top, int unit_bits)
    {
        m = top;
        unit = unit_of(unit_bits);
        const double mc = m * c;
        near = fabs(mc) < 1073741824.0;
        R = near ? (int)rint(mc) : 0;
        part = near ? fma(m, c, -(double)R) : 0.0;
        least = ((double)R - 1000.0) / c;
    }
    __device__ __forceinline__ double log2_of(float z) const { return (double)z == m ? 0.0 : ((double)z - m) * c; }      // (m may be +inf)
    // 2^(z c - R).  Whatever m and c are; of_tile: in two instructions less, where m c is near
    __device__ __forceinline__ double operator()(float z) const
    {
        const double x = fmax(log2_of(z) + part, -1000.0), t = x + ROUND_64;
        return exp2(t, x - (t - ROUND_64), 0);
    }
    __device__ __forceinline__ double of_tile(float z) const
    {
        const double x = fmax((double)z, least), t = fma(x, c, ROUND_64);
        return exp2(t, fma(x, c, -(t - ROUND_64)), R);
    }
    __device__ __forceinline__ unsigned long long units(float z) const { return units_of((*this)(z), unit); }
};
// What a tile's mass is to be multiplied by, as a power of two, in the row's units (a tile that is too far below the row's R weighs nothing).
__device__ __forceinline__ double in_row(double mass, float tile_top, const SampleWeights &row, int bits)
{
    const double R = rint((double)tile_top * row.c);
    return R >= (double)row.R - 1000.0 ? ldexp(mass, bits + (int)(R - (double)row.R)) : 0.0;
}

// What a row asks for.
enum SampleMode { SAMPLE_BAD, SAMPLE_GREEDY, SAMPLE_PLAIN, SAMPLE_TOPK, SAMPLE_STEPPED, SAMPLE_SWEPT };
struct Settings {
    double c;                  // log2(e) / T
    int top_k;                 // 0: off
    double top_p;              // 1: off
    double log2_min_p;         // -inf: off
    double u;
    float step_scale;          // logit -> steps of log2 w
    SampleMode mode;
};
__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int n)
{
    Settings s;
    const float T = a.temperature ? a.temperature[n] : 1.f, p = a.top_p ? a.top_p[n] : 1.f, m = a.min_p ? a.min_p[n] : 0.f, u = a.u[n];
    const int k = a.top_k ? a.top_k[n] : 0;
    const bool bad = !(T >= 0.f && T <= FLT_MAX) || !(p > 0.f) || !(m >= 0.f && m <= 1.f) || !(u >= 0.f && u < 1.f) || k < 0;
    s.c = 1.4426950408889634 / (double)T;
    s.top_k = k < a.V ? k : 0;
    s.top_p = p < 1.f ? (double)p : 1.0;
    s.log2_min_p = m > 0.f ? log2((double)m) : -INFINITY;
    s.u = u;
    // What lies below (1 - top_p) / V of the largest weight has less than 1 - top_p of the mass in all, so the border is above it, and it is not below min_p.  On
    // flat rows, where a step has the more logits the wider it is, this is 25 steps to the octave for top_p 0.9 of 128256, and 118 for min_p 0.05.
    const double octaves = fmin(p < 1.f ? log2((double)a.V / (1.0 - (double)p)) : INFINITY, -s.log2_min_p);
    s.step_scale = (float)(s.c * (double)(SAMPLE_STEPS - 4) / (octaves + 0.5));
    s.mode = bad                      ? SAMPLE_BAD
             : T == 0.f               ? SAMPLE_GREEDY
             : s.top_k > SAMPLE_TOP_K ? SAMPLE_SWEPT
             : s.top_k                ? SAMPLE_TOPK
             : p < 1.f || m > 0.f     ? SAMPLE_STEPPED
                                      : SAMPLE_PLAIN;
    return s;
}

struct SampleLds {
    unsigned long long hist[SAMPLE_BINS];
    unsigned key[SAMPLE_LIST], index[SAMPLE_LIST];
    unsigned long long tile_mass[SAMPLE_MAX_TILES];
    float tile_top[SAMPLE_MAX_TILES];
    unsigned long long wave_tot[SAMPLE_WAVES], wave_sum[3][SAMPLE_WAVES];
    float best[SAMPLE_WAVES];
    unsigned long long found_before, found_upto, total;          // (total: of draw_by_tiles, whose tile has the mass found_upto)
    int found;
    unsigned count, n_list;
    unsigned low;
};

constexpr int DPP_HALF_MIRROR = 0x141;  // row_half_mirror: lane i of 8 has lane 7 - i's
// NaN counts as -inf.
__device__ __forceinline__ float sample_logit(float z) { return z == z ? z : neg_inf(); }

// f(vector index, its N values) for vectors v0 .. v1 - 1 of the row, by all threads in turn; the values behind the row's end and NaN are -inf.
template <typename DT, typename F>
__device__ __forceinline__ void sample_sweep(const DT *row, int V, F f)
{
    constexpr int N = VecOf<DT>::N, U = 8;
    const int nvec = (V + N - 1) / N;
    for (int v0 = threadIdx.x; v0 < nvec; v0 += U * SAMPLE_WG) {
        typename RawOf<DT>::type raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = warp_load<DT>(row, v0 + u * SAMPLE_WG < nvec ? v0 + u * SAMPLE_WG : v0, V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (v0 + u * SAMPLE_WG >= nvec) continue;
            float z[N];
            unpack<DT>(raw[u], z);
#pragma unroll
            for (int e = 0; e < N; ++e) z[e] = sample_logit(z[e]);
            f(v0 + u * SAMPLE_WG, z);
        }
    }
}

// The sum over all threads.  Sums one after the other go through different slots, so that one barrier each does: by the time a slot is written again
// everybody has been through the barrier of another sum.
template <int SLOT>
__device__ __forceinline__ unsigned long long sum_of_all(unsigned long long v, SampleLds &L)
{
    v = wave_reduce(v, OpSum{});
    if ((threadIdx.x & 63) == 0) L.wave_sum[SLOT][threadIdx.x >> 6] = v;
    __syncthreads();
    unsigned long long t = 0ull;
#pragma unroll
    for (int w = 0; w < SAMPLE_WAVES; ++w) t += L.wave_sum[SLOT][w];
    return t;
}

// Of hist[0 .. SAMPLE_BINS), in ascending order if UP and descending if not, the first bin at which the running sum reaches target_of(total) (>= 1), and the sum
// before it; -1 if the total falls short.  All threads, behind a barrier that completes the histogram; ends behind one and leaves the bins at zero, as the
// next histogram finds them.
template <bool UP, typename T>
__device__ __forceinline__ int find_bin(SampleLds &L, T target_of, unsigned long long *before, unsigned long long *total)
{
    constexpr int PER = SAMPLE_BINS / SAMPLE_WG;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long h[PER], sum = 0ull;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        unsigned long long &bin = L.hist[UP ? tid * PER + i : SAMPLE_BINS - 1 - (tid * PER + i)];
        sum += h[i] = bin;
        bin = 0ull;
    }
    const unsigned long long incl = wave_inclusive_sum_u64(sum);
    if (lane == 63) L.wave_tot[wave] = incl;
    __syncthreads();
    unsigned long long run = incl - sum, all = 0ull;
#pragma unroll
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        if (w < wave) run += L.wave_tot[w];
        all += L.wave_tot[w];
    }
    const unsigned long long target = target_of(all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (run < target && run + h[i] >= target) {
            L.found = UP ? tid * PER + i : SAMPLE_BINS - 1 - (tid * PER + i);
            L.found_before = run;
            L.found_upto = run + h[i];
        }
        run += h[i];
    }
    __syncthreads();
    *before = L.found_before;
    *total = all;
    return all < target ? -1 : L.found;
}

// Spans of keys in which a storage type has one number at most are below 2^this.
template <typename DT> constexpr int SPAN_LOW = std::is_same<DT, bf16>::value ? 16 : VecOf<DT>::N == 8 ? 13 : 0;
// The largest key v with measure(keys >= v) >= target, among those between lo and hi that each(f) calls f(key, value) for; lo if all of them fall short.
// A thousandth of the span at a time, down to spans of 2^LOW (where one number of the storage type has room, what is found may be a lower key that
// separates it from the next one as well).  *above: the measure of the keys above it.
template <int LOW, typename Each, typename M>
__device__ __forceinline__ unsigned select_key(Each each, unsigned lo, unsigned hi, unsigned long long target, SampleLds &L, M measure, unsigned long long *above)
{
    *above = 0ull;
    while ((hi - lo) >> LOW) {
        const int shift = max(0, 22 - __clz((int)(hi - lo)));         // (hi - lo) >> shift < 1024
        each([&](unsigned key, float z) {
            if (key >= lo && key <= hi) atomicAdd(&L.hist[(key - lo) >> shift], measure(z));
        });
        __syncthreads();
        unsigned long long before, total;
        const unsigned long long left = target - *above;
        const int bin = find_bin<false>(L, [&](unsigned long long) { return left; }, &before, &total);
        if (bin < 0) return lo;
        *above += before;
        hi = lo + min(hi - lo, (((unsigned)bin + 1u) << shift) - 1u);
        lo += (unsigned)bin << shift;
    }
    return lo;
}

__device__ __forceinline__ void sample_answer(const SampleArgs &a, int n, int token, float prob, int kept)
{
    a.token[n] = token;
    if (a.prob) a.prob[n] = prob;
    if (a.kept) a.kept[n] = kept;
}

// What decides whether a logit stays.
struct Keep {
    unsigned low;              // least key
    double log2_min_p;
    SampleWeights w;
    __device__ __forceinline__ bool operator()(float z) const { return value_key(z) >= low && w.log2_of(z) >= log2_min_p; }
};

// The draw from vectors v0 .. v1 - 1 of the row, whose kept logits have `mass` and which it is to go into at `left`, less than that: the first token at which
// their running sum, over all of it, exceeds left / mass, compared as products of whole numbers.  `measure` says in which units they are summed here: the row's,
// for a mass that is a sum of just these (then it is compared with `left` itself), or, for a tile's mass, which was rounded as a whole, units of the tile's own, so
// that logits of less than a unit of the row's are drawn by their weights too.  A token without a unit is never drawn.  total: of the row, in its units.
template <typename DT>
__device__ __forceinline__ void draw_in_range(const SampleArgs &a, int n, const DT *row, int v0, int v1, const Keep &keep, const SampleWeights &measure,
                                              unsigned long long left, unsigned long long mass, unsigned long long total, int kept, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (v1 - v0 + SAMPLE_WG - 1) / SAMPLE_WG, first = v0 + tid * per, end = min(v1, first + per);
    unsigned long long mine = 0ull;
    for (int v = first; v < end; ++v) {
        float z[N];
        unpack<DT>(warp_load<DT>(row, v, a.V), z);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (keep(sample_logit(z[e]))) mine += measure.units(z[e]);
    }
    const unsigned long long incl = wave_inclusive_sum_u64(mine);
    if (lane == 63) L.wave_tot[wave] = incl;
    __syncthreads();
    unsigned long long run = incl - mine, all = 0ull;
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        if (w < wave) run += L.wave_tot[w];
        all += L.wave_tot[w];
    }
    typedef unsigned __int128 wide_sum;
    const wide_sum at = (wide_sum)left * all;
    const auto reaches = [&](unsigned long long sum) { return (wide_sum)sum * mass > at; };
    if (reaches(run) || !reaches(run + mine)) return;
    for (int v = first; v < end; ++v) {
        float z[N];
        unpack<DT>(warp_load<DT>(row, v, a.V), z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (!keep(sample_logit(z[e]))) continue;
            const unsigned long long x = measure.units(z[e]);
            if (!reaches(run) && reaches(run + x)) sample_answer(a, n, v * N + e, (float)(keep.w(z[e]) / ldexp((double)total, -a.unit_bits)), kept);
            run += x;
        }
    }
}

// Sweeps over the row for every decision: right for whatever it holds.
template <typename DT>
__device__ __forceinline__ void row_by_sweeps(const SampleArgs &a, int n, const DT *row, const Settings &s, const SampleWeights &w, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int V = a.V, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned low = value_key(neg_inf()) + 1u;
    const unsigned high = value_key((float)w.m);
    const auto each = [&](auto f) {
        sample_sweep(row, V, [&](int, const float(&z)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) f(value_key(z[e]), z[e]);
        });
    };
    unsigned long long above;
    if (s.top_k) low = select_key<SPAN_LOW<DT>>(each, low, high, (unsigned long long)s.top_k, L, [](float) { return 1ull; }, &above);
    const auto mass_of = [&](float z) { return w.units(z); };
    if (s.top_p < 1.0) {
        unsigned long long mass = 0ull;
        each([&](unsigned key, float z) { mass += key >= low ? mass_of(z) : 0ull; });
        mass = sum_of_all<0>(mass, L);
        low = select_key<SPAN_LOW<DT>>(each, low, high, max(1ull, (unsigned long long)ceil(s.top_p * (double)mass)), L, mass_of, &above);
    }
    const Keep keep = {low, s.log2_min_p, w};
    // masses of runs of vectors, in index order
    const int nvec = (V + N - 1) / N, chunks = (nvec + 63) / 64, per = (chunks + SAMPLE_BINS - 1) / SAMPLE_BINS;
    unsigned kept = 0u;
    for (int c = wave; c < chunks; c += SAMPLE_WAVES) {
        const int v = c * 64 + lane;
        unsigned long long mass = 0ull;
        if (v < nvec) {
            float z[N];
            unpack<DT>(warp_load<DT>(row, v, V), z);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (keep(sample_logit(z[e]))) mass += w.units(z[e]), ++kept;
        }
        mass = wave_reduce(mass, OpSum{});
        if (lane == 0) atomicAdd(&L.hist[c / per], mass);
    }
    kept = (unsigned)sum_of_all<1>(kept, L);           // (and the barrier behind the histogram)
    unsigned long long before, total;
    const auto at = [&](unsigned long long all) { return (unsigned long long)(s.u * (double)all); };
    const int bin = find_bin<true>(L, [&](unsigned long long all) { return at(all) + 1ull; }, &before, &total);
    draw_in_range<DT>(a, n, row, bin * per * 64, min(nvec, (bin + 1) * per * 64), keep, w, at(total) - before, L.found_upto - before, total, (int)kept, L);
}

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ unsigned dpp_mov_or_zero_u32(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xF, true);
}
// Inclusive prefix sum over the lanes of a wave, as wave_inclusive_sum but on 32-bit integers.
__device__ __forceinline__ unsigned wave_inclusive_sum_u32(unsigned v)
{
    v += dpp_mov_or_zero_u32<0x111, 0xF>(v);
    v += dpp_mov_or_zero_u32<0x112, 0xF>(v);
    v += dpp_mov_or_zero_u32<0x114, 0xF>(v);
    v += dpp_mov_or_zero_u32<0x118, 0xF>(v);
    v += dpp_mov_or_zero_u32<0x142, 0xA>(v);
    v += dpp_mov_or_zero_u32<0x143, 0xC>(v);
    return v;
}

// All settings decided on a list of up to SMALL_LIST candidates, with four threads each: every candidate against every other, in place of selects.
__device__ __forceinline__ void row_by_small_list(const SampleArgs &a, int n, const Settings &s, const SampleWeights &w, SampleLds &L)
{
    static_assert(SAMPLE_WG == 4 * SMALL_LIST && SMALL_LIST <= SAMPLE_BINS, "");
    const int len = (int)L.n_list, i = threadIdx.x >> 2, part = threadIdx.x & 3;
    if (threadIdx.x < SMALL_LIST) L.hist[threadIdx.x] = (int)threadIdx.x < len ? w.units(key_value(L.key[threadIdx.x])) : 0ull;
    __syncthreads();
    const bool mine = i < len;
    const unsigned key = mine ? L.key[i] : 0u, index = mine ? L.index[i] : 0u;
    const unsigned long long units = L.hist[i];
    int over = 0;
    unsigned long long above = 0ull;
    const auto over_four = [](auto v) {
        v += dpp_mov<DPP_QUAD_XOR1>(v);
        return v + dpp_mov<DPP_QUAD_XOR2>(v);
    };
    if (mine)
        for (int j = part; j < len; j += 4)
            if (L.key[j] > key) ++over, above += L.hist[j];
    over = over_four(over);
    above = over_four(above);
    bool keep = mine && over < s.top_k;
    if (s.top_p < 1.0) {
        const unsigned long long mass = sum_of_all<0>(keep && part == 0 ? units : 0ull, L);
        keep = keep && above < max(1ull, (unsigned long long)ceil(s.top_p * (double)mass));
    }
    keep = keep && w.log2_of(key_value(key)) >= s.log2_min_p;
    const unsigned long long total = sum_of_all<1>(keep && part == 0 ? units : 0ull, L), count = sum_of_all<2>(keep && part == 0 ? 1ull : 0ull, L);
    if (part == 0 && !keep) L.hist[i] = 0ull;
    __syncthreads();
    const unsigned long long at = (unsigned long long)(s.u * (double)total);
    unsigned long long before = 0ull;
    if (keep)
        for (int j = part; j < len; j += 4)
            if (L.index[j] < index) before += L.hist[j];
    before = over_four(before);
    if (keep && part == 0 && before <= at && before + units > at)
        sample_answer(a, n, (int)index, (float)(w(key_value(key)) / ldexp((double)total, -a.unit_bits)), (int)count);
}

// The same on any list of candidates.  It holds every logit from the top_k-th largest on.
template <typename DT>
__device__ __forceinline__ void row_by_list(const SampleArgs &a, int n, const DT *row, const Settings &s, const SampleWeights &w, unsigned lo, SampleLds &L)
{
    const unsigned len = L.n_list, high = value_key((float)w.m);
    if (len <= SMALL_LIST) return row_by_small_list(a, n, s, w, L);
    const auto each = [&](auto f) {
        for (unsigned i = threadIdx.x; i < len; i += SAMPLE_WG) f(L.key[i], key_value(L.key[i]));
    };
    const auto mass_of = [&](float z) { return w.units(z); };
    unsigned long long above;
    unsigned low = select_key<SPAN_LOW<DT>>(each, lo, high, (unsigned long long)s.top_k, L, [](float) { return 1ull; }, &above);
    if (s.top_p < 1.0) {
        unsigned long long mass = 0ull;
        each([&](unsigned key, float z) { mass += key >= low ? mass_of(z) : 0ull; });
        mass = sum_of_all<0>(mass, L);
        low = select_key<SPAN_LOW<DT>>(each, low, high, max(1ull, (unsigned long long)ceil(s.top_p * (double)mass)), L, mass_of, &above);
    }
    const Keep keep = {low, s.log2_min_p, w};
    unsigned long long mass = 0ull, count = 0ull;
    each([&](unsigned, float z) {
        if (keep(z)) mass += mass_of(z), ++count;
    });
    mass = sum_of_all<1>(mass, L);
    count = sum_of_all<2>(count, L);
    const unsigned long long at = (unsigned long long)(s.u * (double)mass);
    // by index, upwards: keys are their complements
    const auto by_index = [&](auto f) {
        for (unsigned i = threadIdx.x; i < len; i += SAMPLE_WG) {
            const float z = key_value(L.key[i]);
            if (keep(z)) f(~L.index[i], z);
        }
    };
    const unsigned token = ~select_key<0>(by_index, ~(unsigned)(a.V - 1), ~0u, at + 1ull, L, mass_of, &above);
    if (threadIdx.x == 0) {
        const float z = sample_logit(widen(row[token]));
        sample_answer(a, n, (int)token, (float)(w(z) / ldexp((double)mass, -a.unit_bits)), (int)count);
    }
}

// What of `items` vectors of the row is not below the key `pivot` goes into the list: the indices, with one addition to the list's length for 32 logits of each lane,
// then the keys (64 rows of 128256 with top_k 1000: 28 us, 37 with an addition for 8 logits and the key picked there).  false: the list has no room.
template <typename DT, typename F>
__device__ __forceinline__ bool list_from(const SampleArgs &a, const DT *row, int items, F vector_of, unsigned pivot, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N, AT_ONCE = 32 / N;
    const int tid = threadIdx.x, lane = tid & 63;
    const float least_kept = key_value(pivot);
    for (int i0 = 0; i0 < items; i0 += AT_ONCE * SAMPLE_WG) {
        typename RawOf<DT>::type raw[AT_ONCE];
        bool mine[AT_ONCE];
#pragma unroll
        for (int b = 0; b < AT_ONCE; ++b) {
            if (i0 + b * SAMPLE_WG >= items) break;
            const int i = i0 + b * SAMPLE_WG + tid, at = vector_of(min(i, items - 1));
            mine[b] = i < items && at * N < a.V;
            raw[b] = warp_load<DT>(row, mine[b] ? at : 0, a.V);
        }
        unsigned bits = 0u;
#pragma unroll
        for (int b = 0; b < AT_ONCE; ++b) {
            if (i0 + b * SAMPLE_WG >= items) break;
            float z[N];
            unpack<DT>(raw[b], z);
            unsigned some = 0u;
#pragma unroll
            for (int e = 0; e < N; ++e) some |= z[e] >= least_kept ? 1u << e : 0u;
            bits |= mine[b] ? some << (b * N) : 0u;
        }
        if (!__ballot(bits != 0u)) continue;
        const unsigned count = (unsigned)__popc(bits), incl = wave_inclusive_sum_u32(count), all = (unsigned)read_lane((int)incl, 63);
        unsigned slot = lane == 0 ? lds_add(&L.n_list, all) : 0u;
        slot = (unsigned)__builtin_amdgcn_readfirstlane((int)slot) + incl - count;
        for (; bits; bits &= bits - 1u, ++slot) {
            const int q = __ffs((int)bits) - 1;
            if (slot < SAMPLE_LIST) L.index[slot] = (unsigned)(vector_of(i0 + q / N * SAMPLE_WG + tid) * N + q % N);
        }
    }
    __syncthreads();
    if (L.n_list > SAMPLE_LIST) return false;
    for (unsigned i = tid; i < L.n_list; i += SAMPLE_WG) L.key[i] = value_key(sample_logit(widen(row[L.index[i]])));
    __syncthreads();
    return true;
}

// Candidates of a top_k by the chunks' maxima.  false: they do not fit the list.
template <typename DT>
__device__ __forceinline__ bool list_top_k(const SampleArgs &a, const DT *row, const TileData *tiles, int top_k, float top, unsigned *lowest, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N, U = SAMPLE_CHUNK / N;
    const int tid = threadIdx.x, lane = tid & 63, chunks = a.tiles * 64;
    const unsigned high = value_key(top), none = value_key(neg_inf());
    constexpr int HELD = 4;                // pairs of chunks that a thread keeps; those of more than 4096 chunks are read each time
    const auto pair = [&](int i) { return reinterpret_cast<const float2 *>(tiles[i / 32].chunk_top)[i % 32]; };
    float2 held[HELD];
#pragma unroll
    for (int q = 0; q < HELD; ++q) held[q] = tid + q * SAMPLE_WG < chunks / 2 ? pair(tid + q * SAMPLE_WG) : make_float2(neg_inf(), neg_inf());
    const auto each = [&](auto f) {
#pragma unroll
        for (int q = 0; q < HELD; ++q) {
            f(2 * (tid + q * SAMPLE_WG), held[q].x);
            f(2 * (tid + q * SAMPLE_WG) + 1, held[q].y);
        }
        for (int i0 = HELD * SAMPLE_WG; i0 < chunks / 2; i0 += SAMPLE_WG) {        // (by whole waves)
            const int i = i0 + tid;
            const float2 two = i < chunks / 2 ? pair(i) : make_float2(neg_inf(), neg_inf());
            f(2 * i, two.x);
            f(2 * i + 1, two.y);
        }
    };
    // the least of the maxima, and a thousandth of the span from the largest at a time
    float lowest_top = INFINITY;
    each([&](int, float z) { lowest_top = z > neg_inf() ? fminf(lowest_top, z) : lowest_top; });
    lowest_top = -wave_max(-lowest_top);
    if (tid == 0) L.low = high, L.n_list = 0u, L.count = 0u;
    __syncthreads();
    if ((tid & 63) == 0 && lowest_top < INFINITY) atomicMin(&L.low, value_key(lowest_top));
    __syncthreads();
    const unsigned least = L.low;
    const int shift = high == least ? 0 : max(0, 22 - __clz((int)(high - least)));
    each([&](int, float z) {
        if (z > neg_inf()) atomicAdd(&L.hist[(value_key(z) - least) >> shift], 1ull);
    });
    __syncthreads();
    unsigned long long before, total;
    const int bin = find_bin<false>(L, [&](unsigned long long) { return (unsigned long long)top_k; }, &before, &total);
    if (bin < 0 && total * SAMPLE_CHUNK > SAMPLE_LIST) return false;       // fewer chunks than that
    const unsigned pivot = bin < 0 ? none + 1u : least + ((unsigned)bin << shift);
    // the chunks that reach the pivot (their numbers where other settings have the tiles' masses)
    unsigned short *const reach = reinterpret_cast<unsigned short *>(L.tile_mass);
    constexpr unsigned MOST = sizeof(L.tile_mass) / 2;
    each([&](int chunk, float z) {         // (a slot for each lane from one addition to the count: 64 additions to one address take 64 turns)
        const bool reaches = z > neg_inf() && value_key(z) >= pivot;
        const unsigned long long mask = __ballot(reaches);
        if (!mask) return;
        unsigned slot = lane == 0 ? lds_add(&L.count, (unsigned)__popcll(mask)) : 0u;
        slot = (unsigned)__builtin_amdgcn_readfirstlane((int)slot) + __builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
        if (reaches && slot < MOST) reach[slot] = (unsigned short)chunk;
    });
    __syncthreads();
    if (L.count > MOST || chunks > 65536) return false;
    if (!list_from<DT>(a, row, (int)L.count * U, [&](int i) { return reach[i / U] * U + i % U; }, pivot, L)) return false;
    *lowest = pivot;
    return true;
}

// The same by the row's own keys, for a top_k that the chunks do not decide: from the key `least` on, if there are as many logits, a thousandth of the span at
// a time, until what a bin and those above it hold fits the list.
template <typename DT>
__device__ __forceinline__ bool list_by_row(const SampleArgs &a, const DT *row, unsigned top_k, unsigned least, float top, SampleLds &L, unsigned *lowest)
{
    constexpr int N = VecOf<DT>::N;
    const unsigned first = value_key(neg_inf()) + 1u;
    unsigned lo = least, hi = value_key(top), pivot;
    unsigned long long above = 0ull, before, total;
    __syncthreads();                       // (who still looks at the length of a list that ran over)
    for (;;) {
        const int shift = max(0, 22 - __clz((int)(hi - lo)));
        sample_sweep(row, a.V, [&](int, const float(&z)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const unsigned key = value_key(z[e]);
                if (key >= lo && key <= hi) atomicAdd(&L.hist[(key - lo) >> shift], 1ull);
            }
        });
        if (threadIdx.x == 0) L.n_list = 0u;
        __syncthreads();
        const int bin = find_bin<false>(L, [&](unsigned long long) { return top_k - above; }, &before, &total);
        if (bin < 0 && lo > first) {
            above += total;
            hi = lo - 1u;
            lo = first;
            continue;
        }
        pivot = bin < 0 ? lo : lo + ((unsigned)bin << shift);
        if (above + (bin < 0 ? total : L.found_upto) <= SAMPLE_LIST) break;
        if (shift == 0) return false;
        above += before;
        hi = lo + min(hi - lo, (((unsigned)bin + 1u) << shift) - 1u);
        lo = pivot;
    }
    *lowest = pivot;
    return list_from<DT>(a, row, (a.V + N - 1) / N, [](int i) { return i; }, pivot, L);
}

// Which step of log2 w a logit lies in, counted upwards from an arbitrary zero: one function for all tiles of a row.
__device__ __forceinline__ float step_of(float z, float scale) { return floorf(z * scale); }

// The first token of those with the largest logit, in tile t.
template <typename DT>
__device__ __forceinline__ void first_in_tile(const SampleArgs &a, int n, const DT *row, int t, float top, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int v0 = t * (SAMPLE_TILE / N), v1 = min((a.V + N - 1) / N, v0 + SAMPLE_TILE / N);
    unsigned first = ~0u;
    for (int v = v0 + (int)threadIdx.x; v < v1; v += SAMPLE_WG) {
        float z[N];
        unpack<DT>(warp_load<DT>(row, v, a.V), z);
#pragma unroll
        for (int e = N - 1; e >= 0; --e)
            if (z[e] == top) first = min(first, (unsigned)(v * N + e));
    }
    if (threadIdx.x == 0) L.low = ~0u;
    __syncthreads();
    atomicMin(&L.low, first);
    __syncthreads();
    if (threadIdx.x == 0) sample_answer(a, n, (int)L.low, 1.f, 1);
}

// From the tiles' masses in L.tile_mass: the tile of the draw, and the draw in it.
template <typename DT>
__device__ __forceinline__ void draw_by_tiles(const SampleArgs &a, int n, const DT *row, const Settings &s, const Keep &keep, int kept, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int tid = threadIdx.x;
    if (tid < 64) {
        unsigned long long total = 0ull;
        for (int t = tid; t < a.tiles; t += 64) total += L.tile_mass[t];
        total = wave_reduce(total, OpSum{});
        const unsigned long long at = (unsigned long long)(s.u * (double)total);
        unsigned long long ahead = 0ull;
        for (int t0 = 0; t0 < a.tiles; t0 += 64) {
            const unsigned long long mass = t0 + tid < a.tiles ? L.tile_mass[t0 + tid] : 0ull, incl = wave_inclusive_sum_u64(mass);
            const unsigned long long hit = __ballot(ahead + incl > at);
            if (hit) {
                const int lane = __ffsll((long long)hit) - 1;
                if (tid == lane) {
                    L.found = t0 + lane;
                    L.found_before = at - (ahead + incl - mass);
                    L.found_upto = mass;
                    L.total = total;
                }
                break;
            }
            ahead += read_lane(incl, 63);
        }
    }
    __syncthreads();
    const int t = L.found, v0 = t * (SAMPLE_TILE / N);
    SampleWeights measure = keep.w;        // (one series for both: its coefficients are 20 scalar registers)
    measure.set(L.tile_top[t], max(TILE_UNIT_BITS, a.unit_bits));      // (51 in rows of up to half a tile)
    draw_in_range<DT>(a, n, row, v0, min((a.V + N - 1) / N, v0 + SAMPLE_TILE / N), keep, measure, L.found_before, L.found_upto, L.total, kept, L);
}

// top_p and min_p by what k_sample_border found.
template <typename DT>
__device__ __forceinline__ void row_by_steps(const SampleArgs &a, int n, const DT *row, const Settings &s, const SampleWeights &w, const RowData &found,
                                             const TileData *tiles, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int tid = threadIdx.x, lane = tid & 63;
    unsigned long long above = 0ull, kept = 0ull, len = 0ull;
    for (int t = tid; t < a.tiles; t += SAMPLE_WG) {
        above += L.tile_mass[t] = tiles[t].above;
        kept += (unsigned)tiles[t].kept;
        len += (unsigned)tiles[t].undecided;
    }
    if (tid == 0) L.n_list = 0u;
    above = sum_of_all<0>(above, L);
    kept = sum_of_all<1>(kept, L);
    len = sum_of_all<2>(len, L);
    const unsigned long long target = found.target;
    const bool by_mass = found.by_mass && target > above;
    const auto mass_of = [&](float z) { return w.units(z); };
    unsigned low = value_key(found.lower);
    const unsigned high = value_key(found.upper) - 1u;
    unsigned long long more, stay = 0ull;
    if (len <= SAMPLE_LIST) {
        for (int t = tid >> 6; t < a.tiles; t += SAMPLE_WAVES) {
            unsigned long long word = tiles[t].in_step[lane];
            const unsigned count = (unsigned)__popcll(word), incl = wave_inclusive_sum_u32(count), all = (unsigned)read_lane((int)incl, 63);
            unsigned to = lane == 0 && all ? atomicAdd(&L.n_list, all) : 0u;
            to = (unsigned)__builtin_amdgcn_readfirstlane((int)to) + incl - count;
            const unsigned first = (unsigned)t * SAMPLE_TILE + lane / N * 64 * N + lane % N;
            for (; word; word &= word - 1ull) L.index[to++] = first + (unsigned)(__ffsll((long long)word) - 1) * N;
        }
        __syncthreads();
        constexpr int AT_ONCE = SAMPLE_LIST / SAMPLE_WG;
        float z[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) z[i] = tid + i * SAMPLE_WG < (int)len ? widen(row[L.index[tid + i * SAMPLE_WG]]) : 0.f;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i)
            if (tid + i * SAMPLE_WG < (int)len) L.key[tid + i * SAMPLE_WG] = value_key(z[i]);        // (read by this thread alone)
        const auto each = [&](auto f) {
            for (unsigned i = tid; i < (unsigned)len; i += SAMPLE_WG) f(L.key[i], key_value(L.key[i]));
        };
        if (by_mass && len) low = select_key<SPAN_LOW<DT>>(each, low, high, target - above, L, mass_of, &more);
        for (unsigned i = tid; i < (unsigned)len; i += SAMPLE_WG) {
            if (L.key[i] < low) continue;
            ++stay;
            atomicAdd(&L.tile_mass[L.index[i] / SAMPLE_TILE], w.units(key_value(L.key[i])));
        }
    } else {                               // more than the lists hold: from the row again
        const auto each_index = [&](auto f) {
            sample_sweep(row, a.V, [&](int v, const float(&z)[N]) {
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (z[e] >= found.lower && !(z[e] >= found.upper)) f(v * N + e, z[e]);
            });
        };
        const auto each = [&](auto f) { each_index([&](int, float z) { f(value_key(z), z); }); };
        if (by_mass) low = select_key<SPAN_LOW<DT>>(each, low, high, target - above, L, mass_of, &more);
        each_index([&](int i, float z) {
            if (value_key(z) < low) return;
            ++stay;
            atomicAdd(&L.tile_mass[i / SAMPLE_TILE], w.units(z));
        });
    }
    kept += sum_of_all<0>(stay, L);
    draw_by_tiles<DT>(a, n, row, s, {low, -INFINITY, w}, (int)kept, L);
}

template <typename DT>
__global__ __launch_bounds__(TILES_WG, VecOf<DT>::N == 8 ? 8 : 4) void k_sample_tiles(SampleArgs a)
{
    constexpr int N = VecOf<DT>::N, U = SAMPLE_CHUNK / N, PER = SAMPLE_STEPS / 64;
    __shared__ unsigned long long all_steps[TILES_WAVES][SAMPLE_STEPS - 1 + 64];       // (the last, which many share, for each lane)
    const int n = blockIdx.x / (unsigned)a.groups, group = blockIdx.x - n * a.groups;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), V = a.V;
    const DT *row = static_cast<const DT *>(a.logits) + n * a.row_stride;
    const int tile = group * TILES_WAVES + wave, v0 = tile * (U * 64) + lane;
    if (tile >= a.tiles) return;
    TileData *const mine = tiles_of(row_data(a.data, n, a.tiles)) + tile;
    typename RawOf<DT>::type raw[U];
    if ((tile + 1) * SAMPLE_TILE <= V) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = *(reinterpret_cast<const typename RawOf<DT>::type *>(row) + v0 + u * 64);
    } else {
        load_raw_tail<DT, U, 64>(row, v0, V, raw);
    }
    const Settings s = settings_of(a, n);
    if (s.mode == SAMPLE_BAD) return;
    float top = neg_inf(), chunk_top = neg_inf();
    int count = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[N], most = neg_inf();
        unpack<DT>(raw[u], z);
#pragma unroll
        for (int e = 0; e < N; ++e) most = vmax(most, vmax(z[e], z[e]));       // (a signalling NaN is quiet then, and passed over)
        top = vmax(top, most);
        if (s.mode == SAMPLE_TOPK) {       // a chunk is U lanes side by side: of vector u lane u of each U keeps it
            most = vmax(most, dpp_mov<DPP_QUAD_XOR1>(most));
            most = vmax(most, dpp_mov<DPP_QUAD_XOR2>(most));
            most = vmax(most, dpp_mov<DPP_HALF_MIRROR>(most));
            if (U == 16) most = vmax(most, dpp_mov<DPP_ROW_ROR8>(most));
            chunk_top = lane % U == u ? most : chunk_top;
        }
    }
    if (s.mode == SAMPLE_TOPK) mine->chunk_top[lane % U * (64 / U) + lane / U] = chunk_top;
    top = wave_max(top);
    const SampleWeights w(top, s.c, TILE_UNIT_BITS);
    double mass = 0.0;
    if (s.mode == SAMPLE_PLAIN && top > neg_inf()) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float z[N];
            asm volatile("" : "+v"(raw[u]));           // (or all vectors are widened, and converted, ahead of the first weight: 200 registers)
            unpack<DT>(raw[u], z);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                mass += w.of_tile(z[e]);
                count += __popcll(__ballot(z[e] >= -FLT_MAX));       // (of z > -inf the compiler makes a comparison that is true for NaN)
                if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
        mass = wave_sum(mass);
    }
    if (lane == 0) {
        mine->top = top;
        mine->count = count;
        mine->mass = mass;
    }
    if (s.mode != SAMPLE_STEPPED || !(top > neg_inf())) return;
    unsigned long long *const steps = all_steps[wave];
#pragma unroll
    for (int i = 0; i <= PER; ++i)
        if (lane + 64 * i < SAMPLE_STEPS - 1 + 64) steps[lane + 64 * i] = 0ull;
    __builtin_amdgcn_wave_barrier();
    const float scale = s.step_scale, first = step_of(top, scale);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[N];
        asm volatile("" : "+v"(raw[u]));
        unpack<DT>(raw[u], z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float step = first - step_of(z[e], scale);
            atomicAdd(&steps[step < (float)(SAMPLE_STEPS - 1) ? (int)step : SAMPLE_STEPS - 1 + lane], units_of(w.of_tile(z[e]), w.unit));
            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    }
    __builtin_amdgcn_wave_barrier();
    unsigned long long rest = steps[SAMPLE_STEPS - 1 + lane];
    rest = wave_reduce(rest, OpSum{});
    unsigned long long h[PER], sum = 0ull;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += h[i] = lane * PER + i < SAMPLE_STEPS - 1 ? steps[lane * PER + i] : rest;
    unsigned long long run = wave_inclusive_sum_u64(sum) - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine->down_to[lane * PER + i] = run += h[i];
}

// The least number for which pass(z) holds, a property of all from some number on (of +inf for certain): keys are searched 64 at a time.
template <typename P>
__device__ __forceinline__ float least_that(P pass)
{
    const unsigned end = value_key(INFINITY);
    unsigned at = value_key(neg_inf());
#pragma unroll 1
    for (int bits = 26; bits >= -4; bits -= 6) {       // the last of 64 that does not pass, or the first
        const unsigned unit = 1u << max(0, bits), key = at + min((unsigned)(threadIdx.x & 63) * unit, end - at);
        const unsigned long long reach = __ballot(pass(key_value(key)));
        at += min((unsigned)(reach ? max(0, __ffsll((long long)reach) - 2) : 63) * unit, end - at);
    }
    return key_value(pass(key_value(at)) ? at : at + 1u);
}

// v with lane `lane` set to a uniform value.  (Clang names no builtin for this instruction; as inline assembly it would miss the two wait states that it needs
// behind a vector instruction's write of the scalar register.)
__device__ unsigned llvm_writelane(unsigned value, unsigned lane, unsigned v) __asm("llvm.amdgcn.writelane.i32");
__device__ __forceinline__ unsigned write_lane(unsigned v, unsigned lane, unsigned value) { return llvm_writelane(value, lane, v); }

// Rows with top_p or min_p and no top_k: the step that holds the border, and what the tiles have in it.  BORDER_BOTH: every workgroup of the row finds the step for
// itself, 6 us, while its tiles' logits come.  Where there are many, BORDER_FIND by one workgroup to a row and BORDER_MARK behind it, which reads no tile that lies
// below (top-p 0.9, 512 rows of 128256 in fp32 166 -> 153 us, 250 in bf16 90 -> 81; 64 rows 43 and 45).
enum { BORDER_BOTH, BORDER_FIND, BORDER_MARK };
template <typename DT, int PART>
__global__ __launch_bounds__(TILES_WG) void k_sample_border(SampleArgs a)
{
    constexpr int N = VecOf<DT>::N, U = SAMPLE_CHUNK / N;
    __shared__ float tile_top[SAMPLE_MAX_TILES];
    __shared__ float wave_top[TILES_WAVES];
    __shared__ unsigned long long all;
    __shared__ int first_group;
    const int groups = PART == BORDER_FIND ? 1 : a.groups, n = blockIdx.x / (unsigned)groups, group = blockIdx.x - n * groups;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = a.V;
    const Settings s = settings_of(a, n);
    if (s.mode != SAMPLE_STEPPED) return;
    const DT *row = static_cast<const DT *>(a.logits) + n * a.row_stride;
    typename RawOf<DT>::type raw[U];
    const auto load = [&](int tile) {
        const int v0 = tile * (U * 64) + lane;
        if ((tile + 1) * SAMPLE_TILE <= V) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = *(reinterpret_cast<const typename RawOf<DT>::type *>(row) + v0 + u * 64);
        } else {
            load_raw_tail<DT, U, 64>(row, v0, V, raw);
        }
    };
    const int tile = group * TILES_WAVES + wave;
    if (PART == BORDER_BOTH && tile < a.tiles) load(tile);        // (they arrive while the border is looked for)
    RowData *const found = row_data(a.data, n, a.tiles);
    TileData *const tiles = tiles_of(found);
    if (PART == BORDER_MARK && !found->found) return;
    float top = neg_inf();
    if (PART == BORDER_MARK) {
        top = found->top;
    } else {
        for (int t = tid; t < a.tiles; t += TILES_WG) top = vmax(top, tile_top[t] = tiles[t].top);
        top = wave_max(top);
        if (lane == 0) wave_top[wave] = top;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TILES_WAVES; ++i) top = vmax(top, wave_top[i]);
    }
    const SampleWeights w(top, s.c, a.unit_bits);
    const float scale = s.step_scale, first = step_of(top, scale);
    const auto give_up = [&]() {
        if (group == 0 && tid == 0) found->found = 0;
    };
    if (!(top > neg_inf() && fabsf(first) < 8388608.f && w.near)) return give_up();      // (numbers of steps are whole numbers in fp32)
    // mass of tile t down to the end of the row's step r (counted from its first, downwards; of the last: all of it), in the row's units
    const auto tile_down_to = [&](int t, float its_top, int r) -> unsigned long long {
        if (!(its_top > neg_inf())) return 0ull;
        const float i = r < SAMPLE_STEPS - 1 ? (float)r - (first - step_of(its_top, scale)) : (float)(SAMPLE_STEPS - 1);
        if (!(i >= 0.f)) return 0ull;
        const unsigned long long mass = tiles[t].down_to[(int)i];
        return (unsigned long long)rint(in_row((double)mass, its_top, w, a.unit_bits - TILE_UNIT_BITS));
    };
    // of the row down to the end of eight steps side by side: threads 32 i .. 32 i + 31 have the sum of r(i)
    static_assert(TILES_WG == 8 * 32 && SAMPLE_STEPS == 8 * 8 * 8, "a step each, three times");
    const auto row_down_to = [&](int r) {
        unsigned long long mass = 0ull;
        for (int t = tid & 31; t < a.tiles; t += 32) mass += tile_down_to(t, tile_top[t], r);
        mass = row_reduce(mass, OpSum{});
        const auto lo = __builtin_amdgcn_permlane16_swap((unsigned)mass, (unsigned)mass, false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap((unsigned)(mass >> 32), (unsigned)(mass >> 32), false, false);
        return ((unsigned long long)hi[0] << 32 | lo[0]) + ((unsigned long long)hi[1] << 32 | lo[1]);
    };
    int step = SAMPLE_STEPS;               // above it all stays, below nothing
    float lower = neg_inf(), upper;
    if (PART == BORDER_MARK) {
        step = found->step;
        lower = found->lower;
        upper = found->upper;
    } else {
        unsigned long long target = 0ull;
        if (s.top_p < 1.0) {
            unsigned long long mass = row_down_to(64 * (tid / 32) + 63);
            if (tid == TILES_WG - 1) all = mass;
            __syncthreads();
            target = max(1ull, (unsigned long long)ceil(s.top_p * (double)all));
            step = 0;
#pragma unroll 1
            for (int width = 64;; width /= 8) {
                if (tid == 0) first_group = 8;
                __syncthreads();
                if ((tid & 31) == 0 && mass >= target) atomicMin(&first_group, tid / 32);
                __syncthreads();
                step += first_group * width;
                if (first_group == 8 || width == 1) break;
                mass = row_down_to(step + width / 8 * (tid / 32 + 1) - 1);
                __syncthreads();
            }
        }
        bool by_mass = s.top_p < 1.0;
        if (s.log2_min_p > -INFINITY) {
            lower = least_that([&](float z) { return w.log2_of(z) >= s.log2_min_p; });
            const float its = first - step_of(lower, scale);
            if (its < (float)step) {
                step = (int)its;
                by_mass = false;
            }
        }
        if (step >= SAMPLE_STEPS - 1) return give_up();    // (the last step of a tile is all that lies below it too)
        upper = least_that([&](float z) { return step_of(z, scale) >= first - (float)step + 1.f; });
        lower = fmaxf(lower, least_that([&](float z) { return step_of(z, scale) >= first - (float)step; }));
        if (group == 0 && tid == 0) {
            found->found = 1;
            found->by_mass = by_mass;
            found->upper = upper;
            found->lower = lower;
            found->target = target;
            found->step = step;
            found->top = top;
        }
    }
    if (PART == BORDER_FIND || tile >= a.tiles) return;
    TileData *const mine = tiles + tile;
    const float its_top = mine->top;
    if (!(its_top >= lower)) {             // nothing of it stays
        mine->in_step[lane] = 0ull;
        if (lane == 0) mine->above = 0ull, mine->kept = mine->undecided = 0;
        return;
    }
    if (PART == BORDER_MARK) load(tile);
    int kept = 0;
    unsigned lo = 0u, hi = 0u;             // the word of each lane
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[N];
        unpack<DT>(raw[u], z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            kept += z[e] >= upper;
            const unsigned long long in = __ballot(z[e] >= lower && !(z[e] >= upper));
            lo = write_lane(lo, u * N + e, (unsigned)in);
            hi = write_lane(hi, u * N + e, (unsigned)(in >> 32));
            __builtin_amdgcn_sched_barrier(0);         // (or 128 scalar registers are held for the words)
        }
    }
    mine->in_step[lane] = (unsigned long long)hi << 32 | lo;
    const int undecided = wave_reduce((int)(__popc(lo) + __popc(hi)), OpSum{});
    kept = wave_reduce(kept, OpSum{});
    if (lane == 0) {
        mine->above = tile_down_to(tile, its_top, step - 1);
        mine->kept = kept;
        mine->undecided = undecided;
    }
}

template <typename DT>
__global__ __launch_bounds__(SAMPLE_WG) void k_sample_rows(SampleArgs a)
{
    __shared__ SampleLds L;
    const int n = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const DT *row = static_cast<const DT *>(a.logits) + n * a.row_stride;
    RowData *const found = row_data(a.data, n, a.tiles);
    const TileData *const tiles = tiles_of(found);
    const Settings s = settings_of(a, n);
    if (s.mode == SAMPLE_BAD) {
        if (tid == 0) {
            atomicOr(a.flags, (unsigned)SVIP_FLAG_BAD_SETTING);
            sample_answer(a, n, -1, 0.f, 0);
        }
        return;
    }
    float top = neg_inf();
    unsigned long long count = 0ull;
    for (int t = tid; t < a.tiles; t += SAMPLE_WG) {
        L.tile_top[t] = tiles[t].top;
        top = vmax(top, L.tile_top[t]);
        count += (unsigned)tiles[t].count;
    }
    top = wave_max(top);
    if (lane == 0) L.best[wave] = top;
#pragma unroll
    for (int i = 0; i < SAMPLE_BINS / SAMPLE_WG; ++i) L.hist[tid + i * SAMPLE_WG] = 0ull;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SAMPLE_WAVES; ++i) top = vmax(top, L.best[i]);
    if (!(top > neg_inf())) {
        if (tid == 0) sample_answer(a, n, -1, 0.f, 0);
        return;
    }
    if (s.mode == SAMPLE_GREEDY) {
        if (tid == 0) L.found = a.tiles;
        __syncthreads();
        for (int t = tid; t < a.tiles; t += SAMPLE_WG)
            if (L.tile_top[t] == top) atomicMin(&L.found, t);
        __syncthreads();
        first_in_tile<DT>(a, n, row, L.found, top, L);
        return;
    }
    const SampleWeights w(top, s.c, a.unit_bits);
    if (top < INFINITY && w.near) {
        if (s.mode == SAMPLE_PLAIN) {
            for (int t = tid; t < a.tiles; t += SAMPLE_WG)
                L.tile_mass[t] = L.tile_top[t] > neg_inf() ? (unsigned long long)rint(in_row(tiles[t].mass, L.tile_top[t], w, a.unit_bits)) : 0ull;
            count = sum_of_all<0>(count, L);
            draw_by_tiles<DT>(a, n, row, s, {value_key(neg_inf()) + 1u, -INFINITY, w}, (int)count, L);
            return;
        }
        if (s.top_k && s.top_k <= SAMPLE_LIST) {
            unsigned lowest;
            const bool by_chunks = s.mode == SAMPLE_TOPK;
            const unsigned first = value_key(neg_inf()) + 1u;
            if ((by_chunks && list_top_k<DT>(a, row, tiles, s.top_k, top, &lowest, L)) ||
                list_by_row<DT>(a, row, (unsigned)s.top_k, by_chunks ? L.low : first, top, L, &lowest)) {
                row_by_list<DT>(a, n, row, s, w, lowest, L);
                return;
            }
        }
        if (s.mode == SAMPLE_STEPPED && found->found) {
            row_by_steps<DT>(a, n, row, s, w, *found, tiles, L);
            return;
        }
        __syncthreads();
    }
    row_by_sweeps<DT>(a, n, row, s, w, L);
}

}  // namespace svip
