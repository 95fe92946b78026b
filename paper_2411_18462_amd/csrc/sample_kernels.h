// Kernels of svip_sample: a token for each row of logits, every row with its own temperature, top-k, top-p and min-p (not in the paper).
//
// Weights are w = exp2((z - m) c) with c = log2(e) / T and m the row's largest logit, in 64 bits: which token a uniform falls on, and which
// value the nucleus ends at, are borders between sums of up to V weights, and a rounding of 2^-24 in each weight moves such a border by more than
// the narrowest cells are wide.  The fp64 pipe takes a fused multiply-add in four cycles, as the fp32 pipe does, so a weight costs about
// 17 instructions against 7.  Sums that decide are integers in units of 2^-S of the largest weight (S = 62 - ceil(log2 V)), so that no
// order of additions changes a result and atomics may be used.
//
// Two launches.  k_sample_tiles reads the rows once: a wave has a tile of 4096 logits in registers, a lane a chunk of 64 of them.  k_sample_rows, a workgroup
// each row, does what the row's settings need beside that.  What a wave leaves for the row:
//   T = 0         the tile's maximum
//   no filter     and its mass; the draw finds the tile by the masses and goes through that tile alone again
//   top-k         and the maximum of every chunk.  The k-th largest of those is no larger than the k-th largest logit, so chunks below it hold no
//                 candidate: the others are read again, what is at or above it goes into a list in LDS, and all settings are decided on the list
//   top-p, min-p  and the mass of the tile's logits from the top down to each of 512 steps of 1/16 in log2 w.  From the tiles' masses follows the step
//                 that holds the border, exactly; a sweep over the row without exponentials fetches that step's logits into the list, which decides
//                 what of it stays; the draw goes by the tiles' masses and through one tile.
// Rows that do not fit these (a top_k of more than 1024, a list that runs over, +inf, a border below 2^-31 of the largest weight) are swept as
// often as a radix select over their keys needs (row_by_sweeps).
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
    char *tile_data;           // [N][tiles] TileData
};

constexpr int TILES_WG = 256, TILES_WAVES = TILES_WG / 64;             // k_sample_tiles
constexpr int SAMPLE_WG = 512, SAMPLE_WAVES = SAMPLE_WG / 64;          // k_sample_rows
constexpr int SAMPLE_CHUNK = 64, SAMPLE_TILE = 64 * SAMPLE_CHUNK;       // logits of a lane and of a wave
constexpr int SAMPLE_STEPS = 512;                      // of log2 w, a 16th each
constexpr float STEPS_PER_OCTAVE = 16.f;
constexpr int TILE_UNIT_BITS = 50;                     // masses of a tile, relative to its own largest weight: 2^12 of them fit 64 bits
constexpr int SAMPLE_BINS = 1024;
constexpr int SAMPLE_LIST = 4096;
constexpr int SAMPLE_TOP_K = 1024;
constexpr int SAMPLE_MAX_TILES = (1 << 22) / SAMPLE_TILE;

// What a wave leaves of its tile.
struct TileData {
    float top;                             // the largest logit
    int count;                             // logits above -inf
    double mass;                           // relative to it
    unsigned long long down_to[SAMPLE_STEPS];      // mass from the top down to the end of each step
    float chunk_top[64];
};

// 2^x for x <= 0; below 2^-1000, and for NaN, 2^-1000 (which is nothing in any unit here).  2^n times the series of 2^f = exp(f ln 2), |f| <= 1/2: what it
// leaves out is below 2.3e-13 of the result.  The coefficients are kept in scalar registers: as constants each of them would be moved into
// a vector register pair for every weight, two more instructions to each of ten.
struct Exp2Series {
    double c[11];
    __device__ __forceinline__ Exp2Series()
        : c{1.0,
            6.9314718055994531e-1,
            2.4022650695910072e-1,
            5.5504108664821580e-2,
            9.6181291076284772e-3,
            1.3333558146428443e-3,
            1.5403530393381610e-4,
            1.5252733804059841e-5,
            1.3215486790144309e-6,
            1.0178086009239699e-7,
            7.0549116208011234e-9}
    {
#pragma unroll
        for (int i = 1; i < 11; ++i) asm("" : "+s"(c[i]));
    }
    __device__ __forceinline__ double operator()(double x) const
    {
        x = fmax(x, -1000.0);
        const double t = x + 6755399441055744.0;       // 1.5 * 2^52: x rounded to a whole number in the low bits
        const double f = x - (t - 6755399441055744.0);
        double r = c[10];
#pragma unroll
        for (int i = 9; i >= 0; --i) r = fma(r, f, c[i]);
        return __hiloint2double(__double2hiint(r) + (__double2loint(t) << 20), __double2loint(r));
    }
};
// 2^(52 - bits): added to a weight of at most 1 it leaves the weight in units of 2^-bits, rounded, in the low bits of the sum
__device__ __forceinline__ double unit_of(int bits) { return __longlong_as_double((long long)(1023 + 52 - bits) << 52); }
__device__ __forceinline__ unsigned long long units_of(double w, double unit)
{
    return (unsigned long long)__double_as_longlong(w + unit) - (unsigned long long)__double_as_longlong(unit);
}

struct SampleWeights {
    double m, c;               // the largest logit; log2(e) / T
    double unit;
    Exp2Series exp2;
    __device__ __forceinline__ SampleWeights(float top, double c_, int unit_bits) : m(top), c(c_), unit(unit_of(unit_bits)) {}
    __device__ __forceinline__ double log2_of(float z) const { return (double)z == m ? 0.0 : ((double)z - m) * c; }      // (m may be +inf)
    __device__ __forceinline__ double operator()(float z) const { return exp2(log2_of(z)); }
    __device__ __forceinline__ double of_tile(float z) const { return exp2(((double)z - m) * c); }       // (what a +inf makes of a tile, nobody looks at)
    __device__ __forceinline__ unsigned long long units(float z) const { return units_of((*this)(z), unit); }
};

// What a row asks for.
enum SampleMode { SAMPLE_BAD, SAMPLE_GREEDY, SAMPLE_PLAIN, SAMPLE_TOPK, SAMPLE_STEPPED, SAMPLE_SWEPT };
struct Settings {
    double c;                  // log2(e) / T
    int top_k;                 // 0: off
    double top_p;              // 1: off
    double log2_min_p;         // -inf: off
    double u;
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
    unsigned long long wave_tot[SAMPLE_WAVES];
    float best[SAMPLE_WAVES];
    unsigned long long found_before, total;
    int found;
    unsigned count, n_list;
    unsigned low, high;
    int last;
};

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

template <typename T>
__device__ __forceinline__ T sum_of_all(T v, SampleLds &L)        // ends behind a barrier
{
    v = wave_reduce(v, OpSum{});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) L.wave_tot[threadIdx.x >> 6] = (unsigned long long)v;
    __syncthreads();
    unsigned long long t = 0ull;
#pragma unroll
    for (int w = 0; w < SAMPLE_WAVES; ++w) t += L.wave_tot[w];
    __syncthreads();
    return (T)t;
}

// Of hist[0 .. SAMPLE_BINS), in ascending order if UP and descending if not, the first bin at which the running sum reaches `target` (>= 1), and the sum
// before it; -1 if the total falls short.  All threads; L.hist is complete behind a barrier; ends behind one, and so may a next call begin.
template <bool UP>
__device__ __forceinline__ int find_bin(SampleLds &L, unsigned long long target, unsigned long long *before)
{
    constexpr int PER = SAMPLE_BINS / SAMPLE_WG;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long h[PER], sum = 0ull;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += h[i] = L.hist[UP ? tid * PER + i : SAMPLE_BINS - 1 - (tid * PER + i)];
    const unsigned long long incl = wave_inclusive_sum_u64(sum);
    if (lane == 63) L.wave_tot[wave] = incl;
    if (tid == 0) L.found = -1;
    __syncthreads();
    unsigned long long ahead = 0ull;
    for (int w = 0; w < wave; ++w) ahead += L.wave_tot[w];
    unsigned long long run = ahead + incl - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (run < target && run + h[i] >= target) {
            L.found = UP ? tid * PER + i : SAMPLE_BINS - 1 - (tid * PER + i);
            L.found_before = run;
        }
        run += h[i];
    }
    if (tid == SAMPLE_WG - 1) L.total = run;
    __syncthreads();
    *before = L.found_before;
    const int found = L.found;
    __syncthreads();
    return found;
}
__device__ __forceinline__ void clear_hist(SampleLds &L)
{
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SAMPLE_BINS / SAMPLE_WG; ++i) L.hist[threadIdx.x + i * SAMPLE_WG] = 0ull;
    __syncthreads();
}

// The largest key v with measure(keys >= v) >= target, among those between lo and hi that each(f) calls f(key, value) for; lo if all of them fall short.
// A thousandth of the span at a time, down to spans of 2^LOW (where one number of the storage type has room, what is found may be a lower key that
// separates it from the next one as well).  *above: the measure of the keys above it.
template <int LOW, typename Each, typename M>
__device__ __forceinline__ unsigned select_key(Each each, unsigned lo, unsigned hi, unsigned long long target, SampleLds &L, M measure, unsigned long long *above)
{
    *above = 0ull;
    while ((hi - lo) >> LOW) {
        const int shift = max(0, 22 - __clz((int)(hi - lo)));         // (hi - lo) >> shift < 1024
        clear_hist(L);
        each([&](unsigned key, float z) {
            if (key >= lo && key <= hi) atomicAdd(&L.hist[(key - lo) >> shift], measure(z));
        });
        __syncthreads();
        unsigned long long before;
        const int bin = find_bin<false>(L, target - *above, &before);
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

// The draw from vectors v0 .. v1 - 1 of the row, `left` units behind the mass in front of them: the first token at which the sum exceeds that, or, where
// roundings leave none, the last that has weight.  total: of the row, in units.
template <typename DT>
__device__ __forceinline__ void draw_in_range(const SampleArgs &a, int n, const DT *row, int v0, int v1, const Keep &keep, unsigned long long left,
                                              unsigned long long total, int kept, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (v1 - v0 + SAMPLE_WG - 1) / SAMPLE_WG, first = v0 + tid * per, end = min(v1, first + per);
    unsigned long long mass = 0ull;
    int last = -1;
    for (int v = first; v < end; ++v) {
        float z[N];
        unpack<DT>(warp_load<DT>(row, v, a.V), z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (!keep(sample_logit(z[e]))) continue;
            mass += keep.w.units(z[e]);
            last = v * N + e;
        }
    }
    const unsigned long long incl = wave_inclusive_sum_u64(mass);
    __syncthreads();
    if (lane == 63) L.wave_tot[wave] = incl;
    if (tid == 0) L.last = -1;
    __syncthreads();
    unsigned long long run = incl - mass, all = 0ull;
    for (int w = 0; w < SAMPLE_WAVES; ++w) {
        if (w < wave) run += L.wave_tot[w];
        all += L.wave_tot[w];
    }
    const auto answer = [&](int i) {
        const float z = sample_logit(widen(row[i]));
        sample_answer(a, n, i, (float)(keep.w(z) / ldexp((double)total, -a.unit_bits)), kept);
    };
    if (all <= left) {
        atomicMax(&L.last, last);
        __syncthreads();
        if (tid == 0) answer(L.last);
        return;
    }
    if (run > left || run + mass <= left) return;
    for (int v = first; v < end; ++v) {
        float z[N];
        unpack<DT>(warp_load<DT>(row, v, a.V), z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if (!keep(sample_logit(z[e]))) continue;
            const unsigned long long x = keep.w.units(z[e]);
            if (run <= left && run + x > left) answer(v * N + e);
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
    if (s.top_k) low = select_key<KEY_LOW<DT>>(each, low, high, (unsigned long long)s.top_k, L, [](float) { return 1ull; }, &above);
    const auto mass_of = [&](float z) { return w.units(z); };
    if (s.top_p < 1.0) {
        unsigned long long mass = 0ull;
        each([&](unsigned key, float z) { mass += key >= low ? mass_of(z) : 0ull; });
        mass = sum_of_all(mass, L);
        low = select_key<KEY_LOW<DT>>(each, low, high, max(1ull, (unsigned long long)ceil(s.top_p * (double)mass)), L, mass_of, &above);
    }
    const Keep keep = {low, s.log2_min_p, w};
    // masses of runs of vectors, in index order
    const int nvec = (V + N - 1) / N, chunks = (nvec + 63) / 64, per = (chunks + SAMPLE_BINS - 1) / SAMPLE_BINS;
    clear_hist(L);
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
    kept = (unsigned)sum_of_all((unsigned long long)kept, L);
    unsigned long long before;
    find_bin<true>(L, ~0ull, &before);
    const unsigned long long total = L.total, at = (unsigned long long)(s.u * (double)total);
    __syncthreads();
    const int bin = find_bin<true>(L, at + 1ull, &before);
    draw_in_range<DT>(a, n, row, bin * per * 64, min(nvec, (bin + 1) * per * 64), keep, at - before, total, (int)kept, L);
}

// Appends to the list those of a vector's logits that pass; L.n_list counts them all, also those that have no place.
template <int N, typename P>
__device__ __forceinline__ void append(SampleLds &L, const float (&z)[N], int index, P pass)
{
    unsigned at = 0u;
#pragma unroll
    for (int e = 0; e < N; ++e) at |= pass(z[e]) ? 1u << e : 0u;
    if (!at) return;
    unsigned slot = lds_add(&L.n_list, (unsigned)__popc(at));
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (at >> e & 1u) {
            if (slot < SAMPLE_LIST) {
                L.key[slot] = value_key(z[e]);
                L.index[slot] = (unsigned)(index + e);
            }
            ++slot;
        }
}

// All settings decided on the list of candidates, which holds every logit from the top_k-th largest on.
template <typename DT>
__device__ __forceinline__ void row_by_list(const SampleArgs &a, int n, const DT *row, const Settings &s, const SampleWeights &w, unsigned lo, SampleLds &L)
{
    const unsigned len = L.n_list, high = value_key((float)w.m);
    const auto each = [&](auto f) {
        for (unsigned i = threadIdx.x; i < len; i += SAMPLE_WG) f(L.key[i], key_value(L.key[i]));
    };
    const auto mass_of = [&](float z) { return w.units(z); };
    unsigned long long above;
    unsigned low = select_key<KEY_LOW<DT>>(each, lo, high, (unsigned long long)s.top_k, L, [](float) { return 1ull; }, &above);
    if (s.top_p < 1.0) {
        unsigned long long mass = 0ull;
        each([&](unsigned key, float z) { mass += key >= low ? mass_of(z) : 0ull; });
        mass = sum_of_all(mass, L);
        low = select_key<KEY_LOW<DT>>(each, low, high, max(1ull, (unsigned long long)ceil(s.top_p * (double)mass)), L, mass_of, &above);
    }
    const Keep keep = {low, s.log2_min_p, w};
    unsigned long long mass = 0ull, count = 0ull;
    each([&](unsigned, float z) {
        if (keep(z)) mass += mass_of(z), ++count;
    });
    mass = sum_of_all(mass, L);
    count = sum_of_all(count, L);
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

// Candidates of a top_k by the chunks' maxima.  false: they do not fit the list.
template <typename DT>
__device__ __forceinline__ bool list_top_k(const SampleArgs &a, const DT *row, const TileData *tiles, int top_k, float top, unsigned *lowest, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N, U = SAMPLE_CHUNK / N;
    const int tid = threadIdx.x, chunks = a.tiles * 64;
    const unsigned high = value_key(top), none = value_key(neg_inf());
    const auto each = [&](auto f) {        // two chunks at a time
        for (int i = tid; i < chunks / 2; i += SAMPLE_WG) {
            const unsigned long long two = reinterpret_cast<const unsigned long long *>(tiles[i / 32].chunk_top)[i % 32];
            f(2 * i, value_key(__uint_as_float((unsigned)two)));
            f(2 * i + 1, value_key(__uint_as_float((unsigned)(two >> 32))));
        }
    };
    // the least of the maxima, and a thousandth of the span from the largest at a time
    unsigned least = high;
    each([&](int, unsigned key) { least = key > none ? min(least, key) : least; });
    if (tid == 0) L.low = high, L.n_list = 0u, L.count = 0u;
    clear_hist(L);
    atomicMin(&L.low, least);
    __syncthreads();
    least = L.low;
    const int shift = high == least ? 0 : max(0, 22 - __clz((int)(high - least)));
    each([&](int, unsigned key) {
        if (key > none) atomicAdd(&L.hist[(key - least) >> shift], 1ull);
    });
    __syncthreads();
    unsigned long long before;
    const int bin = find_bin<false>(L, (unsigned long long)top_k, &before);
    const unsigned pivot = bin < 0 ? none + 1u : least + ((unsigned)bin << shift);
    // the chunks that reach the pivot, then their logits (the chunks' numbers where the histogram was)
    unsigned short *const reach = reinterpret_cast<unsigned short *>(L.hist);
    constexpr unsigned MOST = sizeof(L.hist) / 2;
    each([&](int chunk, unsigned key) {
        if (key >= pivot && key > none) {
            const unsigned slot = lds_add(&L.count, 1u);
            if (slot < MOST) reach[slot] = (unsigned short)chunk;
        }
    });
    __syncthreads();
    if (L.count > MOST || chunks > 65536) return false;
    const int items = (int)L.count * U;
    for (int i = tid; i < items; i += SAMPLE_WG) {
        const int chunk = reach[i / U], v = (chunk / 64 * U + i % U) * 64 + chunk % 64;
        if (v * N >= a.V) continue;
        float z[N];
        unpack<DT>(warp_load<DT>(row, v, a.V), z);
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = sample_logit(z[e]);
        append<N>(L, z, v * N, [&](float x) { return x > neg_inf() && value_key(x) >= pivot; });
    }
    __syncthreads();
    *lowest = pivot;
    return L.n_list <= SAMPLE_LIST;
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
                    L.total = total;
                }
                break;
            }
            ahead += read_lane(incl, 63);
        }
    }
    __syncthreads();
    const int t = L.found, v0 = t * (SAMPLE_TILE / N);
    const unsigned long long left = L.found_before, total = L.total;
    draw_in_range<DT>(a, n, row, v0, min((a.V + N - 1) / N, v0 + SAMPLE_TILE / N), keep, left, total, kept, L);
}

// top_p and min_p by the tiles' masses down to each step.  false: for the sweeps.
template <typename DT>
__device__ __forceinline__ bool row_by_steps(const SampleArgs &a, int n, const DT *row, const Settings &s, const SampleWeights &w, const TileData *tiles, SampleLds &L)
{
    constexpr int N = VecOf<DT>::N;
    const int tid = threadIdx.x;
    const float scale = (float)(s.c * (double)STEPS_PER_OCTAVE), first = step_of((float)w.m, scale);
    if (!(fabsf(first) < 8388608.f)) return false;     // (numbers of steps are whole numbers in fp32)
    // mass of tile t down to the end of the row's step r (counted from its first, downwards), in the row's units
    const auto tile_down_to = [&](int t, int r) -> unsigned long long {
        const float top = L.tile_top[t];
        if (!(top > neg_inf())) return 0ull;
        const float i = (float)r - (first - step_of(top, scale));
        if (!(i >= 0.f)) return 0ull;
        const unsigned long long mass = tiles[t].down_to[i < (float)SAMPLE_STEPS ? (int)i : SAMPLE_STEPS - 1];
        return (unsigned long long)rint(ldexp((double)mass, a.unit_bits - TILE_UNIT_BITS) * w(top));
    };
    // of the row down to the end of eight steps side by side: the waves have the sum of a step each
    static_assert(SAMPLE_WAVES == 8, "a step each");
    const int wave = tid >> 6;
    const auto row_down_to = [&](int r) {
        unsigned long long mass = 0ull;
        for (int t = tid & 63; t < a.tiles; t += 64) mass += tile_down_to(t, r);
        return wave_reduce(mass, OpSum{});
    };
    int lo = SAMPLE_STEPS, hi = SAMPLE_STEPS;          // steps from lo to hi are undecided; above all stays, below nothing
    unsigned long long target = ~0ull;
    if (s.top_p < 1.0) {
        int base = 0, found = -1;
        unsigned long long mass = row_down_to(64 * wave + 63);
        if (tid == SAMPLE_WG - 1) L.total = mass;
        __syncthreads();
        target = max(1ull, (unsigned long long)ceil(s.top_p * (double)L.total));
#pragma unroll 1
        for (int width = 64; ; width /= 8) {           // 64, 8, 1
            if (tid == 0) L.found = 8;
            __syncthreads();
            if (mass >= target) atomicMin(&L.found, wave);
            __syncthreads();
            found = L.found;
            __syncthreads();
            if (found == 8) return false;
            base += found * width;
            if (width == 1) break;
            mass = row_down_to(base + width / 8 * (wave + 1) - 1);
        }
        if (base >= SAMPLE_STEPS - 1) return false;    // (the last step of a tile is all that lies below it too)
        lo = hi = base;
    }
    if (s.log2_min_p > -INFINITY) {
        const float step = first - step_of((float)(w.m + s.log2_min_p / w.c), scale);
        if (step < (float)(SAMPLE_STEPS - 2)) {        // one more on either side for the border's own rounding
            lo = min(lo, max(0, (int)step - 1));
            hi = min(hi, (int)step + 1);
        } else if (hi >= SAMPLE_STEPS) {
            return false;
        }
    }
    // masses above the undecided steps, and their logits
    unsigned long long above = 0ull;
    for (int t = tid; t < a.tiles; t += SAMPLE_WG) above += L.tile_mass[t] = tile_down_to(t, lo - 1);
    above = sum_of_all(above, L);
    if (tid == 0) L.n_list = 0u, L.low = ~0u, L.high = 0u;
    __syncthreads();
    unsigned kept = 0u, least = ~0u, most = 0u;
    // the least logit of a step not below `step`: those keys are searched 64 at a time
    const auto least_of = [&](float step) {
        unsigned at = value_key(neg_inf());
#pragma unroll 1
        for (int bits = 26; bits >= -4; bits -= 6) {
            const unsigned unit = 1u << max(0, bits), key = at + min((unsigned)(tid & 63) * unit, value_key(INFINITY) - at);
            const unsigned long long reach = __ballot(step_of(key_value(key), scale) >= step);
            const int before = reach ? max(0, __ffsll((long long)reach) - 2) : 63;      // the last that does not, or the first
            at += min((unsigned)before * unit, value_key(INFINITY) - at);
        }
        return key_value(step_of(key_value(at), scale) >= step ? at : at + 1u);
    };
    const float upper = least_of(first - (float)lo + 1.f), lower = least_of(first - (float)hi);       // from upper on above, from lower on undecided
    sample_sweep(row, a.V, [&](int v, const float(&z)[N]) {
        unsigned over = 0u, from = 0u;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            over += z[e] >= upper;
            from += z[e] >= lower;
        }
        kept += over;
        if (from == over) return;
        unsigned slot = lds_add(&L.n_list, from - over);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (z[e] >= lower && !(z[e] >= upper)) {
                const unsigned key = value_key(z[e]);
                if (slot < SAMPLE_LIST) {
                    L.key[slot] = key;
                    L.index[slot] = (unsigned)(v * N + e);
                }
                ++slot;
                least = min(least, key);
                most = max(most, key);
            }
    });
    atomicMin(&L.low, least);
    atomicMax(&L.high, most);
    __syncthreads();
    unsigned low = L.low;
    const unsigned high = L.high, len = L.n_list;
    unsigned long long more;
    const auto mass_of = [&](float z) { return w.units(z); };
    const bool by_mass = s.top_p < 1.0 && len && target > above;
    if (len <= SAMPLE_LIST) {
        const auto each = [&](auto f) {
            for (unsigned i = tid; i < len; i += SAMPLE_WG) f(L.key[i], key_value(L.key[i]));
        };
        if (by_mass) low = select_key<KEY_LOW<DT>>(each, low, high, target - above, L, mass_of, &more);
        const Keep keep = {len ? low : value_key(neg_inf()) + 1u, s.log2_min_p, w};
        __syncthreads();
        for (unsigned i = tid; i < len; i += SAMPLE_WG) {
            const float z = key_value(L.key[i]);
            if (!keep(z)) continue;
            ++kept;
            atomicAdd(&L.tile_mass[L.index[i] / SAMPLE_TILE], w.units(z));
        }
        kept = (unsigned)sum_of_all((unsigned long long)kept, L);
        draw_by_tiles<DT>(a, n, row, s, keep, (int)kept, L);
        return true;
    }
    // more than the list holds: from the row again
    const auto each_index = [&](auto f) {
        sample_sweep(row, a.V, [&](int v, const float(&z)[N]) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (z[e] >= lower && !(z[e] >= upper)) f(v * N + e, z[e]);
            }
        });
    };
    const auto each = [&](auto f) { each_index([&](int, float z) { f(value_key(z), z); }); };
    if (by_mass) low = select_key<KEY_LOW<DT>>(each, low, high, target - above, L, mass_of, &more);
    const Keep keep = {low, s.log2_min_p, w};
    __syncthreads();
    each_index([&](int i, float z) {
        if (!keep(z)) return;
        ++kept;
        atomicAdd(&L.tile_mass[i / SAMPLE_TILE], w.units(z));
    });
    kept = (unsigned)sum_of_all((unsigned long long)kept, L);
    draw_by_tiles<DT>(a, n, row, s, keep, (int)kept, L);
    return true;
}

template <typename DT>
__global__ __launch_bounds__(TILES_WG, VecOf<DT>::N == 8 ? 8 : 4) void k_sample_tiles(SampleArgs a)
{
    constexpr int N = VecOf<DT>::N, U = SAMPLE_CHUNK / N, PER = SAMPLE_STEPS / 64;
    __shared__ unsigned long long all_steps[TILES_WAVES][SAMPLE_STEPS];
    const int n = blockIdx.x / (unsigned)a.groups, group = blockIdx.x - n * a.groups;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), V = a.V;
    const DT *row = static_cast<const DT *>(a.logits) + n * a.row_stride;
    const int tile = group * TILES_WAVES + wave, v0 = tile * (U * 64) + lane;
    if (tile >= a.tiles) return;
    TileData *const mine = reinterpret_cast<TileData *>(a.tile_data) + (size_t)n * a.tiles + tile;
    typename RawOf<DT>::type raw[U];
    if ((tile + 1) * SAMPLE_TILE <= V) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = *(reinterpret_cast<const typename RawOf<DT>::type *>(row) + v0 + u * 64);
    } else {
        load_raw_tail<DT, U, 64>(row, v0, V, raw);
    }
    const Settings s = settings_of(a, n);
    if (s.mode == SAMPLE_BAD) return;
    float top = neg_inf();
    int count = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[N];
        unpack<DT>(raw[u], z);
#pragma unroll
        for (int e = 0; e < N; ++e) top = vmax(top, vmax(z[e], z[e]));         // (a signalling NaN is quiet then, and passed over)
    }
    if (s.mode == SAMPLE_TOPK) mine->chunk_top[lane] = top;
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
    for (int i = 0; i < PER; ++i) steps[lane + 64 * i] = 0ull;
    __builtin_amdgcn_wave_barrier();
    const float scale = (float)(s.c * (double)STEPS_PER_OCTAVE), first = step_of(top, scale);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float z[N];
        asm volatile("" : "+v"(raw[u]));
        unpack<DT>(raw[u], z);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            atomicAdd(&steps[(int)fminf(first - step_of(z[e], scale), (float)(SAMPLE_STEPS - 1))], units_of(w.of_tile(z[e]), w.unit));
            if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    }
    __builtin_amdgcn_wave_barrier();
    unsigned long long h[PER], sum = 0ull;
#pragma unroll
    for (int i = 0; i < PER; ++i) sum += h[i] = steps[lane * PER + i];
    unsigned long long run = wave_inclusive_sum_u64(sum) - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) mine->down_to[lane * PER + i] = run += h[i];
}

template <typename DT>
__global__ __launch_bounds__(SAMPLE_WG) void k_sample_rows(SampleArgs a)
{
    __shared__ SampleLds L;
    const int n = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const DT *row = static_cast<const DT *>(a.logits) + n * a.row_stride;
    const TileData *const tiles = reinterpret_cast<const TileData *>(a.tile_data) + (size_t)n * a.tiles;
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
    if (top < INFINITY) {
        if (s.mode == SAMPLE_PLAIN) {
            for (int t = tid; t < a.tiles; t += SAMPLE_WG)
                L.tile_mass[t] = L.tile_top[t] > neg_inf() ? (unsigned long long)rint(ldexp(tiles[t].mass * w(L.tile_top[t]), a.unit_bits)) : 0ull;
            count = sum_of_all(count, L);
            draw_by_tiles<DT>(a, n, row, s, {value_key(neg_inf()) + 1u, -INFINITY, w}, (int)count, L);
            return;
        }
        if (s.mode == SAMPLE_TOPK) {
            unsigned lowest;
            if (list_top_k<DT>(a, row, tiles, s.top_k, top, &lowest, L)) {
                row_by_list<DT>(a, n, row, s, w, lowest, L);
                return;
            }
        }
        if (s.mode == SAMPLE_STEPPED && row_by_steps<DT>(a, n, row, s, w, tiles, L)) return;
        __syncthreads();
    }
    row_by_sweeps<DT>(a, n, row, s, w, L);
}

}  // namespace svip
