// Kernels of svip_sample: a token for each row of logits, every row with its own temperature, top-k, top-p and min-p (not in the paper).
//
// Weights are w = exp2((z - m) c) with c = log2(e) / T and m the row's largest logit, in 64 bits: which token a uniform falls on, and which
// value the nucleus ends at, are borders between sums of up to V weights, and a rounding of 2^-24 in each weight moves such a border by more than
// the narrowest cells are wide.  The fp64 pipe takes a fused multiply-add in four cycles, as the fp32 pipe does, so a weight costs about
// 17 instructions against 7.  Sums are integers in units of 2^-S of the largest weight (S = 62 - ceil(log2 V)), so that no
// order of additions changes a result and atomics may be used.
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
};

// 2^x for x <= 0, 0 below 2^-1000.  2^n times the series of 2^f = exp(f ln 2), |f| <= 1/2: what it leaves out is below 2.3e-13 of the result.
__device__ __forceinline__ double exp2_64(double x)
{
    const double t = x + 6755399441055744.0;           // 1.5 * 2^52: x rounded to a whole number in the low bits
    const double f = x - (t - 6755399441055744.0);
    double r = 7.0549116208011234e-9;
    r = fma(r, f, 1.0178086009239699e-7);
    r = fma(r, f, 1.3215486790144309e-6);
    r = fma(r, f, 1.5252733804059841e-5);
    r = fma(r, f, 1.5403530393381610e-4);
    r = fma(r, f, 1.3333558146428443e-3);
    r = fma(r, f, 9.6181291076284772e-3);
    r = fma(r, f, 5.5504108664821580e-2);
    r = fma(r, f, 2.4022650695910072e-1);
    r = fma(r, f, 6.9314718055994531e-1);
    r = fma(r, f, 1.0);
    const double w = __hiloint2double(__double2hiint(r) + (__double2loint(t) << 20), __double2loint(r));
    return x < -1000.0 ? 0.0 : w;
}

struct SampleWeights {
    double m, c;               // the row's largest logit; log2(e) / T
    double unit;               // 2^(52 - S): the units of a double of that size are 2^-S
    __device__ __forceinline__ double log2_of(float z) const { return ((double)z - m) * c; }
    __device__ __forceinline__ double operator()(float z) const { return (double)z == m ? 1.0 : exp2_64(log2_of(z)); }       // (m may be +inf)
    __device__ __forceinline__ unsigned long long units(float z) const
    {
        return (unsigned long long)__double_as_longlong((*this)(z) + unit) - (unsigned long long)__double_as_longlong(unit);
    }
};

// What a row asks for.
struct Settings {
    double T;
    int top_k;                 // 0: off
    double top_p;              // 1: off
    double log2_min_p;         // -inf: off
    double u;
    bool bad;
};
__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int n)
{
    Settings s;
    const float T = a.temperature ? a.temperature[n] : 1.f, p = a.top_p ? a.top_p[n] : 1.f, m = a.min_p ? a.min_p[n] : 0.f, u = a.u[n];
    const int k = a.top_k ? a.top_k[n] : 0;
    s.bad = !(T >= 0.f && T <= FLT_MAX) || !(p > 0.f) || !(m >= 0.f && m <= 1.f) || !(u >= 0.f && u < 1.f) || k < 0;
    s.T = T;
    s.top_k = k < a.V ? k : 0;
    s.top_p = p < 1.f ? (double)p : 1.0;
    s.log2_min_p = m > 0.f ? log2((double)m) : -INFINITY;
    s.u = u;
    return s;
}

constexpr int SAMPLE_WG = 1024, SAMPLE_WAVES = SAMPLE_WG / 64;
constexpr int SAMPLE_BINS = 2048;

struct SampleLds {
    unsigned long long hist[SAMPLE_BINS];
    unsigned long long wave_tot[SAMPLE_WAVES];
    unsigned long long found_before, total;
    int found;
    unsigned long long best[SAMPLE_WAVES];
    int count;
};

// NaN counts as -inf.
__device__ __forceinline__ float sample_logit(float z) { return z == z ? z : neg_inf(); }

// f(vector index, its N values) for the vectors of the row, by all threads in turn; the values behind the row's end and NaN are -inf.
template <typename DT, typename F>
__device__ __forceinline__ void sample_sweep(const DT *row, int V, F f)
{
    constexpr int N = VecOf<DT>::N;
    const int nvec = (V + N - 1) / N;
    for (int v = threadIdx.x; v < nvec; v += SAMPLE_WG) {
        const auto raw = warp_load<DT>(row, v, V);
        float z[N];
        unpack<DT>(raw, z);
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = sample_logit(z[e]);
        f(v, z);
    }
}

// Of hist[0 .. SAMPLE_BINS), in ascending order if UP and descending if not, the first bin at which the running sum reaches `target` (>= 1), and the sum
// before it; -1 if the total falls short.  All threads; L.hist is complete behind a barrier; ends behind one.
template <bool UP>
__device__ __forceinline__ int find_bin(SampleLds &L, unsigned long long target, unsigned long long *before)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int i0 = UP ? 2 * tid : SAMPLE_BINS - 1 - 2 * tid, i1 = UP ? i0 + 1 : i0 - 1;
    const unsigned long long h0 = L.hist[i0], h1 = L.hist[i1], incl = wave_inclusive_sum_u64(h0 + h1);
    if (lane == 63) L.wave_tot[wave] = incl;
    if (tid == 0) L.found = -1;
    __syncthreads();
    unsigned long long ahead = 0ull;
    for (int w = 0; w < wave; ++w) ahead += L.wave_tot[w];
    const unsigned long long b = ahead + incl - h0 - h1;
    if (b < target && b + h0 + h1 >= target) {
        const bool first = b + h0 >= target;
        L.found = first ? i0 : i1;
        L.found_before = first ? b : b + h0;
    }
    if (tid == SAMPLE_WG - 1) L.total = ahead + incl;
    __syncthreads();
    *before = L.found_before;
    return L.found;
}
__device__ __forceinline__ void clear_hist(SampleLds &L)
{
    __syncthreads();
    L.hist[2 * threadIdx.x] = L.hist[2 * threadIdx.x + 1] = 0ull;
    __syncthreads();
}

// The largest key v with measure(keys >= v) >= target, over keys >= low; measure(key, value).  With `part` the target is that share of the total.
// Three digits, most significant first.
template <typename DT, typename M>
__device__ __forceinline__ unsigned select_key(const DT *row, int V, unsigned low, unsigned long long target, double part, SampleLds &L, M measure)
{
    unsigned prefix = 0u, mask = 0u;
    constexpr int SHIFT[3] = {21, 10, 0};
#pragma unroll 1
    for (int d = 0; d < 3; ++d) {
        const int shift = SHIFT[d], width = d == 2 ? 10 : 11;
        clear_hist(L);
        sample_sweep(row, V, [&](int, const float(&z)[VecOf<DT>::N]) {
#pragma unroll
            for (int e = 0; e < VecOf<DT>::N; ++e) {
                const unsigned key = value_key(z[e]);
                if (key >= low && (key & mask) == prefix && z[e] > neg_inf()) atomicAdd(&L.hist[key >> shift & ((1u << width) - 1u)], measure(z[e]));
            }
        });
        __syncthreads();
        unsigned long long before;
        if (d == 0 && part > 0.0) {
            find_bin<false>(L, ~0ull, &before);
            target = (unsigned long long)ceil(part * (double)L.total);
            if (target < 1ull) target = 1ull;
            __syncthreads();
        }
        const int bin = find_bin<false>(L, target, &before);
        if (bin < 0) return low;
        target -= before;
        prefix |= (unsigned)bin << shift;
        mask |= ((1u << width) - 1u) << shift;
    }
    return prefix;
}

__device__ __forceinline__ void sample_answer(const SampleArgs &a, int n, int token, float prob, int kept)
{
    a.token[n] = token;
    if (a.prob) a.prob[n] = prob;
    if (a.kept) a.kept[n] = kept;
}

// A workgroup each row, which it goes through as often as its settings ask for.
template <typename DT>
__global__ __launch_bounds__(SAMPLE_WG) void k_sample_rows(SampleArgs a)
{
    constexpr int N = VecOf<DT>::N;
    __shared__ SampleLds L;
    const int n = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
    const DT *row = static_cast<const DT *>(a.logits) + n * a.row_stride;
    const Settings s = settings_of(a, n);
    if (s.bad) {
        if (tid == 0) {
            atomicOr(a.flags, (unsigned)SVIP_FLAG_BAD_SETTING);
            sample_answer(a, n, -1, 0.f, 0);
        }
        return;
    }
    // the largest logit and the first token that has it
    unsigned long long best = 0ull;
    sample_sweep(row, V, [&](int v, const float(&z)[N]) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned long long k = (unsigned long long)value_key(z[e]) << 32 | (unsigned)~(v * N + e);
            best = k > best ? k : best;
        }
    });
    best = wave_reduce(best, OpMax{});
    if (lane == 0) L.best[wave] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < SAMPLE_WAVES; ++w) best = L.best[w] > best ? L.best[w] : best;
    const float top = key_value((unsigned)(best >> 32));
    if (!(top > neg_inf()) || s.T == 0.0) {
        if (tid == 0) sample_answer(a, n, top > neg_inf() ? (int)~(unsigned)best : -1, top > neg_inf() ? 1.f : 0.f, top > neg_inf() ? 1 : 0);
        return;
    }
    const SampleWeights w = {(double)top, 1.4426950408889634 / s.T, __longlong_as_double((long long)(1023 + 52 - a.unit_bits) << 52)};
    unsigned low = value_key(neg_inf()) + 1u;
    if (s.top_k) low = max(low, select_key(row, V, low, (unsigned long long)s.top_k, 0.0, L, [](float) { return 1ull; }));
    if (s.top_p < 1.0) low = select_key(row, V, low, 0ull, s.top_p, L, [&](float z) { return w.units(z); });
    const auto keep = [&](float z) { return value_key(z) >= low && (z == top || w.log2_of(z) >= s.log2_min_p); };
    // masses of runs of vectors, in index order
    const int nvec = (V + N - 1) / N, chunks = (nvec + 63) / 64, per = (chunks + SAMPLE_BINS - 1) / SAMPLE_BINS;
    clear_hist(L);
    if (tid == 0) L.count = 0;
    __syncthreads();
    int kept = 0;
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
    kept = wave_reduce(kept, OpSum{});
    if (lane == 0) atomicAdd(&L.count, kept);
    __syncthreads();
    unsigned long long before;
    find_bin<true>(L, ~0ull, &before);
    const unsigned long long total = L.total, at = (unsigned long long)(s.u * (double)total);
    __syncthreads();
    const int bin = find_bin<true>(L, at + 1ull, &before);
    if (wave != 0) return;
    unsigned long long left = at - before;
    for (int c = bin * per; c < min(chunks, (bin + 1) * per); ++c) {
        const int v = c * 64 + lane;
        float z[N];
        unsigned long long mass = 0ull;
        if (v < nvec) {
            unpack<DT>(warp_load<DT>(row, v, V), z);
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (keep(sample_logit(z[e]))) mass += w.units(z[e]);
        }
        const unsigned long long incl = wave_inclusive_sum_u64(mass), hit = __ballot(incl > left);
        if (!hit) {
            left -= read_lane(incl, 63);
            continue;
        }
        if (lane == __ffsll((long long)hit) - 1) {
            unsigned long long run = incl - mass;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const unsigned long long units = keep(sample_logit(z[e])) ? w.units(z[e]) : 0ull;
                if (run <= left && run + units > left)
                    sample_answer(a, n, v * N + e, (float)(w(z[e]) / ldexp((double)total, -a.unit_bits)), L.count);
                run += units;
            }
        }
        break;
    }
}

}  // namespace svip
