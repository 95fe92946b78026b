// What the kernels of the head's products share beside the product itself (head_tile.h): storage types, which tile a workgroup makes, and
// how a tile of 16-bit results reaches memory.
#pragma once
#include "head_tile.h"

namespace svip {

// ---- values in and out ---------------------------------------------------------------------------------------------------------------

template <int DT> struct Stored;       // by svip_dtype
template <> struct Stored<0> {
    using type = float;
    static constexpr int VEC = 4;
    __device__ static __forceinline__ void put4(float *p, f32x4 v) { *reinterpret_cast<f32x4 *>(p) = v; }
};
template <> struct Stored<1> {
    using type = __bf16;
    static constexpr int VEC = 8;
    __device__ static __forceinline__ void put4(__bf16 *p, f32x4 v)
    {
        typedef __bf16 v4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<v4 *>(p) = __builtin_convertvector(v, v4);
    }
};
template <> struct Stored<2> {
    using type = _Float16;
    static constexpr int VEC = 8;
    __device__ static __forceinline__ void put4(_Float16 *p, f32x4 v)
    {
        typedef _Float16 v4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<v4 *>(p) = __builtin_convertvector(v, v4);
    }
};
// v[0..count) at p, which is aligned for four
template <int DT>
__device__ __forceinline__ void put_up_to_4(typename Stored<DT>::type *p, f32x4 v, int count)
{
    if (count >= 4) {
        Stored<DT>::put4(p, v);
    } else {
        for (int e = 0; e < count; ++e) p[e] = (typename Stored<DT>::type)v[e];
    }
}

__device__ __forceinline__ unsigned finite_magnitude(float x)
{
    const unsigned a = __float_as_uint(x) & 0x7fffffffu;
    return a < 0x7f800000u ? a : 0u;
}

// ---- which tile a workgroup makes --------------------------------------------------------------------------------------------------------

// Workgroups b, b + 8, ... run on one XCD: it gets a contiguous range of tiles, in groups of GROUP columns of tiles (n) by all of m, n
// first, so that the 32 tiles an XCD works on at a time are about 8 x 4 and share their operands in its L2.
struct Tiles {
    int m, n;
};
__device__ __forceinline__ void tile_of(unsigned block, Tiles t, int group, int &tm, int &tn)
{
    const unsigned total = (unsigned)t.m * (unsigned)t.n, xcd = block & 7u, per = total >> 3, more = total & 7u;
    const unsigned i = xcd * per + (xcd < more ? xcd : more) + (block >> 3);
    const unsigned in_group = (unsigned)group * (unsigned)t.m, g = i / in_group, left = (unsigned)t.n - g * (unsigned)group;
    const unsigned width = left < (unsigned)group ? left : (unsigned)group, j = i - g * in_group;
    tm = (int)(j / width);
    tn = (int)(g * (unsigned)group + j % width);
}

// Stores a tile of 16-bit results, `rows` rows (n) of `cols` values (m) of it, at `out`.  A lane's four neighbours in m are 8 bytes, which stored as they
// are would reach memory 32 bytes to a row at a time; so the tile goes through LDS, and 16 bytes a lane fill whole lines.  Chunk c of
// row n lies at chunk c ^ (n % 16): neither the 16 rows of a fragment nor the chunks of a row meet a bank twice.
// value(i, j): results of fragment (i, j); called by all threads of the workgroup, when no copy into `smem` is under way.
template <typename S, typename X, typename Value>
__device__ __forceinline__ void store_rows(char *smem, int rows, int cols, X *out, long long stride, Value value)
{
    typedef X x4 __attribute__((ext_vector_type(4)));
    typedef X x8 __attribute__((ext_vector_type(8)));
    constexpr int CHUNKS = S::BM / 8, MASK = (CHUNKS < 16 ? CHUNKS : 16) - 1, ROUNDS = S::BN * CHUNKS / S::THREADS;
    static_assert(S::BN * S::BM * 2 <= S::LDS_BYTES && S::BN * CHUNKS % S::THREADS == 0, "");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = (wave % S::WAVES_M) * S::WM, wn = (wave / S::WAVES_M) * S::WN, g = lane >> 4;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < S::FN; ++j) {
        const int n = wn + 16 * j + (lane & 15);
#pragma unroll
        for (int i = 0; i < S::FM; ++i) {
            const int chunk = (wm / 8 + 2 * i + (g >> 1)) ^ (n & MASK);
            *reinterpret_cast<x4 *>(smem + n * (S::BM * 2) + chunk * 16 + (g & 1) * 8) = __builtin_convertvector(value(i, j), x4);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int c = k * S::THREADS + (int)threadIdx.x, n = c / CHUNKS, m = c % CHUNKS * 8;
        if (n >= rows || m >= cols) continue;
        const x8 v = *reinterpret_cast<const x8 *>(smem + n * (S::BM * 2) + ((c % CHUNKS) ^ (n & MASK)) * 16);
        X *p = out + n * stride + m;
        if (m + 8 <= cols) {
            *reinterpret_cast<x8 *>(p) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (m + e < cols) p[e] = v[e];
        }
    }
}

}  // namespace svip
