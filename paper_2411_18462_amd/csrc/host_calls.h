// What the entry points of the head's calls share: limits, checks of arguments, launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/svip.h"

namespace svip {

static inline bool dtype_ok(int d) { return d == SVIP_F32 || d == SVIP_BF16 || d == SVIP_F16; }
static inline int size_of(int d) { return d == SVIP_F32 ? 4 : 2; }
static inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
static inline int up(int n, int to) { return (n + to - 1) / to * to; }
static inline int ceil_div(long long n, long long d) { return (int)((n + d - 1) / d); }

constexpr int HEAD_MAX_ROWS = 1 << 20;                 // of hidden states
constexpr int HEAD_MAX_VOCAB = 1 << 22;
constexpr int HEAD_MAX_WIDTH = 1 << 17;                // hidden channels
constexpr long long HEAD_MAX_STRIDE = 1 << 23;         // elements: 256 rows of a tile lie within 32 bits of bytes

constexpr long long MOST_THREADS = 0xffffffffLL;       // of a launch

template <typename A>
static inline bool launch(void (*kernel)(A), long long grid, unsigned block, hipStream_t st, const A &args)
{
    if (grid <= 0 || grid * block > MOST_THREADS) return false;
    A copy = args;
    void *argv[] = {&copy};
    return hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)grid), dim3(block), argv, 0, st) == hipSuccess;
}

template <typename F>
static inline bool by_dtype(int d, F f)
{
    if (d == SVIP_F32) return f(std::integral_constant<int, SVIP_F32>{});
    if (d == SVIP_BF16) return f(std::integral_constant<int, SVIP_BF16>{});
    return f(std::integral_constant<int, SVIP_F16>{});
}

static inline svip_status check_sizes(int N, int V, int D)
{
    return N <= 0 || N > HEAD_MAX_ROWS || V <= 0 || V > HEAD_MAX_VOCAB || D <= 0 || D > HEAD_MAX_WIDTH ? SVIP_ERR_SHAPE : SVIP_OK;
}
static inline svip_status check_workspace(const void *ws, size_t bytes, size_t need)
{
    return !ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || bytes < need ? SVIP_ERR_WORKSPACE : SVIP_OK;
}

size_t mx_logits_workspace(int N, int V, int K);       // of svip_head_logits_mx

}  // namespace svip
