// What the C entries share on the host: sizes, checks of arguments, launches.
#pragma once
#include "../../include/lshbeam.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "beam_select.h"

namespace lshbeam {
namespace {

constexpr int64_t kMaxRows = 1 << 20;
constexpr int64_t kMaxGrid = (1 << 24) - 1;   // workgroups of 256 threads: fewer than 2^32 threads

size_t round_up(size_t n) { return (n + 255) / 256 * 256; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

lsh_status launched() { return hipGetLastError() == hipSuccess ? LSH_OK : LSH_ERR_HIP; }

template <typename F> void for_type(int32_t dtype, F f) {   // f(std::integral_constant<int, kType...>)
    if (dtype == LSH_F32) f(std::integral_constant<int, kTypeF32>());
    else if (dtype == LSH_BF16) f(std::integral_constant<int, kTypeBf16>());
    else f(std::integral_constant<int, kTypeF16>());
}
bool type_ok(int32_t dtype) { return dtype == LSH_F32 || dtype == LSH_BF16 || dtype == LSH_F16; }
size_t type_bytes(int32_t dtype) { return dtype == LSH_F32 ? 4 : 2; }
bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool pitch_ok(const lsh_rows* x, int32_t head_dim) {
    return x && type_ok(x->dtype) && x->row >= 0 && x->token >= 0 && x->head >= 0 && head_dim > 0;
}

// Do two of the heads of x, D values each, lie on each other?  There is a difference of two rows, tokens and heads, not all 0, with
// |dr row + dt token + dh head| < D.  Pitches that each reach over what lies within them (as views have, in any order) are seen at once; else the two
// dimensions with the fewest members are gone through, and the third's difference follows (at most some 2^18 turns: R T n_heads <= 2^26).
bool heads_overlap(const lsh_rows* x, int64_t R, int64_t T, int64_t n_heads, int32_t D) {
    struct Dim { int64_t n; __int128 pitch; } dim[3] = {{R, x->row}, {T, x->token}, {n_heads, x->head}};
    std::sort(dim, dim + 3, [](const Dim& a, const Dim& b) { return a.pitch < b.pitch; });
    __int128 reach = D;
    bool nested = true;
    for (const Dim& d : dim) {
        if (d.n > 1 && d.pitch < reach) nested = false;
        reach += (d.n - 1) * d.pitch;
    }
    if (nested) return false;
    std::sort(dim, dim + 3, [](const Dim& a, const Dim& b) { return a.n < b.n; });
    for (int64_t i = 0; i < dim[0].n; ++i)
        for (int64_t j = i > 0 ? 1 - dim[1].n : 0; j < dim[1].n; ++j) {
            const __int128 s = i * dim[0].pitch + j * dim[1].pitch, p = dim[2].pitch;
            const __int128 below = p == 0 ? 0 : s > 0 ? -((s + p - 1) / p) : -s / p;   // the largest k with s + k p <= 0
            for (__int128 k = below; k <= below + 1; ++k) {
                const __int128 off = s + k * p;
                if (k > -dim[2].n && k < dim[2].n && off < D && off > -D && (i != 0 || j != 0 || k != 0)) return true;
            }
        }
    return false;
}

// A launch with more than 64 KB of LDS; the limit is raised once per kernel and device.
template <auto KERNEL, int LDS, typename ARGS> bool launch_lds(unsigned grid, unsigned threads, hipStream_t st, const ARGS& a) {
    if constexpr (LDS > 64 * 1024) {
        static std::atomic<uint64_t> done{0};   // a bit per device
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess) return false;
        const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
        if (!(bit && (done.load(std::memory_order_acquire) & bit))) {
            if (hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, LDS) != hipSuccess) return false;
            done.fetch_or(bit, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(KERNEL, dim3(grid), dim3(threads), LDS, st, a);
    return true;
}
// The same where the LDS is known at launch only: the limit is raised to what there is.
template <auto KERNEL, typename ARGS> bool launch_room(dim3 grid, unsigned threads, size_t lds, hipStream_t st, const ARGS& a) {
    if (lds > 64 * 1024) {
        static std::atomic<uint64_t> done{0};
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess) return false;
        const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
        if (!(bit && (done.load(std::memory_order_acquire) & bit))) {
            if (hipFuncSetAttribute((const void*)KERNEL, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxDynLds) != hipSuccess) return false;
            done.fetch_or(bit, std::memory_order_release);
        }
    }
    hipLaunchKernelGGL(KERNEL, grid, dim3(threads), lds, st, a);
    return true;
}

}  // namespace
}  // namespace lshbeam
