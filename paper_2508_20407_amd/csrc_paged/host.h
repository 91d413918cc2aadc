// Host side shared by the paged-cache entry points: launches, device check, argument checks.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "common.h"
#include "tlinpaged.h"

namespace tlin {
namespace {

// One kernel launch, reporting the status of this launch only.  Every kernel takes one argument structure by value.
template <typename Args>
tlin_status launch_kernel(const void *kernel, dim3 grid, dim3 block, size_t lds_bytes, hipStream_t st, const Args &a)
{
    void *argv[] = {const_cast<Args *>(&a)};
    return hipLaunchKernel(kernel, grid, block, argv, lds_bytes, st) == hipSuccess ? TLIN_OK : TLIN_ERR_HIP;
}

// gfx950 with 256 compute units, once per device, after argument checks and before the first launch on it.
tlin_status check_device()
{
    static std::atomic<uint64_t> good{0}, bad{0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return TLIN_ERR_HIP;
    if (dev < 0 || dev >= 64) return TLIN_ERR_UNSUPPORTED;
    const uint64_t bit = (uint64_t)1 << dev;
    if (good.load(std::memory_order_acquire) & bit) return TLIN_OK;
    if (bad.load(std::memory_order_acquire) & bit) return TLIN_ERR_UNSUPPORTED;
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return TLIN_ERR_HIP;
    const bool ok = strncmp(prop.gcnArchName, "gfx950", 6) == 0 && prop.multiProcessorCount == kNumCU;
    (ok ? good : bad).fetch_or(bit, std::memory_order_release);
    return ok ? TLIN_OK : TLIN_ERR_UNSUPPORTED;
}

// Raises a kernel's LDS limit once per device.
tlin_status allow_lds(const void *kernel, int bytes, std::atomic<uint64_t> &done)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return TLIN_ERR_HIP;
    const uint64_t bit = (uint64_t)1 << dev;
    if (done.load(std::memory_order_acquire) & bit) return TLIN_OK;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return TLIN_ERR_HIP;
    done.fetch_or(bit, std::memory_order_release);
    return TLIN_OK;
}

constexpr int kMaxRows = 1 << 30;
constexpr int64_t kMaxBytes = (int64_t)1 << 47;      // of a stride: what device addresses reach (and products of it and a type's size fit)

inline bool is_type(int32_t t) { return t == TLIN_F32 || t == TLIN_BF16; }
inline int bytes_of(int32_t t) { return t == TLIN_F32 ? 4 : 2; }
inline bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }
inline int row_elements(int D, int eb) { const int per16 = 16 / eb; return (D + per16 - 1) / per16 * per16; }
inline bool good_page_rows(int32_t r) { return r >= 16 && r <= 65536 && (r & (r - 1)) == 0; }
inline int log2_of(int32_t r) { return __builtin_ctz((unsigned)r); }

// Strides of a tensor of n axes before D: all 0 = dense (which needs rows of whole 16-byte pieces), else multiples
// of 16 bytes and below kMaxBytes, rows owning their pieces and (32-bit offsets inside a tile) below 32 MiB apart.
template <int N>
tlin_status check_strides(const int64_t (&s)[N], int D, int eb)
{
    bool zero = true;
    for (int i = 0; i < N; ++i) zero = zero && s[i] == 0;
    if (zero) return D % (16 / eb) ? TLIN_ERR_INVALID_ARG : TLIN_OK;
    for (int i = 0; i < N; ++i)
        if (s[i] < 0 || s[i] % (16 / eb) || s[i] >= kMaxBytes / eb) return TLIN_ERR_INVALID_ARG;
    if (s[N - 1] < row_elements(D, eb) || s[N - 1] * eb >= (int64_t)1 << 25) return TLIN_ERR_INVALID_ARG;
    return TLIN_OK;
}
// out: the strides, with those of a dense tensor in the place of zeros; sizes[i] is the number of entries along axis i + 1
template <int N>
void resolve(const int64_t (&s)[N], const int64_t (&sizes)[N - 1], int D, int64_t (&out)[N])
{
    bool zero = true;
    for (int i = 0; i < N; ++i) zero = zero && s[i] == 0;
    for (int i = 0; i < N; ++i) out[i] = s[i];
    if (!zero) return;
    out[N - 1] = D;
    for (int i = N - 2; i >= 0; --i) out[i] = out[i + 1] * sizes[i];
}

// Whether entries that are written lie on one another: sizes[0] entries along the first axis and so on, the rows' axis left
// out (check_strides).
template <int N>
bool written_twice(const int64_t (&s)[N], const int64_t (&sizes)[N - 1])
{
    for (int i = 0; i < N - 1; ++i)
        if (s[i] == 0 && sizes[i] > 1) return true;
    return false;
}

inline bool good_dim(int32_t D) { return D >= 8 && D <= 128 && D % 4 == 0; }

}  // namespace
}  // namespace tlin
