// Launchers that live in translation units of their own (compiled side by side), and what they share.
#pragma once

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>

#include "../../include/bnn.h"
#include "bnn_device.hpp"

#define BNN_EXPORT extern "C" __attribute__((visibility("default")))

namespace bnn {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline bool word_bits_ok(int wb) { return wb == 32 || wb == 64; }
inline int64_t words_per_row(int64_t K, int wb) { return (K + wb - 1) / wb; }
// Row length in 32-bit words (a 64-bit word is two little-endian 32-bit words).
inline int64_t row_w32(int64_t K, int wb) { return words_per_row(K, wb) * (wb / 32); }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    return na && nb && a0 < b0 + nb && b0 < a0 + na;
}
inline int launch_status() { return hipGetLastError() == hipSuccess ? BNN_OK : BNN_EDEVICE; }

constexpr int64_t kMaxDim = (int64_t)1 << 30;
constexpr int64_t kMaxN = (int64_t)1 << 22;   // outputs of a layer: the second grid dimension (65535) counts tiles of 128 or 256 of them

// Dynamic LDS above 64 KiB has to be allowed once per kernel and device.  `bytes` is the most the kernel ever asks for and
// the same in every call, so threads that get here together all set the same value.  false: refused.
template <class Kernel>
bool allow_lds(Kernel kernel, unsigned bytes, std::atomic<uint64_t>& allowed) {
    int dev = 0;
    (void)hipGetDevice(&dev);
    const uint64_t bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;   // (devices past 64: asked for every time)
    if (allowed.load(std::memory_order_relaxed) & bit) return true;
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    allowed.fetch_or(bit);
    return true;
}

// A launch of this grid clears.
inline Clear cleared_by(Clear c, dim3 grid) {
    c.gx = (int)grid.x;
    c.blocks = (int)(grid.x * grid.y);
    return c;
}

// Ascending-k fp32 sums on the matrix cores (f32_chain_launch.hpp); arguments already checked.
struct ChainArgs {
    const float* X;
    const void* W;   // packed bits, or fp32 with real weights
    const float *scale, *bias;
    int M, K, N, w32;
    void* Y;
    int yw32;
    hipStream_t st;
    Clear clear{};   // Sign layers: memory that the launch sets to 0
};
void launch_chain_bits(const ChainArgs& a, int act);   // W packed bits
void launch_chain_real(const ChainArgs& a, int act);   // W fp32

// log-Softmax of every row of Z [M][N], in place (bnn_api.hip).
void launch_log_softmax(float* Z, int M, int N, hipStream_t st);

}  // namespace bnn
