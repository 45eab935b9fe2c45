// Product of two matrices in microscaled 4-bit floating point on V_MFMA_SCALE_F32_32X32X64_F8F6F4: Y[m][n] = f(sum_k x[m][k] w[n][k] +
// bias[n]), sums in fp32.
#pragma once

#include "bnn_device.hpp"
#include "mx4_kernels.hpp"

namespace bnn {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef int v8i __attribute__((ext_vector_type(8)));

template <int ACT>
__device__ __forceinline__ float mx4_act(float h) {
    if constexpr (ACT == ACT_HARDTANH) return hardtanh(h);
    else if constexpr (ACT == ACT_SIGMOID) return sigmoid(h);
    else return h;
}

// Operand layout: lane (r = lane % 32, g = lane / 32) holds the 32 elements 32 g ... of row r, and their scale byte.
// A workgroup is 2 x 2 waves of 64 x 64 outputs.  Rows past M and N repeat the last one and are not stored.
template <int ACT>
__global__ __launch_bounds__(256) void mx4_gemm_simple_kernel(const void* __restrict__ Xq, const void* __restrict__ Wq, const float* __restrict__ bias,
                                                              int M, int K, int N, int chunks, void* __restrict__ Y, int yw32) {
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = lane_id(), r = lane & 31, g = lane >> 5;
    const int m_base = (int)blockIdx.x * 128 + (wave >> 1) * 64, n_base = (int)blockIdx.y * 128 + (wave & 1) * 64;
    if (m_base >= M || n_base >= N) return;
    const unsigned char *xc = static_cast<const unsigned char*>(Xq), *wc = static_cast<const unsigned char*>(Wq);
    const uint32_t *xs = mx4_scales(Xq, M, K), *ws = mx4_scales(Wq, N, K);
    v16f acc[2][2];
    size_t mrow[2], nrow[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        mrow[i] = (size_t)min(m_base + 32 * i + r, M - 1);
        nrow[i] = (size_t)min(n_base + 32 * i + r, N - 1);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
    }
    for (int c = 0; c < chunks; ++c) {
        v8i a[2][2], b[2][2];
        int sa[2], sb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int4 p = *reinterpret_cast<const int4*>(xc + (mrow[i] * chunks + c) * 64 + 32 * s + 16 * g);
                const int4 q = *reinterpret_cast<const int4*>(wc + (nrow[i] * chunks + c) * 64 + 32 * s + 16 * g);
                a[i][s] = v8i{p.x, p.y, p.z, p.w, 0, 0, 0, 0};
                b[i][s] = v8i{q.x, q.y, q.z, q.w, 0, 0, 0, 0};
            }
            sa[i] = (int)(xs[(size_t)c * M + mrow[i]] >> (8 * g));   // bytes 0 and 2: the lane's block of both steps
            sb[i] = (int)(ws[(size_t)c * N + nrow[i]] >> (8 * g));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i][0], b[j][0], acc[i][j], 4, 4, 0, sa[i], 0, sb[j]);
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[i][1], b[j][1], acc[i][j], 4, 4, 2, sa[i], 2, sb[j]);
            }
    }
    // register v of lane (r, g): row 8 (v / 4) + 4 g + v % 4, column r
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int n = n_base + 32 * j + r;
        const float b = n < N && bias ? bias[n] : 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int m = m_base + 32 * i + 8 * (v >> 2) + 4 * g + (v & 3);
                const float h = acc[i][j][v] + b;
                if constexpr (ACT == ACT_SIGN) {
                    const unsigned long long bits = __builtin_amdgcn_ballot_w64(n < N && sign_bit(h));
                    const int word = (n_base >> 5) + j;
                    if (r == 0 && m < M && word < yw32) static_cast<uint32_t*>(Y)[(size_t)m * yw32 + word] = (uint32_t)(bits >> (32 * g));
                } else {
                    if (m < M && n < N) static_cast<float*>(Y)[(size_t)m * N + n] = mx4_act<ACT>(h);
                }
            }
    }
}

}  // namespace bnn
