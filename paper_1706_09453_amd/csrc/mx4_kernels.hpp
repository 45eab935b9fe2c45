// Matrices in microscaled 4-bit floating point (blocks of 32 along a row; layout in include/bnn.h): from fp32 and back.
#pragma once

#include <type_traits>

#include "bnn_device.hpp"
#include "mx_format.hpp"

namespace bnn {

constexpr int kMx4Chunk = 128;        // elements of a chunk: 64 bytes of codes, one word of scale bytes
constexpr int kMx4ChunkBytes = 64;
__host__ __device__ inline int64_t mx4_chunks(int64_t K) { return (K + kMx4Chunk - 1) / kMx4Chunk; }
__host__ __device__ inline size_t mx4_code_bytes(int64_t R, int64_t K) { return ((size_t)R * (size_t)mx4_chunks(K) * kMx4ChunkBytes + 255) / 256 * 256; }
inline size_t mx4_bytes(int64_t R, int64_t K) { return mx4_code_bytes(R, K) + (size_t)R * (size_t)mx4_chunks(K) * 4; }
__host__ __device__ inline uint32_t* mx4_scales(void* q, int64_t R, int64_t K) {
    return reinterpret_cast<uint32_t*>(static_cast<unsigned char*>(q) + mx4_code_bytes(R, K));
}
__host__ __device__ inline const uint32_t* mx4_scales(const void* q, int64_t R, int64_t K) {
    return reinterpret_cast<const uint32_t*>(static_cast<const unsigned char*>(q) + mx4_code_bytes(R, K));
}

// Code of a scaled number y, |y| <= 6: the 4-bit numbers 0, 0.5, 1, 1.5, 2, 3, 4, 6 are codes 0 to 7, which from 1 on are the
// upper bits of the float (exponent and one bit of fraction, 252 = 2 * 126 above the code) and below 2 twice the value.
// Nearest: ties to the even code.  Stochastic: the code below, or the next one up with the probability of how far y is beyond it;
// bits16 are the random bits.  Both add to the bits that fall away and cut them off.
__device__ __forceinline__ uint32_t mx4_code_nearest(float y) {
    const uint32_t a = __float_as_uint(y) & 0x7FFFFFFFu;
    const uint32_t low = (uint32_t)__builtin_rintf(2.0f * __uint_as_float(a));
    const uint32_t high = ((a + 0x1FFFFFu + ((a >> 22) & 1u)) >> 22) - 252u;
    return (a < 0x3F800000u ? low : high) | ((__float_as_uint(y) >> 28) & 8u);
}
__device__ __forceinline__ uint32_t mx4_code_stochastic(float y, uint32_t bits16) {
    const uint32_t a = __float_as_uint(y) & 0x7FFFFFFFu;
    const bool small = a < 0x3F800000u;
    const uint32_t v = small ? (uint32_t)(__uint_as_float(a) * 0x1p23f) : a;
    return ((v + (bits16 << 6)) >> 22) - (small ? 0u : 252u) | ((__float_as_uint(y) >> 28) & 8u);
}

// 4-bit codes of a matrix X [R][C] along its rows (Q: [R][C]) and along its columns (QT: [C][R]); either may be absent.  A workgroup
// takes tiles of 128 x 128, for the rows form with 32 lanes per row (4 consecutive elements each, so that 8 lanes hold a block),
// for the columns form with a column and 32 rows of it per lane.  Elements outside the matrix count as 0: pads are 0.
template <bool VEC, bool STOCHASTIC>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const float* __restrict__ X, int R, int C, uint32_t key, void* __restrict__ Q,
                                                           void* __restrict__ QT, int tiles_r, int tiles_c) {
    const int wave = (int)threadIdx.x >> 6, lane = lane_id();
    for (int64_t t = blockIdx.x; t < (int64_t)tiles_r * tiles_c; t += gridDim.x) {
        const int tc = (int)(t % tiles_c), tr = (int)(t / tiles_c), c0 = tc * 128, r0 = tr * 128;
        if (Q) {
            unsigned char* codes = static_cast<unsigned char*>(Q);
            unsigned char* scales = reinterpret_cast<unsigned char*>(mx4_scales(Q, R, C));
            const int sub = lane & 31, c = c0 + 4 * sub;
            for (int i = 0; i < 16; ++i) {
                const int r = r0 + 8 * i + 2 * wave + (lane >> 5);
                if (r >= R) continue;   // (whole groups of 32 lanes)
                float v[4];
                const float* p = X + (size_t)r * C + c;
                if (VEC && c + 4 <= C) {
                    const float4 q = *reinterpret_cast<const float4*>(p);
                    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = c + j < C ? p[j] : 0.0f;
                }
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
                top = max_of_8_lanes(top);
                const uint32_t e = mx_scale<MxE2M1>(top);
                const float inv = mx_inverse_scale(e);
                const uint32_t row_key = mix32(key + (uint32_t)r);
                uint32_t out = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float y = v[j] * inv;
                    const uint32_t code = STOCHASTIC ? mx4_code_stochastic(y, mix32(row_key + (uint32_t)(c + j)) & 0xFFFFu) : mx4_code_nearest(y);
                    out |= code << (4 * j);
                }
                if (e == 255) out = 0;
                *reinterpret_cast<uint16_t*>(codes + ((size_t)r * tiles_c + tc) * 64 + 2 * sub) = (uint16_t)out;
                if ((sub & 7) == 0) scales[((size_t)tc * R + r) * 4 + (sub >> 3)] = (unsigned char)e;
            }
        }
        if (QT) {
            unsigned char* codes = static_cast<unsigned char*>(QT);
            unsigned char* scales = reinterpret_cast<unsigned char*>(mx4_scales(QT, C, R));
            for (int h = 0; h < 2; ++h) {
                const int c = c0 + 64 * h + lane, rb = r0 + 32 * wave;
                if (c >= C) continue;
                float v[32];
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = rb + j < R ? X[(size_t)(rb + j) * C + c] : 0.0f;
#pragma unroll
                for (int j = 0; j < 32; ++j) top = max(top, __float_as_uint(v[j]) & 0x7FFFFFFFu);
                const uint32_t e = mx_scale<MxE2M1>(top);
                const float inv = mx_inverse_scale(e);
                uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float y = v[j] * inv;
                    const uint32_t code = STOCHASTIC ? mx4_code_stochastic(y, mix32(mix32(key + (uint32_t)(rb + j)) + (uint32_t)c) >> 16) : mx4_code_nearest(y);
                    w[j >> 3] |= code << (4 * (j & 7));
                }
                if (e == 255) w[0] = w[1] = w[2] = w[3] = 0u;
                *reinterpret_cast<uint4*>(codes + ((size_t)c * tiles_r + tr) * 64 + 16 * wave) = make_uint4(w[0], w[1], w[2], w[3]);
                scales[((size_t)tr * C + c) * 4 + wave] = (unsigned char)e;
            }
        }
    }
}

// The values that the codes of a matrix [R][K] stand for, fp32.  A lane takes 4 elements.
template <bool VEC>
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const void* __restrict__ Q, int R, int K, int chunks, float* __restrict__ X) {
    const unsigned char* codes = static_cast<const unsigned char*>(Q);
    const unsigned char* scales = reinterpret_cast<const unsigned char*>(mx4_scales(Q, R, K));
    const int64_t quads = (int64_t)R * chunks * 32, stride = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < quads; i += stride) {
        const int64_t rc = i >> 5;
        const int r = (int)(rc / chunks), chunk = (int)(rc - (int64_t)r * chunks), sub = (int)(i & 31), k = chunk * 128 + 4 * sub;
        if (k >= K) continue;
        const uint32_t c = *reinterpret_cast<const uint16_t*>(codes + 2 * i);
        const float s = mx_scale_value(scales[((size_t)chunk * R + r) * 4 + (sub >> 3)]);
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t n = c >> (4 * j);   // the code's lower bits are a float's exponent and fraction, 2^126 too small
            v[j] = __uint_as_float((n & 7u) << 22 | (n & 8u) << 28) * 0x1p126f * s;
        }
        float* p = X + (size_t)r * K + k;
        if (VEC && k + 4 <= K) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (k + j < K) p[j] = v[j];
        }
    }
}

}  // namespace bnn
