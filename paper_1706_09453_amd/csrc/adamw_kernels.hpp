// AdamW (decoupled weight decay) over many tensors in one launch, states in 32 bits or in 8.
#pragma once

#include <type_traits>

#include "bnn_device.hpp"
#include "mx_format.hpp"

namespace bnn {

constexpr int kAdamwTensors = 40;      // of one launch: 64 bytes of its arguments each
constexpr int kAdamwChunk = 4096;      // elements that a workgroup takes: 4 quads a thread

struct AdamwTensor {
    float* w;
    const float* g;
    void *m, *v;
    unsigned char *m_scale, *v_scale;
    int64_t count;
    int32_t first;     // number of the tensor's first chunk in the launch
    int32_t flags;     // bit 0: clip, bit 1: 16-byte (8-bit states: codes 4-byte) accesses
};
struct AdamwTable {
    AdamwTensor t[kAdamwTensors];
    int n, at;         // tensors; how many tensors with elements the call has had in earlier launches
};

// beta^t by squaring: the same multiplications on the host and on the device
__host__ __device__ inline double power(double beta, int64_t t) {
    double p = 1.0;
    for (; t > 0; t >>= 1, beta = beta * beta)
        if (t & 1) p = p * beta;
    return p;
}
struct AdamwFactors {
    float b1, c1, b2, c2, eps, decay, size, q;
};
__host__ __device__ inline AdamwFactors adamw_factors(double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step) {
    return {(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, (float)(lr * weight_decay),
            (float)(lr / (1.0 - power(beta1, step))), (float)(1.0 / sqrt(1.0 - power(beta2, step)))};
}
struct AdamwParams {
    double lr, beta1, beta2, eps, weight_decay;
    int64_t step;
    const float* lr_at;
    const int64_t* step_at;
    uint32_t key;
};

// the tensor that a chunk belongs to
__device__ __forceinline__ int adamw_tensor_of(const AdamwTable& table, int chunk) {
    int i = 0;
    while (i + 1 < table.n && table.t[i + 1].first <= chunk) ++i;
    return i;
}

struct Quad { float v[4]; };
__device__ __forceinline__ Quad load_quad(const float* p, int64_t e, int64_t count, bool vec) {
    Quad q;
    if (vec && e + 4 <= count) {
        const float4 f = *reinterpret_cast<const float4*>(p + e);
        q.v[0] = f.x; q.v[1] = f.y; q.v[2] = f.z; q.v[3] = f.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) q.v[j] = e + j < count ? p[e + j] : 0.0f;
    }
    return q;
}
__device__ __forceinline__ void store_quad(float* p, int64_t e, int64_t count, bool vec, const Quad& q) {
    if (vec && e + 4 <= count) {
        *reinterpret_cast<float4*>(p + e) = make_float4(q.v[0], q.v[1], q.v[2], q.v[3]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e + j < count) p[e + j] = q.v[j];
    }
}
// 4 codes, one byte each
__device__ __forceinline__ uint32_t load_codes(const unsigned char* p, int64_t e, int64_t count, bool vec) {
    if (vec && e + 4 <= count) return *reinterpret_cast<const uint32_t*>(p + e);
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c |= e + j < count ? (uint32_t)p[e + j] << (8 * j) : 0u;
    return c;
}
__device__ __forceinline__ void store_codes(unsigned char* p, int64_t e, int64_t count, bool vec, uint32_t c) {
    if (vec && e + 4 <= count) {
        *reinterpret_cast<uint32_t*>(p + e) = c;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (e + j < count) p[e + j] = (unsigned char)(c >> (8 * j));
    }
}

__device__ __forceinline__ float signed_code(uint32_t c, int j) { return (float)(int8_t)(c >> (8 * j)); }
__device__ __forceinline__ float unsigned_code(uint32_t c, int j) { return (float)((c >> (8 * j)) & 0xFFu); }

// The update, every operation rounded in fp32 (no contraction: the library is built with -ffp-contract=off):
//     m' = b1 m + c1 g,   v' = b2 v + (c2 g) g,   r = sqrt(v'),   w' = w - (decay w + (size m') / (r q + eps))
template <int BITS>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamwTable table, const AdamwParams p) {
    const int i = adamw_tensor_of(table, (int)blockIdx.x);
    const AdamwTensor& t = table.t[i];
    const AdamwFactors f = adamw_factors(p.lr_at ? (double)*p.lr_at : p.lr, p.beta1, p.beta2, p.eps, p.weight_decay,
                                         p.step_at ? (*p.step_at > 1 ? *p.step_at : 1) : p.step);
    const bool clip = t.flags & 1, vec = t.flags & 2;
    const int64_t chunk = (int64_t)((int)blockIdx.x - t.first) * kAdamwChunk;
    const uint32_t key = mix32(p.key + (uint32_t)(table.at + i));
#pragma unroll
    for (int k = 0; k < kAdamwChunk / 1024; ++k) {
        const int64_t e = chunk + k * 1024 + (int)threadIdx.x * 4;
        if ((e & ~31) >= t.count) break;   // whole groups of 8 lanes
        Quad w = load_quad(t.w, e, t.count, vec), m, v, r;
        const Quad g = load_quad(t.g, e, t.count, vec);
        if constexpr (BITS == 32) {
            m = load_quad(static_cast<const float*>(t.m), e, t.count, vec);
            v = load_quad(static_cast<const float*>(t.v), e, t.count, vec);
        } else {
            const uint32_t cm = load_codes(static_cast<const unsigned char*>(t.m), e, t.count, vec);
            const uint32_t cv = load_codes(static_cast<const unsigned char*>(t.v), e, t.count, vec);
            const float sm = mx_scale_value(t.m_scale[e >> 5]), sv = mx_scale_value(t.v_scale[e >> 5]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                m.v[j] = signed_code(cm, j) * sm;
                const float old = unsigned_code(cv, j) * sv;
                v.v[j] = old * old;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m.v[j] = f.b1 * m.v[j] + f.c1 * g.v[j];
            v.v[j] = f.b2 * v.v[j] + (f.c2 * g.v[j]) * g.v[j];
            r.v[j] = __builtin_sqrtf(v.v[j]);
            w.v[j] = w.v[j] - (f.decay * w.v[j] + (f.size * m.v[j]) / (r.v[j] * f.q + f.eps));
            if (clip) w.v[j] = hardtanh(w.v[j]);
        }
        store_quad(t.w, e, t.count, vec, w);
        if constexpr (BITS == 32) {
            store_quad(static_cast<float*>(t.m), e, t.count, vec, m);
            store_quad(static_cast<float*>(t.v), e, t.count, vec, v);
        } else {
            uint32_t tm = 0, tv = 0;   // (elements past the end are 0)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                tm = max(tm, __float_as_uint(m.v[j]) & 0x7FFFFFFFu);
                tv = max(tv, __float_as_uint(r.v[j]) & 0x7FFFFFFFu);
            }
            const uint32_t em = mx_scale<MxInt8>(max_of_8_lanes(tm)), ev = mx_scale<MxUint8>(max_of_8_lanes(tv));
            const float im = mx_inverse_scale(em), iv = mx_inverse_scale(ev);
            const uint32_t block_key = mix32(key + (uint32_t)(e >> 5));
            uint32_t cm = 0, cv = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t h = mix32(block_key + (uint32_t)((e & 31) + j));
                const int am = (int)(__builtin_fabsf(m.v[j]) * im + (float)(h & 0xFFFFu) * 0x1p-16f);
                const int av = (int)(r.v[j] * iv + (float)(h >> 16) * 0x1p-16f);
                cm |= ((uint32_t)(m.v[j] < 0.0f ? -am : am) & 0xFFu) << (8 * j);
                cv |= ((uint32_t)av & 0xFFu) << (8 * j);
            }
            if (em == 255) cm = 0;
            if (ev == 255) cv = 0;
            store_codes(static_cast<unsigned char*>(t.m), e, t.count, vec, cm);
            store_codes(static_cast<unsigned char*>(t.v), e, t.count, vec, cv);
            if ((threadIdx.x & 7) == 0) {
                t.m_scale[e >> 5] = (unsigned char)em;
                t.v_scale[e >> 5] = (unsigned char)ev;
            }
        }
    }
}

// 8-bit states as the numbers they stand for.  In the table w is where m goes (may be absent) and g where v goes.
__global__ __launch_bounds__(256) void adamw_unpack_kernel(const AdamwTable table) {
    const AdamwTensor& t = table.t[adamw_tensor_of(table, (int)blockIdx.x)];
    const int64_t chunk = (int64_t)((int)blockIdx.x - t.first) * kAdamwChunk;
    const bool vec = t.flags & 2;
#pragma unroll
    for (int k = 0; k < kAdamwChunk / 1024; ++k) {
        const int64_t e = chunk + k * 1024 + (int)threadIdx.x * 4;
        if (e >= t.count) break;
        const uint32_t cm = load_codes(static_cast<const unsigned char*>(t.m), e, t.count, vec);
        const uint32_t cv = load_codes(static_cast<const unsigned char*>(t.v), e, t.count, vec);
        const float sm = mx_scale_value(t.m_scale[e >> 5]), sv = mx_scale_value(t.v_scale[e >> 5]);
        Quad m, v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            m.v[j] = signed_code(cm, j) * sm;
            const float r = unsigned_code(cv, j) * sv;
            v.v[j] = r * r;
        }
        if (t.w) store_quad(t.w, e, t.count, vec, m);
        if (t.g) store_quad(const_cast<float*>(t.g), e, t.count, vec, v);
    }
}

}  // namespace bnn
