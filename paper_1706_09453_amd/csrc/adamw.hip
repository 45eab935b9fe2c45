// C ABI of the AdamW update: argument checks, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/bnn.h"
#include "adamw_kernels.hpp"
#include "launch.hpp"

namespace {

using namespace bnn;

constexpr int64_t kMaxCount = (int64_t)1 << 35;   // 2^25 workgroups; blocks of 32 are counted in 32 bits

struct Range {
    uintptr_t from, to;
    bool written;
};

// Whether no written range meets another one.
bool apart(Range* r, int n) {
    std::sort(r, r + n, [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t any = 0, written = 0;
    for (int i = 0; i < n; ++i) {
        if (r[i].from < (r[i].written ? any : written)) return false;
        any = std::max(any, r[i].to);
        if (r[i].written) written = std::max(written, r[i].to);
    }
    return true;
}

int check_tensor(const bnn_adamw_tensor& t, int bits) {
    if (t.count < 0 || t.count > kMaxCount) return BNN_ESHAPE;
    if (t.clip < 0 || t.clip > 1) return BNN_EINVAL;
    if (t.count == 0) return BNN_OK;
    if (!t.w || !t.g || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale))) return BNN_EINVAL;
    if (!aligned(t.w, 4) || !aligned(t.g, 4) || (bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4)))) return BNN_EALIGN;
    return BNN_OK;
}

// The tensors from `next` on that one launch takes, and its grid; `next` moves on.  `entry` makes a table entry of tensor i.
template <class Entry>
int64_t fill(AdamwTable& table, const bnn_adamw_tensor* tensors, int n, int& next, Entry&& entry) {
    int64_t chunks = 0;
    table.n = 0;
    for (; next < n && table.n < kAdamwTensors; ++next) {
        const int64_t c = (tensors[next].count + kAdamwChunk - 1) / kAdamwChunk;
        if (c == 0) continue;
        if (chunks + c > kMaxCount / kAdamwChunk) break;   // (never a tensor by itself)
        table.first[table.n] = (int32_t)chunks;
        table.t[table.n++] = entry(next);
        chunks += c;
    }
    return chunks;
}

dim3 grid_of(int64_t chunks) {
    const int64_t x = std::min(chunks, (int64_t)1 << 23);
    return dim3((unsigned)x, (unsigned)((chunks + x - 1) / x));
}

int ranges_of(const bnn_adamw_tensor& t, int bits, Range* r) {
    const size_t n = (size_t)t.count, state = bits == 32 ? 4 * n : n, scales = (n + 31) / 32;
    int k = 0;
    auto add = [&](const void* p, size_t bytes, bool written) { r[k++] = {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written}; };
    add(t.w, 4 * n, true);
    add(t.g, 4 * n, false);
    add(t.m, state, true);
    add(t.v, state, true);
    if (bits == 8) {
        add(t.m_scale, scales, true);
        add(t.v_scale, scales, true);
    }
    return k;
}

}  // namespace

BNN_EXPORT int bnn_update_adamw(const bnn_adamw_tensor* tensors, int n_tensors, const bnn_adamw_params* params, void* stream) {
    if (n_tensors < 0) return BNN_ESHAPE;
    if (!params || (n_tensors > 0 && !tensors)) return BNN_EINVAL;
    const bnn_adamw_params& p = *params;
    if (p.state_bits != 32 && p.state_bits != 8) return BNN_EINVAL;
    if (!(p.beta1 >= 0.0 && p.beta1 < 1.0 && p.beta2 >= 0.0 && p.beta2 < 1.0)) return BNN_EINVAL;
    if (!((float)p.eps > 0.0f && std::isfinite((float)p.eps))) return BNN_EINVAL;
    if (!(p.weight_decay >= 0.0 && std::isfinite((float)p.weight_decay))) return BNN_EINVAL;
    if (!p.lr_at && !(p.lr >= 0.0 && std::isfinite((float)p.lr))) return BNN_EINVAL;
    if (!p.step_at && p.step < 1) return BNN_EINVAL;
    if (!aligned(p.lr_at, 4) || !aligned(p.step_at, 8)) return BNN_EALIGN;
    for (int i = 0; i < n_tensors; ++i)
        if (const int rc = check_tensor(tensors[i], p.state_bits); rc != BNN_OK) return rc;

    // The tensors of one launch are updated side by side: what it writes must lie apart.  Checked for every launch before the first.
    const bool on_device = p.lr_at || p.step_at;
    AdamwHost host{};
    const AdamwDevice device{p.lr, p.beta1, p.beta2, p.eps, p.weight_decay, p.step, p.seed, p.lr_at, p.step_at};
    if (!on_device) {
        host = {adamw_factors(p.lr, p.beta1, p.beta2, p.eps, p.weight_decay, p.step), seed_key(p.seed)};
        if (!std::isfinite(host.f.decay) || !std::isfinite(host.f.size) || !std::isfinite(host.f.q)) return BNN_EINVAL;
    }
    for (int pass = 0; pass < 2; ++pass) {
        for (int next = 0, at = 0; next < n_tensors;) {
            AdamwTable table;
            table.at = at;
            Range ranges[6 * kAdamwTensors + 2];
            int k = 0;
            const int64_t chunks = fill(table, tensors, n_tensors, next, [&](int i) {
                const bnn_adamw_tensor& t = tensors[i];
                if (pass == 0) k += ranges_of(t, p.state_bits, ranges + k);
                const bool vec = aligned(t.w, 16) && aligned(t.g, 16) && (p.state_bits == 32 ? aligned(t.m, 16) && aligned(t.v, 16) : aligned(t.m, 4) && aligned(t.v, 4));
                return AdamwTensor{t.w, t.g, t.m, t.v, t.m_scale, t.v_scale, t.count, t.clip, vec};
            });
            if (chunks == 0) break;
            at += table.n;
            if (pass == 0) {
                if (p.lr_at) ranges[k++] = {reinterpret_cast<uintptr_t>(p.lr_at), reinterpret_cast<uintptr_t>(p.lr_at) + 4, false};
                if (p.step_at) ranges[k++] = {reinterpret_cast<uintptr_t>(p.step_at), reinterpret_cast<uintptr_t>(p.step_at) + 8, false};
                if (!apart(ranges, k)) return BNN_EINVAL;
                continue;
            }
            hipStream_t st = static_cast<hipStream_t>(stream);
            auto go = [&](auto bits) {
                constexpr int B = decltype(bits)::value;
                if (on_device) adamw_kernel<B, AdamwDevice><<<grid_of(chunks), 256, 0, st>>>(device, table);
                else adamw_kernel<B, AdamwHost><<<grid_of(chunks), 256, 0, st>>>(host, table);
            };
            if (p.state_bits == 32) go(std::integral_constant<int, 32>{});
            else go(std::integral_constant<int, 8>{});
            if (const int rc = launch_status(); rc != BNN_OK) return rc;
        }
    }
    return BNN_OK;
}

BNN_EXPORT int bnn_unpack_adamw_states(const bnn_adamw_tensor* tensors, int n_tensors, float* const* m_out, float* const* v_out, void* stream) {
    if (n_tensors < 0) return BNN_ESHAPE;
    if (n_tensors > 0 && (!tensors || (!m_out && !v_out))) return BNN_EINVAL;
    for (int i = 0; i < n_tensors; ++i) {
        const bnn_adamw_tensor& t = tensors[i];
        if (t.count < 0 || t.count > kMaxCount) return BNN_ESHAPE;
        if (t.count == 0) continue;
        if (!t.m || !t.v || !t.m_scale || !t.v_scale) return BNN_EINVAL;
        if (!aligned(m_out ? m_out[i] : nullptr, 4) || !aligned(v_out ? v_out[i] : nullptr, 4)) return BNN_EALIGN;
    }
    for (int pass = 0; pass < 2; ++pass) {
        for (int next = 0; next < n_tensors;) {
            AdamwTable table;
            table.at = 0;
            Range ranges[6 * kAdamwTensors];
            int k = 0;
            const int64_t chunks = fill(table, tensors, n_tensors, next, [&](int i) {
                const bnn_adamw_tensor& t = tensors[i];
                float *mo = m_out ? m_out[i] : nullptr, *vo = v_out ? v_out[i] : nullptr;
                if (pass == 0) {
                    Range r[6];
                    ranges_of(t, 8, r);
                    for (int j = 2; j < 6; ++j) ranges[k++] = {r[j].from, r[j].to, false};
                    for (float* o : {mo, vo})
                        if (o) ranges[k++] = {reinterpret_cast<uintptr_t>(o), reinterpret_cast<uintptr_t>(o) + 4 * (size_t)t.count, true};
                }
                const bool vec = aligned(mo, 16) && aligned(vo, 16) && aligned(t.m, 4) && aligned(t.v, 4);
                return AdamwTensor{mo, vo, t.m, t.v, t.m_scale, t.v_scale, t.count, 0, vec};
            });
            if (chunks == 0) break;
            if (pass == 0) {
                if (!apart(ranges, k)) return BNN_EINVAL;
                continue;
            }
            hipStream_t st = static_cast<hipStream_t>(stream);
            adamw_unpack_kernel<<<grid_of(chunks), 256, 0, st>>>(table);
            if (const int rc = launch_status(); rc != BNN_OK) return rc;
        }
    }
    return BNN_OK;
}
