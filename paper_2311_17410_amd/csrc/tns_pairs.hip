// Paired log-ratio loss of true links against sampled ones, and its gradients (include/tns_train.h).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/tns_train.h"
#include "tns_internal.h"
#include "tns_values.h"

using tns::as_float;
using tns::as_value;
using tns::bf16;
using tns::fail;
using tns::fail_hip;

namespace {

template <typename T>
struct Pairs {                        // tns_pairs with its types
    int64_t B, K;
    const T *anchor, *pos, *neg;
    int64_t ld_anchor, ld_pos;
    const float *ref, *weight;
    float beta, smoothing, scale;
    int dim;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int by = 32; by; by >>= 1) v += __shfl_xor(v, by);
    return v;
}

// Loss of a margin and its slope, both times scale and weight.
__device__ __forceinline__ void loss_of(float m, float w, float scale, float smoothing, float& loss, float& slope) {
    const float e = expf(-fabsf(m)), tail = log1pf(e);                      // softplus(-m) = tail + max(-m, 0)
    loss = scale * w * (tail + fmaxf(-m, 0.0f) * (1.0f - smoothing) + fmaxf(m, 0.0f) * smoothing);
    slope = scale * w * (smoothing - (m > 0.0f ? e : 1.0f) / (1.0f + e));   // sigmoid(-m)
    if (m != m) loss = slope = m;
}

// A wave per event, its sampled links one after the other.
template <typename T>
__global__ void __launch_bounds__(64) k_pairs(const Pairs<T> p, float* losses, float* margin, T* danchor, T* dpos, T* dneg) {
    const int64_t b = blockIdx.x;
    const int lane = threadIdx.x;
    const T* const a = p.anchor + b * p.ld_anchor;
    const T* const q = p.pos + b * p.ld_pos;
    float plus = 0.0f;
    for (int c = lane; c < p.dim; c += 64) plus += as_float(a[c]) * as_float(q[c]);
    plus = wave_sum(plus);
    float total = 0.0f, csum = 0.0f;
    bool any = false;
    for (int64_t k = 0; k < p.K; ++k) {
        const int64_t i = b * p.K + k;
        const float w = p.weight ? p.weight[i] : 1.0f;
        const T* const n = p.neg + i * p.dim;
        float m = 0.0f, slope = 0.0f, loss = 0.0f;
        if (w != 0.0f) {
            float minus = 0.0f;
            for (int c = lane; c < p.dim; c += 64) minus += as_float(a[c]) * as_float(n[c]);
            minus = wave_sum(minus);
            m = p.beta * (plus - minus - (p.ref ? p.ref[i] : 0.0f));
            loss_of(m, w, p.scale, p.smoothing, loss, slope);
            slope *= p.beta;
            any = true;
        }
        total += loss;
        csum += slope;
        if (lane == 0 && margin) margin[i] = m;
        if (danchor)
            for (int c = lane; c < p.dim; c += 64) {
                dneg[i * p.dim + c] = as_value<T>(w != 0.0f ? -slope * as_float(a[c]) : 0.0f);
            }
    }
    if (lane == 0) losses[b] = total;
    if (!danchor) return;
    for (int c = lane; c < p.dim; c += 64) {
        float da = 0.0f;
        for (int64_t k = 0; k < p.K; ++k) {
            const int64_t i = b * p.K + k;
            const float w = p.weight ? p.weight[i] : 1.0f;
            if (w != 0.0f) {
                float minus = 0.0f;
                for (int j = 0; j < p.dim; ++j) minus += as_float(a[j]) * as_float(p.neg[i * p.dim + j]);
                float loss, slope;
                loss_of(p.beta * (plus - minus - (p.ref ? p.ref[i] : 0.0f)), w, p.scale, p.smoothing, loss, slope);
                da += slope * p.beta * (as_float(q[c]) - as_float(p.neg[i * p.dim + c]));
            }
        }
        danchor[b * p.dim + c] = as_value<T>(da);
        dpos[b * p.dim + c] = as_value<T>(any ? csum * as_float(a[c]) : 0.0f);
    }
}

__global__ void __launch_bounds__(64) k_pairs_sum(const float* losses, int64_t n, float* out) {
    float sum = 0.0f;
    for (int64_t i = threadIdx.x; i < n; i += 64) sum += losses[i];
    sum = wave_sum(sum);
    if (threadIdx.x == 0) *out = sum;
}

int check(int64_t B, int64_t K, int32_t dim) {
    if (B < 0 || K < 0) return fail(TNS_EINVAL, "negative number of events or links");
    if (B > (int64_t)INT32_MAX || (K && B > ((int64_t)1 << 40) / K)) return fail(TNS_ESIZE, "more than 2^31-1 events or 2^40 links");
    if (dim < 1 || dim > 1 << 16) return fail(TNS_EINVAL, "dim must be in [1, 2^16]");
    return TNS_OK;
}

size_t workspace_bytes_of(int64_t B, int64_t, int32_t) { return (size_t)B * 4; }

}  // namespace

extern "C" {

int tns_pair_loss_workspace(int64_t B, int64_t K, int32_t dim, size_t* bytes) {
    tns::clear_error();
    if (!bytes) return fail(TNS_EINVAL, "null output pointer");
    if (int e = check(B, K, dim)) return e;
    *bytes = workspace_bytes_of(B, K, dim);
    return TNS_OK;
}

int tns_pair_loss(const tns_pairs* p, float* d_loss, float* d_margin, void* d_danchor, void* d_dpos, void* d_dneg, void* d_workspace,
                  size_t workspace_bytes, void* hip_stream) {
    tns::clear_error();
    if (!p || !d_loss) return fail(TNS_EINVAL, "null description of the pairs or loss");
    if (int e = check(p->B, p->K, p->dim)) return e;
    if (p->dtype != TNS_F32 && p->dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if (p->B > 0 && (!p->d_anchor || !p->d_pos || (p->K > 0 && !p->d_neg))) return fail(TNS_EINVAL, "null embeddings");
    if (p->ld_anchor < p->dim || p->ld_pos < p->dim) return fail(TNS_EINVAL, "rows of anchor or pos overlap");
    if (!(p->smoothing >= 0.0 && p->smoothing <= 1.0)) return fail(TNS_EINVAL, "smoothing must be in [0, 1]");
    if (!d_danchor != !d_dpos || (p->K > 0 && !d_danchor != !d_dneg)) return fail(TNS_EINVAL, "gradients come together");
    const size_t need = workspace_bytes_of(p->B, p->K, p->dim);
    if (need && !d_workspace) return fail(TNS_EINVAL, "null workspace");
    if (reinterpret_cast<uintptr_t>(d_workspace) & 255) return fail(TNS_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(TNS_ESIZE, "workspace smaller than tns_pair_loss_workspace()");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    float* const losses = static_cast<float*>(d_workspace);
    auto launch = [&](auto value) {
        using T = decltype(value);
        const Pairs<T> t{p->B, p->K, static_cast<const T*>(p->d_anchor), static_cast<const T*>(p->d_pos), static_cast<const T*>(p->d_neg),
                         p->ld_anchor, p->ld_pos, p->d_ref, p->d_weight, (float)p->beta, (float)p->smoothing, (float)p->scale, p->dim};
        hipLaunchKernelGGL((k_pairs<T>), dim3((unsigned)p->B), dim3(64), 0, stream, t, losses, d_margin, static_cast<T*>(d_danchor),
                           static_cast<T*>(d_dpos), static_cast<T*>(d_dneg));
    };
    if (p->B > 0) {
        if (p->dtype == TNS_F32) launch(float{});
        else launch(bf16{});
    }
    hipLaunchKernelGGL(k_pairs_sum, dim3(1), dim3(64), 0, stream, losses, p->B, d_loss);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, "tns_pair_loss");
}

}  // extern "C"
