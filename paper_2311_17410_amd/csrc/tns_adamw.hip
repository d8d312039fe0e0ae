// AdamW over all tensors of a model in one launch, states in 32 or in 8 bits (include/tns_train.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>
#include <vector>

#include "../../include/tns_train.h"
#include "tns_internal.h"
#include "tns_values.h"

using tns::as_float;
using tns::as_value;
using tns::bf16;
using tns::DeviceGuard;
using tns::fail;
using tns::fail_hip;

namespace {

constexpr int kBlock = 256;           // weights that share a scale: four per lane of a wave
constexpr int kTile = 4096;           // weights per workgroup of four waves
constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull, kMix1 = 0xBF58476D1CE4E5B9ull, kMix2 = 0x94D049BB133111EBull;

__host__ __device__ inline uint64_t mix64(uint64_t z) {        // output function of splitmix64
    z = (z ^ (z >> 30)) * kMix1;
    z = (z ^ (z >> 27)) * kMix2;
    return z ^ (z >> 31);
}

// A workgroup's tile of a tensor, whole in itself: one request, and the addresses of everything else are known.
struct Part {
    float* param;
    bf16* copy;
    const void* grad;
    void *m, *v;
    float *m_scale, *v_scale;
    uint64_t word0;                   // number of the random word of its first four weights
    int32_t n;                        // weights, kTile at most
    int32_t aligned;                  // four weights of every buffer can be read at once
    float decay;
};

struct Step {                         // factors of one step, rounded to fp32 once
    float beta1, rest1, beta2, rest2, lr, rate, root, eps;
    uint64_t key;
};
__device__ __forceinline__ float step_keep(const Step& s, const Part& t) {
#pragma clang fp contract(off)
    return 1.0f - s.lr * t.decay;
}

// Largest of the wave's values, as the bits of magnitudes (a NaN is larger than everything): four steps within the rows of sixteen
// lanes, part of the vector instruction, then the rows' ends.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_with(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max_with<0x111, 0xf>(v);
    v = max_with<0x112, 0xf>(v);
    v = max_with<0x114, 0xf>(v);
    v = max_with<0x118, 0xf>(v);
    v = max_with<0x142, 0xa>(v);
    v = max_with<0x143, 0xc>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Four codes and their values.
__device__ __forceinline__ void from_codes(uint32_t codes, float scale, float (&v)[4]) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    v[0] = lo[0] * scale; v[1] = lo[1] * scale; v[2] = hi[0] * scale; v[3] = hi[1] * scale;
}

// The wave's 256 values as codes and their scale.
template <bool SIGNED>
__device__ __forceinline__ uint32_t to_codes(const float (&v)[4], uint64_t random, float& scale) {
#pragma clang fp contract(off)
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    const float t = __uint_as_float(wave_max(top));
    if (t < 0x1p-100f) { scale = 0.0f; return 0; }
    scale = t * (1.0f / 448.0f);
    const float by = 448.0f / t;
    uint32_t codes = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float y = v[j] * by;
        if (!SIGNED) y = fmaxf(y, 0x1p-6f);
        const uint32_t bits = __float_as_uint(y), size = bits & 0x7fffffffu;
        uint32_t code = ((size + ((uint32_t)(random >> (16 * j)) & 0xffffu) * 16u) >> 20) - (120u << 3);
        code = size < (121u << 23) ? 0u : (min(code, 0x7eu) | (SIGNED ? bits >> 24 & 0x80u : 0u));
        codes |= code << (8 * j);
    }
    return codes;
}

// Four weights of a lane, as they lie in memory, and their step.
template <int BITS, typename G>
struct Four {
    using Grads = typename std::conditional<std::is_same<G, float>::value, float4, uint2>::type;
    float p[4], m[4], v[4];             // (32 bits)
    float g[4];
    uint32_t mc, vc;                    // (8 bits)
    float m_scale, v_scale;

    // All of them, from aligned addresses.
    __device__ void read(const Part& t, int block, int i0) {
        const float4 q = *reinterpret_cast<const float4*>(t.param + i0);
        p[0] = q.x; p[1] = q.y; p[2] = q.z; p[3] = q.w;
        const Grads r = *reinterpret_cast<const Grads*>(static_cast<const G*>(t.grad) + i0);
        if constexpr (std::is_same<G, float>::value) {
            g[0] = r.x; g[1] = r.y; g[2] = r.z; g[3] = r.w;
        } else {
            g[0] = __uint_as_float(r.x << 16); g[1] = __uint_as_float(r.x & 0xffff0000u);
            g[2] = __uint_as_float(r.y << 16); g[3] = __uint_as_float(r.y & 0xffff0000u);
        }
        if (BITS == 32) {
            const float4 a = *reinterpret_cast<const float4*>(static_cast<const float*>(t.m) + i0), b = *reinterpret_cast<const float4*>(static_cast<const float*>(t.v) + i0);
            m[0] = a.x; m[1] = a.y; m[2] = a.z; m[3] = a.w;
            v[0] = b.x; v[1] = b.y; v[2] = b.z; v[3] = b.w;
        } else {
            mc = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + i0);
            vc = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + i0);
            m_scale = t.m_scale[block];
            v_scale = t.v_scale[block];
        }
    }
    __device__ void write(const Part& t, int block, int i0) const {
        *reinterpret_cast<float4*>(t.param + i0) = make_float4(p[0], p[1], p[2], p[3]);
        if (t.copy) {
            bf16 c[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) c[k] = as_value<bf16>(p[k]);
            *reinterpret_cast<uint2*>(t.copy + i0) = __builtin_bit_cast(uint2, c);
        }
        if (BITS == 32) {
            *reinterpret_cast<float4*>(static_cast<float*>(t.m) + i0) = make_float4(m[0], m[1], m[2], m[3]);
            *reinterpret_cast<float4*>(static_cast<float*>(t.v) + i0) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + i0) = mc;
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + i0) = vc;
            if ((threadIdx.x & 63) == 0) { t.m_scale[block] = m_scale; t.v_scale[block] = v_scale; }
        }
    }
    // The first n of them, one by one; the others are zero.
    __device__ void read(const Part& t, int block, int i0, int n) {
        mc = vc = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool is = k < n;
            g[k] = is ? as_float(static_cast<const G*>(t.grad)[i0 + k]) : 0.0f;
            p[k] = is ? t.param[i0 + k] : 0.0f;
            if (BITS == 32) {
                m[k] = is ? static_cast<const float*>(t.m)[i0 + k] : 0.0f;
                v[k] = is ? static_cast<const float*>(t.v)[i0 + k] : 0.0f;
            } else if (is) {
                mc |= (uint32_t)static_cast<const uint8_t*>(t.m)[i0 + k] << (8 * k);
                vc |= (uint32_t)static_cast<const uint8_t*>(t.v)[i0 + k] << (8 * k);
            }
        }
        if (BITS == 8) {
            m_scale = t.m_scale[block];
            v_scale = t.v_scale[block];
        }
    }
    __device__ void write(const Part& t, int block, int i0, int n) const {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= n) continue;
            t.param[i0 + k] = p[k];
            if (t.copy) t.copy[i0 + k] = as_value<bf16>(p[k]);
            if (BITS == 32) {
                static_cast<float*>(t.m)[i0 + k] = m[k];
                static_cast<float*>(t.v)[i0 + k] = v[k];
            } else {
                static_cast<uint8_t*>(t.m)[i0 + k] = (uint8_t)(mc >> (8 * k));
                static_cast<uint8_t*>(t.v)[i0 + k] = (uint8_t)(vc >> (8 * k));
            }
        }
        if (BITS == 8 && (threadIdx.x & 63) == 0) { t.m_scale[block] = m_scale; t.v_scale[block] = v_scale; }
    }

    // n of the lane's four exist (the others stay zero).  The weight's change is divided by the reciprocal of one unit in the last place;
    // what is kept for the next step is rounded operation by operation, so that it is the same wherever it is computed.
    __device__ void step(const Step& s, float keep, float gs, uint64_t word, int n) {
#pragma clang fp contract(off)
        float r[4];
        if (BITS == 8) {
            from_codes(mc, m_scale, m);
            from_codes(vc, v_scale, r);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = r[k] * r[k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float a = g[k] * gs;
            m[k] = s.beta1 * m[k] + s.rest1 * a;
            v[k] = s.beta2 * v[k] + s.rest2 * (a * a);
            r[k] = sqrtf(v[k]);
            p[k] = p[k] * keep - (s.rate * m[k]) * __builtin_amdgcn_rcpf(r[k] * s.root + s.eps);
            if (BITS == 8 && k >= n) m[k] = r[k] = 0.0f;
        }
        if (BITS == 8) {
            const uint64_t random = mix64(s.key + kGolden * (word + 1));
            mc = to_codes<true>(m, random, m_scale);
            vc = to_codes<false>(r, random, v_scale);
        }
    }
};

// A workgroup per tile.  Bound by memory, as everything is read and written once; a wave reads its four blocks before it computes.  128 M
// weights with states of 8 bits, bf16 gradients and copies (16 bytes a weight): 2.06 GB in 382 us (5.4 TB/s); element by element, one block
// after the other, 751.  180 K weights in 28 tensors, states of 32 bits: 4.6 us, the launch and two reads one after the other.
template <int BITS, typename G>
__global__ void __launch_bounds__(256) k_adamw(const Part* __restrict__ tiles, const Step s, const float* __restrict__ grad_scale) {
    const Part t = tiles[blockIdx.x];
    const float gs = grad_scale ? *grad_scale : 1.0f;
    if (gs == 0.0f || !(fabsf(gs) <= 3.402823466e+38f)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int kMine = kTile / kBlock / 4;                // blocks of a wave
    const int first = wave * kMine;
    const float keep = step_keep(s, t);
    Four<BITS, G> f[kMine];
    auto at = [&](int j) { return (first + j) * kBlock + lane * 4; };
    auto whole = [&](int j) { return t.aligned && (first + j + 1) * kBlock <= t.n; };
    auto count = [&](int j) { return min(max(t.n - at(j), 0), 4); };
    if (whole(kMine - 1)) {
#pragma unroll
        for (int j = 0; j < kMine; ++j) f[j].read(t, first + j, at(j));
#pragma unroll
        for (int j = 0; j < kMine; ++j) {
            f[j].step(s, keep, gs, t.word0 + (uint64_t)(at(j) >> 2), 4);
            f[j].write(t, first + j, at(j));
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        if (whole(j)) f[j].read(t, first + j, at(j));
        else if ((first + j) * kBlock < t.n) f[j].read(t, first + j, at(j), count(j));
    }
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
        if ((first + j) * kBlock >= t.n) return;
        f[j].step(s, keep, gs, t.word0 + (uint64_t)(at(j) >> 2), count(j));
        if (whole(j)) f[j].write(t, first + j, at(j));
        else f[j].write(t, first + j, at(j), count(j));
    }
}

}  // namespace

struct tns_adamw {
    tns_adamw_config cfg;
    Part* tiles = nullptr;
    int64_t num_tiles = 0;
};

extern "C" {

int tns_adamw_create(const tns_adamw_config* cfg, int32_t count, const tns_adamw_tensor* tensors, tns_adamw** out) {
    tns::clear_error();
    if (!cfg || !out || (count > 0 && !tensors)) return fail(TNS_EINVAL, "null configuration, tensors or output pointer");
    if (count < 0) return fail(TNS_EINVAL, "negative number of tensors");
    if (!(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0 && cfg->beta2 >= 0.0 && cfg->beta2 < 1.0)) return fail(TNS_EINVAL, "beta1 and beta2 must be in [0, 1)");
    if (!(cfg->eps >= 0.0 && std::isfinite(cfg->eps))) return fail(TNS_EINVAL, "eps must be finite and not negative");
    if (cfg->state_bits != 8 && cfg->state_bits != 32) return fail(TNS_EINVAL, "states have 8 or 32 bits");
    if (cfg->grad_dtype != TNS_F32 && cfg->grad_dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown grad_dtype");
    if (cfg->device < 0 || cfg->reserved) return fail(TNS_EINVAL, "negative device ordinal or reserved field in use");
    int64_t total = 0;
    for (int32_t i = 0; i < count; ++i) {
        const tns_adamw_tensor& t = tensors[i];
        if (t.n < 0) return fail(TNS_EINVAL, "negative number of weights");
        if (t.n > (int64_t)1 << 36) return fail(TNS_ESIZE, "more than 2^36 weights in one tensor");
        if (t.n && (!t.d_param || !t.d_grad || !t.d_m || !t.d_v)) return fail(TNS_EINVAL, "null weights, gradient or state");
        if (t.n && cfg->state_bits == 8 && (!t.d_m_scale || !t.d_v_scale)) return fail(TNS_EINVAL, "null scales of a state of 8 bits");
        if (!std::isfinite(t.weight_decay)) return fail(TNS_EINVAL, "weight_decay must be finite");
        total += (t.n + kTile - 1) / kTile;
        if (total >= (int64_t)1 << 24) return fail(TNS_ESIZE, "more than 2^36 weights in all");      // a launch has fewer than 2^32 threads
    }
    DeviceGuard guard(cfg->device);
    if (guard.error() != hipSuccess) return fail_hip(guard.error(), "selecting the optimizer's device");
    tns_adamw* opt = nullptr;
    try {
        opt = new tns_adamw();
        opt->cfg = *cfg;
        opt->num_tiles = total;
        std::vector<Part> tiles;
        tiles.reserve(total);
        uint64_t word = 0;
        for (int32_t i = 0; i < count; ++i) {
            const tns_adamw_tensor& t = tensors[i];
            auto at = [](const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; };
            const size_t state = cfg->state_bits / 2, grad = cfg->grad_dtype == TNS_F32 ? 16 : 8;      // bytes of four values
            const bool all = at(t.d_param, 16) && at(t.d_copy, 8) && at(t.d_grad, grad) && at(t.d_m, state) && at(t.d_v, state);
            for (int64_t k = 0; k < t.n; k += kTile) {
                auto from = [&](const void* p, size_t bytes) { return p ? (void*)((char*)p + k * bytes) : nullptr; };
                auto scales = [&](float* p) { return p ? p + k / kBlock : nullptr; };
                tiles.push_back({(float*)from(t.d_param, 4), (bf16*)from(t.d_copy, 2), from(t.d_grad, grad / 4), from(t.d_m, state / 4), from(t.d_v, state / 4),
                                 scales(t.d_m_scale), scales(t.d_v_scale), word + (uint64_t)k / 4, (int32_t)std::min<int64_t>(t.n - k, kTile), all, (float)t.weight_decay});
            }
            word += (uint64_t)((t.n + kBlock - 1) / kBlock) * (kBlock / 4);
        }
        if (total) {
            hipError_t e = tns::device_malloc((void**)&opt->tiles, tiles.size() * sizeof(Part));
            if (e == hipSuccess) e = hipMemcpy(opt->tiles, tiles.data(), tiles.size() * sizeof(Part), hipMemcpyHostToDevice);
            if (e != hipSuccess) {
                tns_adamw_destroy(opt);
                return fail_hip(e, "copying the optimizer's table");
            }
        }
    } catch (const std::bad_alloc&) {
        tns_adamw_destroy(opt);
        return fail(TNS_ENOMEM, "host allocation failed");
    }
    *out = opt;
    return TNS_OK;
}

int tns_adamw_step(tns_adamw* opt, double lr, int64_t t, const float* d_grad_scale, void* hip_stream) {
    tns::clear_error();
    if (!opt) return fail(TNS_EINVAL, "null optimizer");
    if (t < 1) return fail(TNS_EINVAL, "steps count from 1");
    if (!std::isfinite(lr)) return fail(TNS_EINVAL, "lr must be finite");
    if (opt->num_tiles == 0) return TNS_OK;
    DeviceGuard guard(opt->cfg.device);
    if (guard.error() != hipSuccess) return fail_hip(guard.error(), "selecting the optimizer's device");
    const tns_adamw_config& c = opt->cfg;
    const Step s{(float)c.beta1, (float)(1.0 - c.beta1), (float)c.beta2, (float)(1.0 - c.beta2), (float)lr,
                 (float)(lr / (1.0 - std::pow(c.beta1, (double)t))), (float)(1.0 / std::sqrt(1.0 - std::pow(c.beta2, (double)t))), (float)c.eps,
                 mix64(c.seed + kGolden * (uint64_t)t)};
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)opt->num_tiles), dim3(256), 0, static_cast<hipStream_t>(hip_stream), opt->tiles, s, d_grad_scale);
    };
    if (c.state_bits == 32) c.grad_dtype == TNS_F32 ? launch(k_adamw<32, float>) : launch(k_adamw<32, bf16>);
    else c.grad_dtype == TNS_F32 ? launch(k_adamw<8, float>) : launch(k_adamw<8, bf16>);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, "tns_adamw_step");
}

int tns_adamw_destroy(tns_adamw* opt) {
    if (!opt) return TNS_OK;
    DeviceGuard guard(opt->cfg.device);
    if (guard.error() == hipSuccess) {
        (void)hipDeviceSynchronize();
        if (opt->tiles) (void)hipFree(opt->tiles);
    }
    delete opt;
    return TNS_OK;
}

}  // extern "C"
