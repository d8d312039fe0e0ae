// Paired log-ratio loss of true links against sampled ones, and its gradients (include/tns_train.h).
#include <hip/hip_runtime.h>

#include <algorithm>
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

constexpr int kWaves = 4;
constexpr int64_t kMostGroups = 1 << 16;   // workgroups of a launch; they go round the events
constexpr int kWide = 2048, kWideSingle = 512;      // channels that a wave holds at most, in vectors of four and one by one

// Sums over lanes as vector instructions (a shuffle through the LDS unit is some sixty cycles, and every row of a product waits for one
// sum).  Lanes that have the same sum read each other's in mirrored order, so all of them add the same two values.
template <int CTRL>
__device__ __forceinline__ float moved(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ float add_row16(float v) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_row32(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum over the G lanes that share a row.
template <int G>
__device__ __forceinline__ float row_sum(float v) {
    static_assert(G >= 8);
    v += moved<0xB1>(v);               // quad_perm 1, 0, 3, 2
    v += moved<0x4E>(v);               // quad_perm 2, 3, 0, 1
    v += moved<0x141>(v);              // the other four of eight
    if (G >= 16) v += moved<0x140>(v); // the other eight of sixteen
    if (G >= 32) v = add_row16(v);
    if (G >= 64) v = add_row32(v);
    return v;
}
// Sum over the rows of a wave, of values that are the same for the lanes of a row.
template <int G>
__device__ __forceinline__ float sum_of_rows(float v) {
    if (G <= 8) v += __shfl_xor(v, 8);
    if (G <= 16) v = add_row16(v);
    if (G <= 32) v = add_row32(v);
    return v;
}
// Lane r's of every four lanes.
__device__ __forceinline__ float of_quad(float v, int r) {
    return r == 0 ? moved<0x00>(v) : r == 1 ? moved<0x55>(v) : r == 2 ? moved<0xAA>(v) : moved<0xFF>(v);
}

// Loss of a margin and its slope, both times scale and weight.  softplus(-m) = log(1 + e) + max(-m, 0) with e = exp(-|m|); the logarithm is
// twice the inverse hyperbolic tangent of e / (2 + e), which is a third at most: nine terms of its series leave 1e-10 of it.  The exponent
// is rounded to 32 bits before it is raised: e, which is what loss and slope of a far margin are, has a relative error of (1.5 |m| + 2) 2^-24 at
// most; to put it back costs 4000 events of 50 links half a microsecond of 35, for pairs that hardly count.  A side
// whose factor is 0 is left out: its margin may be infinite.
__device__ __forceinline__ void loss_of(float m, float w, float scale, float smoothing, float& loss, float& slope) {
    const float e = __builtin_amdgcn_exp2f(-fabsf(m) * tns::kLog2e), t = e * __builtin_amdgcn_rcpf(2.0f + e), q = t * t;
    float tail = 1.0f / 17;
    tail = tail * q + 1.0f / 15;
    tail = tail * q + 1.0f / 13;
    tail = tail * q + 1.0f / 11;
    tail = tail * q + 1.0f / 9;
    tail = tail * q + 1.0f / 7;
    tail = tail * q + 1.0f / 5;
    tail = tail * q + 1.0f / 3;
    tail = 2.0f * t * (tail * q + 1.0f);
    const float down = smoothing < 1.0f ? fmaxf(-m, 0.0f) : 0.0f, up = smoothing > 0.0f ? fmaxf(m, 0.0f) : 0.0f;
    loss = scale * w * (tail + down * (1.0f - smoothing) + up * smoothing);
    slope = scale * w * (smoothing - (m > 0.0f ? e : 1.0f) * __builtin_amdgcn_rcpf(1.0f + e));      // sigmoid(-m)
    if (m != m) loss = slope = m;
}

// VEC channels of a row as they lie in memory.
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
    T v[VEC];
};
// (`p` is the same for the wave, `bytes` the lane's part of the address: 32 bits.)
template <typename T, int VEC>
__device__ __forceinline__ void load(const T* p, uint32_t bytes, bool there, float (&v)[VEC]) {
    if (there) {
        const Vec<T, VEC> raw = *reinterpret_cast<const Vec<T, VEC>*>(reinterpret_cast<const char*>(p) + bytes);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = as_float(raw.v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = 0.0f;
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void load(const T* p, uint32_t bytes, bool there, Vec<T, VEC>& v) {
    v = Vec<T, VEC>{};
    if (there) v = *reinterpret_cast<const Vec<T, VEC>*>(reinterpret_cast<const char*>(p) + bytes);
}
template <typename T, int VEC>
__device__ __forceinline__ void store(T* p, uint32_t bytes, const float (&v)[VEC]) {
    Vec<T, VEC> raw;
#pragma unroll
    for (int i = 0; i < VEC; ++i) raw.v[i] = as_value<T>(v[i]);
    *reinterpret_cast<Vec<T, VEC>*>(reinterpret_cast<char*>(p) + bytes) = raw;
}

struct Work {                         // how the links of an event are shared out
    int64_t chunks, links;            // parts of an event that workgroups take, links of each
    int waves;                        // of a workgroup on one part: 1 or 4 (and so four parts a workgroup, or one)
    float *losses, *parts, *sums;     // per workgroup; [B * chunks, dim] and [B * chunks, 2] where there are parts to join
};

// The loss and all gradients in one pass over the sampled links: G lanes hold a row, NV vectors of VEC channels each, and the next R rows
// are on their way while R are computed; the anchor and the sum for its gradient stay in registers.  The margins' losses and slopes, a
// hundred instructions each, are computed for R rows at once, by a lane of every four each.  Bound by memory, (2 + K) rows read and written
// for every event: 200 events of 10000 links, 128 fp32 channels, 2.06 GB in 425 us (4.9 TB/s).  Where an event has few links its first and
// last steps show: 4000 of 50, 172 bf16 channels, 146 MB in 34 us (4.3 TB/s; 54 with the
// library's exponential and logarithm and 64-bit indices: bound by instructions); 600 of one: 5.0 us.
template <typename T, int VEC, int G, int NV, bool GRADS>
__global__ void __launch_bounds__(256) k_pairs(const Pairs<T> p, const Work w, float* margin, T* danchor, T* dpos, T* dneg) {
    constexpr int kRows = 64 / G, R = NV * VEC <= 4 ? 4 : NV * VEC <= 8 ? 2 : 1;
    __shared__ float s_acc[kWaves][GRADS ? G * VEC * NV : 1], s_sum[kWaves][3];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), row = lane / G;
    const int part_of = wave % w.waves;                      // which of the part's waves this is
    int at[NV];
    bool there[NV];
    uint32_t col[NV], mine_at[NV];     // bytes of the lane's vectors from a row's begin, and from the begin of the rows side by side
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        at[j] = (j * G + lane % G) * VEC;
        there[j] = at[j] < p.dim;
        col[j] = (uint32_t)at[j] * sizeof(T);
        mine_at[j] = ((uint32_t)row * (uint32_t)p.dim + (uint32_t)at[j]) * sizeof(T);
    }
    float total = 0.0f;
    const int64_t units = p.B * w.chunks, per = kWaves / w.waves;
    for (int64_t first = (int64_t)blockIdx.x * per; first < units; first += (int64_t)gridDim.x * per) {
        const int64_t unit = first + wave / w.waves;
        const bool real = unit < units;
        const int64_t b = real ? unit / w.chunks : 0, k_begin = real ? unit % w.chunks * w.links : 0, k_end = real ? min(k_begin + w.links, p.K) : 0;
        float a[NV][VEC], acc[NV][VEC], dot = 0.0f;
        // The part's links, fewer than 2^30.  Row r of an iteration is link k0 + r * kRows + row; the lane sees to the weight and the loss of
        // one of the R.  (What lanes read of each other is computed without branches.)
        const int count = (int)(k_end - k_begin), r_mine = lane % 4 % R, by = w.waves * kRows * R, of_mine = r_mine * kRows + row;
        const int64_t base = b * p.K + k_begin;
        const T* const neg = p.neg + base * p.dim;
        T* const to = GRADS ? dneg + base * p.dim : nullptr;
        auto weight_of = [&](int k0) {
            const int k = k0 + of_mine;
            const float v = p.weight && count > 0 ? p.weight[base + min(k, count - 1)] : 1.0f;
            return k < count ? v : 0.0f;
        };
        auto ref_of = [&](int k0) { return p.ref && count > 0 ? p.ref[base + min(k0 + of_mine, count - 1)] : 0.0f; };
        auto read = [&](int k0, float weight, Vec<T, VEC> (&n)[R][NV]) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool is = of_quad(weight, r) != 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j) load<T, VEC>(neg + (int64_t)(k0 + r * kRows) * p.dim, mine_at[j], there[j] && is, n[r][j]);
            }
        };
        const int k_first = part_of * kRows * R;
        float weight = weight_of(k_first), weight_next = weight_of(k_first + by), ref = ref_of(k_first), ref_next = ref_of(k_first + by);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float q[VEC];
            load<T, VEC>(p.anchor + b * p.ld_anchor, col[j], there[j], a[j]);
            load<T, VEC>(p.pos + b * p.ld_pos, col[j], there[j], q);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                dot += a[j][i] * q[i];
                acc[j][i] = 0.0f;
            }
        }
        Vec<T, VEC> n[R][NV];
        read(k_first, weight, n);
        const float plus = row_sum<G>(dot);
        float loss_sum = 0.0f, slope_sum = 0.0f, any = 0.0f;
        for (int k0 = k_first; k0 < count; k0 += by) {
            const float weight_after = weight_of(k0 + 2 * by), ref_after = ref_of(k0 + 2 * by);
            Vec<T, VEC> next[R][NV];
            read(k0 + by, weight_next, next);
            float minus = 0.0f;                              // of the lane's row
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int c = 0; c < VEC; ++c) sum += a[j][c] * as_float(n[r][j].v[c]);
                sum = row_sum<G>(sum);
                if (r == r_mine) minus = sum;
            }
            float m = p.beta * (plus - minus - ref), loss, slope;
            loss_of(m, weight, p.scale, p.smoothing, loss, slope);
            const bool read_it = weight != 0.0f;
            m = read_it ? m : 0.0f;
            slope = read_it ? slope * p.beta : 0.0f;
            loss_sum += read_it ? loss : 0.0f;
            any = read_it ? 1.0f : any;
            slope_sum += slope;
            if (margin && k0 + of_mine < count && lane % G < R) margin[base + k0 + of_mine] = m;
            if (GRADS) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float s = of_quad(slope, r);
                    const bool is = of_quad(weight, r) != 0.0f;
#pragma unroll
                    for (int j = 0; j < NV; ++j) {
                        float out[VEC];
#pragma unroll
                        for (int c = 0; c < VEC; ++c) {
                            acc[j][c] -= s * as_float(n[r][j].v[c]);
                            out[c] = is ? -s * a[j][c] : 0.0f;
                        }
                        if (k0 + r * kRows + row < count && there[j]) store<T, VEC>(to + (int64_t)(k0 + r * kRows) * p.dim, mine_at[j], out);
                    }
                }
            }
            weight = weight_next;
            weight_next = weight_after;
            ref = ref_next;
            ref_next = ref_after;
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < NV; ++j) n[r][j] = next[r][j];
        }
        auto sum_up = [&](float v) {                         // over the lanes' rows, and the rows side by side
            if (R >= 2) v += moved<0xB1>(v);
            if (R >= 4) v += moved<0x4E>(v);
            return sum_of_rows<G>(v);
        };
        loss_sum = sum_up(loss_sum);
        slope_sum = sum_up(slope_sum);
        any = sum_up(any);
        if (real) total += loss_sum;
        if (GRADS) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int c = 0; c < VEC; ++c) acc[j][c] = sum_of_rows<G>(acc[j][c]);
            if (w.waves > 1) {                               // the waves' shares, in their order
                __syncthreads();                             // (the part before has been read)
                if (part_of) {
                    if (row == 0)
#pragma unroll
                        for (int j = 0; j < NV; ++j)
#pragma unroll
                            for (int c = 0; c < VEC; ++c) s_acc[wave][at[j] + c] = acc[j][c];
                    if (lane == 0) { s_sum[wave][0] = slope_sum; s_sum[wave][1] = any; }
                }
                __syncthreads();
                if (part_of == 0)
                    for (int k = wave + 1; k < wave + w.waves; ++k) {
                        slope_sum += s_sum[k][0];
                        any += s_sum[k][1];
#pragma unroll
                        for (int j = 0; j < NV; ++j)
#pragma unroll
                            for (int c = 0; c < VEC; ++c) acc[j][c] += s_acc[k][at[j] + c];
                    }
            }
            if (real && part_of == 0 && row == 0) {
                if (w.chunks > 1 && lane == 0) { w.sums[unit * 2] = slope_sum; w.sums[unit * 2 + 1] = any; }
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    if (!there[j]) continue;
                    if (w.chunks > 1) {
#pragma unroll
                        for (int c = 0; c < VEC; ++c) w.parts[unit * p.dim + at[j] + c] = acc[j][c];
                    } else {
                        float q[VEC], da[VEC], dp[VEC];
                        load<T, VEC>(p.pos + b * p.ld_pos, col[j], true, q);
#pragma unroll
                        for (int c = 0; c < VEC; ++c) {
                            da[c] = any != 0.0f ? slope_sum * q[c] + acc[j][c] : 0.0f;
                            dp[c] = any != 0.0f ? slope_sum * a[j][c] : 0.0f;
                        }
                        store<T, VEC>(danchor + b * p.dim, col[j], da);
                        store<T, VEC>(dpos + b * p.dim, col[j], dp);
                    }
                }
            }
        }
    }
    __syncthreads();
    if (lane == 0) s_sum[wave][2] = total;
    __syncthreads();
    if (threadIdx.x == 0) w.losses[blockIdx.x] = (s_sum[0][2] + s_sum[1][2]) + (s_sum[2][2] + s_sum[3][2]);
}

// Rows too wide for a wave's registers: margins and slopes first, a wave for a part of an event's links ...
template <typename T>
__global__ void __launch_bounds__(256) k_pairs_wide(const Pairs<T> p, const Work w, float* margin, float* slopes) {
    __shared__ float s_sum[kWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float total = 0.0f;
    const int64_t units = p.B * w.chunks;
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
        const int64_t b = unit / w.chunks, k_begin = unit % w.chunks * w.links, k_end = min(k_begin + w.links, p.K);
        const T* const a = p.anchor + b * p.ld_anchor;
        float plus = 0.0f;
        for (int c = lane; c < p.dim; c += 64) plus += as_float(a[c]) * as_float(p.pos[b * p.ld_pos + c]);
        plus = row_sum<64>(plus);
        for (int64_t k = k_begin; k < k_end; ++k) {
            const int64_t i = b * p.K + k;
            const float weight = p.weight ? p.weight[i] : 1.0f;
            float m = 0.0f, loss = 0.0f, slope = 0.0f;
            if (weight != 0.0f) {
                float minus = 0.0f;
                for (int c = lane; c < p.dim; c += 64) minus += as_float(a[c]) * as_float(p.neg[i * p.dim + c]);
                m = p.beta * (plus - row_sum<64>(minus) - (p.ref ? p.ref[i] : 0.0f));
                loss_of(m, weight, p.scale, p.smoothing, loss, slope);
            }
            total += loss;
            if (lane == 0 && margin) margin[i] = m;
            if (lane == 0) slopes[i] = slope * p.beta;
        }
    }
    if (lane == 0) s_sum[wave] = total;
    __syncthreads();
    if (threadIdx.x == 0) w.losses[blockIdx.x] = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
}
// ... and the gradients of 256 channels of an event a workgroup.
template <typename T>
__global__ void __launch_bounds__(256) k_pairs_wide_grads(const Pairs<T> p, const float* slopes, T* danchor, T* dpos, T* dneg) {
    const int tiles = (p.dim + 255) / 256;
    for (int64_t at = blockIdx.x; at < p.B * tiles; at += gridDim.x) {
        const int64_t b = at / tiles;
        const int c = (int)(at % tiles) * 256 + threadIdx.x;
        if (c >= p.dim) continue;
        const float a = as_float(p.anchor[b * p.ld_anchor + c]), q = as_float(p.pos[b * p.ld_pos + c]);
        float acc = 0.0f, sum = 0.0f;
        bool any = false;
        for (int64_t i = b * p.K; i < (b + 1) * p.K; ++i) {
            const bool is = !p.weight || p.weight[i] != 0.0f;
            if (is) {
                acc += slopes[i] * as_float(p.neg[i * p.dim + c]);
                sum += slopes[i];
                any = true;
            }
            dneg[i * p.dim + c] = as_value<T>(is ? -slopes[i] * a : 0.0f);
        }
        danchor[b * p.dim + c] = as_value<T>(any ? sum * q - acc : 0.0f);
        dpos[b * p.dim + c] = as_value<T>(any ? sum * a : 0.0f);
    }
}

// Sum of the workgroups' losses (the first workgroup) and, where events were taken in parts, the gradients of anchor and pos from them:
// kColumns channels of an event a workgroup, the parts shared by its threads (2 us without parts, 5 with eleven parts of 200 events).
constexpr int kColumns = 64, kShares = 1024 / kColumns;
template <typename T>
__global__ void __launch_bounds__(1024) k_pairs_join(const Pairs<T> p, const Work w, int64_t groups, float* loss, T* danchor, T* dpos) {
    __shared__ float s_v[1024], s_sum[kShares], s_any[kShares];
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        float sum = 0.0f;
        for (int64_t k = threadIdx.x; k < groups; k += 8 * 1024) {
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = k + r * 1024 < groups ? w.losses[k + r * 1024] : 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) sum += v[r];
        }
        s_v[threadIdx.x] = sum;
        for (int n = 512; n; n /= 2) {
            __syncthreads();
            if ((int)threadIdx.x < n) s_v[threadIdx.x] += s_v[threadIdx.x + n];
        }
        if (threadIdx.x == 0) *loss = s_v[0];
        __syncthreads();
    }
    if (!danchor) return;
    const int64_t b = blockIdx.y;
    const int share = threadIdx.x / kColumns, c = blockIdx.x * kColumns + threadIdx.x % kColumns;
    float acc = 0.0f, sum = 0.0f, any = 0.0f;
    for (int64_t k = share; k < w.chunks; k += 8 * kShares) {
        float v[8], s[8], n[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const int64_t unit = b * w.chunks + min(k + r * kShares, w.chunks - 1);
            const bool is = k + r * kShares < w.chunks;
            v[r] = is && c < p.dim ? w.parts[unit * p.dim + c] : 0.0f;
            s[r] = is ? w.sums[unit * 2] : 0.0f;
            n[r] = is ? w.sums[unit * 2 + 1] : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < 8; ++r) { acc += v[r]; sum += s[r]; any += n[r]; }
    }
    s_v[threadIdx.x] = acc;
    if (threadIdx.x % kColumns == 0) { s_sum[share] = sum; s_any[share] = any; }
    __syncthreads();
    if (share || c >= p.dim) return;
    acc = sum = any = 0.0f;
    for (int k = 0; k < kShares; ++k) {
        acc += s_v[k * kColumns + threadIdx.x];
        sum += s_sum[k];
        any += s_any[k];
    }
    const float a = as_float(p.anchor[b * p.ld_anchor + c]), q = as_float(p.pos[b * p.ld_pos + c]);
    danchor[b * p.dim + c] = as_value<T>(any != 0.0f ? sum * q + acc : 0.0f);
    dpos[b * p.dim + c] = as_value<T>(any != 0.0f ? sum * a : 0.0f);
}

int check(int64_t B, int64_t K, int32_t dim) {
    if (B < 0 || K < 0) return fail(TNS_EINVAL, "negative number of events or links");
    if (B > (int64_t)INT32_MAX || (K && B > ((int64_t)1 << 40) / K)) return fail(TNS_ESIZE, "more than 2^31-1 events or 2^40 links");
    if (dim < 1 || dim > 1 << 16) return fail(TNS_EINVAL, "dim must be in [1, 2^16]");
    return TNS_OK;
}

size_t aligned(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Few events are cut into parts, so that there are some 2048 workgroups of four waves (two for every wave's place of the chip); a part
// has 64 links at least.  A part of few links is one wave's where there are enough of them (4000 events of 50 links, 172 channels in 16
// bits: 34 us, four waves a part 39; 200 events of 10000, 128 channels in 32 bits: 474 us, four waves 423).
struct Workspace {
    Work w;
    float* slopes;                    // [B, K], of rows that may be too wide for a wave
    size_t bytes;
};
Workspace carve(int64_t B, int64_t K, int32_t dim, void* base) {
    Workspace s{};
    const int64_t most = std::max<int64_t>((K + 63) / 64, 1), want = B ? (2048 + B - 1) / B : 1;
    s.w.chunks = std::min(most, want);
    s.w.links = std::max<int64_t>((K + s.w.chunks - 1) / s.w.chunks, 1);
    s.w.chunks = std::max<int64_t>((K + s.w.links - 1) / s.w.links, 1);
    s.w.waves = s.w.links <= (B * s.w.chunks >= 2048 ? 64 : 16) ? 1 : kWaves;
    char* p = static_cast<char*>(base);
    auto take = [&](size_t floats) {
        void* const at = p;
        p += aligned(floats * 4);
        s.bytes += aligned(floats * 4);
        return static_cast<float*>(at);
    };
    const int64_t units = B * s.w.chunks;
    s.w.losses = take(std::min(units, kMostGroups));
    if (s.w.chunks > 1) {
        s.w.parts = take(units * dim);
        s.w.sums = take(units * 2);
    }
    if (dim > kWideSingle) s.slopes = take(B * K);
    return s;
}

template <typename T>
struct Out {
    float *loss, *margin;
    T *danchor, *dpos, *dneg;
};

template <typename T, int VEC, int G, int NV>
int64_t launch(const Pairs<T>& p, const Work& w, const Out<T>& o, hipStream_t stream) {
    const int64_t per = kWaves / w.waves, groups = std::min((p.B * w.chunks + per - 1) / per, kMostGroups);
    if (o.danchor) hipLaunchKernelGGL((k_pairs<T, VEC, G, NV, true>), dim3((unsigned)groups), dim3(256), 0, stream, p, w, o.margin, o.danchor, o.dpos, o.dneg);
    else hipLaunchKernelGGL((k_pairs<T, VEC, G, NV, false>), dim3((unsigned)groups), dim3(256), 0, stream, p, w, o.margin, o.danchor, o.dpos, o.dneg);
    return groups;
}

// Vectors of four channels where every row begins at a multiple of them, else one by one; as few lanes to a row as hold it.
template <typename T>
void run(const Pairs<T>& p, const Workspace& s, const Out<T>& o, hipStream_t stream) {
    const Work& w = s.w;
    auto fits = [](const void* at) { return (reinterpret_cast<uintptr_t>(at) & (4 * sizeof(T) - 1)) == 0; };
    const bool four = p.dim % 4 == 0 && p.ld_anchor % 4 == 0 && p.ld_pos % 4 == 0 && fits(p.anchor) && fits(p.pos) && fits(p.neg) && fits(o.danchor) && fits(o.dpos) && fits(o.dneg);
    int64_t groups = 0;
    bool joined = w.chunks == 1;
    if (p.B > 0) {
        const int d = p.dim;
        if (d > (four ? kWide : kWideSingle)) {
            groups = std::min((p.B * w.chunks + kWaves - 1) / kWaves, kMostGroups);
            hipLaunchKernelGGL((k_pairs_wide<T>), dim3((unsigned)groups), dim3(256), 0, stream, p, w, o.margin, s.slopes);
            if (o.danchor)
                hipLaunchKernelGGL((k_pairs_wide_grads<T>), dim3((unsigned)std::min<int64_t>(p.B * ((d + 255) / 256), kMostGroups)), dim3(256), 0, stream, p, s.slopes,
                                   o.danchor, o.dpos, o.dneg);
            joined = true;
        } else if (four) {
            groups = d <= 32 ? launch<T, 4, 8, 1>(p, w, o, stream) : d <= 64 ? launch<T, 4, 16, 1>(p, w, o, stream) : d <= 128 ? launch<T, 4, 32, 1>(p, w, o, stream)
                     : d <= 256 ? launch<T, 4, 64, 1>(p, w, o, stream) : d <= 512 ? launch<T, 4, 64, 2>(p, w, o, stream)
                     : d <= 1024 ? launch<T, 4, 64, 4>(p, w, o, stream) : launch<T, 4, 64, 8>(p, w, o, stream);
        } else {
            groups = d <= 64 ? launch<T, 1, 64, 1>(p, w, o, stream) : d <= 128 ? launch<T, 1, 64, 2>(p, w, o, stream)
                     : d <= 256 ? launch<T, 1, 64, 4>(p, w, o, stream) : launch<T, 1, 64, 8>(p, w, o, stream);
        }
    }
    T* const da = joined ? nullptr : o.danchor;
    const dim3 grid = da ? dim3((p.dim + kColumns - 1) / kColumns, (unsigned)p.B) : dim3(1);
    hipLaunchKernelGGL((k_pairs_join<T>), grid, dim3(1024), 0, stream, p, w, groups, o.loss, da, o.dpos);
}

}  // namespace

extern "C" {

int tns_pair_loss_workspace(int64_t B, int64_t K, int32_t dim, size_t* bytes) {
    tns::clear_error();
    if (!bytes) return fail(TNS_EINVAL, "null output pointer");
    if (int e = check(B, K, dim)) return e;
    *bytes = carve(B, K, dim, nullptr).bytes;
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
    const Workspace s = carve(p->B, p->K, p->dim, d_workspace);
    const size_t need = s.bytes;
    if (need && !d_workspace) return fail(TNS_EINVAL, "null workspace");
    if (reinterpret_cast<uintptr_t>(d_workspace) & 255) return fail(TNS_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(TNS_ESIZE, "workspace smaller than tns_pair_loss_workspace()");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto go = [&](auto value) {
        using T = decltype(value);
        run(Pairs<T>{p->B, p->K, static_cast<const T*>(p->d_anchor), static_cast<const T*>(p->d_pos), static_cast<const T*>(p->d_neg),
                     p->ld_anchor, p->ld_pos, p->d_ref, p->d_weight, (float)p->beta, (float)p->smoothing, (float)p->scale, p->dim},
            s, Out<T>{d_loss, d_margin, static_cast<T*>(d_danchor), static_cast<T*>(d_dpos), static_cast<T*>(d_dneg)}, stream);
    };
    if (p->dtype == TNS_F32) go(float{});
    else go(bf16{});
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, "tns_pair_loss");
}

}  // extern "C"
