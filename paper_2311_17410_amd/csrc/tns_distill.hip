// Loss of a student's scores of all candidates against a teacher's highest ones, and its gradient (include/tns_layer.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "../../include/tns_layer.h"
#include "tns_internal.h"
#include "tns_sums.h"
#include "tns_values.h"

using tns::Add;
using tns::as_float;
using tns::as_value;
using tns::bf16;
using tns::fail;
using tns::fail_hip;
using tns::kLog2e;
using tns::Max;
using tns::over_lanes;

namespace {

constexpr int kWave = 64, kMostIds = 1024;
constexpr float kInf = __builtin_inff();

template <typename T>
struct Distill {                        // tns_distill_desc with its types; a launch has the rows from `first` on
    int64_t first, V, ld;
    int K;
    const T* logits;
    const int32_t* ids;
    const float *teacher, *lse, *weight;
    float rate, scale;                  // rate: 1 / temperature
};

// Over a workgroup, in a fixed order; the same value for all threads.
template <int THREADS, typename Op>
__device__ __forceinline__ float over_workgroup(float v, float* s_part, const Op& op) {
    v = over_lanes(v, kWave, op);
    if constexpr (THREADS > kWave) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s_part[0];
#pragma unroll
        for (int w = 1; w < THREADS / kWave; ++w) v = op(v, s_part[w]);
    }
    return v;
}

// Values of a row from `begin` on, `count` of them, as THREADS threads hold them: sixteen bytes at a time from the row's aligned addresses on,
// so the first vector begins `skew` values before the piece.  What lies outside the piece is not touched.
template <typename T, int THREADS, int NV>
struct Held {
    static constexpr int VEC = 16 / sizeof(T), N = VEC * NV;
    struct alignas(16) Vec { T v[VEC]; };
    Vec raw[NV];

    __device__ static int skew_of(const T* at) { return (int)((reinterpret_cast<uintptr_t>(at) / sizeof(T)) % VEC); }
    __device__ static int first(int j, int skew) { return (j * THREADS + (int)threadIdx.x) * VEC - skew; }      // place of a vector's first value in the piece
    __device__ __forceinline__ void read(const T* piece, int count, int skew) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int at = first(j, skew);
            raw[j] = Vec{};
            if (at >= 0 && at + VEC <= count) raw[j] = *reinterpret_cast<const Vec*>(piece + at);
            else if (at > -VEC && at < count)
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (at + i >= 0 && at + i < count) raw[j].v[i] = piece[at + i];
        }
    }
    // With the same skew as the vectors were read with, or value by value.
    __device__ __forceinline__ static void write(T* piece, int count, int skew, bool same, int j, const float (&v)[VEC]) {
        const int at = first(j, skew);
        if (same && at >= 0 && at + VEC <= count) {
            Vec out;
#pragma unroll
            for (int i = 0; i < VEC; ++i) out.v[i] = as_value<T>(v[i]);
            *reinterpret_cast<Vec*>(piece + at) = out;
        } else if (at > -VEC && at < count) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (at + i >= 0 && at + i < count) piece[at + i] = as_value<T>(v[i]);
        }
    }
};

// A piece's bits of the candidates that some id names.
template <int PIECE>
struct Names {
    uint32_t word[PIECE / 32];
    __device__ bool has(int at) const { return word[at >> 5] >> (at & 31) & 1; }
};
// What all pieces of a row know of the teacher: ids and p in LDS, p's sum, what its entropy adds to the loss, and whether an id of the
// piece is named twice.
struct Teacher {
    float mass, rest, entropy;          // sum of p; of the others; sum of p log p
    bool twice;
};

template <typename T, int THREADS, int PIECE>
__device__ __forceinline__ Teacher teach(const Distill<T>& d, int64_t row, int64_t begin, int count, int32_t* s_id, float* s_p, Names<PIECE>& names, int* s_twice, float* s_part) {
    for (int i = threadIdx.x; i < PIECE / 32; i += THREADS) names.word[i] = 0;
    if (threadIdx.x == 0) *s_twice = 0;
    float top = -kInf;
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const int32_t id = d.ids[row * d.K + k];
        const bool is = id >= 0 && id < d.V;
        const float t = is ? d.teacher[row * d.K + k] * d.rate : -kInf;
        s_id[k] = is ? id : -1;
        s_p[k] = t;
        top = fmaxf(top, t);
    }
    float lse;
    if (d.lse) {
        lse = d.lse[row];
        __syncthreads();
    } else {
        top = over_workgroup<THREADS>(top, s_part, Max{});
        const float base = top == -kInf ? 0.0f : top;
        float sum = 0.0f;
        for (int k = threadIdx.x; k < d.K; k += THREADS) sum += expf(s_p[k] - base);
        sum = over_workgroup<THREADS>(sum, s_part, Add{});
        lse = sum > 0.0f || sum != sum ? base + logf(sum) : 0.0f;      // (no entry: every p is exp(-infinity))
        __syncthreads();
    }
    float mass = 0.0f, entropy = 0.0f;
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const float l = s_p[k] - lse, p = expf(l);
        s_p[k] = p;
        mass += p;
        entropy += p == 0.0f ? 0.0f : p * l;
        const int64_t at = s_id[k] - begin;
        if (s_id[k] >= 0 && at >= 0 && at < count)
            if (atomicOr(&names.word[at >> 5], 1u << (at & 31)) >> (at & 31) & 1) *s_twice = 1;
    }
    Teacher t;
    t.mass = over_workgroup<THREADS>(mass, s_part, Add{});
    t.entropy = over_workgroup<THREADS>(entropy, s_part, Add{});
    t.rest = d.lse ? fmaxf(1.0f - t.mass, 0.0f) : 0.0f;
    if (t.mass != t.mass) t.rest = t.mass;
    __syncthreads();
    t.twice = *s_twice != 0;
    return t;
}

// Of a row's scores, or a piece of them: the largest, and the sums of exp(rate (score - largest)) over all and over those that no id names.
struct Stats {
    float top, all, others;
};
template <typename T, int THREADS, int NV, int PIECE>
__device__ __forceinline__ Stats stats_of(const Distill<T>& d, const Held<T, THREADS, NV>& held, int count, int skew, bool split, const Names<PIECE>& names, float* s_part) {
    using H = Held<T, THREADS, NV>;
    Stats s = {-kInf, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < H::VEC; ++i) {
            const int at = H::first(j, skew) + i;
            const float v = as_float(held.raw[j].v[i]);
            if (at >= 0 && at < count) s.top = fmaxf(s.top, v);
        }
    s.top = over_workgroup<THREADS>(s.top, s_part, Max{});
    const float base = s.top == -kInf ? 0.0f : s.top, by = d.rate * kLog2e;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < H::VEC; ++i) {
            const int at = H::first(j, skew) + i;
            if (at < 0 || at >= count) continue;
            const float e = __builtin_amdgcn_exp2f((as_float(held.raw[j].v[i]) - base) * by);
            s.all += e;
            if (split && !names.has(at)) s.others += e;
        }
    s.all = over_workgroup<THREADS>(s.all, s_part, Add{});
    if (split) s.others = over_workgroup<THREADS>(s.others, s_part, Add{});
    return s;
}

// Gradient of a row's piece and (`loss`) the row's loss, from the whole row's statistics.
template <typename T, int THREADS, int NV, int PIECE>
__device__ __forceinline__ void finish(const Distill<T>& d, const Held<T, THREADS, NV>& held, int64_t row, int64_t begin, int count, int skew, const Teacher& t, const Stats& s,
                                       float weight, const int32_t* s_id, const float* s_p, const Names<PIECE>& names, float* s_part, bool loss, float* rows, T* dlogits) {
    using H = Held<T, THREADS, NV>;
    const float base = s.top == -kInf ? 0.0f : s.top, by = d.rate * kLog2e, inverse = 1.0f / s.all, c = d.scale * d.rate * weight;
    const T* const logits = d.logits + row * d.ld;
    if (loss) {
        const float log_all = logf(s.all);
        float sum = 0.0f;
        for (int k = threadIdx.x; k < d.K; k += THREADS)
            if (s_p[k] != 0.0f) sum -= s_p[k] * ((as_float(logits[s_id[k]]) - base) * d.rate - log_all);
        sum = over_workgroup<THREADS>(sum, s_part, Add{});
        if (threadIdx.x == 0) {
            float l = t.entropy + sum;
            if (t.rest != 0.0f) l += t.rest * (logf(t.rest) - (logf(s.others) - log_all));
            rows[row] = weight * l;
        }
    }
    if (!dlogits) return;
    // by a named candidate q (mass + rest) - p, by another one q (mass + rest) - rest exp(.) / others, both times c
    const float named = c * (t.mass + t.rest) * inverse, other = t.rest != 0.0f ? named - c * t.rest / s.others : named;
    T* const to = dlogits + row * d.V + begin;
    const bool same = H::skew_of(to) == skew, split = other != named;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float g[H::VEC];
#pragma unroll
        for (int i = 0; i < H::VEC; ++i) {
            const int at = H::first(j, skew) + i;
            const float e = __builtin_amdgcn_exp2f((as_float(held.raw[j].v[i]) - base) * by);
            g[i] = e * (split && at >= 0 && at < count && names.has(at) ? named : other);
        }
        H::write(to, count, skew, same, j, g);
    }
    // then the named ones once more, whole: the workgroup's stores of one address stay in order over the barrier
    __syncthreads();
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const int64_t at = s_id[k] - begin;
        if (s_id[k] < 0 || at < 0 || at >= count) continue;
        float p = s_p[k];
        if (t.twice) {                  // (threads of the same id add up the same terms in the same order)
            p = 0.0f;
            for (int i = 0; i < d.K; ++i) p += s_id[i] == s_id[k] ? s_p[i] : 0.0f;
        }
        const float e = __builtin_amdgcn_exp2f((as_float(logits[s_id[k]]) - base) * by);
        to[at] = as_value<T>(e * named - c * p);
    }
}

// A row of weight 0, or without any p: zeros.
template <typename T, int THREADS>
__device__ __forceinline__ void nothing(const Distill<T>& d, int64_t row, int64_t begin, int64_t count, float* rows, T* dlogits) {
    if (threadIdx.x == 0 && begin == 0) rows[row] = 0.0f;
    if (dlogits)
        for (int64_t i = threadIdx.x; i < count; i += THREADS) dlogits[row * d.V + begin + i] = T{};
}

// A whole row in a workgroup's registers: read once, written once.
template <typename T, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS) k_distill_row(const Distill<T> d, float* rows, T* dlogits) {
    constexpr int PIECE = THREADS * NV * (16 / (int)sizeof(T));
    __shared__ Names<PIECE> names;
    __shared__ int32_t s_id[kMostIds];
    __shared__ float s_p[kMostIds], s_part[16];
    __shared__ int s_twice;
    const int64_t row = d.first + blockIdx.x;
    const float weight = d.weight ? d.weight[row] : 1.0f;
    if (weight == 0.0f) return nothing<T, THREADS>(d, row, 0, d.V, rows, dlogits);
    const T* const piece = d.logits + row * d.ld;
    const int count = (int)d.V, skew = Held<T, THREADS, NV>::skew_of(piece);
    Held<T, THREADS, NV> held;
    held.read(piece, count, skew);
    const Teacher t = teach<T, THREADS>(d, row, 0, count, s_id, s_p, names, &s_twice, s_part);
    if (t.mass == 0.0f && !d.lse) return nothing<T, THREADS>(d, row, 0, d.V, rows, dlogits);
    const Stats s = stats_of(d, held, count, skew, t.rest != 0.0f, names, s_part);
    finish(d, held, row, 0, count, skew, t, s, weight, s_id, s_p, names, s_part, true, rows, dlogits);
}

// Rows of several pieces: the pieces' statistics, then their gradients.
constexpr int kThreads = 1024, kPieceBytes = 1 << 16;
template <typename T> constexpr int kVectors = kPieceBytes / 16 / kThreads;
template <typename T> constexpr int kPiece = kPieceBytes / (int)sizeof(T) - 16 / (int)sizeof(T);      // (a vector less: where the row is not aligned)
template <typename T>
__global__ void __launch_bounds__(kThreads) k_distill_stats(const Distill<T> d, unsigned pieces, Stats* stats) {
    constexpr int NV = kVectors<T>;
    __shared__ Names<kPieceBytes / (int)sizeof(T)> names;
    __shared__ int32_t s_id[kMostIds];
    __shared__ float s_p[kMostIds], s_part[16];
    __shared__ int s_twice;
    const int64_t row = d.first + blockIdx.x / pieces, begin = (int64_t)(blockIdx.x % pieces) * kPiece<T>;
    const int count = (int)min(d.V - begin, (int64_t)kPiece<T>);
    if (d.weight && d.weight[row] == 0.0f) return;
    const T* const piece = d.logits + row * d.ld + begin;
    const int skew = Held<T, kThreads, NV>::skew_of(piece);
    Held<T, kThreads, NV> held;
    held.read(piece, count, skew);
    if (d.lse) teach<T, kThreads>(d, row, begin, count, s_id, s_p, names, &s_twice, s_part);
    const Stats s = stats_of(d, held, count, skew, d.lse != nullptr, names, s_part);
    if (threadIdx.x == 0) stats[row * pieces + blockIdx.x % pieces] = s;
}
template <typename T>
__global__ void __launch_bounds__(kThreads) k_distill_grad(const Distill<T> d, unsigned pieces, unsigned written, const Stats* stats, float* rows, T* dlogits) {
    constexpr int NV = kVectors<T>;
    __shared__ Names<kPieceBytes / (int)sizeof(T)> names;
    __shared__ int32_t s_id[kMostIds];
    __shared__ float s_p[kMostIds], s_part[16];
    __shared__ int s_twice;
    const int64_t row = d.first + blockIdx.x / written, begin = (int64_t)(blockIdx.x % written) * kPiece<T>;
    const int count = (int)min(d.V - begin, (int64_t)kPiece<T>);
    const float weight = d.weight ? d.weight[row] : 1.0f;
    if (weight == 0.0f) return nothing<T, kThreads>(d, row, begin, count, rows, dlogits);
    const T* const piece = d.logits + row * d.ld + begin;
    const int skew = Held<T, kThreads, NV>::skew_of(piece);
    Held<T, kThreads, NV> held;
    if (dlogits) held.read(piece, count, skew);
    const Teacher t = teach<T, kThreads>(d, row, begin, count, s_id, s_p, names, &s_twice, s_part);
    if (t.mass == 0.0f && !d.lse) return nothing<T, kThreads>(d, row, begin, count, rows, dlogits);
    Stats s = {-kInf, 0.0f, 0.0f};
    for (int64_t i = threadIdx.x; i < pieces; i += kThreads) s.top = fmaxf(s.top, stats[row * pieces + i].top);
    s.top = over_workgroup<kThreads>(s.top, s_part, Max{});
    const float base = s.top == -kInf ? 0.0f : s.top;
    for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
        const Stats o = stats[row * pieces + i];
        const float f = __builtin_amdgcn_exp2f((o.top == -kInf ? 0.0f - base : o.top - base) * d.rate * kLog2e);
        s.all += f * o.all;
        s.others += f * o.others;
    }
    s.all = over_workgroup<kThreads>(s.all, s_part, Add{});
    s.others = over_workgroup<kThreads>(s.others, s_part, Add{});
    finish(d, held, row, begin, count, skew, t, s, weight, s_id, s_p, names, s_part, begin == 0, rows, dlogits);
}

// Sum of the rows' losses, in a fixed order.
__global__ void __launch_bounds__(1024) k_distill_sum(const float* rows, int64_t n, float scale, float* loss) {
    __shared__ float s_part[16];
    float sum = 0.0f;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += 1024) sum += rows[i];
    sum = over_workgroup<1024>(sum, s_part, Add{});
    if (threadIdx.x == 0) *loss = scale * sum;
}

// ---- host -------------------------------------------------------------------------------------------------

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }
size_t aligned(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

int check_sizes(int64_t B, int64_t V, int32_t K) {
    if (B < 0) return fail(TNS_EINVAL, "negative number of rows");
    if (B > (int64_t)INT32_MAX || V > (int64_t)INT32_MAX) return fail(TNS_ESIZE, "more than 2^31-1 rows or candidates");
    if (V < 1) return fail(TNS_EINVAL, "no candidates");
    if (K < 0 || K > kMostIds) return fail(TNS_EINVAL, "K must be in [0, 1024]");
    return TNS_OK;
}

// Pieces of a row (the workspace is sized without the type: by the smaller piece of the two).
template <typename T> int64_t pieces_of(int64_t V) { return (V + kPiece<T> - 1) / kPiece<T>; }

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, what);
}

template <typename T>
int launch(const tns_distill_desc& a, float* loss, float* rows, T* dlogits, void* workspace, hipStream_t stream) {
    Distill<T> d = {0, a.V, a.ld_logits, a.K, static_cast<const T*>(a.d_logits), a.d_ids, a.d_teacher, a.d_lse, a.d_weight, (float)(1.0 / a.temperature), (float)a.scale};
    constexpr int VEC = 16 / (int)sizeof(T);
    Stats* const stats = reinterpret_cast<Stats*>(static_cast<char*>(workspace) + aligned(a.B * 4));
    if (!rows) rows = static_cast<float*>(workspace);
    // Launches of at most 2^31 threads, `per` workgroups a row.
    auto in_pieces = [&](int threads, int64_t per, const auto& go) {
        const int64_t most = std::max<int64_t>(((int64_t)1 << 31) / threads / per, 1);
        for (d.first = 0; d.first < a.B; d.first += most) go(dim3((unsigned)(std::min(a.B - d.first, most) * per)));
    };
    // As few threads as hold the row in two vectors each (a vector less: where it is not aligned).
    auto row = [&](auto threads, auto vectors) {
        in_pieces(threads(), 1, [&](dim3 grid) { hipLaunchKernelGGL((k_distill_row<T, threads(), vectors()>), grid, dim3(threads()), 0, stream, d, rows, dlogits); });
    };
    using Two = std::integral_constant<int, 2>;
    using Four = std::integral_constant<int, 4>;
    if (a.V <= 64 * 2 * VEC - VEC) row(std::integral_constant<int, 64>{}, Two{});
    else if (a.V <= 256 * 2 * VEC - VEC) row(std::integral_constant<int, 256>{}, Two{});
    else if (a.V <= 1024 * 2 * VEC - VEC) row(std::integral_constant<int, 1024>{}, Two{});
    else if (a.V <= kPiece<T>) row(std::integral_constant<int, 1024>{}, Four{});
    else {
        const unsigned pieces = (unsigned)pieces_of<T>(a.V), written = dlogits ? pieces : 1;
        in_pieces(kThreads, pieces, [&](dim3 grid) { hipLaunchKernelGGL((k_distill_stats<T>), grid, dim3(kThreads), 0, stream, d, pieces, stats); });
        in_pieces(kThreads, written, [&](dim3 grid) { hipLaunchKernelGGL((k_distill_grad<T>), grid, dim3(kThreads), 0, stream, d, pieces, written, stats, rows, dlogits); });
    }
    hipLaunchKernelGGL(k_distill_sum, dim3(1), dim3(1024), 0, stream, rows, a.B, d.scale, loss);
    return launched("tns_distill");
}

}  // namespace

extern "C" {

int tns_distill_workspace(int64_t B, int64_t V, int32_t K, size_t* bytes) {
    tns::clear_error();
    if (int e = check_sizes(B, V, K)) return e;
    if (bytes) *bytes = aligned((size_t)B * 4) + (V > kPiece<float> ? aligned((size_t)B * pieces_of<float>(V) * sizeof(Stats)) : 0);
    return TNS_OK;
}

int tns_distill(const tns_distill_desc* d, float* d_loss, float* d_rows, void* d_dlogits, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    tns::clear_error();
    if (!d) return fail(TNS_EINVAL, "null description of the scores");
    if (int e = check_sizes(d->B, d->V, d->K)) return e;
    if (d->dtype != TNS_F32 && d->dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if (d->ld_logits < d->V) return fail(TNS_EINVAL, "rows of logits overlap");
    if (!d_loss) return fail(TNS_EINVAL, "null loss");
    if (d->B > 0 && !d->d_logits) return fail(TNS_EINVAL, "null logits");
    if (d->B > 0 && d->K > 0 && (!d->d_ids || !d->d_teacher)) return fail(TNS_EINVAL, "null ids or teacher");
    if (!(d->temperature > 1e-30) || d->temperature > 1e30) return fail(TNS_EINVAL, "temperature must be above 0");
    const size_t size = d->dtype == TNS_F32 ? 4 : 2;
    if (misaligned(d->d_logits, size) || misaligned(d_dlogits, size)) return fail(TNS_EINVAL, "logits or dlogits is not aligned to its type");
    size_t need = 0;
    if (int e = tns_distill_workspace(d->B, d->V, d->K, &need)) return e;
    if (need && !d_workspace) return fail(TNS_EINVAL, "null workspace");
    if (misaligned(d_workspace, 256)) return fail(TNS_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(TNS_ESIZE, "workspace smaller than asked for");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (d->B == 0) {
        hipLaunchKernelGGL(k_distill_sum, dim3(1), dim3(1024), 0, stream, nullptr, 0, 0.0f, d_loss);
        return launched("tns_distill");
    }
    if (d->dtype == TNS_F32) return launch<float>(*d, d_loss, d_rows, static_cast<float*>(d_dlogits), d_workspace, stream);
    return launch<bf16>(*d, d_loss, d_rows, static_cast<bf16*>(d_dlogits), d_workspace, stream);
}

}  // extern "C"
