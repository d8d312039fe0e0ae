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

// K values at once over a workgroup, in a fixed order; the same values for all threads.  `s_part` is used for this alone (so that one barrier is enough).
template <int THREADS, int K, typename Op>
__device__ __forceinline__ void over_workgroup(float (&v)[K], float (&s_part)[K][16], const Op& op) {
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = over_lanes(v[k], kWave, op);
    if constexpr (THREADS > kWave) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) s_part[k][threadIdx.x >> 6] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k] = s_part[k][0];
#pragma unroll
            for (int w = 1; w < THREADS / kWave; ++w) v[k] = op(v[k], s_part[k][w]);
        }
    } else {
        __syncthreads();
    }
}

// `count` values of a row from `piece` on, as THREADS threads hold them: sixteen bytes at a time from aligned addresses on, so the first vector
// begins `skew` values before the piece.  What lies outside the piece is not touched; its places hold -infinity.
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
            if (at >= 0 && at + VEC <= count) {
                raw[j] = *reinterpret_cast<const Vec*>(piece + at);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i) raw[j].v[i] = at + i >= 0 && at + i < count ? piece[at + i] : as_value<T>(-kInf);
            }
        }
    }
    __device__ __forceinline__ float get(int j, int i) const { return as_float(raw[j].v[i]); }
    __device__ __forceinline__ float top() const {
        float v = -kInf;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) v = fmaxf(v, get(j, i));
        return v;
    }
    __device__ __forceinline__ float sum(float base, float by) const {
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) v += __builtin_amdgcn_exp2f((get(j, i) - base) * by);
        return v;
    }
    // With the same skew as the vectors were read with, or value by value.  STREAM: with the non-temporal hint.
    template <bool STREAM>
    __device__ __forceinline__ static void write(T* piece, int count, int skew, bool same, int j, const float (&v)[VEC]) {
        const int at = first(j, skew);
        if (same && at >= 0 && at + VEC <= count) {
            Vec out;
#pragma unroll
            for (int i = 0; i < VEC; ++i) out.v[i] = as_value<T>(v[i]);
            using Words = uint32_t __attribute__((ext_vector_type(4)));
            if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(Words, out), reinterpret_cast<Words*>(piece + at));
            else *reinterpret_cast<Vec*>(piece + at) = out;
        } else if (at > -VEC && at < count) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (at + i >= 0 && at + i < count) piece[at + i] = as_value<T>(v[i]);
        }
    }
};

__device__ __forceinline__ float base_of(float top) { return top == -kInf ? 0.0f : top; }

// What is known of a row's ids, in LDS.
struct Ids {
    int32_t* id;                        // -1 outside the candidates
    float *p, *x;                       // teacher's probability (before it: score); student's score
    __device__ Ids(float* mem, int K) : id(reinterpret_cast<int32_t*>(mem)), p(mem + K), x(mem + 2 * K) {}
};
constexpr size_t ids_bytes(int K) { return (size_t)K * 12; }

// Reads them; the largest of the teacher's scores that the thread has seen.
template <typename T, int THREADS>
__device__ __forceinline__ float read_ids(const Distill<T>& d, int64_t row, const Ids& ids) {
    float top = -kInf;
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const int32_t id = d.ids[row * d.K + k];
        const bool is = id >= 0 && id < d.V;
        const float t = is ? d.teacher[row * d.K + k] : -kInf;
        ids.id[k] = is ? id : -1;
        ids.p[k] = t;
        ids.x[k] = is ? as_float(d.logits[row * d.ld + id]) : 0.0f;
        top = fmaxf(top, t);
    }
    return top;
}

// Sums over a row: of p, of p log p, of p (student's score - largest) / temperature.
struct Terms {
    float mass, entropy, score;
};
// log p = (teacher's score - from) / temperature - lse: without d_lse from the largest of them on and with the logarithm of their sum by it, since that
// logarithm added to a far one, and one over the temperature times the lowest number, would be rounded away or infinite.
template <typename T, int THREADS>
__device__ __forceinline__ Terms terms_of(const Distill<T>& d, const Ids& ids, float from, float lse, float base) {
    Terms t = {0.0f, 0.0f, 0.0f};
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const float l = (ids.p[k] - from) * d.rate - lse, p = expf(l);
        ids.p[k] = p;
        t.mass += p;
        if (p != 0.0f) {
            t.entropy += p * l;
            t.score += p * ((ids.x[k] - base) * d.rate);
        }
    }
    return t;
}
template <typename T>
__device__ __forceinline__ float teacher_sum(const Distill<T>& d, const Ids& ids, float base, int threads) {
    float sum = 0.0f;
    for (int k = threadIdx.x; k < d.K; k += threads) sum += expf((ids.p[k] - base) * d.rate);
    return sum;
}
// (no entry: every p is exp(-infinity))
__device__ __forceinline__ float teacher_lse(float sum) { return sum > 0.0f || sum != sum ? logf(sum) : 0.0f; }
// The others' mass, and 0 without d_lse.
template <typename T>
__device__ __forceinline__ float rest_of(const Distill<T>& d, float mass) { return !d.lse ? 0.0f : mass == mass ? fmaxf(1.0f - mass, 0.0f) : mass; }

// Of a row's scores, or a piece of them: the largest, and the sum of exp(rate (score - largest)).  With d_lse the same of those that no id names: their
// sum by their own largest, since by that of all it would be zero where a named one lies some ninety temperatures above them.
struct Stats {
    float top, others_top, all, others;
};
// exp(rate (others' largest - largest)): what the others' exponentials are by the largest of all.  0 where there are none.
__device__ __forceinline__ float others_scale(const Stats& s, float by) { return s.others == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((base_of(s.others_top) - base_of(s.top)) * by); }
__device__ __forceinline__ float loss_of(const Terms& t, float rest, const Stats& s, float rate) {
    const float log_all = logf(s.all);
    float l = t.entropy - t.score + (t.mass != 0.0f ? t.mass * log_all : 0.0f);
    if (rest != 0.0f) l += rest * (logf(rest) - (logf(s.others) + (base_of(s.others_top) - base_of(s.top)) * rate - log_all));
    return l;
}

// Gradient of a row's piece from the whole row's statistics.  By a named candidate it is q (mass + rest) - p, by another one q (mass + rest) -
// rest exp(.) / others, both times c; with d_lse (REST) the latter's exponential is by the others' largest, and q's factor is brought there.  All are written
// as others first, then the named ones once more, by the threads that have them: a workgroup's stores of one address stay in order over the barrier.
template <bool REST, bool STREAM, typename T, int THREADS, int NV>
__device__ __forceinline__ void write_grad(const Distill<T>& d, const Held<T, THREADS, NV>& held, int64_t row, int64_t begin, int count, int skew, const Stats& s, float mass, float rest,
                                           float weight, const Ids& ids, bool twice, T* dlogits) {
    using H = Held<T, THREADS, NV>;
    const float base = base_of(s.top), by = d.rate * kLog2e, c = d.scale * d.rate * weight, named = c * (mass + rest) * (1.0f / s.all);
    float other = named, other_base = base;
    if (REST) {
        other = named * others_scale(s, by);
        if (rest != 0.0f && s.others != 0.0f) other -= c * rest / s.others;
        other_base = base_of(s.others_top);
    }
    T* const to = dlogits + row * d.V + begin;
    const bool same = H::skew_of(to) == skew;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float g[H::VEC];
#pragma unroll
        for (int i = 0; i < H::VEC; ++i) g[i] = __builtin_amdgcn_exp2f((held.get(j, i) - other_base) * by) * other;
        H::template write<STREAM>(to, count, skew, same, j, g);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const int64_t at = ids.id[k] - begin;
        if (ids.id[k] < 0 || at < 0 || at >= count) continue;
        float p = ids.p[k];
        if (twice) {                    // (threads of the same id add up the same terms in the same order)
            p = 0.0f;
            for (int i = 0; i < d.K; ++i) p += ids.id[i] == ids.id[k] ? ids.p[i] : 0.0f;
        }
        to[at] = as_value<T>(__builtin_amdgcn_exp2f((ids.x[k] - base) * by) * named - c * p);
    }
}

// A row of weight 0, or without any p: zeros.
template <typename T, int THREADS>
__device__ __forceinline__ void nothing(const Distill<T>& d, int64_t row, int64_t begin, int64_t count, float* rows, T* dlogits) {
    if (threadIdx.x == 0 && begin == 0) rows[row] = 0.0f;
    if (dlogits) tns::zero_values(dlogits + row * d.V + begin, count, threadIdx.x, THREADS);
}

// Whether no lower k has the same id: of a candidate that is named more than once the lowest k's thread adds it to the named, whichever comes first.
__device__ __forceinline__ bool first_of(const int32_t* ids, int k) {
    for (int i = 0; i < k; ++i)
        if (ids[i] == ids[k]) return false;
    return true;
}

// Which candidates of a piece some id names, a bit each, and whether some id came twice.
template <int PLACES>
struct Names {
    uint32_t twice, word[(PLACES + 31) / 32];
    template <int THREADS>
    __device__ __forceinline__ void clear() {
        for (int i = threadIdx.x; i < (PLACES + 31) / 32; i += THREADS) word[i] = 0;
        if (threadIdx.x == 0) twice = 0;
    }
    __device__ __forceinline__ void add(int at) {
        if (atomicOr(&word[at >> 5], 1u << (at & 31)) >> (at & 31) & 1) twice = 1;
    }
};

// A whole row in a workgroup's registers: read once, written once.  Bound by memory where there are many rows: 4000 of 10000 bf16 scores with
// fifty ids, 161 MB in 31 us (5.2 TB/s); with 1024 threads to a row, a bit looked up for every score and bounds checked at every use it was 126 us,
// bound by instructions.  600 rows of 1000 fp32 scores: 4.6 us, four waits one after the other.  REST: the scores that no id names are added up by themselves (what is left
// of the sum over all without the named ones would lose them where they are few) and by their own largest: the row lies in LDS too, the named ones are
// crossed out there, and the threads take their values from it again (one exchange more: a call of 50000 rows of 50 fp32
// scores 34 -> 37 us, one of 4000 rows of 10000 bf16 scores 37 -> 34).
template <typename T, int THREADS, int NV, bool REST>
__global__ void __launch_bounds__(THREADS) k_distill_row(const Distill<T> d, float* rows, T* dlogits) {
    using H = Held<T, THREADS, NV>;
    constexpr int PLACES = THREADS * H::N;
    extern __shared__ float s_mem[];
    __shared__ typename H::Vec s_row[REST ? THREADS * NV : 1];
    __shared__ Names<PLACES> names;
    __shared__ float s_top[2][16], s_lse[1][16], s_sum[5][16];
    const Ids ids(s_mem, d.K);
    const int64_t row = d.first + blockIdx.x;
    const float weight = d.weight ? d.weight[row] : 1.0f;
    if (weight == 0.0f) return nothing<T, THREADS>(d, row, 0, d.V, rows, dlogits);
    const T* const piece = d.logits + row * d.ld;
    const int count = (int)d.V, skew = H::skew_of(piece);
    H held;
    held.read(piece, count, skew);
    names.template clear<THREADS>();
    float top[2];                       // of the row (REST: of the others); of the teacher's (REST: of the named)
    top[1] = read_ids<T, THREADS>(d, row, ids);
    float sum[5] = {};                  // over the row (REST: without the named), over the named, mass, entropy, score
    if (REST) {
#pragma unroll
        for (int j = 0; j < NV; ++j) s_row[j * THREADS + threadIdx.x] = held.raw[j];
        __syncthreads();
        top[1] = -kInf;
    } else {
        top[0] = held.top();
        over_workgroup<THREADS>(top, s_top, Max{});
    }
    for (int k = threadIdx.x; k < d.K; k += THREADS) {
        const int at = ids.id[k];
        if (at < 0) continue;
        names.add(at);
        if (REST) {
            reinterpret_cast<T*>(s_row)[at + skew] = as_value<T>(-kInf);
            top[1] = fmaxf(top[1], ids.x[k]);
        }
    }
    float lse, from = 0.0f, others_top = -kInf;
    if (REST) {
        lse = d.lse[row];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j) held.raw[j] = s_row[j * THREADS + threadIdx.x];
        top[0] = held.top();
        over_workgroup<THREADS>(top, s_top, Max{});
        others_top = top[0];
        top[0] = fmaxf(top[0], top[1]);
    } else {
        from = base_of(top[1]);
        float t[1] = {teacher_sum(d, ids, from, THREADS)};
        over_workgroup<THREADS>(t, s_lse, Add{});
        lse = teacher_lse(t[0]);
    }
    const float base = base_of(top[0]), by = d.rate * kLog2e;
    if (REST)
        for (int k = threadIdx.x; k < d.K; k += THREADS)
            if (ids.id[k] >= 0 && (!names.twice || first_of(ids.id, k))) sum[1] += __builtin_amdgcn_exp2f((ids.x[k] - base) * by);
    const Terms mine = terms_of<T, THREADS>(d, ids, from, lse, base);
    sum[0] = held.sum(REST ? base_of(others_top) : base, by);
    sum[2] = mine.mass;
    sum[3] = mine.entropy;
    sum[4] = mine.score;
    over_workgroup<THREADS>(sum, s_sum, Add{});
    const Terms t = {sum[2], sum[3], sum[4]};
    if (!REST && t.mass == 0.0f) return nothing<T, THREADS>(d, row, 0, d.V, rows, dlogits);
    Stats s = {top[0], REST ? others_top : top[0], sum[0], sum[0]};
    if (REST) s.all = sum[1] + others_scale(s, by) * sum[0];
    const float rest = rest_of(d, t.mass);
    if (threadIdx.x == 0) rows[row] = weight * loss_of(t, rest, s, d.rate);
    if (dlogits) write_grad<REST, false>(d, held, row, 0, count, skew, s, t.mass, rest, weight, ids, names.twice, dlogits);
}

// Rows of several pieces: the pieces' statistics, then their gradients.  200 rows of 500009 fp32 scores: 95 and 142 us before the second pass
// was made to find the rows in the caches (below).
constexpr int kThreads = 256, kVectors = 8, kPieceBytes = kThreads * kVectors * 16;
template <typename T> constexpr int kPiece = (kPieceBytes - 16) / (int)sizeof(T);      // (a vector less: where the row is not aligned)
template <typename T, bool REST>
__global__ void __launch_bounds__(kThreads) k_distill_stats(const Distill<T> d, unsigned pieces, Stats* stats) {
    using H = Held<T, kThreads, kVectors>;
    __shared__ typename H::Vec s_row[REST ? kThreads * kVectors : 1];
    __shared__ Names<kThreads * H::N> names;
    __shared__ float s_top[2][16], s_sum[2][16];
    const int64_t row = d.first + blockIdx.x / pieces, begin = (int64_t)(blockIdx.x % pieces) * kPiece<T>;
    const int count = (int)min(d.V - begin, (int64_t)kPiece<T>);
    if (d.weight && d.weight[row] == 0.0f) return;
    const T* const piece = d.logits + row * d.ld + begin;
    const int skew = H::skew_of(piece);
    H held;
    held.read(piece, count, skew);
    float top[2] = {-kInf, -kInf}, sum[2] = {};      // of all (REST: of the others), of the named
    const float by = d.rate * kLog2e;
    constexpr int NAMED = REST ? kMostIds / kThreads : 0;
    int at[NAMED + 1];                  // the thread's named candidates of the piece, or -1
    float x[NAMED + 1];
    if (REST) {
#pragma unroll
        for (int i = 0; i < NAMED; ++i) {
            const int k = threadIdx.x + i * kThreads;
            const int64_t place = k < d.K ? d.ids[row * d.K + k] - begin : -1;
            at[i] = place >= 0 && place < count ? (int)place : -1;
            x[i] = at[i] >= 0 ? as_float(piece[at[i]]) : -kInf;
            top[1] = fmaxf(top[1], x[i]);
        }
        names.template clear<kThreads>();
#pragma unroll
        for (int j = 0; j < kVectors; ++j) s_row[j * kThreads + threadIdx.x] = held.raw[j];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NAMED; ++i) {
            if (at[i] < 0) continue;
            names.add(at[i]);
            reinterpret_cast<T*>(s_row)[at[i] + skew] = as_value<T>(-kInf);
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kVectors; ++j) held.raw[j] = s_row[j * kThreads + threadIdx.x];
    }
    top[0] = held.top();
    over_workgroup<kThreads>(top, s_top, Max{});
    const float others_top = top[0], base = base_of(fmaxf(top[0], top[1]));
#pragma unroll
    for (int i = 0; i < NAMED; ++i)
        if (at[i] >= 0 && (!names.twice || first_of(d.ids + row * d.K, threadIdx.x + i * kThreads))) sum[1] += __builtin_amdgcn_exp2f((x[i] - base) * by);
    sum[0] = held.sum(base_of(others_top), by);
    over_workgroup<kThreads>(sum, s_sum, Add{});
    if (threadIdx.x) return;
    Stats s = {fmaxf(top[0], top[1]), others_top, sum[0], sum[0]};
    if (REST) s.all = sum[1] + others_scale(s, by) * sum[0];
    stats[row * pieces + blockIdx.x % pieces] = s;
}
template <typename T, bool REST, bool STREAM>
__global__ void __launch_bounds__(kThreads) k_distill_grad(const Distill<T> d, unsigned pieces, unsigned written, const Stats* stats, float* rows, T* dlogits) {
    using H = Held<T, kThreads, kVectors>;
    extern __shared__ float s_mem[];
    __shared__ Names<kThreads * H::N> names;
    __shared__ float s_top[3][16], s_lse[1][16], s_sum[5][16];
    const Ids ids(s_mem, d.K);
    const int64_t row = d.first + blockIdx.x / written, begin = (int64_t)(blockIdx.x % written) * kPiece<T>;
    const int count = (int)min(d.V - begin, (int64_t)kPiece<T>);
    const float weight = d.weight ? d.weight[row] : 1.0f;
    if (weight == 0.0f) return nothing<T, kThreads>(d, row, begin, count, rows, dlogits);
    const T* const piece = d.logits + row * d.ld + begin;
    const int skew = H::skew_of(piece);
    H held;
    if (dlogits) held.read(piece, count, skew);
    names.template clear<kThreads>();
    float top[3] = {-kInf, -kInf, -kInf};      // of all, of the teacher's, of the others
    top[1] = read_ids<T, kThreads>(d, row, ids);
    for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
        top[0] = fmaxf(top[0], stats[row * pieces + i].top);
        top[2] = fmaxf(top[2], stats[row * pieces + i].others_top);
    }
    over_workgroup<kThreads>(top, s_top, Max{});
    const float base = base_of(top[0]), others_base = base_of(top[2]), by = d.rate * kLog2e;
    float sum[5] = {};                  // all, others, mass, entropy, score
    for (int64_t i = threadIdx.x; i < pieces; i += kThreads) {
        const Stats o = stats[row * pieces + i];
        sum[0] += o.all == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((base_of(o.top) - base) * by) * o.all;
        sum[1] += o.others == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((base_of(o.others_top) - others_base) * by) * o.others;
    }
    for (int k = threadIdx.x; k < d.K; k += kThreads) {
        const int64_t at = ids.id[k] - begin;
        if (ids.id[k] >= 0 && at >= 0 && at < count) names.add((int)at);
    }
    float lse, from = 0.0f;
    if (REST) {
        lse = d.lse[row];
    } else {
        from = base_of(top[1]);
        float t[1] = {teacher_sum(d, ids, from, kThreads)};
        over_workgroup<kThreads>(t, s_lse, Add{});
        lse = teacher_lse(t[0]);
    }
    const Terms mine = terms_of<T, kThreads>(d, ids, from, lse, base);
    sum[2] = mine.mass;
    sum[3] = mine.entropy;
    sum[4] = mine.score;
    over_workgroup<kThreads>(sum, s_sum, Add{});
    const Terms t = {sum[2], sum[3], sum[4]};
    if (!REST && t.mass == 0.0f) return nothing<T, kThreads>(d, row, begin, count, rows, dlogits);
    const Stats s = {top[0], top[2], sum[0], sum[1]};
    const float rest = rest_of(d, t.mass);
    if (threadIdx.x == 0 && begin == 0) rows[row] = weight * loss_of(t, rest, s, d.rate);
    if (dlogits) write_grad<REST, STREAM>(d, held, row, begin, count, skew, s, t.mass, rest, weight, ids, names.twice, dlogits);
}

// Sum of the rows' losses, in a fixed order.
__global__ void __launch_bounds__(1024) k_distill_sum(const float* rows, int64_t n, float scale, float* loss) {
    __shared__ float s_part[1][16];
    float sum[1] = {};
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < n; i += 1024) sum[0] += rows[i];
    over_workgroup<1024>(sum, s_part, Add{});
    if (threadIdx.x == 0) *loss = scale * sum[0];
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
    const size_t lds = ids_bytes(a.K);
    auto row = [&](auto threads, auto vectors) {
        auto with = [&](auto kernel) {  // launches of at most 2^31 threads
            const int64_t most = ((int64_t)1 << 31) / threads();
            for (d.first = 0; d.first < a.B; d.first += most)
                hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(a.B - d.first, most)), dim3(threads()), lds, stream, d, rows, dlogits);
        };
        if (a.d_lse) with(k_distill_row<T, threads(), vectors(), true>);
        else with(k_distill_row<T, threads(), vectors(), false>);
    };
    using std::integral_constant;
    // (a vector less: where the row is not aligned)
    if (a.V <= (64 * 1 - 1) * VEC) row(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    else if (a.V <= (64 * 4 - 1) * VEC) row(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    else if (a.V <= (256 * 2 - 1) * VEC) row(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    else if (a.V <= (256 * 4 - 1) * VEC) row(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    else if (a.V <= (256 * 6 - 1) * VEC) row(integral_constant<int, 256>{}, integral_constant<int, 6>{});
    else if (a.V <= (512 * 4 - 1) * VEC) row(integral_constant<int, 512>{}, integral_constant<int, 4>{});
    else if (a.V <= (512 * 6 - 1) * VEC) row(integral_constant<int, 512>{}, integral_constant<int, 6>{});
    else {
        const unsigned pieces = (unsigned)pieces_of<T>(a.V), written = dlogits ? pieces : 1;
        // Scores beyond the last-level cache (256 MiB) go through in parts that it holds: the second kernel finds there what the first has
        // read, and writes past it.  200 rows of 500009 fp32 scores, 400 MB: 241 us at once, 225 with the hint on the stores, 213 in parts of
        // 192 MiB (now 214), 228 of 96, 266 of 48 (without the hint 251, 246, 278).
        const size_t bytes = (size_t)a.B * a.V * sizeof(T);
        const int64_t parts = bytes > size_t(256) << 20 ? (int64_t)(bytes / (size_t(192) << 20)) + 1 : 1;
        const int64_t most = std::max<int64_t>(std::min((a.B + parts - 1) / parts, ((int64_t)1 << 31) / kThreads / pieces), 1);
        for (d.first = 0; d.first < a.B; d.first += most) {
            const unsigned n = (unsigned)std::min(a.B - d.first, most);
            auto with = [&](auto rest) {
                hipLaunchKernelGGL((k_distill_stats<T, rest()>), dim3(n * pieces), dim3(kThreads), 0, stream, d, pieces, stats);
                if (parts > 1) hipLaunchKernelGGL((k_distill_grad<T, rest(), true>), dim3(n * written), dim3(kThreads), lds, stream, d, pieces, written, stats, rows, dlogits);
                else hipLaunchKernelGGL((k_distill_grad<T, rest(), false>), dim3(n * written), dim3(kThreads), lds, stream, d, pieces, written, stats, rows, dlogits);
            };
            if (a.d_lse) with(std::true_type{});
            else with(std::false_type{});
        }
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
