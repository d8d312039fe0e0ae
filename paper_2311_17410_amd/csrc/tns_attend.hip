// Attention of targets over ragged lists of events with a bias by buckets of their age, and its gradients (include/tns_layer.h).
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
using tns::gap_of;
using tns::kLog2e;
using tns::Max;
using tns::over_lanes;
using tns::over_strided;

namespace {

constexpr int kWave = 64, kWaves = 4;      // lanes of a wave, waves of a workgroup
constexpr float kInf = __builtin_inff();
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// tns_attend with its types.  Whatever rowptr holds, a row that is read lies in [0, rows) and a list in [0, S).
template <typename T>
struct Attend {
    int64_t S, rows, num;
    const int64_t* rowptr;
    const T *q, *k, *v;
    int64_t ld_q, ld_k, ld_v;
    const int32_t* index;
    const uint8_t* mask;
    const float *t, *ts, *edges, *table;
    int heads, kv_heads, dim, group, buckets;
    bool newest_first, zero_beyond;
    float scale;

    __device__ int64_t edge(int64_t s) const { return uniform(min(max(rowptr[s], (int64_t)0), rows)); }
    __device__ int64_t total() const { return S ? edge(S) : 0; }
};

// How the work is cut.  A list's first part begins with the list and ends with the first whole block of `1 << part` rows behind its
// begin, or with the list; every further block, as far as the list reaches, is a part of its own.  So a part has less than two blocks,
// lists up to a block are one part, and the parts of a list that has several are numbered by the blocks they end with.
//
// A wave takes a part for some of the heads: `lanes` lanes hold a row of a head of k or v, sixteen bytes each, `wide` heads side by
// side, and the rest of the wave are `slots` events at a time.
struct Cut {
    int part;                           // log2 of a block's rows
    int64_t blocks;                     // of the rows
    int lanes, wide, slots, turns;      // turns: waves that the heads of k and v take
};
struct Part {
    int64_t list, begin, end, slot;     // slot: block that the part is numbered by
    bool any, whole;                    // whole: the list has no other part
};

// The list that holds row p < total: the last one that begins at or before it.  Called by the whole wave, which looks at 64 lists a step.
// (What a ballot votes on is computed without branches.)
template <typename T>
__device__ int64_t find_list(const Attend<T>& a, int64_t p) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = a.S;
    while (hi - lo > 1) {
        const int64_t by = (hi - lo + kWave - 1) / kWave, j = lo + (lane + 1) * by;
        const int64_t at = min(max(a.rowptr[min(j, hi)], (int64_t)0), a.rows);
        const int c = __popcll(__ballot((j < hi) & (at <= p)));
        lo += c * by;
        hi = min(lo + by, hi);
    }
    return uniform(lo);
}

// Of the units, the first S are the lists' first parts, the others the blocks.  The unit of a block also says (`first`) which list has
// its first part end with the block and goes on behind it, or -1.
template <typename T>
__device__ __forceinline__ Part part_of(const Attend<T>& a, const Cut& cut, int64_t unit, int32_t* first) {
    Part w = {};
    const int64_t size = (int64_t)1 << cut.part;
    if (unit < a.S) {
        const int64_t begin = a.edge(unit), end = max(a.edge(unit + 1), begin);
        w.list = unit;
        w.begin = begin;
        w.slot = (begin + size - 1) >> cut.part;
        const int64_t most = (w.slot + 1) << cut.part;
        w.end = min(end, most);
        w.whole = end <= most;
        w.any = true;
        return w;
    }
    w.slot = unit - a.S;
    w.begin = w.slot << cut.part;
    int32_t starts = -1;
    if (w.begin < a.total()) {
        w.list = find_list(a, w.begin);
        const int64_t begin = a.edge(w.list), end = a.edge(w.list + 1), block = (begin + size - 1) >> cut.part;
        w.end = min(end, w.begin + size);
        w.any = block < w.slot && w.begin < end;
        if (block == w.slot && end > w.begin + size) starts = (int32_t)w.list;
    }
    if (first && (threadIdx.x & 63) == 0) first[w.slot] = starts;
    return w;
}

// The lane's sixteen bytes of a row of a head: pieces of VEC channels, the p-th at ((p lanes) + lane) VEC.
template <typename T, int VEC>
struct Row {
    static constexpr int N = 16 / sizeof(T), PIECES = N / VEC;
    struct alignas(VEC * sizeof(T)) Piece { T v[VEC]; };
    union {
        Piece piece[PIECES];
        uint32_t word[4];
    };
    __device__ Row() {}
    __device__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(word[i]);
        else return __uint_as_float(i & 1 ? word[i / 2] & 0xffff0000u : word[i / 2] << 16);
    }
    __device__ __forceinline__ void read(const T* base, const int (&at)[PIECES]) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) piece[p] = *reinterpret_cast<const Piece*>(base + at[p]);
    }
    __device__ __forceinline__ void clear_unless(bool keep) {
#pragma unroll
        for (int i = 0; i < 4; ++i) word[i] = keep ? word[i] : 0u;
    }
    __device__ __forceinline__ void set(const float (&v)[N]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) word[i] = __float_as_uint(v[i]);
        } else {
            using Two = float __attribute__((ext_vector_type(2)));
            using Halves = __bf16 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < 4; ++i) word[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((Two{v[2 * i], v[2 * i + 1]}), Halves));
        }
    }
    __device__ __forceinline__ void write(T* base, const int (&at)[PIECES], const bool (&there)[PIECES]) const {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (there[p]) *reinterpret_cast<Piece*>(base + at[p]) = piece[p];
    }
};

// Where a lane stands in its wave.
template <typename T, int VEC>
struct Place {
    static constexpr int PIECES = Row<T, VEC>::PIECES;
    int lane, slot, kv;                 // kv: head of k and v, the last one again where there are no more (`head`: there is)
    bool head;
    int at[PIECES];                     // channels of the pieces, 0 where there are no more (`there`)
    bool there[PIECES];

    __device__ Place(const Attend<T>& a, const Cut& cut, int turn) {
        lane = threadIdx.x & 63;
        const int of = lane % (cut.lanes * cut.wide);
        slot = lane / (cut.lanes * cut.wide);
        kv = turn * cut.wide + of / cut.lanes;
        head = kv < a.kv_heads;
        kv = min(kv, a.kv_heads - 1);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            at[p] = (p * cut.lanes + of % cut.lanes) * VEC;
            there[p] = at[p] < a.dim;
            at[p] = there[p] ? at[p] : 0;
        }
    }
    // Row of head g of the lane's group in an array [S, heads, dim], zero where there is no such head or channel.
    template <int G, typename U>
    __device__ __forceinline__ void heads(const Attend<T>& a, const U* base, float (&to)[G][Row<T, VEC>::N]) const {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const bool is = head && g < a.group;
            const U* const row = base + (int64_t)(kv * a.group + min(g, a.group - 1)) * a.dim;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                struct alignas(VEC * sizeof(U)) { U v[VEC]; } piece = *reinterpret_cast<const decltype(piece)*>(row + at[p]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) to[g][p * VEC + i] = is && there[p] ? as_float(piece.v[i]) : 0.0f;
            }
        }
    }
};

// Bucket, or -1 for an event that is left out, and row of k and v, of the 64 rows from `row0` on, `n` of them the part's: one a lane.
struct Known {
    int bucket, index;
};
template <typename T>
__device__ __forceinline__ Known known_of(const Attend<T>& a, const Part& w, int64_t list_begin, int64_t list_end, float t, int64_t row0, int n, const float* s_edges, int steps) {
    const int lane = threadIdx.x & 63;
    const int64_t row = row0 + min(lane, n - 1);
    Known o = {0, 0};
    const bool kept = a.mask ? a.mask[row] != 0 : true;
    bool inside = true;
    if (a.index) {
        o.index = a.index[row];
        inside = o.index >= 0 && o.index < a.num;
        o.index = inside ? o.index : 0;
    }
    if (a.buckets > 1) {
        const float age = a.ts ? gap_of(t, a.ts[row]) : (float)(a.newest_first ? row - list_begin : list_end - 1 - row);
        const int edges = a.buckets - 1;
        for (int by = steps; by; by >>= 1) {
            const int to = o.bucket + by;
            const float edge = s_edges[min(to, edges) - 1];
            o.bucket = to <= edges && edge <= age ? to : o.bucket;
        }
    }
    if (!(kept && inside)) o.bucket = -1;
    return o;
}

// Edges and table in LDS, the table in powers of two.
template <typename T>
__device__ __forceinline__ void stage(const Attend<T>& a, float* s_edges, float* s_table) {
    for (int i = threadIdx.x; i < a.buckets - 1; i += kWaves * kWave) s_edges[i] = a.edges[i];
    for (int i = threadIdx.x; i < a.buckets * a.heads; i += kWaves * kWave) s_table[i] = a.table[i] * kLog2e;
    __syncthreads();
}
__device__ __forceinline__ int search_steps(int edges) {
    int by = 1;
    while (by * 2 <= edges) by *= 2;
    return by;
}

struct Work {
    int32_t* first;                     // [blocks]
    float *stats, *acc;                 // [blocks, heads, 2], [blocks, heads, dim]: of the parts of lists that have several
    float* tables;                      // [workgroups of the gradients, buckets * heads]
};

// Scores, running maximum and sum, and the weighted sum of the values in one pass over k and v; what the slots found is joined at the end.
template <typename T, int VEC, int G>
__global__ void __launch_bounds__(kWaves* kWave) k_attend(const Attend<T> a, const Cut cut, const Work work, T* out, float* saved_out, float* saved_lse) {
    extern __shared__ float s_mem[];
    float *const s_edges = s_mem, *const s_table = s_mem + a.buckets;
    constexpr int N = Row<T, VEC>::N, U = 2;
    stage(a, s_edges, s_table);
    const int steps = search_steps(a.buckets - 1), wave = uniform((int)(threadIdx.x >> 6));
    const int64_t units = (a.S + cut.blocks) * cut.turns;
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
        const int turn = (int)(unit % cut.turns);
        const Part w = part_of(a, cut, unit / cut.turns, turn == 0 ? work.first : nullptr);
        if (!w.any) continue;
        const Place<T, VEC> at(a, cut, turn);
        float q[G][N], acc[G][N], m[G], l[G];
        at.template heads<G>(a, a.q + w.list * a.ld_q, q);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            m[g] = -kInf;
            l[g] = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                q[g][i] *= a.scale * kLog2e;
                acc[g][i] = 0.0f;
            }
        }
        const float t = a.t ? a.t[w.list] : 0.0f;
        const int64_t list_begin = a.edge(w.list), list_end = a.edge(w.list + 1);
        for (int64_t row0 = w.begin; row0 < w.end; row0 += kWave) {
            const int n = (int)min(w.end - row0, (int64_t)kWave);
            const Known known = known_of(a, w, list_begin, list_end, t, row0, n, s_edges, steps);
            for (int i0 = 0; i0 < n; i0 += cut.slots * U) {
                Row<T, VEC> k[U], v[U];
                int bucket[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * cut.slots + at.slot, place = min(i, n - 1);
                    bucket[u] = __shfl(known.bucket, place);
                    if (i >= n) bucket[u] = -1;
                    const int64_t row = a.index ? (int64_t)__shfl(known.index, place) : row0 + place;
                    k[u].read(a.k + row * a.ld_k + at.kv * a.dim, at.at);
                    v[u].read(a.v + row * a.ld_v + at.kv * a.dim, at.at);
                }
                float s[U][G];
                bool mixed = false;     // an event that is left out by some of the lane's heads only
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    bool some = false, all = true;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        float dot = 0.0f;
#pragma unroll
                        for (int i = 0; i < N; ++i) dot += q[g][i] * k[u].get(i);
                        dot = over_lanes(dot, cut.lanes, Add{});
                        const float bias = a.buckets && bucket[u] >= 0 ? s_table[bucket[u] * a.heads + at.kv * a.group + min(g, a.group - 1)] : 0.0f;
                        const bool counts = bucket[u] >= 0 && bias != -kInf;
                        s[u][g] = counts ? dot + bias : -kInf;
                        some |= counts;
                        all &= counts;
                    }
                    v[u].clear_unless(some);
                    mixed |= some && !all;
                }
                const bool careful = G > 1 && __ballot(mixed) != 0;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float top = m[g];
#pragma unroll
                    for (int u = 0; u < U; ++u) top = fmaxf(top, s[u][g]);
                    const float base = top == -kInf ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m[g] - base);
                    m[g] = top;
                    l[g] *= keep;
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[g][i] *= keep;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const float p = __builtin_amdgcn_exp2f(s[u][g] - base);
                        l[g] += p;
                        if (careful) {
#pragma unroll
                            for (int i = 0; i < N; ++i) acc[g][i] += s[u][g] == -kInf ? 0.0f : p * v[u].get(i);
                        } else {
#pragma unroll
                            for (int i = 0; i < N; ++i) acc[g][i] += p * v[u].get(i);
                        }
                    }
                }
            }
        }
        const int width = cut.lanes * cut.wide;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float top = over_strided(m[g], width, Max{}), f = m[g] == -kInf ? 0.0f : __builtin_amdgcn_exp2f(m[g] - top);
            l[g] = over_strided(l[g] * f, width, Add{});
            m[g] = top;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[g][i] = over_strided(acc[g][i] * f, width, Add{});
        }
        if (at.slot || !at.head) continue;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g >= a.group) break;
            const int64_t h = at.kv * a.group + g;
            if (!w.whole) {
                const int64_t to = w.slot * a.heads + h;
                if (at.at[0] == 0 && at.there[0]) {
                    work.stats[2 * to] = m[g];
                    work.stats[2 * to + 1] = l[g];
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (at.there[i / VEC]) work.acc[to * a.dim + at.at[i / VEC] + i % VEC] = acc[g][i];
                continue;
            }
            const int64_t to = w.list * a.heads + h;
            const float inverse = l[g] == 0.0f ? 0.0f : 1.0f / l[g];
#pragma unroll
            for (int i = 0; i < N; ++i) acc[g][i] *= inverse;
            Row<T, VEC> row;
            row.set(acc[g]);
            row.write(out + to * a.dim, at.at, at.there);
            if (saved_out) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (at.there[i / VEC]) saved_out[to * a.dim + at.at[i / VEC] + i % VEC] = acc[g][i];
                if (at.at[0] == 0 && at.there[0]) saved_lse[to] = l[g] == 0.0f ? kInf : m[g] + __log2f(l[g]);
            }
        }
    }
}

// The blocks of the calling workgroup's share that a list with several parts begins with, `count` of them, in s_list (of 1024 threads).
__device__ __forceinline__ int starts_of(const Work& work, int64_t blocks, int64_t first, int64_t by, int32_t* s_list, int64_t* s_block, int* s_count) {
    if (threadIdx.x == 0) *s_count = 0;
    __syncthreads();
    const int64_t block = first + threadIdx.x * by;
    const int32_t list = block < blocks ? work.first[block] : -1;
    if (list >= 0) {
        const int at = atomicAdd(s_count, 1);              // (in any order: each is taken on its own)
        s_list[at] = list;
        s_block[at] = block;
    }
    __syncthreads();
    return *s_count;
}
// Sum over the parts that the threads of a channel have, in a fixed order; s_sum has 1024 places.
__device__ __forceinline__ float over_parts(float v, int wide, float* s_sum) {
    __syncthreads();
    s_sum[threadIdx.x] = v;
    for (int n = 512; n >= wide; n /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < n) s_sum[threadIdx.x] += s_sum[threadIdx.x + n];
    }
    __syncthreads();
    return s_sum[threadIdx.x % wide];
}

// Joins the parts of the lists that have several: a workgroup for a head of a list, a thread for a channel of every so many parts.
template <typename T>
__global__ void __launch_bounds__(1024) k_attend_join(const Attend<T> a, const Cut cut, const Work work, int groups, int channels, T* out, float* saved_out, float* saved_lse) {
    __shared__ float s_sum[1024];
    __shared__ int32_t s_list[1024];
    __shared__ int64_t s_block[1024];
    __shared__ int s_count;
    const int64_t h = blockIdx.x % a.heads, share = blockIdx.x / a.heads;
    const int ch = threadIdx.x % channels, mine = threadIdx.x / channels, parts = 1024 / channels;
    for (int64_t first = share; first < cut.blocks; first += (int64_t)groups * 1024) {
        const int count = starts_of(work, cut.blocks, first, groups, s_list, s_block, &s_count);
        for (int j = 0; j < count; ++j) {
            const int64_t list = s_list[j], begin = s_block[j], end = min((a.edge(list + 1) + ((int64_t)1 << cut.part) - 1) >> cut.part, cut.blocks);
            float top = -kInf;
            for (int64_t b = begin + threadIdx.x; b < end; b += 1024) top = fmaxf(top, work.stats[2 * (b * a.heads + h)]);
            top = over_lanes(top, kWave, Max{});
            __syncthreads();
            if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = top;
            __syncthreads();
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s_sum[i]);
            const float base = top == -kInf ? 0.0f : top;
            float l = 0.0f, acc = 0.0f;
            const int c = min(ch, a.dim - 1);
#pragma unroll 4
            for (int64_t b = begin + mine; b < end; b += parts) {
                const int64_t at = b * a.heads + h;
                const float f = __builtin_amdgcn_exp2f(work.stats[2 * at] - base);
                l += f * work.stats[2 * at + 1];
                acc += f * work.acc[at * a.dim + c];
            }
            l = over_parts(l, channels, s_sum);
            acc = over_parts(acc, channels, s_sum);
            if (mine == 0 && ch < a.dim) {
                const int64_t to = list * a.heads + h;
                acc = l == 0.0f ? 0.0f : acc / l;
                out[to * a.dim + ch] = as_value<T>(acc);
                if (saved_out) {
                    saved_out[to * a.dim + ch] = acc;
                    if (ch == 0) saved_lse[to] = l == 0.0f ? kInf : top + __log2f(l);
                }
            }
        }
        __syncthreads();
    }
}

// Zeros in the values from..to of an array, by a wave.
template <typename T>
__device__ void zero_values(T* base, int64_t from, int64_t to) {
    for (int64_t i = from + (threadIdx.x & 63); i < to; i += kWave) base[i] = T{};
}

// One pass over k and v: the scores again, p from the saved logarithm of their sum, and all gradients of the event while its rows are in
// registers.  The table's gradient is summed up by every wave in LDS, one slot after the other, so in a fixed order.
template <typename T, int VEC, int G>
__global__ void __launch_bounds__(kWaves* kWave) k_attend_grad(const Attend<T> a, const Cut cut, const Work work, const float* saved_out, const float* saved_lse, const T* dout, T* dq,
                                                               T* dk, T* dv, bool tables) {
    extern __shared__ float s_mem[];
    const int entries = a.buckets * a.heads;
    float *const s_edges = s_mem, *const s_table = s_mem + a.buckets, *const s_sums = s_table + entries;
    constexpr int N = Row<T, VEC>::N, U = 1;
    if (tables)
        for (int i = threadIdx.x; i < kWaves * entries; i += kWaves * kWave) s_sums[i] = 0.0f;
    stage(a, s_edges, s_table);
    const int steps = search_steps(a.buckets - 1), wave = uniform((int)(threadIdx.x >> 6));
    float* const s_mine = s_sums + wave * entries;
    const int64_t units = (a.S + cut.blocks) * cut.turns, row_of = (int64_t)a.kv_heads * a.dim;
    for (int64_t unit = (int64_t)blockIdx.x * kWaves + wave; unit < units; unit += (int64_t)gridDim.x * kWaves) {
        const int turn = (int)(unit % cut.turns);
        const Part w = part_of(a, cut, unit / cut.turns, turn == 0 ? work.first : nullptr);
        if (a.zero_beyond && turn == 0 && unit / cut.turns >= a.S) {
            const int64_t from = max(w.slot << cut.part, a.total()), to = min((w.slot + 1) << cut.part, a.rows);
            zero_values(dk, from * row_of, to * row_of);
            zero_values(dv, from * row_of, to * row_of);
        }
        if (!w.any) continue;
        const Place<T, VEC> at(a, cut, turn);
        float q[G][N], d[G][N], acc[G][N], lse[G], delta[G];
        at.template heads<G>(a, saved_out + w.list * a.heads * a.dim, acc);
        at.template heads<G>(a, dout + w.list * a.heads * a.dim, d);
        at.template heads<G>(a, a.q + w.list * a.ld_q, q);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                dot += d[g][i] * acc[g][i];
                q[g][i] *= a.scale * kLog2e;
                acc[g][i] = 0.0f;
            }
            delta[g] = over_lanes(dot, cut.lanes, Add{});
            lse[g] = g < a.group ? saved_lse[w.list * a.heads + at.kv * a.group + g] : kInf;
        }
        const float t = a.t ? a.t[w.list] : 0.0f;
        const int64_t list_begin = a.edge(w.list), list_end = a.edge(w.list + 1);
        for (int64_t row0 = w.begin; row0 < w.end; row0 += kWave) {
            const int n = (int)min(w.end - row0, (int64_t)kWave);
            const Known known = known_of(a, w, list_begin, list_end, t, row0, n, s_edges, steps);
            for (int i0 = 0; i0 < n; i0 += cut.slots * U) {
                Row<T, VEC> k[U], v[U];
                int bucket[U], row[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    row[u] = i0 + u * cut.slots + at.slot;
                    const int place = min(row[u], n - 1);
                    bucket[u] = __shfl(known.bucket, place);
                    if (row[u] >= n) bucket[u] = -1;
                    k[u].read(a.k + (row0 + place) * a.ld_k + at.kv * a.dim, at.at);
                    v[u].read(a.v + (row0 + place) * a.ld_v + at.kv * a.dim, at.at);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float p[G], ds[G], to_k[N], to_v[N];
                    bool counts[G], some = false, all = true;
#pragma unroll
                    for (int i = 0; i < N; ++i) to_k[i] = to_v[i] = 0.0f;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float bias = a.buckets && bucket[u] >= 0 ? s_table[bucket[u] * a.heads + at.kv * a.group + min(g, a.group - 1)] : 0.0f;
                        counts[g] = bucket[u] >= 0 && bias != -kInf && g < a.group;
                        some |= counts[g];
                        all &= counts[g] || g >= a.group;
                        ds[g] = bias;
                    }
                    k[u].clear_unless(some);
                    v[u].clear_unless(some);
                    const bool careful = G > 1 && __ballot(some && !all) != 0;
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        float score = 0.0f, dp = 0.0f;
#pragma unroll
                        for (int i = 0; i < N; ++i) {
                            score += q[g][i] * k[u].get(i);
                            dp += d[g][i] * v[u].get(i);
                        }
                        score = over_lanes(score, cut.lanes, Add{});
                        dp = over_lanes(dp, cut.lanes, Add{});
                        p[g] = counts[g] ? __builtin_amdgcn_exp2f(score + ds[g] - lse[g]) : 0.0f;
                        ds[g] = counts[g] ? p[g] * (dp - delta[g]) : 0.0f;
                        if (careful) {
#pragma unroll
                            for (int i = 0; i < N; ++i) {
                                to_k[i] += counts[g] ? ds[g] * q[g][i] : 0.0f;
                                to_v[i] += counts[g] ? p[g] * d[g][i] : 0.0f;
                                acc[g][i] += counts[g] ? ds[g] * k[u].get(i) : 0.0f;
                            }
                        } else {
#pragma unroll
                            for (int i = 0; i < N; ++i) {
                                to_k[i] += ds[g] * q[g][i];
                                to_v[i] += p[g] * d[g][i];
                                acc[g][i] += ds[g] * k[u].get(i);
                            }
                        }
                    }
                    if (at.head && row[u] < n) {
                        const int64_t to = (row0 + row[u]) * row_of + at.kv * a.dim;
                        Row<T, VEC> back;
#pragma unroll
                        for (int i = 0; i < N; ++i) to_k[i] *= kLn2;
                        back.set(to_k);
                        back.clear_unless(some);
                        back.write(dk + to, at.at, at.there);
                        back.set(to_v);
                        back.clear_unless(some);
                        back.write(dv + to, at.at, at.there);
                    }
                    if (tables)         // (the LDS unit takes a wave's requests in order, and those of one slot go to different entries)
                        for (int e = 0; e < cut.slots; ++e) {
                            if (at.slot == e && at.head && at.at[0] == 0 && at.there[0])
#pragma unroll
                                for (int g = 0; g < G; ++g)
                                    if (counts[g])
                                        __hip_atomic_fetch_add(&s_mine[bucket[u] * a.heads + at.kv * a.group + g], ds[g], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                            __builtin_amdgcn_wave_barrier();
                        }
                }
            }
        }
        const int width = cut.lanes * cut.wide;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < N; ++i) acc[g][i] = over_strided(acc[g][i] * a.scale, width, Add{});
        if (at.slot || !at.head) continue;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g >= a.group) break;
            const int64_t h = at.kv * a.group + g;
            if (!w.whole) {
#pragma unroll
                for (int i = 0; i < N; ++i)
                    if (at.there[i / VEC]) work.acc[(w.slot * a.heads + h) * a.dim + at.at[i / VEC] + i % VEC] = acc[g][i];
                continue;
            }
            Row<T, VEC> row;
            row.set(acc[g]);
            row.write(dq + (w.list * a.heads + h) * a.dim, at.at, at.there);
        }
    }
    if (!tables) return;
    __syncthreads();
    for (int i = threadIdx.x; i < entries; i += kWaves * kWave) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kWaves; ++k) sum += s_sums[k * entries + i];
        work.tables[(int64_t)blockIdx.x * entries + i] = sum;
    }
}

// Adds up the parts' gradients of q, and (the workgroups behind those) the workgroups' of the table, eight entries each.
constexpr int kEntries = 8;
template <typename T>
__global__ void __launch_bounds__(1024) k_attend_grad_join(const Attend<T> a, const Cut cut, const Work work, int groups, int channels, T* dq, int64_t shares, float* dtable) {
    __shared__ float s_sum[1024];
    __shared__ int32_t s_list[1024];
    __shared__ int64_t s_block[1024];
    __shared__ int s_count;
    const int64_t own = (int64_t)groups * a.heads;
    if (blockIdx.x >= own) {
        const int entries = a.buckets * a.heads, e = (int)(blockIdx.x - own) * kEntries + threadIdx.x % kEntries;
        float sum = 0.0f;
#pragma unroll 4
        for (int64_t k = threadIdx.x / kEntries; k < shares; k += 1024 / kEntries) sum += work.tables[k * entries + min(e, entries - 1)];
        sum = over_parts(sum, kEntries, s_sum);
        if ((int)threadIdx.x < kEntries && e < entries) dtable[e] = sum;
        return;
    }
    const int64_t h = blockIdx.x % a.heads, share = blockIdx.x / a.heads;
    const int ch = threadIdx.x % channels, mine = threadIdx.x / channels, parts = 1024 / channels;
    for (int64_t first = share; first < cut.blocks; first += (int64_t)groups * 1024) {
        const int count = starts_of(work, cut.blocks, first, groups, s_list, s_block, &s_count);
        for (int j = 0; j < count; ++j) {
            const int64_t list = s_list[j], begin = s_block[j], end = min((a.edge(list + 1) + ((int64_t)1 << cut.part) - 1) >> cut.part, cut.blocks);
            float acc = 0.0f;
            const int c = min(ch, a.dim - 1);
#pragma unroll 4
            for (int64_t b = begin + mine; b < end; b += parts) acc += work.acc[(b * a.heads + h) * a.dim + c];
            acc = over_parts(acc, channels, s_sum);
            if (mine == 0 && ch < a.dim) dq[(list * a.heads + h) * a.dim + ch] = as_value<T>(acc);
        }
        __syncthreads();
    }
}

// ---- host -------------------------------------------------------------------------------------------------

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }
size_t aligned(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
int power_of_two(int n) {
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

int check(const tns_attend* a) {
    if (!a) return fail(TNS_EINVAL, "null description of the lists");
    if (a->S < 0 || a->rows < 0 || a->num < 0) return fail(TNS_EINVAL, "negative number of lists or rows");
    if (a->S > (int64_t)INT32_MAX || a->num > (int64_t)INT32_MAX || a->rows > (int64_t)1 << 40) return fail(TNS_ESIZE, "more than 2^31-1 lists or gathered rows, or 2^40 rows");
    if (a->heads < 1 || a->heads > 1024 || a->kv_heads < 1 || a->heads % a->kv_heads || a->heads / a->kv_heads > 8)
        return fail(TNS_EINVAL, "heads must be in [1, 1024] and one to eight times kv_heads");
    if (a->head_dim < 1 || a->head_dim > 256) return fail(TNS_EINVAL, "head_dim must be in [1, 256]");
    if (a->dtype != TNS_F32 && a->dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if (a->buckets < 0 || a->buckets > 256 || (int64_t)a->buckets * a->heads > 2048) return fail(TNS_EINVAL, "buckets must be in [0, 256] and buckets * heads at most 2048");
    if (a->flags & ~(TNS_NEWEST_FIRST | TNS_ZERO_BEYOND)) return fail(TNS_EINVAL, "unknown flag");
    return TNS_OK;
}

int check_arrays(const tns_attend* a) {
    if (int e = check(a)) return e;
    const int64_t q_row = (int64_t)a->heads * a->head_dim, k_row = (int64_t)a->kv_heads * a->head_dim;
    if (a->ld_q < q_row || a->ld_k < k_row || a->ld_v < k_row) return fail(TNS_EINVAL, "rows of q, k or v overlap");
    if (a->S > 0 && (!a->d_rowptr || !a->d_q)) return fail(TNS_EINVAL, "null rowptr or q");
    if (!a->d_index && a->num) return fail(TNS_EINVAL, "num without index");
    if ((a->d_index ? a->num : a->rows) > 0 && (!a->d_k || !a->d_v)) return fail(TNS_EINVAL, "null k or v");
    if (a->S > 0 && a->rows > 0 && !a->d_t != !a->d_ts) return fail(TNS_EINVAL, "t and ts come together");
    if (a->buckets > 0 && !a->d_table) return fail(TNS_EINVAL, "null table");
    if (a->buckets > 1 && !a->d_edges) return fail(TNS_EINVAL, "null edges");
    if (a->buckets == 0 && (a->d_table || a->d_edges)) return fail(TNS_EINVAL, "edges or table without buckets");
    const size_t size = a->dtype == TNS_F32 ? 4 : 2;
    if (misaligned(a->d_q, size) || misaligned(a->d_k, size) || misaligned(a->d_v, size)) return fail(TNS_EINVAL, "q, k or v is not aligned to its type");
    return TNS_OK;
}

int check_workspace(const void* p, size_t have, size_t need) {
    if (need && !p) return fail(TNS_EINVAL, "null workspace");
    if (misaligned(p, 256)) return fail(TNS_EINVAL, "workspace must be 256-byte aligned");
    if (have < need) return fail(TNS_ESIZE, "workspace smaller than asked for");
    return TNS_OK;
}

// Lanes of a head as many as hold a row of it, sixteen bytes each.
Cut cut_of(const tns_attend& a) {
    Cut c{};
    const int n = a.dtype == TNS_F32 ? 4 : 8;
    c.lanes = power_of_two((a.head_dim + n - 1) / n);
    c.wide = std::min(power_of_two(a.kv_heads), kWave / c.lanes);
    c.slots = kWave / (c.lanes * c.wide);
    c.turns = (a.kv_heads + c.wide - 1) / c.wide;
    c.part = 6;
    while (c.part < 9 && ((a.rows * c.turns) >> c.part) > 8192) ++c.part;
    c.blocks = (a.rows + ((int64_t)1 << c.part) - 1) >> c.part;
    return c;
}

int groups_of(const tns_attend& a, const Cut& c, int most) {
    const int64_t units = (a.S + c.blocks) * c.turns;
    return (int)std::min<int64_t>((units + kWaves - 1) / kWaves, most);
}
constexpr int kGroups = 2048, kGradGroups = 1024;      // workgroups of a launch, which go round the units
int join_groups(const Cut& c) { return c.blocks > 1 ? (int)std::min<int64_t>(c.blocks, 256) : 0; }

struct Layout {
    Work w;
    size_t bytes;
};
Layout carve(const tns_attend& a, const Cut& c, bool grad, void* base) {
    Layout l{};
    char* p = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        void* const at = p;
        p += aligned(bytes);
        l.bytes += aligned(bytes);
        return at;
    };
    const size_t heads = (size_t)c.blocks * a.heads;
    l.w.first = static_cast<int32_t*>(take(c.blocks * 4));
    l.w.acc = static_cast<float*>(take(heads * a.head_dim * 4));
    if (grad) l.w.tables = static_cast<float*>(take((size_t)kGradGroups * a.buckets * a.heads * 4));
    else l.w.stats = static_cast<float*>(take(heads * 8));
    return l;
}
size_t saved_out_bytes(const tns_attend& a) { return aligned((size_t)a.S * a.heads * a.head_dim * 4); }
size_t saved_bytes(const tns_attend& a) { return saved_out_bytes(a) + aligned((size_t)a.S * a.heads * 4); }

template <typename T>
Attend<T> typed(const tns_attend& a) {
    // (without a row to gather no event counts: the lists are read as empty ones)
    const bool none = a.d_index && a.num == 0;
    return {a.S, none ? 0 : a.rows, a.num, a.d_rowptr, static_cast<const T*>(a.d_q), static_cast<const T*>(a.d_k), static_cast<const T*>(a.d_v), a.ld_q, a.ld_k, a.ld_v,
            a.d_index, a.d_mask, a.d_t, a.d_ts, a.d_edges, a.d_table, a.heads, a.kv_heads, a.head_dim, a.heads / a.kv_heads, a.buckets,
            (a.flags & TNS_NEWEST_FIRST) != 0, (a.flags & TNS_ZERO_BEYOND) != 0, (float)a.scale};
}

// Calls `go` with the type, the channels that a lane reads at once and the heads that share a key.  `fits(n)`: n values at once are aligned everywhere.
template <typename F, typename A>
void choose(const tns_attend& a, const A& fits, const F& go) {
    const int group = power_of_two(a.heads / a.kv_heads);
    auto with = [&](auto value, auto vec) {
        if (group == 1) go(value, vec, std::integral_constant<int, 1>{});
        else if (group == 2) go(value, vec, std::integral_constant<int, 2>{});
        else if (group == 4) go(value, vec, std::integral_constant<int, 4>{});
        else go(value, vec, std::integral_constant<int, 8>{});
    };
    if (a.dtype == TNS_F32) {
        if (fits(4)) with(float{}, std::integral_constant<int, 4>{});
        else if (fits(2)) with(float{}, std::integral_constant<int, 2>{});
        else with(float{}, std::integral_constant<int, 1>{});
    } else {
        if (fits(8)) with(bf16{}, std::integral_constant<int, 8>{});
        else if (fits(4)) with(bf16{}, std::integral_constant<int, 4>{});
        else if (fits(2)) with(bf16{}, std::integral_constant<int, 2>{});
        else with(bf16{}, std::integral_constant<int, 1>{});
    }
}
bool fits(const tns_attend& a, int n, std::initializer_list<const void*> arrays, std::initializer_list<const void*> floats) {
    const size_t size = a.dtype == TNS_F32 ? 4 : 2;
    if (a.head_dim % n || (a.S > 1 && a.ld_q % n) || (a.rows > 1 && (a.ld_k % n || a.ld_v % n))) return false;
    for (const void* p : arrays)
        if (misaligned(p, n * size)) return false;
    for (const void* p : floats)
        if (misaligned(p, n * 4)) return false;
    return true;
}

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, what);
}

}  // namespace

extern "C" {

int tns_attend_workspace(const tns_attend* a, size_t* run, size_t* grad, size_t* saved) {
    tns::clear_error();
    if (int e = check(a)) return e;
    const Cut c = cut_of(*a);
    if (run) *run = carve(*a, c, false, nullptr).bytes;
    if (grad) *grad = carve(*a, c, true, nullptr).bytes;
    if (saved) *saved = saved_bytes(*a);
    return TNS_OK;
}

int tns_attend_run(const tns_attend* a, void* d_out, void* d_saved, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    tns::clear_error();
    if (int e = check_arrays(a)) return e;
    if (a->S > 0 && !d_out) return fail(TNS_EINVAL, "null out");
    if (misaligned(d_out, a->dtype == TNS_F32 ? 4 : 2)) return fail(TNS_EINVAL, "out is not aligned to its type");
    if (misaligned(d_saved, 256)) return fail(TNS_EINVAL, "saved values must be 256-byte aligned");
    const Cut c = cut_of(*a);
    const Layout l = carve(*a, c, false, d_workspace);
    if (int e = check_workspace(d_workspace, workspace_bytes, l.bytes)) return e;
    if (a->S == 0) return TNS_OK;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    float* const saved = static_cast<float*>(d_saved);
    float* const lse = saved ? saved + saved_out_bytes(*a) / 4 : nullptr;
    const size_t lds = (size_t)(a->buckets + a->buckets * a->heads) * 4;
    choose(*a, [&](int n) { return fits(*a, n, {a->d_q, a->d_k, a->d_v, d_out}, {}); }, [&](auto value, auto vec, auto group) {
        using T = decltype(value);
        const Attend<T> t = typed<T>(*a);
        hipLaunchKernelGGL((k_attend<T, vec(), group()>), dim3(groups_of(*a, c, kGroups)), dim3(kWaves * kWave), lds, stream, t, c, l.w, static_cast<T*>(d_out), saved, lse);
        if (const int groups = join_groups(c))
            hipLaunchKernelGGL((k_attend_join<T>), dim3(groups * a->heads), dim3(1024), 0, stream, t, c, l.w, groups, power_of_two(a->head_dim), static_cast<T*>(d_out), saved, lse);
    });
    return launched("tns_attend_run");
}

int tns_attend_grad(const tns_attend* a, const void* d_saved, const void* d_dout, void* d_dq, void* d_dk, void* d_dv, float* d_dtable, void* d_workspace,
                    size_t workspace_bytes, void* hip_stream) {
    tns::clear_error();
    if (int e = check_arrays(a)) return e;
    if (a->d_index) return fail(TNS_EINVAL, "no gradients by rows that are gathered");
    if (a->S > 0 && (!d_saved || !d_dout || !d_dq)) return fail(TNS_EINVAL, "null saved values, dout or dq");
    if (a->rows > 0 && (!d_dk || !d_dv)) return fail(TNS_EINVAL, "null dk or dv");
    if (!d_dtable != !a->buckets) return fail(TNS_EINVAL, "dtable and buckets come together");
    const size_t size = a->dtype == TNS_F32 ? 4 : 2;
    if (misaligned(d_dout, size) || misaligned(d_dq, size) || misaligned(d_dk, size) || misaligned(d_dv, size)) return fail(TNS_EINVAL, "dout, dq, dk or dv is not aligned to its type");
    if (misaligned(d_saved, 256)) return fail(TNS_EINVAL, "saved values must be 256-byte aligned");
    const Cut c = cut_of(*a);
    const Layout l = carve(*a, c, true, d_workspace);
    if (int e = check_workspace(d_workspace, workspace_bytes, l.bytes)) return e;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const float* const saved = static_cast<const float*>(d_saved);
    const float* const lse = saved + saved_out_bytes(*a) / 4;
    const size_t lds = (size_t)(a->buckets + (1 + kWaves) * a->buckets * a->heads) * 4;
    const int shares = groups_of(*a, c, kGradGroups), groups = join_groups(c), sums = (a->buckets * a->heads + kEntries - 1) / kEntries;
    choose(*a, [&](int n) { return fits(*a, n, {a->d_q, a->d_k, a->d_v, d_dout, d_dq, d_dk, d_dv}, {}); }, [&](auto value, auto vec, auto group) {
        using T = decltype(value);
        const Attend<T> t = typed<T>(*a);
        if (shares)
            hipLaunchKernelGGL((k_attend_grad<T, vec(), group()>), dim3(shares), dim3(kWaves * kWave), lds, stream, t, c, l.w, saved, lse, static_cast<const T*>(d_dout),
                               static_cast<T*>(d_dq), static_cast<T*>(d_dk), static_cast<T*>(d_dv), d_dtable != nullptr);
        if (groups * a->heads + sums)
            hipLaunchKernelGGL((k_attend_grad_join<T>), dim3(groups * a->heads + sums), dim3(1024), 0, stream, t, c, l.w, groups, power_of_two(a->head_dim), static_cast<T*>(d_dq),
                               (int64_t)shares, d_dtable);
    });
    return launched("tns_attend_grad");
}

}  // extern "C"
