// What the kernels of the attention over event lists share (include/tns_layer.h).  Included by tns_attend.hip and tns_attend_grad.hip only.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "../../include/tns_layer.h"
#include "tns_internal.h"
#include "tns_parts.h"
#include "tns_sums.h"
#include "tns_values.h"

using tns::Add;
using tns::add_either;
using tns::as_float;
using tns::as_value;
using tns::bf16;
using tns::fail;
using tns::fail_hip;
using tns::gap_of;
using tns::is_many;
using tns::kLog2e;
using tns::Max;
using tns::over_lanes;
using tns::over_row_strided;
using tns::over_strided;
using tns::parts_end;

namespace {

constexpr int kWave = 64, kWaves = 4;      // lanes of a wave, waves of a workgroup
constexpr float kInf = __builtin_inff();
constexpr float kLn2 = 0.69314718055994530942f;

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ int64_t read_lane64(int64_t v, int lane) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v >> 32), lane);
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
    int heads, kv_heads, dim, group, buckets, steps;      // steps: of the search, the largest power of two that is no more than the edges
    bool newest_first, zero_beyond;
    float scale;                        // times log2 e: scores are in powers of two

    __device__ int64_t edge(int64_t s) const { return uniform(min(max(rowptr[s], (int64_t)0), rows)); }
    __device__ int64_t total() const { return S ? edge(S) : 0; }
};

// How the work is cut.  Lists of more rows than a block (`1 << part` rows, counted from row 0) are cut where blocks end.  Of such lists a block has the
// first part of one at most and another part of one at most; parts are numbered by their block, first ones as many further as there are blocks.
//
// A wave takes a part for some of the heads: `lanes` lanes hold a row of a head of k or v, sixteen bytes each, `wide` heads side by
// side, and the rest of the wave are `slots` events at a time.
struct Cut {
    int part;                           // log2 of a block's rows
    int64_t blocks;                     // of the rows
    int lanes, wide, slots, turns;      // powers of two but for turns, the waves that the heads of k and v take (the grid's second dimension)
    int log_lanes, log_width;           // of lanes, and of lanes * wide
    bool exact;                         // every lane of every wave has a head and all its channels
    int log_copies;                     // of the table's gradient that a wave has, for its slots in turn
    int brief;                          // lists of so many events at most are taken a slot each; -1: none
};
struct Part {
    int64_t list, begin, end, slot;     // slot: the part's number
    int64_t list_begin, list_end;
    bool whole;                         // the list has no other part
};

// The lists that hold the K rows p[] < total: the last ones that begin at or before them.  Called by the whole wave, which looks at 64 lists a step, for
// all K at once.  (What a ballot votes on is computed without branches.)
template <int K, typename T>
__device__ void find_lists(const Attend<T>& a, const int64_t (&p)[K], int64_t (&list)[K]) {
    const int lane = threadIdx.x & 63;
    int64_t lo[K], hi[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        lo[k] = 0;
        hi[k] = a.S;
    }
    for (int64_t wide = a.S; wide > 1;) {
        const int64_t by = (wide + kWave - 1) / kWave;
        int64_t at[K];
#pragma unroll
        for (int k = 0; k < K; ++k) at[k] = a.rowptr[min(lo[k] + (lane + 1) * by, hi[k])];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int64_t j = lo[k] + (lane + 1) * by;
            const int c = __popcll(__ballot((j < hi[k]) & (min(max(at[k], (int64_t)0), a.rows) <= p[k])));
            lo[k] += c * by;
            hi[k] = min(lo[k] + by, hi[k]);
        }
        wide = by;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) list[k] = uniform(lo[k]);
}
template <typename T>
__device__ int64_t find_list(const Attend<T>& a, int64_t p) {
    const int64_t row[1] = {p};
    int64_t list[1];
    find_lists(a, row, list);
    return list[0];
}

// A list's edges as they lie in memory, the lane's or the wave's.
struct Edges {
    int64_t begin = 0, end = 0;
    __device__ Edges() {}
    template <typename T>
    __device__ Edges(const Attend<T>& a, int64_t list) : begin(a.rowptr[min(list, a.S)]), end(a.rowptr[min(list + 1, a.S)]) {}
    template <typename T>
    __device__ void tidy(const Attend<T>& a) {
        begin = min(max(begin, (int64_t)0), a.rows);
        end = max(min(max(end, (int64_t)0), a.rows), begin);
    }
};

// The parts that a wave takes: of every `stride`-th list the first, lists that are taken a slot each left out; then every `stride`-th block.
template <typename T>
struct Walk {
    int64_t next, block, from = 0, stride;     // next: list of lane 0 when 64 more are looked at; from: that of those that were
    uint64_t left = 0;                  // of the 64, a bit each
    Edges edges;                        // lane i's: of list from + i stride
    // (Waves that have no list, or one fewer, are the last ones: they begin with the blocks.)
    __device__ Walk(int64_t begin, int64_t stride) : next(begin), block(stride - 1 - begin), stride(stride) {}

    // The next part, false if there is none.  For every block it also says (`first`) which list that is cut has its first part there, or -1, and calls
    // beyond(block).
    template <typename Beyond>
    __device__ __forceinline__ bool get(const Attend<T>& a, const Cut& cut, int32_t* first, Part& w, const Beyond& beyond) {
        const int64_t size = (int64_t)1 << cut.part;
        while (!left && next < a.S) {
            const int64_t list = next + (threadIdx.x & 63) * stride;
            edges = Edges(a, list);
            edges.tidy(a);
            left = __ballot((list < a.S) & (edges.end - edges.begin > cut.brief));
            from = next;
            next += kWave * stride;
        }
        if (left) {
            const int i = __builtin_ctzll(left);
            left &= left - 1;
            w.list = from + i * stride;
            w.begin = w.list_begin = read_lane64(edges.begin, i);
            w.list_end = read_lane64(edges.end, i);
            w.whole = w.list_end - w.begin <= size;
            w.slot = (w.begin >> cut.part) + cut.blocks;
            w.end = w.whole ? w.list_end : ((w.begin >> cut.part) + 1) << cut.part;
            return true;
        }
        for (; block < cut.blocks; block += stride) {
            beyond(block);
            w.slot = block;
            w.begin = block << cut.part;
            int32_t starts = -1;
            bool any = false;
            const int64_t total = a.total();
            if (w.begin < total) {
                const int64_t row[2] = {w.begin, min(w.begin + size, total - 1)};
                int64_t list[2];
                find_lists(a, row, list);
                Edges here(a, list[0]), on(a, list[1]);      // of the list that the block begins in, and of the one that goes on behind it
                here.tidy(a);
                on.tidy(a);
                if (w.begin + size < total && uniform(on.begin) >= w.begin && uniform(on.begin) < w.begin + size && uniform(on.end - on.begin) > size) starts = (int32_t)list[1];
                w.list = list[0];
                w.list_begin = uniform(here.begin);
                w.list_end = uniform(here.end);
                w.end = min(w.list_end, w.begin + size);
                w.whole = false;
                any = w.list_begin < w.begin && w.begin < w.list_end && w.list_end - w.list_begin > size;
            }
            if (first && (threadIdx.x & 63) == 0) first[block] = starts;
            if (any) {
                block += stride;
                return true;
            }
        }
        return false;
    }
};

// Where there are many lists, those of `brief` events at most are taken a slot each: what a list costs apart from its events (its query, its
// edges, its result) is then paid once for all slots, and nothing is joined.  131072 lists of ten, two heads of 64 bf16 channels, outputs: 169 us
// either way; gathered, four heads of 32, 66600 lists: 63 us, a wave to a list 74.
struct Own {
    int64_t list, begin;
    int n, events;                      // of the list; that are taken here, 0 of lists that are not (`here`)
    bool here;
    template <typename T>
    __device__ Own(const Attend<T>& a, const Cut& cut, int64_t of, Edges edges) {
        edges.tidy(a);
        n = (int)min(edges.end - edges.begin, (int64_t)INT32_MAX);
        here = of < a.S && n <= cut.brief;
        events = here ? n : 0;
        list = min(of, a.S - 1);
        begin = min(edges.begin, a.rows - 1);      // (where there is a row)
    }
};

// A lane's sixteen bytes of a row of a head, at any address that is aligned to T: N channels side by side (VEC = N), where a head has no whole number of
// them the last lane's begin further to the front, so that they end with the row; or one by one (VEC = 1) where a head has fewer.
template <typename T, int VEC>
struct Row {
    static constexpr int N = 16 / sizeof(T), PIECES = N / VEC;
    struct Piece { T v[VEC]; };
    union {
        Piece piece[PIECES];
        uint32_t word[4];
    };
    __device__ Row() {}
    __device__ float get(int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(word[i]);
        else return __uint_as_float(i & 1 ? word[i / 2] & 0xffff0000u : word[i / 2] << 16);
    }
    __device__ __forceinline__ void read(const char* base, uint32_t more, const uint32_t (&at)[PIECES]) {      // (the base is the same for the wave, 32 bits more the lane's)
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            uint32_t bytes = more + at[p];
            asm("" : "+v"(bytes));
            piece[p] = *reinterpret_cast<const Piece*>(base + bytes);
        }
    }
    __device__ __forceinline__ void gather(const char* base, uint64_t more, const uint32_t (&at)[PIECES]) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) piece[p] = *reinterpret_cast<const Piece*>(base + more + at[p]);
    }
    // The lane's part of the product with another row.  Two products of 16 bits and their sum are one instruction, off by 2.4 * 2^-24 of the
    // terms' magnitudes where two rounded sums would be off by 2: measured over values 2^12 apart.
    // MASK: of the channels that are in `mask`, each once for all lanes.
    template <bool MASK>
    __device__ __forceinline__ float dot(const Row& o, const uint32_t (&mask)[4]) const {
        float v = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                v += __uint_as_float(MASK ? word[i] & mask[i] : word[i]) * __uint_as_float(o.word[i]);
            } else {
                using Pair = __bf16 __attribute__((ext_vector_type(2)));
                v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair, MASK ? word[i] & mask[i] : word[i]), __builtin_bit_cast(Pair, o.word[i]), v, false);
            }
        }
        return v;
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
    __device__ __forceinline__ void write(char* base, uint32_t more, const uint32_t (&at)[PIECES], const bool (&there)[PIECES]) const {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            uint32_t bytes = more + at[p];
            asm("" : "+v"(bytes));
            if (there[p]) *reinterpret_cast<Piece*>(base + bytes) = piece[p];
        }
    }
};

// `base[more]` where the base is the same for the wave and what is added the lane's, in 32 bits.
template <typename V, typename U>
__device__ __forceinline__ V* lane_at(U* base, uint32_t bytes) {
    asm("" : "+v"(bytes));
    using Char = std::conditional_t<std::is_const_v<U>, const char, char>;
    return reinterpret_cast<V*>(reinterpret_cast<Char*>(base) + bytes);
}

// Where a lane stands in its wave.  EXACT: every lane has a head and all its channels.
template <typename T, int VEC, bool EXACT>
struct Place {
    static constexpr int N = Row<T, VEC>::N, PIECES = Row<T, VEC>::PIECES;
    int lane, slot, kv, mine;           // kv: head of k and v, the last one again where there are no more (`head`: there is); mine: which of its lanes
    bool head;
    uint32_t at[PIECES];                // bytes of the pieces from the begin of a row of k or v on, those of channel 0 where there are no more (`there`)
    uint32_t in_q[PIECES];              // values from the begin of a row of q on, of the group's first head
    bool there[PIECES];
    int channel;                        // of the lane's first value (VEC = N)
    uint32_t mask[4];                   // of the values that no other lane has

    __device__ Place(const Attend<T>& a, const Cut& cut, int turn) {
        lane = threadIdx.x & 63;
        const int of = lane & ((1 << cut.log_width) - 1);
        mine = of & (cut.lanes - 1);
        slot = lane >> cut.log_width;
        kv = turn * cut.wide + (of >> cut.log_lanes);
        head = EXACT || kv < a.kv_heads;
        kv = min(kv, a.kv_heads - 1);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int own = VEC == N ? mine * N : p;
            there[p] = EXACT || own < a.dim;
            const int c = VEC == N ? min(own, a.dim - N) : there[p] ? p : 0;
            at[p] = (uint32_t)(kv * a.dim + c) * sizeof(T);
            in_q[p] = (uint32_t)(kv * a.group * a.dim + c);
            if (VEC == N) channel = c;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            constexpr int PER = 4 / sizeof(T);
            mask[i] = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) mask[i] |= counts(i * PER + k) ? (PER == 1 ? ~0u : 0xffffu << 16 * k) : 0u;
        }
    }
    // Whether no other lane has the lane's i-th value.
    __device__ __forceinline__ bool counts(int i) const { return EXACT || (VEC == N ? there[0] && channel + i >= mine * N : there[VEC == N ? 0 : i]); }
    // Rows of the lane's group of heads of an array's list, zero where there is no such head or channel.
    template <int G>
    __device__ __forceinline__ void heads(const Attend<T>& a, const T* list, Row<T, VEC> (&to)[G]) const {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                to[g].piece[p] = *lane_at<const typename Row<T, VEC>::Piece>(list, (in_q[p] + (uint32_t)(min(g, a.group - 1) * a.dim)) * (uint32_t)sizeof(T));
                if (!(head && there[p])) to[g].piece[p] = {};
                if (g >= a.group) to[g].piece[p] = {};
            }
    }
    template <int G>
    __device__ __forceinline__ void heads(const Attend<T>& a, const float* list, float (&to)[G][N]) const {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                struct Floats { float v[VEC]; } piece = *lane_at<const Floats>(list, (in_q[p] + (uint32_t)(min(g, a.group - 1) * a.dim)) * 4u);
#pragma unroll
                for (int i = 0; i < VEC; ++i) to[g][p * VEC + i] = head && there[p] && g < a.group ? piece.v[i] : 0.0f;
            }
    }
    // The lane's values of a head of the group, `more` values from the group's first one on, to an array's list.
    template <typename U>
    __device__ __forceinline__ void write(U* list, int more, const float (&v)[N]) const {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            struct Some { U v[VEC]; } some;
#pragma unroll
            for (int i = 0; i < VEC; ++i) some.v[i] = as_value<U>(v[p * VEC + i]);
            if (there[p]) *lane_at<Some>(list, (in_q[p] + (uint32_t)more) * (uint32_t)sizeof(U)) = some;
        }
    }
    // Sums of the lane's N values over the slots, go(values from the begin of a row of q on, sum, next sum or nothing) for those that come to lie with
    // the lane.  Rows of lanes that are slots share the values: a step costs a value half an addition, and in the end every lane has some to write.
    template <typename Go>
    __device__ __forceinline__ void joined(const Attend<T>& a, const Cut& cut, int g, float (&v)[N], const Go& go) const {
        int first = 0;
        auto write = [&](auto count) {
            constexpr int R = count();
            if (!head || (lane & 15) >> min(cut.log_width, 4)) return;
            constexpr int STEP = sizeof(T) == 2 && VEC >= 2 && R >= 2 ? 2 : 1;
            if (VEC == N && !there[0]) return;
#pragma unroll
            for (int i = 0; i < R; i += STEP) {
                const int c = VEC == N ? channel + first + i : first + i;
                if (VEC == N || c < a.dim) go((uint32_t)((kv * a.group + g) * a.dim + c), v[i], v[i + STEP - 1], std::integral_constant<int, STEP>{});
            }
        };
        if (cut.slots == 1) return write(std::integral_constant<int, N>{});
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = add_either<32>(v[i], v[i + N / 2]);
        first = lane & 32 ? N / 2 : 0;
        if (cut.slots == 2) return write(std::integral_constant<int, N / 2>{});
#pragma unroll
        for (int i = 0; i < N / 4; ++i) v[i] = add_either<16>(v[i], v[i + N / 4]);
        if (cut.log_width < 4)
#pragma unroll
            for (int i = 0; i < N / 4; ++i) v[i] = over_row_strided(v[i], 1 << cut.log_width, Add{});
        first += lane & 16 ? N / 4 : 0;
        write(std::integral_constant<int, N / 4>{});
    }
};
// Writes one or two values.
template <typename U, typename Two>
__device__ __forceinline__ void put(U* base, uint32_t at, float a, float b, Two) {
    struct Some { U v[Two()]; } some;
    some.v[0] = as_value<U>(a);
    if constexpr (Two() == 2) some.v[1] = as_value<U>(b);
    *lane_at<Some>(base, at * (uint32_t)sizeof(U)) = some;
}

// What is read of an event.
struct Event {
    float ts;
    int32_t index;
    uint8_t mask;
    template <typename T>
    __device__ __forceinline__ Event(const Attend<T>& a, int64_t row0, uint32_t more) {      // row0: of the wave, or the lane's own
        index = a.index ? *lane_at<const int32_t>(a.index + row0, 4 * more) : 0;
        mask = a.mask ? *lane_at<const uint8_t>(a.mask + row0, more) : 1;
        ts = a.ts ? *lane_at<const float>(a.ts + row0, 4 * more) : 0.0f;
    }
};
// Bucket, or -1 for an event that is left out, and row of k and v with an index.
struct Known {
    int bucket = 0, index = 0;
    __device__ Known() {}
    // `newer`: events of the list that are.
    template <typename T>
    __device__ __forceinline__ Known(const Attend<T>& a, const Event& event, float t, int64_t newer, const float* s_edges) {
        const bool inside = !a.index || (event.index >= 0 && event.index < a.num);
        index = inside ? event.index : 0;
        if (a.buckets > 1) {
            const float age = a.ts ? gap_of(t, event.ts) : __ll2float_rz(newer);      // (rounded down: fp32 edges at or below a place are those at or below this)
            const int edges = a.buckets - 1;
            for (int by = a.steps; by; by >>= 1) {
                const int to = bucket + by;
                const float edge = s_edges[min(to, edges) - 1];
                bucket = to <= edges && edge <= age ? to : bucket;
            }
        }
        if (!(event.mask && inside)) bucket = -1;
    }
};

// A table's entry in powers of two.  Times log2 e, the largest finite numbers (the lowest one as a mask is one) would become infinite, and only an infinite
// entry leaves its events out: from 2^126 on the factor is smaller.  Entries that differ differ by 2^103 or more there, so p is 0 or 1 by any factor.
__device__ __forceinline__ float in_powers(float v) {
    constexpr float from = 0x1p126f, by = 0.85f;      // (by * FLT_MAX + from * (log2 e - by) is 3.397e38)
    return fabsf(v) < from ? v * kLog2e : v * by + copysignf(from * (kLog2e - by), v);
}
// Edges and table in LDS, the table in powers of two.
template <typename T>
__device__ __forceinline__ void stage(const Attend<T>& a, float* s_edges, float* s_table) {
    for (int i = threadIdx.x; i < a.buckets - 1; i += kWaves * kWave) s_edges[i] = a.edges[i];
    for (int i = threadIdx.x; i < max(a.buckets, 1) * a.heads; i += kWaves * kWave) s_table[i] = a.buckets ? in_powers(a.table[i]) : 0.0f;
    __syncthreads();
}

struct Work {
    int32_t* first;                     // [blocks]: the list that is cut and has its first part there, or -1
    float *stats, *acc;                 // [2 blocks, heads, 2], [2 blocks, heads, dim]: of the parts of lists that have several
    float* tables;                      // [workgroups of the gradients, buckets * heads]
};

// What the gradients need of a list's softmax to have its p again: the largest score, in powers of two, and one over the sum of exponentials by it (0 where
// no event counts).  The logarithm of the sum, added to the largest score, would be rounded to that one's last place: beside a table of -1e4 p
// would be off by 7e-4, beside one of -1e9 by any factor.
struct Norm {
    float top, inverse;
    __device__ Norm() {}
    __device__ Norm(float top, float sum, float inverse) : top(sum == 0.0f ? 0.0f : top), inverse(inverse) {}
};

// What a kernel is called with, read again where it is used: some sixty scalar registers would hold it otherwise, and as many values of the loops
// would be moved to vector registers and back.
template <typename T>
struct Args {
    Attend<T> a;
    Cut cut;
    Work work;
    T* out;
    float* saved_out;                   // (the gradients read what is saved)
    Norm* saved_norm;
    const T* dout;
    T *dq, *dk, *dv;
    int tables;                         // whether the table's gradient is wanted
};
template <typename T>
__device__ __forceinline__ const Args<T>& args_now() {
#if defined(__HIP_DEVICE_COMPILE__)
    using Const = const __attribute__((address_space(4))) Args<T>;
    auto p = (Const*)__builtin_amdgcn_kernarg_segment_ptr();      // (the kernels' only argument)
    asm volatile("" : "+s"(p));
    return *(const Args<T>*)p;
#else
    __builtin_unreachable();            // (the host's pass over the kernels)
#endif
}
// Over the lanes of a head: LANES, or `lanes` where that is 0.
template <int LANES>
__device__ __forceinline__ float over_head(float v, int lanes) {
    if constexpr (LANES) return over_lanes(v, LANES, Add{});
    else return over_lanes(v, lanes, Add{});
}

// U events of every slot: their rows of k and v, on their way while others are computed.
template <typename T, int VEC, int U, bool EXACT>
struct Batch {
    Row<T, VEC> k[U], v[U];
    // Of the events from row0 + i0 on; rows beyond the n of the part are the last one's.
    __device__ __forceinline__ void read(const Attend<T>& a, const Cut& cut, const Place<T, VEC, EXACT>& at, int64_t row0, int i0, int n, const Known* known) {
        const char* const k_row = reinterpret_cast<const char*>(a.k + (known ? 0 : row0 * a.ld_k));
        const char* const v_row = reinterpret_cast<const char*>(a.v + (known ? 0 : row0 * a.ld_v));
        const uint32_t k_step = (uint32_t)a.ld_k * sizeof(T), v_step = (uint32_t)a.ld_v * sizeof(T);      // (below 2^24)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int place = min(i0 + u * cut.slots + at.slot, n - 1);
            if (known) {
                const uint32_t row = (uint32_t)__shfl(known->index, place);
                k[u].gather(k_row, (uint64_t)row * k_step, at.at);
                v[u].gather(v_row, (uint64_t)row * v_step, at.at);
            } else {
                k[u].read(k_row, __umul24(place, k_step), at.at);
                v[u].read(v_row, __umul24(place, v_step), at.at);
            }
        }
    }
    // Of the slot's own list, from event i0 on; with `known`, of the lanes from `lane0` on.
    __device__ __forceinline__ void read_own(const Attend<T>& a, const Place<T, VEC, EXACT>& at, const char* k_row, const char* v_row, const Own& own, int i0, const Known* known, int lane0) {
        const uint32_t k_step = (uint32_t)a.ld_k * sizeof(T), v_step = (uint32_t)a.ld_v * sizeof(T);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (known) {
                const uint32_t row = (uint32_t)__shfl(known->index, lane0 + u);
                k[u].gather(k_row, (uint64_t)row * k_step, at.at);
                v[u].gather(v_row, (uint64_t)row * v_step, at.at);
            } else {
                const int place = max(min(i0 + u, own.events - 1), 0);
                k[u].gather(k_row, __umul24(place, k_step), at.at);
                v[u].gather(v_row, __umul24(place, v_step), at.at);
            }
        }
    }
};

// A part's events in order, `by` at a time: go(batch, first event), with the next batch on its way.  (From behind a read that may not have been made
// the compiler could only wait for everything; so the last batch is taken by itself.)
template <typename B, typename Read, typename Go>
__device__ __forceinline__ void each_batch(B& batch, int n, int by, const Read& read, const Go& go) {
    int i = 0;
    for (; i + by < n; i += by) {
        B next;
        read(next, i + by);
        go(batch, i);
        batch = next;
    }
    go(batch, i);
}

// ---- lists of several parts ---------------------------------------------------------------------------------
// A workgroup joins the lists whose first part lies in one of sixteen blocks, one after the other: a wave has every sixteenth part, a lane kOwn
// channels, and every so many channels a workgroup of their own.  Lists of more than kMany parts are joined by a workgroup for every kSlice
// channels of a head, at the place that stands for them (tns_parts.h).
constexpr int kOwn = 4, kSlice = 16;
template <typename T>
struct ListsOf {
    const Attend<T>& a;
    __device__ int64_t total() const { return a.total(); }
    __device__ int64_t edge(int64_t list) const { return a.edge(list); }
    __device__ int64_t find(int64_t row) const { return find_list(a, row); }
};
template <typename T>
__device__ __forceinline__ int64_t many_of(const Attend<T>& a, const Cut& cut, int64_t place, int64_t& first, int64_t& end) {
    return tns::many_at(place, cut.part, cut.blocks, ListsOf<T>{a}, first, end);
}

// The number of a list's part that lies in block b, the list's first part in block `first`.
__device__ __forceinline__ int64_t slot_of(int64_t b, int64_t first, const Cut& cut) { return b == first ? b + cut.blocks : b; }

// Sum over the threads that have the same number modulo `wide`, a power of two, of 1024, in a fixed order.
__device__ __forceinline__ float over_parts(float v, int wide, float* s_sum) {
    __syncthreads();
    s_sum[threadIdx.x] = v;
    for (int n = 512; n >= wide; n /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < n) s_sum[threadIdx.x] += s_sum[threadIdx.x + n];
    }
    __syncthreads();
    return s_sum[threadIdx.x & (wide - 1)];
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
    if (a->ld_k >= (int64_t)1 << 22 || a->ld_v >= (int64_t)1 << 22) return fail(TNS_ESIZE, "rows of k or v are 2^22 values apart or more");
    if (a->S > 0 && (!a->d_rowptr || !a->d_q)) return fail(TNS_EINVAL, "null rowptr or q");
    if (!a->d_index && a->num && a->rows > 0) return fail(TNS_EINVAL, "num without index");      // (an index of no rows may have no address)
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
    c.log_lanes = __builtin_ctz(c.lanes);
    c.exact = c.lanes * n == a.head_dim && a.kv_heads % c.wide == 0;
    c.log_width = __builtin_ctz(c.lanes * c.wide);
    // Blocks: of 64 rows; of fewer where that leaves few of them for the chip, and a call is as long as its blocks; of more where there would be more
    // than 16384.
    c.part = 6;
    while (c.part > 4 && ((a.rows * c.turns) >> (c.part - 1)) <= 2048) --c.part;
    while (c.part < 9 && ((a.rows * c.turns) >> c.part) > 16384) ++c.part;
    // Brief lists a slot each: where there are enough of them, and short ones by what rows there are (8300 lists of 64, two heads of 64 bf16 channels,
    // gradients: 99 us, 85 otherwise; of ten, outputs: 12 and 15).
    c.brief = c.log_width >= 2 && a.S / c.slots * c.turns >= 2048 && a.rows <= 16 * a.S ? std::min(64, 1 << c.part) : -1;
    c.log_copies = std::min(__builtin_ctz(c.slots), 3);
    while (c.log_copies && ((size_t)a.buckets * a.heads * kWaves << c.log_copies) > 4096) --c.log_copies;
    c.blocks = (a.rows + ((int64_t)1 << c.part) - 1) >> c.part;
    return c;
}

// Workgroups of a launch for each turn: as many as the chip holds at once.  They go round the units; with a few more than it holds the last ones would start
// when the first are done, and the launch take twice as long.
constexpr int kCus = 256, kMostPerCu = 8, kLdsPerCu = 160 << 10;
template <typename K>
int resident(K kernel, size_t lds, int& per_cu) {      // per_cu: what was found the first time, by the registers
    int n = __atomic_load_n(&per_cu, __ATOMIC_RELAXED);
    if (!n) {
        n = hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, kWaves * kWave, 0) == hipSuccess && n > 0 ? std::min(n, kMostPerCu) : 2;
        __atomic_store_n(&per_cu, n, __ATOMIC_RELAXED);
    }
    return kCus * std::min<int>(n, std::max<int>(kLdsPerCu / (int)(lds + 256), 1));
}
int groups_of(const tns_attend& a, const Cut& c, int most) {
    return (int)std::min<int64_t>((a.S + c.blocks + kWaves - 1) / kWaves, std::max(most / c.turns, 1));
}
int64_t slices_of(const tns_attend& a) { return (a.head_dim + kSlice - 1) / kSlice; }
int64_t few_of(const tns_attend& a, const Cut& c) { return c.blocks > 1 ? (c.blocks + 15) / 16 * ((a.heads * a.head_dim + kOwn * kWave - 1) / (kOwn * kWave)) : 0; }
int64_t many_of(const tns_attend& a, const Cut& c) { return tns::many_places(c.blocks) * a.heads * slices_of(a); }
// (A launch has fewer than 2^32 threads: 2^34 rows of up to 256 channels.)
int check_joins(const tns_attend& a, const Cut& c) {
    return few_of(a, c) + many_of(a, c) > (int64_t)1 << 21 ? fail(TNS_ESIZE, "more rows times channels than one call can join") : (int)TNS_OK;
}

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
    const size_t heads = (size_t)2 * c.blocks * a.heads;
    l.w.first = static_cast<int32_t*>(take(c.blocks * 4));
    l.w.acc = static_cast<float*>(take(heads * a.head_dim * 4));
    if (grad) l.w.tables = static_cast<float*>(take((size_t)groups_of(a, c, kCus * kMostPerCu) * c.turns * a.buckets * a.heads * 4));
    else l.w.stats = static_cast<float*>(take(heads * 8));
    return l;
}
size_t saved_out_bytes(const tns_attend& a) { return aligned((size_t)a.S * a.heads * a.head_dim * 4); }
inline size_t saved_bytes(const tns_attend& a) { return saved_out_bytes(a) + aligned((size_t)a.S * a.heads * sizeof(Norm)); }

template <typename T>
Attend<T> typed(const tns_attend& a) {
    // (without a row to gather no event counts: the lists are read as empty ones)
    const bool none = a.d_index && a.num == 0;
    return {a.S, none ? 0 : a.rows, a.num, a.d_rowptr, static_cast<const T*>(a.d_q), static_cast<const T*>(a.d_k), static_cast<const T*>(a.d_v), a.ld_q, a.ld_k, a.ld_v,
            a.d_index, a.d_mask, a.d_t, a.d_ts, a.d_edges, a.d_table, a.heads, a.kv_heads, a.head_dim, a.heads / a.kv_heads, a.buckets, a.buckets > 1 ? 1 << (31 - __builtin_clz(a.buckets - 1)) : 0,
            (a.flags & TNS_NEWEST_FIRST) != 0, (a.flags & TNS_ZERO_BEYOND) != 0, (float)(a.scale * 1.4426950408889634)};
}

// Calls `go` with the type, the channels that a lane reads at once, the heads that share a key, and the lanes of a head: where no lane is idle or has
// another one's channels the compiler knows them, 0 otherwise.
template <typename F>
void choose(const tns_attend& a, const Cut& c, const F& go) {
    using std::integral_constant;
    const int group = power_of_two(a.heads / a.kv_heads);
    auto with = [&](auto value, auto vec, auto lanes) {
        if (group == 1) go(value, vec, integral_constant<int, 1>{}, lanes);
        else if (group == 2) go(value, vec, integral_constant<int, 2>{}, lanes);
        else if (group == 4) go(value, vec, integral_constant<int, 4>{}, lanes);
        else go(value, vec, integral_constant<int, 8>{}, integral_constant<int, 0>{});
    };
    auto of = [&](auto value) {
        constexpr int N = 16 / (int)sizeof(value);
        using Whole = integral_constant<int, N>;
        if (a.head_dim < N) with(value, integral_constant<int, 1>{}, integral_constant<int, 0>{});
        else if (c.exact && c.lanes == 4) with(value, Whole{}, integral_constant<int, 4>{});
        else if (c.exact && c.lanes == 8) with(value, Whole{}, integral_constant<int, 8>{});
        else if (c.exact && c.lanes == 16) with(value, Whole{}, integral_constant<int, 16>{});
        else with(value, Whole{}, integral_constant<int, 0>{});
    };
    if (a.dtype == TNS_F32) of(float{});
    else of(bf16{});
}
// LDS of a kernel: edges, table, and `more` tables.
size_t lds_of(const tns_attend& a, int more) { return (size_t)(a.buckets + std::max(a.buckets, 1) * a.heads + more * a.buckets * a.heads) * 4; }
int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, what);
}

}  // namespace
