// Gated linear recurrence over ragged lists of events (include/tns_train.h): states, gradients, and the step of one event per node.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "../../include/tns_train.h"
#include "tns_internal.h"
#include "tns_values.h"

using tns::as_float;
using tns::as_value;
using tns::bf16;
using tns::fail;
using tns::fail_hip;
using tns::gap_of;
using tns::gate_of;
using tns::kLog2e;

namespace {

constexpr int kWave = 64, kWaves = 4;  // lanes of a wave, waves of a workgroup
constexpr int kSaved = 16;             // rows from one saved state to the next, and rows that a wave has in its registers
constexpr int kBatch = 64;             // rows whose lists and gaps the lanes of a wave hold, and rows of a tile at most
constexpr uint32_t kGroupMask = (1u << kSaved) - 1;

// Values of the V channels of a lane, as they lie in memory.
template <typename T, int V> struct Pack;
template <> struct Pack<float, 1> {
    float raw;
    __device__ float get(int) const { return raw; }
};
template <> struct Pack<bf16, 1> {
    bf16 raw;
    __device__ float get(int) const { return as_float(raw); }
};
template <> struct Pack<bf16, 2> {
    uint32_t raw;
    __device__ float get(int i) const { return __uint_as_float(i ? raw & 0xffff0000u : raw << 16); }
};
template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = p[i];
}
template <int V>
__device__ __forceinline__ void load_or_zero(const float* p, float (&v)[V]) {      // (p is the same or null for the whole wave)
    if (p) load_floats<V>(p, v);
    else
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.0f;
}
template <int V>
__device__ __forceinline__ void store_floats(float* p, const float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = v[i];
}

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint64_t)v >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ float read_lane(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// The lists (tns_recur with its types) as one walk over all events: place p of the walk is row p, or, newest first, row total - 1 - p; the
// j-th list of the walk is list j or S - 1 - j.  Whatever rowptr holds, a place below `total` has a row below `rows` and a list below S.
template <typename T>
struct Lists {
    int64_t S, rows;
    const int64_t* rowptr;
    const T *u, *x;
    int64_t ld_u, ld_x;
    const float *ts, *decay, *h0, *t0;
    int dim;
    bool newest_first, zero_beyond;

    __device__ int64_t total() const { return S ? uniform(min(max(rowptr[S], (int64_t)0), rows)) : 0; }
    __device__ int64_t begin_of(int64_t j, int64_t total) const {         // 0 <= j <= S
        const int64_t at = min(max(rowptr[newest_first ? S - j : j], (int64_t)0), total);
        return newest_first ? total - at : at;
    }
    __device__ int64_t row(int64_t p, int64_t total) const { return newest_first ? total - 1 - p : p; }
    __device__ int64_t list(int64_t j) const { return newest_first ? S - 1 - j : j; }
    __device__ const float* h0_of(int64_t j) const { return h0 ? h0 + list(j) * dim : nullptr; }
};

// The list that holds place p: the last one that begins at or before it.  Called by the whole wave, which looks at 64 lists a step.
// (What a ballot votes on is computed without branches here and below: behind a load that some lanes skipped, the compiler folded the
// skipping lanes' vote away and the two sides saw different results.)
template <typename T>
__device__ int find_list(const Lists<T>& l, int64_t total, int64_t p, int64_t* begin = nullptr) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = l.S, first = 0;
    while (hi - lo > 1) {
        const int64_t by = (hi - lo + kWave - 1) / kWave, j = lo + (lane + 1) * by;
        const int64_t at = l.begin_of(min(j, hi), total);
        const int c = __popcll(__ballot((j < hi) & (at <= p)));
        if (c) {
            const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)at, c - 1), high = (uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)at >> 32), c - 1);
            first = (int64_t)((uint64_t)high << 32 | low);
        }
        lo += c * by;
        hi = min(lo + by, hi);
    }
    if (begin) *begin = first;                // of the list (the walk's first one begins at 0)
    return uniform((int)lo);
}

// What the lanes know of the 64 places from a tile's first one on: lane i the list of the i-th and the gap before its event; bit i of
// `starts` and `ends`, whether that place is the first and the last of its list.
struct Batch {
    int list;
    float gap;
    uint64_t starts, ends;
};

// Of lane i: list base + 1 + i begins at that place of the 64 from p0 on (FORWARD), or list base - i.
template <bool FORWARD, typename T>
__device__ __forceinline__ int border_at(const Lists<T>& l, int64_t total, int64_t p0, int64_t base) {
    const int lane = threadIdx.x & 63;
    const int64_t j = FORWARD ? base + 1 + lane : base - lane;
    const int64_t at = l.begin_of(FORWARD ? min(j, l.S) : max(j, (int64_t)0), total) - p0;
    const int64_t rel = FORWARD ? (j <= l.S ? at : kBatch + 1) : (j >= 0 ? at : -1);
    return (int)min(max(rel, (int64_t)(FORWARD ? 0 : -1)), (int64_t)(kBatch + (FORWARD ? 1 : 0)));
}

// The tile at p0, 0 <= p0 < total.  FORWARD: `from` is its first place's list, `edge` whether that place is the list's first; backward: its
// last place's (the place `last` of the tile), and whether that place is the list's last.
template <bool FORWARD, bool DECAY, typename T>
__device__ __forceinline__ Batch locate(const Lists<T>& l, int64_t total, int64_t p0, int64_t from, bool edge, int last) {
    const int lane = threadIdx.x & 63;
    int passed = 0, more = 0;                   // borders between `from` and the lane's place; and the place after lane 63's (FORWARD), before lane 0's
    int at = border_at<FORWARD>(l, total, p0, from);
    const float time = DECAY ? l.ts[l.row(min(p0 + lane, total - 1), total)] : 0.0f, before = DECAY ? l.ts[l.row(max(p0 - 1, (int64_t)0), total)] : 0.0f;
    bool all = false;                           // every border looked at lies in the batch
    for (int64_t base = from, window = 0;; ++window) {
        const uint64_t some = __ballot(FORWARD ? at <= kBatch : at >= 0);
        if (some) {                             // they come in order: how many lie at or before (beyond) the lane's place
            int n = 0;
#pragma unroll
            for (int by = 32; by; by >>= 1) {
                const int border = __shfl(at, n + by - 1);
                if (FORWARD ? border <= lane : border > lane) n += by;
            }
            const int border = __shfl(at, 63);
            if (n == 63 && (FORWARD ? border <= lane : border > lane)) n = 64;
            passed += n;
            more += __popcll(some);
        }
        all = some == ~0ull;
        if (!all || window == 3) break;
        base += FORWARD ? kWave : -kWave;
        at = border_at<FORWARD>(l, total, p0, base);
    }
    Batch b;
    int list = (int)min(max(from + (FORWARD ? passed : -passed), (int64_t)0), l.S - 1);
    if (all) {                                  // many lists without events: every lane looks for its own
        const int64_t p = p0 + lane;
        int64_t lo = 0, hi = l.S;
        for (int k = 0; k < 31; ++k) {
            const int64_t mid = (lo + hi) >> 1;
            const bool at_or_before = l.begin_of(mid, total) <= p, go = hi - lo > 1;
            lo = (go & at_or_before) ? mid : lo;
            hi = (go & !at_or_before) ? mid : hi;
        }
        list = (int)lo;
    }
    b.list = (int)l.list(list);
    if (all) {
        const int64_t p = p0 + lane, begin = l.begin_of(list, total), end = l.begin_of((int64_t)list + 1, total);
        b.starts = __ballot((p < total) & (begin == p));
        b.ends = __ballot((p < total) & (end == p + 1));
    } else if (FORWARD) {
        const int prev = __shfl_up(passed, 1);
        b.starts = __ballot((lane != 0) & (passed != prev)) | (uint64_t)(edge | (uniform(passed) != 0));
        b.ends = b.starts >> 1 | (uint64_t)(more != __builtin_amdgcn_readlane(passed, 63)) << 63;
    } else {
        const int prev = __shfl_up(passed, 1);
        b.starts = __ballot((lane != 0) & (passed != prev)) | (uint64_t)(more != uniform(passed));
        b.ends = b.starts >> 1 | (uint64_t)edge << last;
    }
    b.gap = 0.0f;
    if (DECAY) {
        float t = __shfl_up(time, 1);
        if (lane == 0) t = before;
        if (b.starts >> lane & 1) t = l.t0 ? l.t0[b.list] : time;
        b.gap = gap_of(time, t);
    }
    return b;
}

// Has the wave wait for values that it has read, here rather than at their first use: the code of a group branches, and from behind a
// branch the compiler can only wait for as few requests on their way as its shortest path has, the next group's among them.
template <typename P>
__device__ __forceinline__ void arrive(P& v) {
    if constexpr (sizeof(P) == 2) {
        uint32_t bits = __builtin_bit_cast(uint16_t, v);
        asm volatile("" : "+v"(bits));
        v = __builtin_bit_cast(P, (uint16_t)bits);
    } else {
        float word = __builtin_bit_cast(float, v);
        asm volatile("" : "+v"(word));
        v = __builtin_bit_cast(P, word);
    }
}
template <typename P, int N>
__device__ __forceinline__ void arrive(P (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) arrive(v[i]);
}

// Rows of an fp32 array [S, dim] (h0 at the first events of lists, dlast at the last ones) that a group of rows needs: the first two are
// read with the group's rows, any more when their event comes.
template <int V>
struct Edges {
    float v[2][V] = {};
    int left;                           // of the two

    template <bool FORWARD>
    __device__ void read(const float* base, const Batch& b, uint32_t mask, int q, int dim, int c) {
        left = 2;
        if (!base) {
            left = 1 << 30;
            return;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (!mask) break;
            const int r = FORWARD ? __builtin_ctz(mask) : 31 - __builtin_clz(mask);
            mask &= ~(1u << r);
            load_floats<V>(at(base, b, q + r, dim) + c, v[k]);
        }
    }
    __device__ static const float* at(const float* base, const Batch& b, int place, int dim) {
        return base + (uint64_t)(uint32_t)__builtin_amdgcn_readlane(b.list, place) * (uint32_t)dim;
    }
    __device__ void take(const float* base, const Batch& b, int place, int dim, int c, float (&to)[V]) {
        if (left > 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                to[i] = base ? v[0][i] : 0.0f;
                v[0][i] = v[1][i];
            }
            --left;
        } else {
            load_floats<V>(at(base, b, place, dim) + c, to);
            arrive(to);
        }
    }
};

// f and z of a lane's channels.
template <int V, bool DECAY, typename P>
__device__ __forceinline__ void gates(const P& u, const float (&rate)[V], float gap, float (&z)[V], float (&rest)[V], float (&f)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        gate_of(u.get(i), z[i], rest[i]);
        f[i] = DECAY ? rest[i] * __builtin_amdgcn_exp2f(rate[i] * gap) : rest[i];
    }
}

// Channels of a lane, V from c on, in a block of 64 V.  Lanes beyond the last channel repeat it (they store what it stores).
template <int V>
__device__ __forceinline__ int channel_of(int dim, int block) { return min(block * kWave * V + (int)(threadIdx.x & 63) * V, dim - V); }

// An array's rows along the walk: place p lies at origin + p * step bytes.  Everything but the channel is the same for the whole wave:
// the addresses are the scalar unit's work, two additions a row.
#if defined(__HIP_DEVICE_COMPILE__)
#define TNS_GLOBAL __attribute__((address_space(1)))
#else
#define TNS_GLOBAL                      // (the host's pass over the kernels knows no address spaces)
#endif
using Global = TNS_GLOBAL char*;
struct Along {
    Global origin;
    int64_t step;
    template <typename L, typename T>
    __device__ Along(const L& l, T* base, int64_t ld, int64_t total) {
        T* const first = l.newest_first ? base + (total - 1) * ld : base;
        origin = (Global)(char*)const_cast<std::remove_const_t<T>*>(first);
        step = (l.newest_first ? -ld : ld) * (int64_t)sizeof(T);
    }
    __device__ Global at(int64_t p) const { return origin + p * step; }
    // The next row (the one before).  Opaque to the compiler, which would keep the sixteen multiples of the step that a group takes in
    // scalar registers, for every array, and move them to vector registers and back as there are not that many.
    __device__ Global next(Global q) const { q += step; asm("" : "+s"(q)); return q; }
    __device__ Global back(Global q) const { q -= step; asm("" : "+s"(q)); return q; }
};
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_row(Global row, uint32_t bytes) {
    asm("" : "+v"(bytes));              // (stays 32 bits: address = scalar base + vector offset)
    return *(const TNS_GLOBAL Pack<T, V>*)(row + bytes);
}
// STREAM: with the non-temporal hint (streams_out).
template <bool STREAM, typename T, int V>
__device__ __forceinline__ void store_row(Global row, uint32_t bytes, const float (&v)[V]) {
    asm("" : "+v"(bytes));
    using Bits = std::conditional_t<sizeof(T) * V == 4, uint32_t, uint16_t>;
    Bits bits;
    if constexpr (V == 2) {
        using Two = float __attribute__((ext_vector_type(2)));
        using Halves = __bf16 __attribute__((ext_vector_type(2)));
        bits = __builtin_bit_cast(Bits, __builtin_convertvector((Two{v[0], v[1]}), Halves));
    } else {
        bits = __builtin_bit_cast(Bits, as_value<T>(v[0]));
    }
    if constexpr (STREAM) __builtin_nontemporal_store(bits, (TNS_GLOBAL Bits*)(row + bytes));
    else *(TNS_GLOBAL Bits*)(row + bytes) = bits;
}
// The kSaved rows from place p on, 0 <= p < total; the walk's last row again where there are no more.
template <typename T, int V>
__device__ __forceinline__ void read_rows(Pack<T, V> (&a)[kSaved], const Along& rows, int64_t total, int64_t p, int c) {
    const uint32_t bytes = (uint32_t)c * sizeof(T);
    Global q = rows.at(p);
    if (p + kSaved <= total) {
#pragma unroll
        for (int r = 0; r < kSaved; ++r, q = rows.next(q)) a[r] = load_row<T, V>(q, bytes);
    } else {
        const int n = (int)(total - p);
#pragma unroll
        for (int r = 0; r < kSaved; ++r) {
            a[r] = load_row<T, V>(q, bytes);
            if (r + 1 < n) q = rows.next(q);
        }
    }
}
// Runs go(r) for the first n of a group's rows, in order or from the last one back.
template <typename F>
__device__ __forceinline__ void each_row(int n, const F& go) {
#pragma unroll
    for (int r = 0; r < kSaved; ++r)
        if (r < n) go(r);
}
template <typename F>
__device__ __forceinline__ void each_row_back(int n, const F& go) {
#pragma unroll
    for (int r = kSaved - 1; r >= 0; --r)
        if (r < n) go(r);
}

// Rate of the decay in powers of two.  Rounded, as its product with the gap is: exp(-decay gap) has a relative error of (2.5 decay gap + 3) 2^-24
// at most, of which the product alone, in whatever base, would leave 1 (gate_of says what more bits would cost).
template <int V, bool DECAY, typename T>
__device__ __forceinline__ void rates(const Lists<T>& l, int c, float (&rate)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) rate[i] = DECAY ? -kLog2e * l.decay[c + i] : 0.0f;
}

// A workgroup's share: block of channels and the q-th group of tiles.  Workgroups go round the eight XCDs; those of one group of tiles come
// eight apart and so meet in one L2, as their blocks of channels share cache lines wherever rows are no multiple of them (172 channels of
// fp32, 0.8 M rows: states 452 -> 338 us, gradients 776 -> 599 us).
constexpr int kXcds = 8;
struct Share {
    int64_t q;
    int block;
    __device__ Share(int64_t workgroup, int blocks) {
        const int64_t at = workgroup % (kXcds * blocks);
        q = workgroup / (kXcds * blocks) * kXcds + at % kXcds;
        block = (int)(at / kXcds);
    }
};
constexpr int64_t workgroups_of(int64_t groups, int blocks) { return (groups + kXcds - 1) / kXcds * kXcds * blocks; }
// One of the launches that a walk takes (a launch has fewer than 2^32 threads): the groups of tiles from `first` on; workgroups from
// `workgroups` on have no share of the walk.
struct Piece {
    int64_t first;
    unsigned workgroups;
    int blocks;
};

// ---- carries -------------------------------------------------------------------------------------------
// The walk is cut into tiles, eight tiles to a span.  What enters a tile is the state before its first event, or (backward) what the
// events after its last one send back.  A tile whose part of the crossing list begins (ends) inside it knows what it hands on, B (closed);
// one that lies inside a list altogether hands on A * what enters + B (open).  A workgroup of a wave for every tile of a span finds both
// and puts them together: for every tile what its span's entering carry becomes on the way to it, and what it becomes behind the span;
// k_recur_join then goes along the spans.  All in a fixed order, so that a result does not depend on which wave was first.
constexpr int kSpan = 8;
constexpr uint32_t kCrosses = 0x80000000u;
struct Carries {
    float *b, *a;                       // [tiles, dim]: what enters a tile is b, or a * (what enters its span) + b where `open`
    float *span_b, *span_a;             // [spans, dim]: what the span before hands on; after the join, span_b is what enters
    uint8_t *open, *span_open;
    uint32_t* list;                     // list of a tile's first place, or (backward) its last one; kCrosses: it reaches into the tile beside
    int64_t tile_rows, tiles;
};

template <int V>
struct Effect {
    float a[V], b[V];
    bool open;
};
// `e` followed by an effect that lies in LDS.
template <int V>
__device__ __forceinline__ void follow(Effect<V>& e, const float* a, const float* b, bool open) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        e.b[i] = open ? a[i] * e.b[i] + b[i] : b[i];
        e.a[i] *= a[i];
    }
    e.open = e.open && open;
}

template <int V, bool FORWARD>
__device__ __forceinline__ void join_span(const Carries& t, const Effect<V>& mine, int64_t span, int64_t tile, int dim, int c, bool lead) {
    __shared__ float s_a[kSpan][kWave * V], s_b[kSpan][kWave * V];
    __shared__ int s_open[kSpan];
    const int lane = threadIdx.x & 63, w = uniform((int)(threadIdx.x >> 6));
    store_floats<V>(&s_a[w][lane * V], mine.a);
    store_floats<V>(&s_b[w][lane * V], mine.b);
    if (lane == 0) s_open[w] = mine.open;
    __syncthreads();
    Effect<V> e;
#pragma unroll
    for (int i = 0; i < V; ++i) { e.a[i] = 1.0f; e.b[i] = 0.0f; }
    e.open = true;
    const int before = FORWARD ? w : kSpan - 1 - w;      // tiles of the span on the way to this one
    for (int k = 0; k < before; ++k) {
        const int from = FORWARD ? k : kSpan - 1 - k;
        follow<V>(e, &s_a[from][lane * V], &s_b[from][lane * V], s_open[from]);
    }
    if (tile < t.tiles) {
        store_floats<V>(t.b + tile * dim + c, e.b);
        if (e.open) store_floats<V>(t.a + tile * dim + c, e.a);
        if (lead) t.open[tile] = e.open;
    }
    const int64_t to = FORWARD ? span + 1 : span - 1;
    if (before == kSpan - 1 && to >= 0 && to * kSpan < t.tiles) {
        follow<V>(e, mine.a, mine.b, mine.open);
        store_floats<V>(t.span_b + to * dim + c, e.b);
        if (e.open) store_floats<V>(t.span_a + to * dim + c, e.a);
        if (lead) t.span_open[to] = e.open;
    }
}
// What enters a tile, where its list crosses the border: read before that is known (whatever lies there then), so that it is no request more to wait for.
template <int V>
struct Entering {
    float a[V], b[V], e[V];
    int open;
    __device__ Entering(const Carries& t, int64_t tile, int dim, int c) {
        open = t.open[tile];
        load_floats<V>(t.b + tile * dim + c, b);
        load_floats<V>(t.a + tile * dim + c, a);
        load_floats<V>(t.span_b + tile / kSpan * dim + c, e);
    }
    __device__ void take(bool crosses, float (&v)[V]) const {
        const bool all = uniform(open);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = !crosses ? 0.0f : all ? a[i] * e[i] + b[i] : b[i];
    }
};

// First pass of the states: reads the rows of every list that crosses the end of a tile, from the list's begin or the tile's on.  For short
// lists that is half a list a tile (1.14 M rows of 128 bf16 channels in lists of ten: 29 us), for long ones all rows, and then bound by memory
// (0.79 M rows of 256 bf16 channels: 0.82 GB in 165 us, 5.0 TB/s).  Sixteen tiles a workgroup took a sixth more: two workgroups fill a compute unit,
// and their waves wait for each other.
template <typename T, int V, bool DECAY>
__global__ void __launch_bounds__(kSpan * kWave) k_recur_tails(const Lists<T> l, const Carries t, const Piece piece) {
    const Share share(blockIdx.x, piece.blocks);
    const int64_t span = piece.first + share.q, tile = span * kSpan + uniform((int)(threadIdx.x >> 6));
    if (span * kSpan >= t.tiles) return;
    const int c = channel_of<V>(l.dim, share.block);
    const bool lead = share.block == 0 && (threadIdx.x & 63) == 0;
    const int64_t total = l.total(), begin = tile * t.tile_rows, end = begin + t.tile_rows;
    Effect<V> e = {};
    if (end < total) {
        int64_t first;
        const int j = find_list(l, total, end, &first);
        if (lead) t.list[tile + 1] = (uint32_t)j | (first < end ? kCrosses : 0u);
        if (first < end) {
            e.open = first < begin;
            float rate[V];
            rates<V, DECAY>(l, c, rate);
            load_or_zero<V>(e.open || !l.h0 ? nullptr : l.h0_of(j) + c, e.b);
#pragma unroll
            for (int i = 0; i < V; ++i) e.a[i] = 1.0f;
            Pack<T, V> u[kSaved], x[kSaved];
            const Along rows_u(l, l.u, l.ld_u, total), rows_x(l, l.x, l.ld_x, total);
            for (int64_t p = max(first, begin); p < end; p += kSaved) {
                read_rows<T, V>(u, rows_u, end, p, c);
                read_rows<T, V>(x, rows_x, end, p, c);
                float gap = 0.0f;
                if (DECAY) {
                    const int64_t q = min(p + (threadIdx.x & (kSaved - 1)), end - 1);
                    const float t1 = l.ts[l.row(q, total)], t0 = l.ts[l.row(max(q - 1, (int64_t)0), total)];
                    gap = gap_of(t1, q != first ? t0 : l.t0 ? l.t0[l.list(j)] : t1);
                }
                const int n = (int)min(end - p, (int64_t)kSaved);
                each_row(n, [&](int r) {
                    float z[V], rest[V], f[V];
                    gates<V, DECAY>(u[r], rate, DECAY ? read_lane(gap, r) : 0.0f, z, rest, f);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        e.b[i] = f[i] * e.b[i] + z[i] * x[r].get(i);
                        e.a[i] *= f[i];
                    }
                });
            }
        }
    }
    join_span<V, true>(t, e, span, tile, l.dim, c, lead);
}

// First pass of the gradients: what the rows behind a tile's begin send back over it, from u and dh.  As k_recur_tails (0.79 M rows of 256
// bf16 channels: 167 us).
template <typename T, int V, bool DECAY>
__global__ void __launch_bounds__(kSpan * kWave) k_recur_heads(const Lists<T> l, const Carries t, const Piece piece, const T* dh, int64_t ld_dh, const float* dlast) {
    const Share share(blockIdx.x, piece.blocks);
    const int64_t span = piece.first + share.q, tile = span * kSpan + uniform((int)(threadIdx.x >> 6));
    if (span * kSpan >= t.tiles) return;
    const int c = channel_of<V>(l.dim, share.block);
    const bool lead = share.block == 0 && (threadIdx.x & 63) == 0;
    const int64_t total = l.total(), begin = tile * t.tile_rows;
    Effect<V> e = {};
    if (begin > 0 && begin < total) {
        const int j = find_list(l, total, begin - 1);
        const int64_t last = uniform(l.begin_of((int64_t)j + 1, total)), end = min(last, begin + t.tile_rows);
        if (lead) t.list[tile - 1] = (uint32_t)j | (last > begin ? kCrosses : 0u);
        if (last > begin) {
            e.open = end < last;
            float rate[V];
            rates<V, DECAY>(l, c, rate);
            load_or_zero<V>(e.open || !dlast ? nullptr : dlast + l.list(j) * l.dim + c, e.b);
#pragma unroll
            for (int i = 0; i < V; ++i) e.a[i] = 1.0f;
            Pack<T, V> u[kSaved], d[kSaved] = {};
            const Along rows_u(l, l.u, l.ld_u, total), rows_d(l, dh, ld_dh, total);
            for (int64_t p = begin + (end - 1 - begin) / kSaved * kSaved; p >= begin; p -= kSaved) {
                read_rows<T, V>(u, rows_u, end, p, c);
                if (dh) read_rows<T, V>(d, rows_d, end, p, c);
                float gap = 0.0f;
                if (DECAY) {
                    const int64_t q = min(p + (threadIdx.x & (kSaved - 1)), end - 1);
                    gap = gap_of(l.ts[l.row(q, total)], l.ts[l.row(q - 1, total)]);      // (the list's first event is not here)
                }
                const int n = (int)min(end - p, (int64_t)kSaved);
                each_row_back(n, [&](int r) {
                    float z[V], rest[V], f[V];
                    gates<V, DECAY>(u[r], rate, DECAY ? read_lane(gap, r) : 0.0f, z, rest, f);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        e.b[i] += d[r].get(i);
                        e.b[i] *= f[i];
                        e.a[i] *= f[i];
                    }
                });
            }
        }
    }
    join_span<V, false>(t, e, span, tile, l.dim, c, lead);
}

// Puts the open spans' carries together, from span 1 on or (BACKWARD) from the last but one down: kChannels channels a workgroup, each
// with kParts parts of the spans: every thread joins its part, the parts are scanned, every thread goes through its part again.  Bound by
// how fast a few compute units read 32 bytes of a row each: 22 us for 1536 spans of 256 channels, 2 to 5 where no list is that long.
constexpr int kChannels = 8, kParts = 1024 / kChannels, kAtOnce = 8;
template <bool BACKWARD>
__global__ void __launch_bounds__(1024) k_recur_join(int64_t spans, int dim, float* carry, const float* factor, const uint8_t* open) {
    __shared__ float s_a[2][kParts][kChannels], s_b[2][kParts][kChannels];
    __shared__ int s_any;
    if (threadIdx.x == 0) s_any = 0;
    __syncthreads();
    const int64_t n = spans - 1;                            // carries that spans have written
    auto at = [&](int64_t i) { return BACKWARD ? n - 1 - i : i + 1; };
    int any = 0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) any |= open[at(i)];
    if (any) s_any = 1;
    __syncthreads();
    if (!s_any) return;
    const int part = threadIdx.x / kChannels, ch = threadIdx.x % kChannels, c = min((int)blockIdx.x * kChannels + ch, dim - 1);
    const bool mine = (int)blockIdx.x * kChannels + ch < dim;
    const int64_t per = (n + kParts - 1) / kParts, begin = min(part * per, n), end = min(begin + per, n);
    float v[kAtOnce], f[kAtOnce];
    uint8_t is[kAtOnce];
    auto read = [&](int64_t i) {
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r) {
            const int64_t k = at(min(i + r, end - 1));
            is[r] = open[k];
            v[r] = carry[k * dim + c];
            f[r] = factor[k * dim + c];                     // (whatever lies there if the span was closed)
        }
    };
    float a = 1.0f, b = 0.0f;                               // what the part does to the carry that enters it: b alone once a span was closed
    bool all = true;
    for (int64_t i = begin; i < end; i += kAtOnce) {
        read(i);
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r)
            if (i + r < end) {
                b = is[r] ? f[r] * b + v[r] : v[r];
                a = is[r] ? a * f[r] : 1.0f;
                all = all && is[r];
            }
    }
    if (!all) a = __uint_as_float(0x7fc00000u);             // marks a part that lets nothing through
    auto join = [](float la, float lb, float ra, float rb, float& oa, float& ob) {      // left part, then right part; a NaN marks "closed"
        ob = ra == ra ? ra * lb + rb : rb;
        oa = ra == ra && la == la ? ra * la : __uint_as_float(0x7fc00000u);
    };
    s_a[0][part][ch] = a;
    s_b[0][part][ch] = b;
    int from = 0;
    for (int by = 1; by < kParts; by *= 2, from ^= 1) {
        __syncthreads();
        float oa = s_a[from][part][ch], ob = s_b[from][part][ch];
        if (part >= by) join(s_a[from][part - by][ch], s_b[from][part - by][ch], oa, ob, oa, ob);
        s_a[from ^ 1][part][ch] = oa;
        s_b[from ^ 1][part][ch] = ob;
    }
    __syncthreads();
    float enter = part ? s_b[from][part - 1][ch] : 0.0f;    // (the first span is never open: no list crosses the walk's ends)
    for (int64_t i = begin; i < end; i += kAtOnce) {
        read(i);
#pragma unroll
        for (int r = 0; r < kAtOnce; ++r)
            if (i + r < end) {
                enter = is[r] ? f[r] * enter + v[r] : v[r];
                if (mine && is[r]) carry[at(i + r) * dim + c] = enter;
            }
    }
}

// ---- states --------------------------------------------------------------------------------------------

// Rows of an array [S, dim] that belong to lists without events: those of h0, or zero.  64 lists a wave.
template <typename T>
__device__ void fill_empty(const Lists<T>& l, int64_t first, const float* from, float* to) {
    const int lane = threadIdx.x & 63;
    const int64_t total = l.total(), s = first + lane;
    const int64_t begin = min(max(l.rowptr[min(s, l.S)], (int64_t)0), total), end = min(max(l.rowptr[min(s + 1, l.S)], (int64_t)0), total);
    uint64_t empty = __ballot((s < l.S) & (begin >= end));
    for (; empty; empty &= empty - 1) {
        const int64_t at = (first + __ffsll((unsigned long long)empty) - 1) * l.dim;
        for (int c = lane; c < l.dim; c += kWave) to[at + c] = from ? from[at + c] : 0.0f;
    }
}

// Zeros in the rows of a tile that belong to no list (the tile's rows along memory: they lie behind the walk in either order).
template <typename T, int V>
__device__ void zero_rows(const Lists<T>& l, T* out, int64_t ld, int64_t begin, int64_t end, int64_t total, int c) {
    end = min(end, l.rows);
    for (int64_t p = max(begin, total); p < end; ++p)
#pragma unroll
        for (int i = 0; i < V; ++i) out[p * ld + c + i] = T{};
}

// h = f h + z x along the rows of a tile, V channels a lane, 16 rows in registers and the next 16 on their way.  The list a row belongs to, and
// the gap before it, lie in the lanes (64 rows at a time); what is the same for the wave (addresses, first and last rows) is the scalar
// unit's.  Bound by memory: 0.79 M rows of 256 bf16 channels, all states written and saved, 1.26 GB in 219 us (5.8 TB/s); 0.80 M rows of
// 172 fp32 channels, 1.70 GB in 334 us (5.1); 0.91 M of 128 fp32, 1.39 GB in 233 us (6.0); lists of ten, last states only, 1.14 M rows of 128
// bf16: 0.69 GB in 141 us (4.9).  Four waves a SIMD: with the fifth that the registers have room for, the walk met less of what the first pass left
// in the caches (0.80 M rows of 172 fp32: 348 us instead of 333; the others the same or 1 % more).
template <typename T, int V, bool DECAY, bool STREAM>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(4, 4))) k_recur_states(const Lists<T> l, const Carries t, const Piece piece, T* h_out, int64_t ld_h, float* last, float* saved) {
    const int wave = uniform((int)(threadIdx.x >> 6));
    if (blockIdx.x >= piece.workgroups) {
        const int64_t first = ((int64_t)(blockIdx.x - piece.workgroups) * kWaves + wave) * kWave;
        if (last && first < l.S) fill_empty(l, first, l.h0, last);
        return;
    }
    const Share share(blockIdx.x, piece.blocks);
    const int64_t quad = piece.first + share.q, tile = ((t.tiles + kWaves - 1) / kWaves - 1 - quad) * kWaves + wave;
    const int c = channel_of<V>(l.dim, share.block);
    if (tile < 0 || tile >= t.tiles) return;
    const Entering<V> entering(t, tile, l.dim, c);
    const uint32_t known = tile ? t.list[tile] : 0u;
    const int64_t total = l.total(), begin = tile * t.tile_rows, end = min(begin + t.tile_rows, total);
    if (l.zero_beyond && h_out) zero_rows<T, V>(l, h_out, ld_h, begin, begin + t.tile_rows, total, c);
    if (begin >= end) return;
    Pack<T, V> u[kSaved], x[kSaved];
    const Along rows_u(l, l.u, l.ld_u, total), rows_x(l, l.x, l.ld_x, total);
    const Along rows_h(l, h_out, ld_h, total);
    read_rows<T, V>(u, rows_u, total, begin, c);
    read_rows<T, V>(x, rows_x, total, begin, c);
    float rate[V], h[V];
    rates<V, DECAY>(l, c, rate);
    const int j = tile ? uniform((int)(known & ~kCrosses)) : find_list(l, total, 0);
    const bool fresh = !uniform((int)(known & kCrosses));
    entering.take(!fresh, h);
    const Batch b = locate<true, DECAY>(l, total, begin, j, fresh, 0);
    Edges<V> enter;
    enter.template read<true>(l.h0, b, (uint32_t)b.starts & kGroupMask, 0, l.dim, c);
    for (int64_t p = begin; p < end; p += kSaved) {
        const int q = (int)(p - begin);
        const bool more = p + kSaved < end;
        arrive(u);
        arrive(x);
        arrive(enter.v);
        Pack<T, V> next_u[kSaved], next_x[kSaved];
        Edges<V> next_enter;
        if (more) {
            read_rows<T, V>(next_u, rows_u, total, p + kSaved, c);
            read_rows<T, V>(next_x, rows_x, total, p + kSaved, c);
            next_enter.template read<true>(l.h0, b, (uint32_t)(b.starts >> (q + kSaved)) & kGroupMask, q + kSaved, l.dim, c);
        }
        const int n = (int)min(end - p, (int64_t)kSaved);
        const uint32_t starts = (uint32_t)(b.starts >> q), ends = (uint32_t)(b.ends >> q);
        if (saved) store_floats<V>(saved + p / kSaved * l.dim + c, h);
        Global to = rows_h.at(p);
        each_row(n, [&](int r) {
            if (starts >> r & 1) enter.take(l.h0, b, q + r, l.dim, c, h);
            float z[V], rest[V], f[V];
            gates<V, DECAY>(u[r], rate, DECAY ? read_lane(b.gap, q + r) : 0.0f, z, rest, f);
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = f[i] * h[i] + z[i] * x[r].get(i);
            if (h_out) store_row<STREAM, T, V>(to, (uint32_t)c * sizeof(T), h);
            to = rows_h.next(to);
            if (ends >> r & 1)
                if (last) store_floats<V>(last + (Edges<V>::at(last, b, q + r, l.dim) - last) + c, h);
        });
#pragma unroll
        for (int r = 0; r < kSaved; ++r) { u[r] = next_u[r]; x[r] = next_x[r]; }
        enter = next_enter;
    }
}

// ---- gradients -----------------------------------------------------------------------------------------

// The gradients of a tile's rows, group by group from the last one back.  A group's states are computed again from the one saved before it
// (a sixteenth of what reading them all would cost, and they stay in fp32), then the group is walked back.  The next rows of u and x are on
// their way during the walk back, those of dh during the walk forward: a second set of registers for them left one wave a SIMD instead of
// two.  Bound by memory: 0.79 M rows of 256 bf16 channels, 2.05 GB in 394 us (5.2 TB/s); 0.80 M of 172 fp32, 2.78 GB in 607 us (4.6); lists
// of ten, 1.14 M rows of 128 bf16, 1.28 GB in 272 us (4.7).
template <typename T, int V, bool DECAY, bool STREAM>
__global__ void __launch_bounds__(256) k_recur_grads(const Lists<T> l, const Carries t, const Piece piece, const float* saved, const T* dh, int64_t ld_dh, const float* dlast,
                                                     T* du, int64_t ld_du, T* dx, int64_t ld_dx, float* dh0, float* sums) {
    const int wave = uniform((int)(threadIdx.x >> 6));
    if (blockIdx.x >= piece.workgroups) {
        const int64_t first = ((int64_t)(blockIdx.x - piece.workgroups) * kWaves + wave) * kWave;
        if (dh0 && first < l.S) fill_empty(l, first, dlast, dh0);
        return;
    }
    const Share share(blockIdx.x, piece.blocks);
    const int64_t quad = piece.first + share.q, tile = ((t.tiles + kWaves - 1) / kWaves - 1 - quad) * kWaves + wave;
    const int c = channel_of<V>(l.dim, share.block);
    const int64_t total = l.total(), begin = tile * t.tile_rows, end = min(begin + t.tile_rows, total);
    float sum[V] = {};
    if (l.zero_beyond && tile >= 0) {
        zero_rows<T, V>(l, du, ld_du, begin, begin + t.tile_rows, total, c);
        zero_rows<T, V>(l, dx, ld_dx, begin, begin + t.tile_rows, total, c);
    }
    if (tile >= 0 && begin < end) {         // (and so tile < t.tiles)
        const Entering<V> entering(t, tile, l.dim, c);
        const uint32_t known = end < total ? t.list[tile] : 0u;
        const int64_t last_group = begin + (end - 1 - begin) / kSaved * kSaved;
        Pack<T, V> u[kSaved], x[kSaved], d[kSaved] = {};      // (d stays zero without dh)
        float enter[V];                                     // state before the group
        const Along rows_u(l, l.u, l.ld_u, total), rows_x(l, l.x, l.ld_x, total), rows_d(l, dh, ld_dh, total);
        const Along rows_du(l, du, ld_du, total), rows_dx(l, dx, ld_dx, total);
        auto read_inputs = [&](int64_t p) {
            read_rows<T, V>(u, rows_u, total, p, c);
            read_rows<T, V>(x, rows_x, total, p, c);
            load_floats<V>(saved + p / kSaved * l.dim + c, enter);
        };
        auto read_grads = [&](int64_t p) {
            if (dh) read_rows<T, V>(d, rows_d, total, p, c);
        };
        read_inputs(last_group);
        read_grads(last_group);
        float rate[V], back[V];
        rates<V, DECAY>(l, c, rate);
        const int j = end < total ? uniform((int)(known & ~kCrosses)) : find_list(l, total, end - 1);
        const bool over = end == total || !uniform((int)(known & kCrosses));
        entering.take(!over, back);
        const Batch b = locate<false, DECAY>(l, total, begin, j, over, (int)(end - 1 - begin));
        Edges<V> start, leave;
        auto part = [](uint64_t bits, int q) { return (uint32_t)(bits >> q) & kGroupMask; };
        int q = (int)(last_group - begin);
        start.template read<true>(l.h0, b, part(b.starts, q), q, l.dim, c);
        leave.template read<false>(dlast, b, part(b.ends, q), q, l.dim, c);
        for (int64_t p = last_group; p >= begin; p -= kSaved) {
            const bool more = p > begin;
            const int n = (int)min(end - p, (int64_t)kSaved);
            const uint32_t starts = (uint32_t)(b.starts >> q), ends = (uint32_t)(b.ends >> q);
            arrive(u);
            arrive(x);
            arrive(enter);
            arrive(start.v);
            float h[V];
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = enter[i];
            // Forward through the group: dx = z back, du = slope back, and what the event keeps of the state before it.
            float z[kSaved][V], f[kSaved][V], slope[kSaved][V], kept[kSaved][V];
            each_row(n, [&](int r) {
                if (starts >> r & 1) start.take(l.h0, b, q + r, l.dim, c, h);
                float rest[V];
                gates<V, DECAY>(u[r], rate, DECAY ? read_lane(b.gap, q + r) : 0.0f, z[r], rest, f[r]);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float in = x[r].get(i);
                    kept[r][i] = f[r][i] * h[i];
                    slope[r][i] = z[r][i] * (rest[i] * in - kept[r][i]);
                    h[i] = kept[r][i] + z[r][i] * in;
                }
            });
            arrive(d);
            arrive(leave.v);
            if (more) {
                read_inputs(p - kSaved);
                start.template read<true>(l.h0, b, part(b.starts, q - kSaved), q - kSaved, l.dim, c);
            }
            Global to_x = rows_dx.at(p + n - 1), to_u = rows_du.at(p + n - 1);
            each_row_back(n, [&](int r) {
                if (ends >> r & 1) leave.take(dlast, b, q + r, l.dim, c, back);
                const float g = DECAY ? read_lane(b.gap, q + r) : 0.0f;
                float vu[V], vx[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    back[i] += d[r].get(i);
                    vx[i] = z[r][i] * back[i];
                    vu[i] = slope[r][i] * back[i];
                    if (DECAY) sum[i] -= kept[r][i] * back[i] * g;
                    back[i] *= f[r][i];
                }
                store_row<STREAM, T, V>(to_x, (uint32_t)c * sizeof(T), vx);
                store_row<STREAM, T, V>(to_u, (uint32_t)c * sizeof(T), vu);
                to_x = rows_dx.back(to_x);
                to_u = rows_du.back(to_u);
                if (starts >> r & 1)
                    if (dh0) store_floats<V>(dh0 + (Edges<V>::at(dh0, b, q + r, l.dim) - dh0) + c, back);
            });
            if (more) {
                read_grads(p - kSaved);
                leave.template read<false>(dlast, b, part(b.ends, q - kSaved), q - kSaved, l.dim, c);
            }
            q -= kSaved;
        }
    }
    if (DECAY && sums) {                // the workgroup's share
        __shared__ float s_sum[kWaves][kWave * V];
        store_floats<V>(&s_sum[wave][(threadIdx.x & 63) * V], sum);
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (int k = 1; k < kWaves; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += s_sum[k][(threadIdx.x & 63) * V + i];
        if (quad * kWaves < t.tiles) store_floats<V>(sums + quad * l.dim + c, sum);
    }
}

// Sums of the workgroups' shares, kChannels channels a workgroup, in a fixed order (4469 shares of 128 channels: 13 us).
__global__ void __launch_bounds__(1024) k_recur_sums(const float* sums, int64_t shares, int dim, float* out) {
    __shared__ float s_sum[kParts][kChannels];
    const int part = threadIdx.x / kChannels, ch = threadIdx.x % kChannels, c = (int)blockIdx.x * kChannels + ch;
    float sum = 0.0f;
    if (c < dim)
        for (int64_t k = part; k < shares; k += kParts * kAtOnce) {
            float v[kAtOnce];
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) v[r] = k + r * kParts < shares ? sums[(k + r * kParts) * dim + c] : 0.0f;
#pragma unroll
            for (int r = 0; r < kAtOnce; ++r) sum += v[r];
        }
    s_sum[part][ch] = sum;
    for (int n = kParts / 2; n; n /= 2) {
        __syncthreads();
        if (part < n) s_sum[part][ch] += s_sum[part + n][ch];
    }
    if (part == 0 && c < dim) out[c] = s_sum[0][ch];
}

// ---- one event per node ----------------------------------------------------------------------------------

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
    T v[N];
};
// G lanes to an event, VEC channels a lane at a time.  Bound by memory; the states lie anywhere, so a row of them is read in as few
// requests as there are: 66600 events of 172 bf16 channels, 161 MB in 33 us (4.9 TB/s); a workgroup of 256 threads to an event, a channel
// each, took 63.  600 events of 100: 3.4 us, the launch and three reads one after the other.
template <typename T, int VEC, int G>
__global__ void __launch_bounds__(256) k_recur_step(int64_t B, int64_t num_ids, int dim, const int32_t* __restrict__ ids, const T* __restrict__ u, int64_t ld_u,
                                                    const T* __restrict__ x, int64_t ld_x, const float* __restrict__ ts, const float* __restrict__ decay, float* state,
                                                    float* state_ts, T* __restrict__ out, int64_t ld_out) {
    for (int64_t b = ((int64_t)blockIdx.x * 256 + threadIdx.x) / G; b < B; b += (int64_t)gridDim.x * (256 / G)) {
        const int64_t id = ids[b];
        const bool held = id >= 0 && id < num_ids;
        float gap = 0.0f;
        if (held && ts) {
            gap = gap_of(ts[b], state_ts[id]);
            if (threadIdx.x % G == 0) state_ts[id] = ts[b];      // (the lanes of an event are in one wave: all have read it)
        }
        for (int c = threadIdx.x % G * VEC; c < dim; c += G * VEC) {
            const Vec<T, VEC> vu = *reinterpret_cast<const Vec<T, VEC>*>(u + b * ld_u + c), vx = *reinterpret_cast<const Vec<T, VEC>*>(x + b * ld_x + c);
            Vec<float, VEC> h = {}, rate = {};
            if (held) h = *reinterpret_cast<const Vec<float, VEC>*>(state + id * dim + c);
            if (ts) rate = *reinterpret_cast<const Vec<float, VEC>*>(decay + c);
            Vec<T, VEC> to;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float z, f;
                gate_of(as_float(vu.v[i]), z, f);
                if (ts) f *= __builtin_amdgcn_exp2f(-kLog2e * rate.v[i] * gap);
                h.v[i] = held ? f * h.v[i] + z * as_float(vx.v[i]) : 0.0f;
                to.v[i] = as_value<T>(h.v[i]);
            }
            if (held) *reinterpret_cast<Vec<float, VEC>*>(state + id * dim + c) = h;
            if (out) *reinterpret_cast<Vec<T, VEC>*>(out + b * ld_out + c) = to;
        }
    }
}

int check(const tns_recur* r) {
    if (!r) return fail(TNS_EINVAL, "null description of the lists");
    if (r->S < 0 || r->rows < 0) return fail(TNS_EINVAL, "negative number of lists or rows");
    if (r->S > (int64_t)INT32_MAX || r->rows > (int64_t)1 << 40) return fail(TNS_ESIZE, "more than 2^31-1 lists or 2^40 rows");
    if (r->dim < 1 || r->dim > 1 << 16) return fail(TNS_EINVAL, "dim must be in [1, 2^16]");
    if (r->dtype != TNS_F32 && r->dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if ((r->flags & ~(TNS_NEWEST_FIRST | TNS_ZERO_BEYOND)) || r->reserved) return fail(TNS_EINVAL, "unknown flag");
    return TNS_OK;
}

// The arrays of the lists (checked where there are any).
int check_arrays(const tns_recur* r) {
    if (int e = check(r)) return e;
    if (r->S > 0 && !r->d_rowptr) return fail(TNS_EINVAL, "null rowptr");
    if (r->rows > 0 && (!r->d_u || !r->d_x)) return fail(TNS_EINVAL, "null u or x");
    if (r->ld_u < r->dim || r->ld_x < r->dim) return fail(TNS_EINVAL, "rows of u or x overlap");
    if (r->rows > 0 && !r->d_ts != !r->d_decay) return fail(TNS_EINVAL, "ts and decay come together");
    if (r->rows > 0 && r->d_t0 && !r->d_ts) return fail(TNS_EINVAL, "t0 without ts");
    return TNS_OK;
}

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }

int check_workspace(const void* p, size_t have, size_t need) {
    if (need && !p) return fail(TNS_EINVAL, "null workspace");
    if (misaligned(p, 256)) return fail(TNS_EINVAL, "workspace must be 256-byte aligned");
    if (have < need) return fail(TNS_ESIZE, "workspace smaller than asked for");
    return TNS_OK;
}

// Rows of a tile.  A wave takes a tile's rows one after the other, so a small call is as long as its tiles; the fewer waves a large one
// has, the less their reads overlap and the more unevenly they fill the chip; and every tile has its carry to find.  Tiles of 16, 32 and 64
// rows: 35 K rows of 100 fp32 channels, states 13.6, 12.2, 15.2 us, gradients 21.2, 19.3, 24.5.  Of 64, 128 and 256 (more
// than a wave's lanes hold lists and gaps of; measured with code, since gone, that went from 64 places to the next): 0.79 M rows of 256 bf16
// channels, states 219, 238, 246, gradients 378, 399, 413.
int64_t tile_rows_of(int64_t rows, int dim) {
    const int64_t blocks = (dim + kWave - 1) / kWave;
    return rows / kBatch * blocks < 2048 ? 32 : kBatch;
}

size_t aligned(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

struct Workspace {
    Carries t;
    int64_t spans;
    float* sums;                        // [workgroups of a gradient, dim]
    size_t bytes;
};
Workspace carve(const tns_recur& r, void* base) {
    Workspace w{};
    w.t.tile_rows = tile_rows_of(r.rows, r.dim);
    w.t.tiles = (r.rows + w.t.tile_rows - 1) / w.t.tile_rows;
    w.spans = (w.t.tiles + kSpan - 1) / kSpan;
    char* p = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        void* const at = p;
        p += aligned(bytes);
        w.bytes += aligned(bytes);
        return at;
    };
    const size_t row = (size_t)r.dim * 4;
    w.t.b = static_cast<float*>(take(w.t.tiles * row));
    w.t.a = static_cast<float*>(take(w.t.tiles * row));
    w.t.span_b = static_cast<float*>(take(w.spans * row));
    w.t.span_a = static_cast<float*>(take(w.spans * row));
    w.t.open = static_cast<uint8_t*>(take(w.t.tiles));
    w.t.span_open = static_cast<uint8_t*>(take(w.spans));
    w.t.list = static_cast<uint32_t*>(take(w.t.tiles * 4));
    w.sums = static_cast<float*>(take((w.t.tiles + kWaves - 1) / kWaves * row));
    return w;
}
size_t saved_bytes(const tns_recur& r) { return (size_t)((r.rows + kSaved - 1) / kSaved) * r.dim * 4; }

template <typename T>
Lists<T> typed(const tns_recur& r) {
    return {r.S, r.rows, r.d_rowptr, static_cast<const T*>(r.d_u), static_cast<const T*>(r.d_x), r.ld_u, r.ld_x,
            r.d_ts, r.d_decay, r.d_h0, r.d_t0, r.dim, (r.flags & TNS_NEWEST_FIRST) != 0, (r.flags & TNS_ZERO_BEYOND) != 0};
}

// Calls go(piece, workgroups) for the launches of a walk of `groups` groups of tiles, 2^30 threads each at most; the last one has `more`
// workgroups beyond the walk's.
template <typename F>
void in_pieces(int64_t groups, int blocks, int threads, int64_t more, const F& go) {
    const int64_t most = ((int64_t)1 << 30) / threads / blocks / kXcds * kXcds;      // (2^16 channels are 1024 blocks: 2048 groups at least)
    for (int64_t first = 0; first < groups || (first == 0 && more); first += most) {
        const int64_t n = std::min(groups - first, most), own = workgroups_of(n, blocks);
        go(Piece{first, (unsigned)own, blocks}, dim3((unsigned)(own + (first + n == groups ? more : 0))));
    }
}
int64_t quads_of(const Workspace& w) { return (w.t.tiles + kWaves - 1) / kWaves; }
int64_t fills_of(const tns_recur& r, bool lists) { return lists ? (r.S + kWaves * kWave - 1) / (kWaves * kWave) : 0; }      // 256 lists a workgroup
template <int V> int blocks_of(const tns_recur& r) { return (r.dim + kWave * V - 1) / (kWave * V); }

// Whether rows are written past the caches: where one call's rows of u and x alone are more than the last-level cache holds (256 MiB), so that
// nothing written stays there for a later call anyway and what is read twice has the room, and only rows that are whole lines of 128
// bytes (others come in parts, which would each go to memory).  0.79 M rows of 256 bf16 channels, both directions: 1011 -> 957 us; 1.14 M of 128 in
// lists of ten: 484 -> 466; with rows of 688 bytes, 0.80 M of them: 1444 -> 1650.
template <typename T>
bool streams_out(const tns_recur& r, const void* out, int64_t ld) {
    const size_t line = 128;
    return 2 * (size_t)r.rows * r.dim * sizeof(T) > size_t(256) << 20 && r.dim * sizeof(T) % line == 0 && ld * sizeof(T) % line == 0 && !misaligned(out, line);
}

template <bool BACKWARD>
void launch_join(const tns_recur& r, const Workspace& w, hipStream_t stream) {
    if (w.spans > 1)
        hipLaunchKernelGGL((k_recur_join<BACKWARD>), dim3((r.dim + kChannels - 1) / kChannels), dim3(1024), 0, stream, w.spans, r.dim, w.t.span_b, w.t.span_a, w.t.span_open);
}

template <typename T, int V, bool DECAY>
void launch_run(const tns_recur& r, void* h, int64_t ld_h, float* last, void* saved, void* workspace, hipStream_t stream) {
    const Workspace w = carve(r, workspace);
    const int blocks = blocks_of<V>(r);
    const Lists<T> l = typed<T>(r);
    if (w.t.tiles > 1) {
        in_pieces(w.spans, blocks, kSpan * kWave, 0, [&](Piece piece, dim3 grid) {
            hipLaunchKernelGGL((k_recur_tails<T, V, DECAY>), grid, dim3(kSpan * kWave), 0, stream, l, w.t, piece);
        });
        launch_join<false>(r, w, stream);
    }
    in_pieces(quads_of(w), blocks, 256, fills_of(r, last != nullptr), [&](Piece piece, dim3 grid) {
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, l, w.t, piece, static_cast<T*>(h), ld_h, last, static_cast<float*>(saved));
        };
        if (streams_out<T>(r, h, ld_h)) go(k_recur_states<T, V, DECAY, true>);
        else go(k_recur_states<T, V, DECAY, false>);
    });
}

template <typename T, int V, bool DECAY>
void launch_grad(const tns_recur& r, const void* saved, const void* dh, int64_t ld_dh, const float* dlast, void* du, int64_t ld_du, void* dx,
                 int64_t ld_dx, float* ddecay, float* dh0, void* workspace, hipStream_t stream) {
    const Workspace w = carve(r, workspace);
    const int blocks = blocks_of<V>(r);
    const Lists<T> l = typed<T>(r);
    const T* const d = static_cast<const T*>(dh);
    if (w.t.tiles > 1) {
        in_pieces(w.spans, blocks, kSpan * kWave, 0, [&](Piece piece, dim3 grid) {
            hipLaunchKernelGGL((k_recur_heads<T, V, DECAY>), grid, dim3(kSpan * kWave), 0, stream, l, w.t, piece, d, ld_dh, dlast);
        });
        launch_join<true>(r, w, stream);
    }
    in_pieces(quads_of(w), blocks, 256, fills_of(r, dh0 != nullptr), [&](Piece piece, dim3 grid) {
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, l, w.t, piece, static_cast<const float*>(saved), d, ld_dh, dlast,
                               static_cast<T*>(du), ld_du, static_cast<T*>(dx), ld_dx, dh0, ddecay ? w.sums : nullptr);
        };
        if (streams_out<T>(r, du, ld_du) && streams_out<T>(r, dx, ld_dx)) go(k_recur_grads<T, V, DECAY, true>);
        else go(k_recur_grads<T, V, DECAY, false>);
    });
    if (ddecay)
        hipLaunchKernelGGL(k_recur_sums, dim3((r.dim + kChannels - 1) / kChannels), dim3(1024), 0, stream, w.sums, (w.t.tiles + kWaves - 1) / kWaves, r.dim, ddecay);
}

// Calls `go` with the type, the channels a lane has and whether there is a decay.  Two channels in 16 bits where every row allows reads of
// four bytes and the lanes of the last wave are not fewer for it.
template <typename F>
void choose(const tns_recur& r, bool pairs, const F& go) {
    const bool decay = r.d_decay && r.rows > 0;
    auto with = [&](auto value, auto v) {
        if (decay) go(value, v, std::true_type{});
        else go(value, v, std::false_type{});
    };
    pairs = pairs && r.dim % 2 == 0 && r.ld_u % 2 == 0 && r.ld_x % 2 == 0 && !misaligned(r.d_u, 4) && !misaligned(r.d_x, 4) &&
            (r.dim + 127) / 128 * 2 <= (r.dim + 63) / 64;
    if (r.dtype == TNS_F32) with(float{}, std::integral_constant<int, 1>{});
    else if (pairs) with(bf16{}, std::integral_constant<int, 2>{});
    else with(bf16{}, std::integral_constant<int, 1>{});
}

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, what);
}

}  // namespace

extern "C" {

int tns_recur_workspace(const tns_recur* r, size_t* run, size_t* grad, size_t* saved) {
    tns::clear_error();
    if (int e = check(r)) return e;
    if (run) *run = carve(*r, nullptr).bytes;
    if (grad) *grad = carve(*r, nullptr).bytes;
    if (saved) *saved = saved_bytes(*r);
    return TNS_OK;
}

int tns_recur_run(const tns_recur* r, void* d_h, int64_t ld_h, float* d_h_last, void* d_saved, void* d_workspace, size_t workspace_bytes,
                  void* hip_stream) {
    tns::clear_error();
    if (int e = check_arrays(r)) return e;
    if (d_h && ld_h < r->dim) return fail(TNS_EINVAL, "rows of h overlap");
    if (misaligned(d_saved, 256)) return fail(TNS_EINVAL, "saved states must be 256-byte aligned");
    if (int e = check_workspace(d_workspace, workspace_bytes, carve(*r, nullptr).bytes)) return e;
    if (r->S == 0 && !(r->flags & TNS_ZERO_BEYOND)) return TNS_OK;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    choose(*r, !d_h || (ld_h % 2 == 0 && !misaligned(d_h, 4)), [&](auto value, auto v, auto decay) {
        launch_run<decltype(value), v(), decay()>(*r, d_h, ld_h, d_h_last, d_saved, d_workspace, stream);
    });
    return launched("tns_recur_run");
}

int tns_recur_grad(const tns_recur* r, const void* d_saved, const void* d_dh, int64_t ld_dh, const float* d_dh_last, void* d_du, int64_t ld_du,
                   void* d_dx, int64_t ld_dx, float* d_ddecay, float* d_dh0, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    tns::clear_error();
    if (int e = check_arrays(r)) return e;
    if (r->rows > 0 && (!d_saved || !d_du || !d_dx)) return fail(TNS_EINVAL, "null saved states, du or dx");
    if (misaligned(d_saved, 256)) return fail(TNS_EINVAL, "saved states must be 256-byte aligned");
    if (ld_du < r->dim || ld_dx < r->dim || (d_dh && ld_dh < r->dim)) return fail(TNS_EINVAL, "rows of dh, du or dx overlap");
    if (d_ddecay && !r->d_decay) return fail(TNS_EINVAL, "gradient of a decay that is not there");
    if (int e = check_workspace(d_workspace, workspace_bytes, carve(*r, nullptr).bytes)) return e;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (r->S == 0 && !(r->flags & TNS_ZERO_BEYOND)) {
        if (d_ddecay) hipLaunchKernelGGL(k_recur_sums, dim3((r->dim + kChannels - 1) / kChannels), dim3(1024), 0, stream, nullptr, 0, r->dim, d_ddecay);
        return launched("tns_recur_grad");
    }
    const bool pairs = ld_du % 2 == 0 && ld_dx % 2 == 0 && (!d_dh || ld_dh % 2 == 0) && !misaligned(d_du, 4) && !misaligned(d_dx, 4) && !misaligned(d_dh, 4);
    choose(*r, pairs, [&](auto value, auto v, auto decay) {
        launch_grad<decltype(value), v(), decay()>(*r, d_saved, d_dh, ld_dh, d_dh_last, d_du, ld_du, d_dx, ld_dx, d_ddecay, d_dh0, d_workspace, stream);
    });
    return launched("tns_recur_grad");
}

int tns_recur_step(int64_t B, int64_t num_ids, int32_t dim, int32_t dtype, const int32_t* d_ids, const void* d_u, int64_t ld_u, const void* d_x,
                   int64_t ld_x, const float* d_ts, const float* d_decay, float* d_state, float* d_state_ts, void* d_out, int64_t ld_out,
                   void* hip_stream) {
    tns::clear_error();
    if (B < 0 || num_ids < 0) return fail(TNS_EINVAL, "negative B or num_ids");
    if (B > (int64_t)INT32_MAX || num_ids > (int64_t)INT32_MAX) return fail(TNS_ESIZE, "more than 2^31-1 events or states");
    if (dim < 1 || dim > 1 << 16) return fail(TNS_EINVAL, "dim must be in [1, 2^16]");
    if (dtype != TNS_F32 && dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if (ld_u < dim || ld_x < dim || (d_out && ld_out < dim)) return fail(TNS_EINVAL, "rows of u, x or out overlap");
    if (B == 0) return TNS_OK;
    if (!d_ts != !d_decay || (num_ids > 0 && !d_ts != !d_state_ts)) return fail(TNS_EINVAL, "ts, decay and state_ts come together");
    if (!d_ids || !d_u || !d_x || (num_ids > 0 && !d_state)) return fail(TNS_EINVAL, "null ids, u, x or state");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto launch = [&](auto value, auto vec, auto lanes) {
        using T = decltype(value);
        const int64_t groups = std::min<int64_t>((B + 256 / lanes() - 1) / (256 / lanes()), 1 << 20);
        hipLaunchKernelGGL((k_recur_step<T, vec(), lanes()>), dim3((unsigned)groups), dim3(256), 0, stream, B, num_ids, dim, d_ids, static_cast<const T*>(d_u), ld_u,
                           static_cast<const T*>(d_x), ld_x, d_ts, d_decay, d_state, d_state_ts, static_cast<T*>(d_out), ld_out);
    };
    // Four channels at a time where all rows allow it, and as few lanes to an event as hold it at once.
    auto choose_step = [&](auto value) {
        using T = decltype(value);
        auto fits = [](const void* p, size_t to) { return !misaligned(p, to); };
        const bool four = dim % 4 == 0 && ld_u % 4 == 0 && ld_x % 4 == 0 && (!d_out || ld_out % 4 == 0) && fits(d_u, 4 * sizeof(T)) && fits(d_x, 4 * sizeof(T)) &&
                          fits(d_out, 4 * sizeof(T)) && fits(d_state, 16) && fits(d_decay, 16);
        using One = std::integral_constant<int, 1>;
        using Four = std::integral_constant<int, 4>;
        if (!four) launch(value, One{}, std::integral_constant<int, 64>{});
        else if (dim <= 32) launch(value, Four{}, std::integral_constant<int, 8>{});
        else if (dim <= 64) launch(value, Four{}, std::integral_constant<int, 16>{});
        else if (dim <= 128) launch(value, Four{}, std::integral_constant<int, 32>{});
        else launch(value, Four{}, std::integral_constant<int, 64>{});
    };
    if (dtype == TNS_F32) choose_step(float{});
    else choose_step(bf16{});
    return launched("tns_recur_step");
}

}  // extern "C"
