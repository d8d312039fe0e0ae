// Attention of targets over ragged lists of events with a bias by buckets of their age (include/tns_layer.h): outputs.
#include "tns_attend.h"

namespace {

// A lane's running maximum, sum and weighted sum of values, for a group of heads.
template <typename T, int VEC, int G, bool EXACT>
struct Running {
    static constexpr int N = Row<T, VEC>::N;
    float m[G], l[G], acc[G][N];
    __device__ Running() {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            m[g] = -kInf;
            l[g] = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) acc[g][i] = 0.0f;
        }
    }
    // Takes U events of these buckets, the first ones or more.
    template <int LANES, int U>
    __device__ __forceinline__ void take(const Attend<T>& a, const Cut& cut, const Place<T, VEC, EXACT>& at, Batch<T, VEC, U, EXACT>& b, const Row<T, VEC> (&q)[G], const int (&bucket)[U],
                                         const float* s_table, bool more) {
        float s[U][G];
        bool mixed = false;             // an event that is left out by some of the lane's heads only
#pragma unroll
        for (int u = 0; u < U; ++u) {
            bool some = false, all = true;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float dot = over_head<LANES>(b.k[u].template dot<!EXACT>(q[g], at.mask), cut.lanes);
                const float bias = s_table[max(bucket[u], 0) * a.heads + at.kv * a.group + min(g, a.group - 1)];
                const bool counts = bucket[u] >= 0 && bias != -kInf;
                s[u][g] = counts ? dot * a.scale + bias : -kInf;
                some |= counts;
                all &= counts;
            }
            b.v[u].clear_unless(some);
            mixed |= some && !all;
        }
        const bool careful = G > 1 && __ballot(mixed) != 0;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float top = m[g];
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, s[u][g]);
            const float base = top == -kInf ? 0.0f : top;
            if (more && __ballot(top > m[g])) {
                const float keep = __builtin_amdgcn_exp2f(m[g] - base);
                l[g] *= keep;
#pragma unroll
                for (int c = 0; c < N; ++c) acc[g][c] *= keep;
            }
            m[g] = top;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float p = __builtin_amdgcn_exp2f(s[u][g] - base);
                l[g] += p;
                if (careful) {
#pragma unroll
                    for (int c = 0; c < N; ++c) acc[g][c] += s[u][g] == -kInf ? 0.0f : p * b.v[u].get(c);
                } else {
#pragma unroll
                    for (int c = 0; c < N; ++c) acc[g][c] += p * b.v[u].get(c);
                }
            }
        }
    }
};

// Scores, running maximum and sum, and the weighted sum of the values in one pass over k and v.  Bound by memory, and before that by the waves that the
// registers leave room for: 131072 lists of ten, two heads of 64 bf16 channels, with what the gradients need, 0.73 GB in 169 us (4.3 TB/s); 66600
// lists gathered from a table, four heads of 32, 0.34 GB in 56 us (6.1); seven lists of 120000, eight heads of 64 on four, 0.81 GB in 156 us (5.2).
// What it took: products of two bf16 pairs an instruction; the arguments read again where they are used; one event of every slot ahead rather than two
// (fewer registers, seven waves instead of five: 63 -> 74 us); no more workgroups than fit (the others would start when these end); flags that the
// compiler knows instead of branches, from behind which it waits for every request.  600 lists: 7.7 us, five reads one after the other.
// GATHER: rows of k and v by their index; 2: looked up when it is needed to be known.
template <typename T, int VEC, int G, int LANES, int GATHER>
__global__ void __launch_bounds__(kWaves* kWave) k_attend(const Args<T>) {
    extern __shared__ float s_mem[];
    constexpr bool EXACT = LANES != 0;
    constexpr int N = Row<T, VEC>::N, U = G == 2 || G == 4 ? 2 : 1, OWN = 1;
    const Args<T>& start = args_now<T>();
    float *const s_edges = s_mem, *const s_table = s_mem + start.a.buckets;
    const int64_t stride = (int64_t)gridDim.x * kWaves, begin = (int64_t)blockIdx.x * kWaves + uniform((int)(threadIdx.x >> 6));
    const Place<T, VEC, EXACT> at(start.a, start.cut, blockIdx.y);
    const int log_slots = 6 - start.cut.log_width, lane0 = at.lane & ~((1 << start.cut.log_width) - 1);
    Edges edges;
    if (start.cut.brief >= 0) edges = Edges(start.a, (begin << log_slots) + at.slot);
    stage(start.a, s_edges, s_table);
    if (start.cut.brief >= 0)
        for (int64_t group = begin; group << log_slots < args_now<T>().a.S; group += stride) {
            const Args<T>& now = args_now<T>();
            const Attend<T>& a = now.a;
            const Cut& cut = now.cut;
            const Own own(a, cut, (group << log_slots) + at.slot, edges);
            edges = Edges(a, ((group + stride) << log_slots) + at.slot);
            const int most = (int)over_lanes((float)own.events, kWave, Max{}), width = 1 << cut.log_width;
            const float t = a.t ? a.t[own.list] : 0.0f;
            const bool gather = GATHER == 2 ? a.index != nullptr : GATHER;
            const char* const k_row = reinterpret_cast<const char*>(a.k + (gather ? 0 : own.begin * a.ld_k));
            const char* const v_row = reinterpret_cast<const char*>(a.v + (gather ? 0 : own.begin * a.ld_v));
            Row<T, VEC> q[G];
            Running<T, VEC, G, EXACT> sums;
            Batch<T, VEC, OWN, EXACT> batch;
            for (int i0 = 0; i0 < most; i0 += width) {
                const int place = max(min(i0 + at.lane - lane0, own.events - 1), 0);
                const Event event(a, own.begin, place);
                Known known;
                auto read = [&](Batch<T, VEC, OWN, EXACT>& b, int i) { b.read_own(a, at, k_row, v_row, own, i0 + i, gather ? &known : nullptr, lane0 + i); };
                if (!gather) read(batch, 0);
                if (i0 == 0) at.heads(a, a.q + own.list * a.ld_q, q);
                known = Known(a, event, t, a.newest_first ? place : own.n - 1 - place, s_edges);
                if (gather) read(batch, 0);
                each_batch(batch, min(width, most - i0), OWN, read, [&](Batch<T, VEC, OWN, EXACT>& b, int i) {
                    int bucket[OWN];
#pragma unroll
                    for (int u = 0; u < OWN; ++u) {
                        const int found = __shfl(known.bucket, lane0 + min(i + u, width - 1));
                        bucket[u] = i0 + i + u < own.events && i + u < width ? found : -1;
                    }
                    sums.template take<LANES, OWN>(a, cut, at, b, q, bucket, s_table, i0 + i > 0);
                });
            }
            if (!own.here || !at.head) continue;
            const Args<T>& end = args_now<T>();
            const int64_t to = own.list * end.a.heads, row = to * end.a.dim;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if (g >= end.a.group) break;
                const float weight = sums.l[g] == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sums.l[g]);
#pragma unroll
                for (int i = 0; i < N; ++i) sums.acc[g][i] *= weight;
                at.write(end.out + row, g * end.a.dim, sums.acc[g]);
                if (!end.saved_out) continue;
                at.write(end.saved_out + row, g * end.a.dim, sums.acc[g]);
                if (at.mine == 0) end.saved_norm[to + at.kv * end.a.group + g] = Norm(sums.m[g], sums.l[g], weight);
            }
        }
    Walk<T> walk(begin, stride);
    for (;;) {
        const Args<T>& now = args_now<T>();
        const Attend<T>& a = now.a;
        const Cut& cut = now.cut;
        Part w;
        if (!walk.get(a, cut, blockIdx.y == 0 ? now.work.first : nullptr, w, [](int64_t) {})) return;
        Row<T, VEC> q[G];
        Running<T, VEC, G, EXACT> sums;
        Batch<T, VEC, U, EXACT> batch;
        const bool gather = GATHER == 2 ? a.index != nullptr : GATHER;
        const float t = a.t ? a.t[w.list] : 0.0f;
        for (int64_t row0 = w.begin; row0 < w.end; row0 += kWave) {
            const int n = (int)min(w.end - row0, (int64_t)kWave), place = min(at.lane, n - 1);
            Known known;
            auto read = [&](Batch<T, VEC, U, EXACT>& b, int i0) { b.read(a, cut, at, row0, i0, n, gather ? &known : nullptr); };
            const Event event(a, row0, place);
            if (!gather) read(batch, 0);
            if (row0 == w.begin) at.heads(a, a.q + w.list * a.ld_q, q);
            known = Known(a, event, t, a.newest_first ? row0 - w.list_begin + place : w.list_end - 1 - row0 - place, s_edges);
            if (gather) read(batch, 0);
            each_batch(batch, n, cut.slots * U, read, [&](Batch<T, VEC, U, EXACT>& b, int i0) {
                int bucket[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * cut.slots + at.slot, found = __shfl(known.bucket, min(i, n - 1));
                    bucket[u] = i < n ? found : -1;
                }
                sums.template take<LANES, U>(a, cut, at, b, q, bucket, s_table, row0 != w.begin || i0);
            });
        }
        // what the slots found is joined
        const Args<T>& end = args_now<T>();
        const int width = 1 << end.cut.log_width, heads = end.a.heads, group = end.a.group;
        const int64_t to = (w.whole ? w.list : w.slot) * heads, row = to * end.a.dim;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g >= group) break;
            const float top = over_strided(sums.m[g], width, Max{}), f = sums.m[g] == -kInf ? 0.0f : __builtin_amdgcn_exp2f(sums.m[g] - top);
            const float sum = over_strided(sums.l[g] * f, width, Add{}), inverse = sum == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(sum), weight = w.whole ? f * inverse : f;
#pragma unroll
            for (int i = 0; i < N; ++i) sums.acc[g][i] *= weight;
            if (at.head && at.slot == 0 && at.mine == 0) {
                const uint32_t h = at.kv * group + g;
                if (!w.whole) {
                    *lane_at<float>(end.work.stats + 2 * to, 8 * h) = top;
                    *lane_at<float>(end.work.stats + 2 * to, 8 * h + 4) = sum;
                } else if (end.saved_out) {
                    *lane_at<Norm>(end.saved_norm + to, (uint32_t)sizeof(Norm) * h) = Norm(top, sum, inverse);
                }
            }
            at.joined(end.a, end.cut, g, sums.acc[g], [&](uint32_t c, float x, float y, auto two_) {
                if (!w.whole) return put(end.work.acc + row, c, x, y, two_);
                put(end.out + row, c, x, y, two_);
                if (end.saved_out) put(end.saved_out + row, c, x, y, two_);
            });
        }
    }
}

// 6563 parts of 3001 histories: 25 us; 13125 of seven lists: 26.
template <typename T>
__global__ void __launch_bounds__(1024) k_attend_join(const Attend<T> a, const Cut cut, const Work work, unsigned few, T* out, float* saved_out, Norm* saved_norm) {
    __shared__ float s_sum[1024];
    auto write = [&](int64_t list, int64_t h, int c, float top, float l, float acc) {
        const int64_t to = list * a.heads + h;
        const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
        acc *= inverse;
        out[to * a.dim + c] = as_value<T>(acc);
        if (saved_out) {
            saved_out[to * a.dim + c] = acc;
            if (c == 0) saved_norm[to] = Norm(top, l, inverse);
        }
    };
    if (blockIdx.x < few) {
        __shared__ float s_top[16][kOwn * kWave], s_l[16][kOwn * kWave], s_acc[16][kOwn * kWave];
        const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, all = a.heads * a.dim;
        const int chunks = (all + kOwn * kWave - 1) / (kOwn * kWave), c0 = (int)(blockIdx.x % chunks) * kOwn * kWave;
        const int64_t block0 = (int64_t)(blockIdx.x / chunks) * 16;
        const int32_t begins = lane < 16 && block0 + lane < cut.blocks ? work.first[block0 + lane] : -1;
        for (uint64_t left = __ballot(begins >= 0); left; left &= left - 1) {
            const int k = __builtin_ctzll(left);
            const int64_t block = block0 + k, list = __builtin_amdgcn_readlane(begins, k);
            const int64_t end = parts_end(a.edge(list + 1), cut.part, cut.blocks);
            if (is_many(block, end)) continue;
            __syncthreads();
            int c[kOwn], h[kOwn];
            float top[kOwn], l[kOwn] = {}, acc[kOwn] = {};
#pragma unroll
            for (int j = 0; j < kOwn; ++j) {
                c[j] = min(c0 + j * kWave + lane, all - 1);
                h[j] = c[j] / a.dim;
                top[j] = -kInf;
            }
#pragma unroll 2
            for (int64_t b = block + wave; b < end; b += 16) {
                const int64_t at = slot_of(b, block, cut);
#pragma unroll
                for (int j = 0; j < kOwn; ++j) {
                    const float m = work.stats[2 * (at * a.heads + h[j])], n = work.stats[2 * (at * a.heads + h[j]) + 1], v = work.acc[at * all + c[j]];
                    const float both = fmaxf(top[j], m), base = both == -kInf ? 0.0f : both, keep = __builtin_amdgcn_exp2f(top[j] - base), f = __builtin_amdgcn_exp2f(m - base);
                    l[j] = keep * l[j] + f * n;
                    acc[j] = keep * acc[j] + f * v;
                    top[j] = both;
                }
            }
#pragma unroll
            for (int j = 0; j < kOwn; ++j) {
                s_top[wave][j * kWave + lane] = top[j];
                s_l[wave][j * kWave + lane] = l[j];
                s_acc[wave][j * kWave + lane] = acc[j];
            }
            __syncthreads();
            const int mine = c0 + (int)threadIdx.x;
            if ((int)threadIdx.x >= kOwn * kWave || mine >= all) continue;
            float most = -kInf, sum = 0.0f, value = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s_top[i][threadIdx.x]);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float m = s_top[i][threadIdx.x], f = m == -kInf ? 0.0f : __builtin_amdgcn_exp2f(m - most);
                sum += f * s_l[i][threadIdx.x];
                value += f * s_acc[i][threadIdx.x];
            }
            write(list, mine / a.dim, mine % a.dim, most, sum, value);
        }
        return;
    }
    const unsigned slices = (a.dim + kSlice - 1) / kSlice, slice = (blockIdx.x - few) % slices;
    const int64_t h = (blockIdx.x - few) / slices % a.heads;
    int64_t begin = 0, end = 0;
    const int64_t list = many_of(a, cut, (blockIdx.x - few) / slices / a.heads, begin, end);
    if (list < 0) return;
    const int ch = (int)(slice * kSlice + (threadIdx.x & (kSlice - 1))), c = min(ch, a.dim - 1), mine = threadIdx.x / kSlice, parts = 1024 / kSlice;
    float top = -kInf;
    for (int64_t b = begin + threadIdx.x; b < end; b += 1024) top = fmaxf(top, work.stats[2 * (slot_of(b, begin, cut) * a.heads + h)]);
    top = over_lanes(top, kWave, Max{});
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = top;
    __syncthreads();
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s_sum[i]);
    const float base = top == -kInf ? 0.0f : top;
    float l = 0.0f, acc = 0.0f;
#pragma unroll 8
    for (int64_t b = begin + mine; b < end; b += parts) {
        const int64_t at = slot_of(b, begin, cut) * a.heads + h;
        const float f = __builtin_amdgcn_exp2f(work.stats[2 * at] - base);
        l += f * work.stats[2 * at + 1];
        acc += f * work.acc[at * a.dim + c];
    }
    l = over_parts(l, kSlice, s_sum);
    acc = over_parts(acc, kSlice, s_sum);
    if (mine == 0 && ch < a.dim) write(list, h, ch, top, l, acc);
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
    if (int e = check_joins(*a, c)) return e;
    if (a->S == 0) return TNS_OK;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    float* const saved = static_cast<float*>(d_saved);
    Norm* const norms = saved ? reinterpret_cast<Norm*>(saved + saved_out_bytes(*a) / 4) : nullptr;
    const size_t lds = lds_of(*a, 0);
    choose(*a, c, [&](auto value, auto vec, auto group, auto lanes) {
        using T = decltype(value);
        const Attend<T> t = typed<T>(*a);
        const Args<T> args = {t, c, l.w, static_cast<T*>(d_out), saved, norms, nullptr, nullptr, nullptr, nullptr, 0};
        auto launch = [&](auto kernel, int& per_cu) {
            hipLaunchKernelGGL(kernel, dim3(groups_of(*a, c, resident(kernel, lds, per_cu)), c.turns), dim3(kWaves * kWave), lds, stream, args);
        };
        static int per_cu[3];           // (of these types; the same whoever writes it)
        if constexpr (lanes() == 0) launch(k_attend<T, vec(), group(), 0, 2>, per_cu[2]);
        else if (a->d_index) launch(k_attend<T, vec(), group(), lanes(), 1>, per_cu[1]);
        else launch(k_attend<T, vec(), group(), lanes(), 0>, per_cu[0]);
        if (const unsigned few = (unsigned)few_of(*a, c))
            hipLaunchKernelGGL((k_attend_join<T>), dim3(few + (unsigned)many_of(*a, c)), dim3(1024), 0, stream, t, c, l.w, few, static_cast<T*>(d_out), saved, norms);
    });
    return launched("tns_attend_run");
}

}  // extern "C"
