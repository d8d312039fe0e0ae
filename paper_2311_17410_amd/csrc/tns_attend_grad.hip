// Attention of targets over ragged lists of events (include/tns_layer.h): gradients.
#include "tns_attend.h"

namespace {

// A lane's share of the gradients of a list, for a group of heads.
template <typename T, int VEC, int G, bool EXACT>
struct Back {
    static constexpr int N = Row<T, VEC>::N;
    Row<T, VEC> q[G], d[G];             // query, gradient by the output
    float acc[G][N], delta[G];          // gradient by the query; gradient by the output times the output
    Norm norm[G];
    __device__ Back() {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < N; ++i) acc[g][i] = 0.0f;
    }
    template <int LANES>
    __device__ __forceinline__ void read(const Args<T>& now, const Place<T, VEC, EXACT>& at, int64_t list) {
        const Attend<T>& a = now.a;
        const int64_t row = list * a.heads * a.dim;
        float out[G][N];
        at.heads(a, now.saved_out + row, out);
        at.heads(a, now.dout + row, d);
        at.heads(a, a.q + list * a.ld_q, q);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            norm[g] = now.saved_norm[list * a.heads + at.kv * a.group + min(g, a.group - 1)];
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) dot += at.counts(i) ? d[g].get(i) * out[g][i] : 0.0f;
            delta[g] = over_head<LANES>(dot, now.cut.lanes);
        }
    }
    // Takes an event of that bucket: its gradients by k and v, and what its score's gradient is (ds), head by head; false if it counts for none.
    template <int LANES>
    __device__ __forceinline__ bool take(const Attend<T>& a, const Cut& cut, const Place<T, VEC, EXACT>& at, Row<T, VEC>& k, Row<T, VEC>& v, int bucket, const float* s_table, float scale,
                                         bool (&counts)[G], float (&ds)[G], float (&to_k)[N], float (&to_v)[N]) {
        if constexpr (G > 1 && sizeof(T) == 2)      // (opaque here: the compiler would keep all heads' values widened, 32 registers a head, and fewer waves)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) asm("" : "+v"(q[g].word[i]), "+v"(d[g].word[i]));
        bool some = false, all = true;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            ds[g] = s_table[max(bucket, 0) * a.heads + at.kv * a.group + min(g, a.group - 1)];
            counts[g] = bucket >= 0 && ds[g] != -kInf && g < a.group;
            some |= counts[g];
            all &= counts[g] || g >= a.group;
        }
        k.clear_unless(some);
        v.clear_unless(some);
        const bool careful = G > 1 && __ballot(some && !all) != 0;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float score = over_head<LANES>(k.template dot<!EXACT>(q[g], at.mask), cut.lanes), dp = over_head<LANES>(v.template dot<!EXACT>(d[g], at.mask), cut.lanes);
            const float p = counts[g] ? __builtin_amdgcn_exp2f(score * a.scale + ds[g] - norm[g].top) * norm[g].inverse : 0.0f;
            ds[g] = counts[g] ? p * (dp - delta[g]) : 0.0f;
            const float by = ds[g] * scale;
            if (careful) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    to_k[i] = (g ? to_k[i] : 0.0f) + (counts[g] ? by * q[g].get(i) : 0.0f);
                    to_v[i] = (g ? to_v[i] : 0.0f) + (counts[g] ? p * d[g].get(i) : 0.0f);
                    acc[g][i] += counts[g] ? by * k.get(i) : 0.0f;
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    to_k[i] = g ? to_k[i] + by * q[g].get(i) : by * q[g].get(i);
                    to_v[i] = g ? to_v[i] + p * d[g].get(i) : p * d[g].get(i);
                    acc[g][i] += by * k.get(i);
                }
            }
        }
        return some;
    }
};

// Adds to the wave's part of the table's gradient.  Slots take turns, as many at once as the wave has copies of the table: requests of one turn go to
// different entries, and the LDS unit takes a wave's requests in order, so the order of the sums is the same every time.
template <typename T, int VEC, int G, bool EXACT>
__device__ __forceinline__ void add_to_table(const Attend<T>& a, const Cut& cut, const Place<T, VEC, EXACT>& at, int bucket, const bool (&counts)[G], const float (&ds)[G], float* s_mine) {
    for (int e = 0; e < cut.slots >> cut.log_copies; ++e) {
        if (at.slot >> cut.log_copies == e && at.head && at.mine == 0)
#pragma unroll
            for (int g = 0; g < G; ++g)
                if (counts[g]) __hip_atomic_fetch_add(&s_mine[bucket * a.heads + at.kv * a.group + g], ds[g], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// One pass over k and v: the scores again, p from the largest and the sum that were saved, and all gradients of an event while its rows are in
// registers.  ds = p (dp - delta) with dp = dout . v; delta = dout . out from outputs saved in fp32 (of bf16 ones the difference would keep their rounding,
// and the table's gradient, in which most of it cancels, would show it).  Bound by memory: 131072 lists of ten, two heads of 64 bf16 channels, 1.36 GB in
// 262 us (5.2 TB/s); 3001 histories, eight heads of 32 fp32 channels on four, 1.68 GB in 343 us (4.9).  Heads that share a key in fours and eights
// are bound by instructions and by the few waves that their registers leave room for: 30000 lists of ten, eight heads of 64 bf16 channels on two, 0.42 GB
// in 118 us (3.6 TB/s), on one, 0.29 GB in 220 (1.3).
template <typename T, int VEC, int G, int LANES>
__global__ void __launch_bounds__(kWaves* kWave) k_attend_grad(const Args<T>) {
    extern __shared__ float s_mem[];
    constexpr bool EXACT = LANES != 0;
    constexpr int N = Row<T, VEC>::N, U = G == 2 && sizeof(T) == 4 ? 2 : 1, OWN = 1;
    const Args<T>& start = args_now<T>();
    const int entries = start.a.buckets * start.a.heads, wave = uniform((int)(threadIdx.x >> 6));
    float *const s_edges = s_mem, *const s_table = s_mem + start.a.buckets, *const s_sums = s_table + max(entries, start.a.heads);
    const int64_t stride = (int64_t)gridDim.x * kWaves, begin = (int64_t)blockIdx.x * kWaves + wave;
    const Place<T, VEC, EXACT> at(start.a, start.cut, blockIdx.y);
    const int copies = kWaves << start.cut.log_copies;
    float* const s_mine = s_sums + ((wave << start.cut.log_copies) + (at.slot & ((1 << start.cut.log_copies) - 1))) * entries;      // the slot's
    const int log_slots = 6 - start.cut.log_width, lane0 = at.lane & ~((1 << start.cut.log_width) - 1);
    Edges edges;
    if (start.cut.brief >= 0) edges = Edges(start.a, (begin << log_slots) + at.slot);
    if (start.tables)
        for (int i = threadIdx.x; i < copies * entries; i += kWaves * kWave) s_sums[i] = 0.0f;
    stage(start.a, s_edges, s_table);
    if (start.cut.brief >= 0)
        for (int64_t group = begin; group << log_slots < args_now<T>().a.S; group += stride) {
            const Args<T>& now = args_now<T>();
            const Attend<T>& a = now.a;
            const Cut& cut = now.cut;
            const Own own(a, cut, (group << log_slots) + at.slot, edges);
            edges = Edges(a, ((group + stride) << log_slots) + at.slot);
            const int most = (int)over_lanes((float)own.events, kWave, Max{}), width = 1 << cut.log_width;
            const uint32_t row_bytes = (uint32_t)(a.kv_heads * a.dim) * (uint32_t)sizeof(T);
            const float t = a.t ? a.t[own.list] : 0.0f, scale = a.scale * kLn2;
            const char *const k_row = reinterpret_cast<const char*>(a.k + own.begin * a.ld_k), *const v_row = reinterpret_cast<const char*>(a.v + own.begin * a.ld_v);
            char *const dk_row = reinterpret_cast<char*>(now.dk) + own.begin * row_bytes, *const dv_row = reinterpret_cast<char*>(now.dv) + own.begin * row_bytes;
            Back<T, VEC, G, EXACT> back;
            Batch<T, VEC, OWN, EXACT> batch;
            for (int i0 = 0; i0 < most; i0 += width) {
                const int place = max(min(i0 + at.lane - lane0, own.events - 1), 0);
                const Event event(a, own.begin, place);
                auto read = [&](Batch<T, VEC, OWN, EXACT>& b, int i) { b.read_own(a, at, k_row, v_row, own, i0 + i, nullptr, 0); };
                read(batch, 0);
                if (i0 == 0) back.template read<LANES>(now, at, own.list);
                const Known known(a, event, t, a.newest_first ? place : own.n - 1 - place, s_edges);
                each_batch(batch, min(width, most - i0), OWN, read, [&](Batch<T, VEC, OWN, EXACT>& b, int i) {
#pragma unroll
                    for (int u = 0; u < OWN; ++u) {
                        const int row = i0 + i + u, found = __shfl(known.bucket, lane0 + min(i + u, width - 1));
                        const bool is = row < own.events && i + u < width;
                        const int bucket = is ? found : -1;
                        bool counts[G];
                        float ds[G], to_k[N], to_v[N];
                        const bool some = back.template take<LANES>(a, cut, at, b.k[u], b.v[u], bucket, s_table, scale, counts, ds, to_k, to_v);
                        if (at.head && is) {
                            Row<T, VEC> to;
                            to.set(to_k);
                            to.clear_unless(some);
                            to.write(dk_row, __umul24(row, row_bytes), at.at, at.there);
                            to.set(to_v);
                            to.clear_unless(some);
                            to.write(dv_row, __umul24(row, row_bytes), at.at, at.there);
                        }
                        if (now.tables) add_to_table<T, VEC, G, EXACT>(a, cut, at, bucket, counts, ds, s_mine);
                    }
                });
            }
            if (!own.here || !at.head) continue;
            const Args<T>& end = args_now<T>();
#pragma unroll
            for (int g = 0; g < G; ++g)
                if (g < end.a.group) at.write(end.dq + own.list * end.a.heads * end.a.dim, g * end.a.dim, back.acc[g]);
        }
    Walk<T> walk(begin, stride);
    for (;;) {
        const Args<T>& now = args_now<T>();
        const Attend<T>& a = now.a;
        const Cut& cut = now.cut;
        const int64_t row_of = a.kv_heads * a.dim;
        Part w;
        const bool any = walk.get(a, cut, blockIdx.y == 0 ? now.work.first : nullptr, w, [&](int64_t block) {
            if (!a.zero_beyond || blockIdx.y) return;
            const int64_t from = max(block << cut.part, a.total()), to = min((block + 1) << cut.part, a.rows);
            tns::zero_values(now.dk + from * row_of, max(to - from, (int64_t)0) * row_of, at.lane, kWave);
            tns::zero_values(now.dv + from * row_of, max(to - from, (int64_t)0) * row_of, at.lane, kWave);
        });
        if (!any) break;
        const float t = a.t ? a.t[w.list] : 0.0f, scale = a.scale * kLn2;
        Back<T, VEC, G, EXACT> back;
        Batch<T, VEC, U, EXACT> batch;
        for (int64_t row0 = w.begin; row0 < w.end; row0 += kWave) {
            const int n = (int)min(w.end - row0, (int64_t)kWave), place = min(at.lane, n - 1);
            char *const dk_row = reinterpret_cast<char*>(now.dk + row0 * row_of), *const dv_row = reinterpret_cast<char*>(now.dv + row0 * row_of);
            auto read = [&](Batch<T, VEC, U, EXACT>& b, int i0) { b.read(a, cut, at, row0, i0, n, nullptr); };
            const Event event(a, row0, place);
            read(batch, 0);
            if (row0 == w.begin) back.template read<LANES>(now, at, w.list);
            const Known known(a, event, t, a.newest_first ? row0 - w.list_begin + place : w.list_end - 1 - row0 - place, s_edges);
            each_batch(batch, n, cut.slots * U, read, [&](Batch<T, VEC, U, EXACT>& b, int i0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int row = i0 + u * cut.slots + at.slot, found = __shfl(known.bucket, min(row, n - 1)), bucket = row < n ? found : -1;
                    bool counts[G];
                    float ds[G], to_k[N], to_v[N];
                    const bool some = back.template take<LANES>(a, cut, at, b.k[u], b.v[u], bucket, s_table, scale, counts, ds, to_k, to_v);
                    if (at.head && row < n) {
                        const uint32_t more = __umul24(row, (uint32_t)row_of * (uint32_t)sizeof(T));
                        Row<T, VEC> to;
                        to.set(to_k);
                        to.clear_unless(some);
                        to.write(dk_row, more, at.at, at.there);
                        to.set(to_v);
                        to.clear_unless(some);
                        to.write(dv_row, more, at.at, at.there);
                    }
                    if (now.tables) add_to_table<T, VEC, G, EXACT>(a, cut, at, bucket, counts, ds, s_mine);
                }
            });
        }
        const Args<T>& end = args_now<T>();
        const int64_t row = (w.whole ? w.list : w.slot) * end.a.heads * end.a.dim;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            if (g >= end.a.group) break;
            at.joined(end.a, end.cut, g, back.acc[g], [&](uint32_t c, float x, float y, auto two_) {
                if (!w.whole) put(end.work.acc + row, c, x, y, two_);
                else put(end.dq + row, c, x, y, two_);
            });
        }
    }
    const Args<T>& last = args_now<T>();
    if (!last.tables) return;
    __syncthreads();
    const int64_t share = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    for (int i = threadIdx.x; i < entries; i += kWaves * kWave) {
        float sum = 0.0f;
        for (int k = 0; k < copies; ++k) sum += s_sums[k * entries + i];
        last.work.tables[share * entries + i] = sum;
    }
}

// Adds up the parts' gradients of q, as k_attend_join, and (the first `sums` workgroups) the workgroups' of the table, eight entries each.
constexpr int kEntries = 8;
template <typename T>
__global__ void __launch_bounds__(1024) k_attend_grad_join(const Attend<T> a, const Cut cut, const Work work, unsigned sums, unsigned few, T* dq, int64_t shares, float* dtable) {
    __shared__ float s_sum[1024];
    if (blockIdx.x < sums) {
        const int entries = a.buckets * a.heads, e = (int)blockIdx.x * kEntries + threadIdx.x % kEntries;
        float sum = 0.0f;
#pragma unroll 8
        for (int64_t k = threadIdx.x / kEntries; k < shares; k += 1024 / kEntries) sum += work.tables[k * entries + min(e, entries - 1)];
        sum = over_parts(sum, kEntries, s_sum);
        if ((int)threadIdx.x < kEntries && e < entries) dtable[e] = sum;
        return;
    }
    const unsigned group = blockIdx.x - sums;
    if (group < few) {
        __shared__ float s_acc[16][kOwn * kWave];
        const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, all = a.heads * a.dim;
        const int chunks = (all + kOwn * kWave - 1) / (kOwn * kWave), c0 = (int)(group % chunks) * kOwn * kWave;
        const int64_t block0 = (int64_t)(group / chunks) * 16;
        const int32_t begins = lane < 16 && block0 + lane < cut.blocks ? work.first[block0 + lane] : -1;
        for (uint64_t left = __ballot(begins >= 0); left; left &= left - 1) {
            const int k = __builtin_ctzll(left);
            const int64_t block = block0 + k, list = __builtin_amdgcn_readlane(begins, k);
            const int64_t end = parts_end(a.edge(list + 1), cut.part, cut.blocks);
            if (is_many(block, end)) continue;
            __syncthreads();
            float acc[kOwn] = {};
#pragma unroll 4
            for (int64_t b = block + wave; b < end; b += 16) {
                const float* const row = work.acc + slot_of(b, block, cut) * all;
#pragma unroll
                for (int j = 0; j < kOwn; ++j) acc[j] += row[min(c0 + j * kWave + lane, all - 1)];
            }
#pragma unroll
            for (int j = 0; j < kOwn; ++j) s_acc[wave][j * kWave + lane] = acc[j];
            __syncthreads();
            const int mine = c0 + (int)threadIdx.x;
            if ((int)threadIdx.x >= kOwn * kWave || mine >= all) continue;
            float value = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) value += s_acc[i][threadIdx.x];
            dq[list * all + mine] = as_value<T>(value);
        }
        return;
    }
    const unsigned slices = (a.dim + kSlice - 1) / kSlice, slice = (group - few) % slices;
    const int64_t h = (group - few) / slices % a.heads;
    int64_t begin = 0, end = 0;
    const int64_t list = many_of(a, cut, (group - few) / slices / a.heads, begin, end);
    if (list < 0) return;
    const int ch = (int)(slice * kSlice + (threadIdx.x & (kSlice - 1))), c = min(ch, a.dim - 1), mine = threadIdx.x / kSlice, parts = 1024 / kSlice;
    float acc = 0.0f;
#pragma unroll 8
    for (int64_t b = begin + mine; b < end; b += parts) acc += work.acc[(slot_of(b, begin, cut) * a.heads + h) * a.dim + c];
    acc = over_parts(acc, kSlice, s_sum);
    if (mine == 0 && ch < a.dim) dq[(list * a.heads + h) * a.dim + ch] = as_value<T>(acc);
}

}  // namespace

extern "C" {

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
    const Norm* const norms = reinterpret_cast<const Norm*>(saved + saved_out_bytes(*a) / 4);
    const size_t lds = lds_of(*a, kWaves << c.log_copies);
    if (int e = check_joins(*a, c)) return e;
    const unsigned few = (unsigned)few_of(*a, c), sums = (a->buckets * a->heads + kEntries - 1) / kEntries, joins = sums + few + (unsigned)many_of(*a, c);
    choose(*a, c, [&](auto value, auto vec, auto group, auto lanes) {
        using T = decltype(value);
        const Attend<T> t = typed<T>(*a);
        const Args<T> args = {t, c, l.w, nullptr, const_cast<float*>(saved), const_cast<Norm*>(norms), static_cast<const T*>(d_dout), static_cast<T*>(d_dq),
                              static_cast<T*>(d_dk), static_cast<T*>(d_dv), d_dtable != nullptr};
        const auto kernel = k_attend_grad<T, vec(), group(), lanes()>;
        static int per_cu;
        const int shares = groups_of(*a, c, resident(kernel, lds, per_cu));
        if (shares) hipLaunchKernelGGL(kernel, dim3(shares, c.turns), dim3(kWaves * kWave), lds, stream, args);
        if (joins)
            hipLaunchKernelGGL((k_attend_grad_join<T>), dim3(joins), dim3(1024), 0, stream, t, c, l.w, sums, few, static_cast<T*>(d_dq),
                               (int64_t)shares * c.turns, d_dtable);
    });
    return launched("tns_attend_grad");
}

}  // extern "C"
