// Gated linear recurrence over ragged lists of events (include/tns_train.h): states, gradients, and the step of one event per node.
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
using tns::gap_of;
using tns::gate_of;
using tns::kLog2e;

namespace {

constexpr int kSaved = 16;            // rows from one saved state to the next
constexpr int kGroups = 1024;         // workgroups that share the lists of a gradient

template <typename T>
struct Lists {                        // tns_recur with its types
    int64_t S, rows;
    const int64_t* rowptr;
    const T *u, *x;
    int64_t ld_u, ld_x;
    const float *ts, *decay, *h0, *t0;
    int dim;
    bool newest_first;
};

// Rows of a list in the order of time: row(i) for i = 0 .. n-1, and the place of that event in the walk over all lists.
struct Walk {
    int64_t begin, n, total;
    bool newest_first;
    template <typename T>
    __device__ Walk(const Lists<T>& l, int64_t s) : newest_first(l.newest_first) {
        total = min(max(l.rowptr[l.S], (int64_t)0), l.rows);
        begin = min(max(l.rowptr[s], (int64_t)0), total);
        n = min(max(l.rowptr[s + 1], begin), total) - begin;
    }
    __device__ int64_t row(int64_t i) const { return newest_first ? begin + n - 1 - i : begin + i; }
    __device__ int64_t place(int64_t i) const { return newest_first ? total - 1 - row(i) : row(i); }
};

template <typename T>
__device__ float gap_at(const Lists<T>& l, const Walk& w, int64_t s, int64_t i) {
    const float t = l.ts[w.row(i)];
    return gap_of(t, i ? l.ts[w.row(i - 1)] : l.t0 ? l.t0[s] : t);
}

template <typename T>
__global__ void __launch_bounds__(256) k_recur_run(const Lists<T> l, T* h_out, int64_t ld_h, float* last, float* saved) {
    const int64_t s = blockIdx.x;
    const Walk w(l, s);
    for (int c = threadIdx.x; c < l.dim; c += 256) {
        float h = l.h0 ? l.h0[s * l.dim + c] : 0.0f;
        const float rate = l.ts ? -kLog2e * l.decay[c] : 0.0f;
        for (int64_t i = 0; i < w.n; ++i) {
            const int64_t r = w.row(i);
            if (saved && w.place(i) % kSaved == 0) saved[w.place(i) / kSaved * l.dim + c] = h;
            float z, f;
            gate_of(as_float(l.u[r * l.ld_u + c]), z, f);
            if (l.ts) f *= __builtin_amdgcn_exp2f(rate * gap_at(l, w, s, i));
            h = f * h + z * as_float(l.x[r * l.ld_x + c]);
            if (h_out) h_out[r * ld_h + c] = as_value<T>(h);
        }
        if (last) last[s * l.dim + c] = h;
    }
}

template <typename T>
__global__ void __launch_bounds__(256) k_recur_grad(const Lists<T> l, const float* saved, const T* dh, int64_t ld_dh, const float* dlast,
                                                    T* du, int64_t ld_du, T* dx, int64_t ld_dx, float* dh0, float* sums) {
    for (int c = threadIdx.x; c < l.dim; c += 256) {
        float sum = 0.0f;
        const float rate = l.ts ? -kLog2e * l.decay[c] : 0.0f;
        for (int64_t s = blockIdx.x; s < l.S; s += gridDim.x) {
            const Walk w(l, s);
            float back = dlast ? dlast[s * l.dim + c] : 0.0f;
            int64_t end = w.n;
            while (end > 0) {
                const int64_t first = max(end - 1 - w.place(end - 1) % kSaved, (int64_t)0);
                float before[kSaved], h = w.place(first) % kSaved == 0 && first ? saved[w.place(first) / kSaved * l.dim + c] : l.h0 ? l.h0[s * l.dim + c] : 0.0f;
                for (int64_t i = first; i < end; ++i) {
                    before[i - first] = h;
                    float z, f;
                    gate_of(as_float(l.u[w.row(i) * l.ld_u + c]), z, f);
                    if (l.ts) f *= __builtin_amdgcn_exp2f(rate * gap_at(l, w, s, i));
                    h = f * h + z * as_float(l.x[w.row(i) * l.ld_x + c]);
                }
                for (int64_t i = end - 1; i >= first; --i) {
                    const int64_t r = w.row(i);
                    float z, rest;
                    gate_of(as_float(l.u[r * l.ld_u + c]), z, rest);
                    const float gap = l.ts ? gap_at(l, w, s, i) : 0.0f;
                    const float f = l.ts ? rest * __builtin_amdgcn_exp2f(rate * gap) : rest;
                    if (dh) back += as_float(dh[r * ld_dh + c]);
                    dx[r * ld_dx + c] = as_value<T>(z * back);
                    const float keep = f * before[i - first];
                    du[r * ld_du + c] = as_value<T>(z * back * (rest * as_float(l.x[r * l.ld_x + c]) - keep));
                    sum -= back * keep * gap;
                    back *= f;
                }
                end = first;
            }
            if (dh0) dh0[s * l.dim + c] = back;
        }
        if (sums) sums[(int64_t)blockIdx.x * l.dim + c] = sum;
    }
}

__global__ void __launch_bounds__(256) k_recur_sums(const float* sums, int groups, int dim, float* out) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= dim) return;
    float sum = 0.0f;
    for (int g = 0; g < groups; ++g) sum += sums[(int64_t)g * dim + c];
    out[c] = sum;
}

template <typename T>
__global__ void __launch_bounds__(256) k_recur_step(int64_t num_ids, int dim, const int32_t* ids, const T* u, int64_t ld_u, const T* x, int64_t ld_x,
                                                    const float* ts, const float* decay, float* state, float* state_ts, T* out, int64_t ld_out) {
    const int64_t b = blockIdx.x;
    const int64_t id = ids[b];
    const bool held = id >= 0 && id < num_ids;
    const float gap = held && ts ? gap_of(ts[b], state_ts[id]) : 0.0f;
    __syncthreads();                  // every wave has read the time before one writes it
    if (held && ts && threadIdx.x == 0) state_ts[id] = ts[b];
    for (int c = threadIdx.x; c < dim; c += 256) {
        float h = 0.0f;
        if (held) {
            float z, f;
            gate_of(as_float(u[b * ld_u + c]), z, f);
            if (ts) f *= __builtin_amdgcn_exp2f(-kLog2e * decay[c] * gap);
            h = f * state[id * dim + c] + z * as_float(x[b * ld_x + c]);
            state[id * dim + c] = h;
        }
        if (out) out[b * ld_out + c] = as_value<T>(h);
    }
}

int check(const tns_recur* r) {
    if (!r) return fail(TNS_EINVAL, "null description of the lists");
    if (r->S < 0 || r->rows < 0) return fail(TNS_EINVAL, "negative number of lists or rows");
    if (r->S > (int64_t)INT32_MAX || r->rows > (int64_t)1 << 40) return fail(TNS_ESIZE, "more than 2^31-1 lists or 2^40 rows");
    if (r->dim < 1 || r->dim > 1 << 16) return fail(TNS_EINVAL, "dim must be in [1, 2^16]");
    if (r->dtype != TNS_F32 && r->dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if ((r->flags & ~TNS_NEWEST_FIRST) || r->reserved) return fail(TNS_EINVAL, "unknown flag");
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

size_t run_bytes(const tns_recur&) { return 0; }
size_t grad_bytes(const tns_recur& r) { return (size_t)kGroups * r.dim * 4; }
size_t saved_bytes(const tns_recur& r) { return (size_t)((r.rows + kSaved - 1) / kSaved) * r.dim * 4; }

template <typename T>
Lists<T> typed(const tns_recur& r) {
    return {r.S, r.rows, r.d_rowptr, static_cast<const T*>(r.d_u), static_cast<const T*>(r.d_x), r.ld_u, r.ld_x,
            r.d_ts, r.d_decay, r.d_h0, r.d_t0, r.dim, (r.flags & TNS_NEWEST_FIRST) != 0};
}

template <typename T>
void launch_run(const tns_recur& r, void* h, int64_t ld_h, float* last, void* saved, hipStream_t stream) {
    hipLaunchKernelGGL((k_recur_run<T>), dim3((unsigned)r.S), dim3(256), 0, stream, typed<T>(r), static_cast<T*>(h), ld_h, last, static_cast<float*>(saved));
}

template <typename T>
void launch_grad(const tns_recur& r, const void* saved, const void* dh, int64_t ld_dh, const float* dlast, void* du, int64_t ld_du, void* dx,
                 int64_t ld_dx, float* ddecay, float* dh0, void* workspace, hipStream_t stream) {
    const int groups = (int)std::min<int64_t>(r.S, kGroups);
    float* const sums = ddecay ? static_cast<float*>(workspace) : nullptr;
    if (groups)
        hipLaunchKernelGGL((k_recur_grad<T>), dim3(groups), dim3(256), 0, stream, typed<T>(r), static_cast<const float*>(saved), static_cast<const T*>(dh), ld_dh,
                           dlast, static_cast<T*>(du), ld_du, static_cast<T*>(dx), ld_dx, dh0, sums);
    if (ddecay) hipLaunchKernelGGL(k_recur_sums, dim3((r.dim + 255) / 256), dim3(256), 0, stream, sums, groups, r.dim, ddecay);
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
    if (run) *run = run_bytes(*r);
    if (grad) *grad = grad_bytes(*r);
    if (saved) *saved = saved_bytes(*r);
    return TNS_OK;
}

int tns_recur_run(const tns_recur* r, void* d_h, int64_t ld_h, float* d_h_last, void* d_saved, void* d_workspace, size_t workspace_bytes,
                  void* hip_stream) {
    tns::clear_error();
    if (int e = check_arrays(r)) return e;
    if (d_h && ld_h < r->dim) return fail(TNS_EINVAL, "rows of h overlap");
    if (misaligned(d_saved, 256)) return fail(TNS_EINVAL, "saved states must be 256-byte aligned");
    if (int e = check_workspace(d_workspace, workspace_bytes, run_bytes(*r))) return e;
    if (r->S == 0) return TNS_OK;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    (r->dtype == TNS_F32 ? launch_run<float> : launch_run<bf16>)(*r, d_h, ld_h, d_h_last, d_saved, stream);
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
    if (int e = check_workspace(d_workspace, workspace_bytes, grad_bytes(*r))) return e;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    (r->dtype == TNS_F32 ? launch_grad<float> : launch_grad<bf16>)(*r, d_saved, d_dh, ld_dh, d_dh_last, d_du, ld_du, d_dx, ld_dx, d_ddecay, d_dh0,
                                                                   d_workspace, stream);
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
    auto launch = [&](auto value) {
        using T = decltype(value);
        hipLaunchKernelGGL((k_recur_step<T>), dim3((unsigned)B), dim3(256), 0, stream, num_ids, dim, d_ids, static_cast<const T*>(d_u), ld_u,
                           static_cast<const T*>(d_x), ld_x, d_ts, d_decay, d_state, d_state_ts, static_cast<T*>(d_out), ld_out);
    };
    if (dtype == TNS_F32) launch(float{});
    else launch(bf16{});
    return launched("tns_recur_step");
}

}  // extern "C"
