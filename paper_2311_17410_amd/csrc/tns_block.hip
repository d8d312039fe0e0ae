// What stands between two layers: norm of a branch, its gate and scale, the sum with the residual, the norm before the next branch; and
// the gradients (include/tns_layer.h).
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
using tns::gate_of;
using tns::over_lanes;
using tns::over_strided;

namespace {

constexpr int kWave = 64;

template <typename T>
struct Block {                          // tns_block with its types
    int64_t rows;
    const T *x, *branch, *gate;
    int64_t ld_x, ld_branch, ld_gate;
    const float *scale, *post, *pre;
    float eps, inverse;                 // inverse: 1 / dim
    int dim;
    bool center;
};

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
    T v[VEC];
};

// G lanes, or a workgroup of G threads, hold a row: NV vectors of VEC channels each.
template <typename T, int VEC, int G, int NV>
struct Team {
    static constexpr int THREADS = G > 256 ? G : 256, ROWS = THREADS / G, N = VEC * NV;
    int at[NV];
    bool there[NV], whole;              // whole: every lane has all its channels

    __device__ Team(int dim) : whole(dim == G * N) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            at[j] = (j * G + (int)(threadIdx.x % G)) * VEC;
            there[j] = at[j] < dim;
        }
    }
    // (Without branches, so that all arrays' rows are on their way at once: lanes beyond the row read its first channels.)
    __device__ __forceinline__ void read(const T* row, Vec<T, VEC> (&to)[NV]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) to[j] = *reinterpret_cast<const Vec<T, VEC>*>(row + (there[j] ? at[j] : 0));
    }
    // Values of a row that `is`, zero beyond it.
    __device__ __forceinline__ void widen(const Vec<T, VEC> (&v)[NV], bool is, float (&to)[N]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) to[j * VEC + i] = is && there[j] ? as_float(v[j].v[i]) : 0.0f;
    }
    __device__ __forceinline__ void write(T* row, bool is, const float (&v)[N]) const {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            Vec<T, VEC> raw;
#pragma unroll
            for (int i = 0; i < VEC; ++i) raw.v[i] = as_value<T>(v[j * VEC + i]);
            if (is && there[j]) *reinterpret_cast<Vec<T, VEC>*>(row + at[j]) = raw;
        }
    }
    __device__ __forceinline__ void weights(const float* w, float (&to)[N]) const {      // 1 without, and 0 beyond the row
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) to[j * VEC + i] = !there[j] ? 0.0f : w ? w[at[j] + i] : 1.0f;
    }
    // Sums over a row, by all its lanes; K of them at once.
    template <int K>
    __device__ __forceinline__ void sums(float (&v)[K]) const {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = over_lanes(v[k], G < kWave ? G : kWave, Add{});
        if constexpr (G > kWave) {
            __shared__ float s_sum[K][G / kWave];
            __syncthreads();
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) s_sum[k][threadIdx.x >> 6] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                v[k] = 0.0f;
                for (int w = 0; w < G / kWave; ++w) v[k] += s_sum[k][w];
            }
        }
    }
    // v becomes the normed row (zero beyond it); returns one over the norm.  The mean first and then the squares of what is left: their
    // difference, mean(v^2) - mean^2, would lose the spread of rows that are far from zero.
    __device__ __forceinline__ float norm(const Block<T>& b, float (&v)[N]) const {
        if (b.center) {
            float mean[1] = {};
#pragma unroll
            for (int i = 0; i < N; ++i) mean[0] += v[i];
            sums(mean);
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = there[i / VEC] ? v[i] - mean[0] * b.inverse : 0.0f;
        }
        float square[1] = {};
#pragma unroll
        for (int i = 0; i < N; ++i) square[0] += v[i] * v[i];
        sums(square);
        const float r = 1.0f / sqrtf(square[0] * b.inverse + b.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= r;
        return r;
    }
    // Gradient by a norm's input: g, given that by its output, y the normed row and r one over the norm.
    __device__ __forceinline__ void through_norm(const Block<T>& b, float (&g)[N], const float (&y)[N], float r) const {
        float sum[2] = {};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            sum[0] += g[i] * y[i];
            sum[1] += g[i];
        }
        sums(sum);
        const float along = sum[0] * b.inverse, mean = b.center ? sum[1] * b.inverse : 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = there[i / VEC] ? (g[i] - y[i] * along - mean) * r : 0.0f;
    }
};

// Bound by memory: a million rows of 128 fp32 channels without a gate, 2.05 GB in 395 us (5.2 TB/s); 66600 of 172 bf16, 116 MB in 29 us (4.0): there
// the instructions of sums and gates are as many as memory leaves time for.
template <typename T, int VEC, int G, int NV, bool GATE>
__global__ void __launch_bounds__(G > 256 ? G : 256) k_block(const Block<T> b, T* out, T* next) {
    using Rows = Team<T, VEC, G, NV>;
    constexpr int N = Rows::N;
    const Rows team(b.dim);
    float factor[N], other[N], pre[N];
    team.weights(b.scale, factor);
    team.weights(b.post, other);
    team.weights(b.pre, pre);
#pragma unroll
    for (int i = 0; i < N; ++i) factor[i] *= other[i];
    struct Raw {
        Vec<T, VEC> branch[NV], x[NV], gate[GATE ? NV : 1];
    };
    auto read = [&](int64_t row, Raw& raw) {
        row = min(row, b.rows - 1);
        team.read(b.branch + row * b.ld_branch, raw.branch);
        team.read(b.x + row * b.ld_x, raw.x);
        if constexpr (GATE) team.read(b.gate + row * b.ld_gate, raw.gate);
    };
    const int64_t stride = (int64_t)gridDim.x * Rows::ROWS;
    int64_t row = (int64_t)blockIdx.x * Rows::ROWS + threadIdx.x / G;
    Raw raw;
    // (every lane makes every turn: the sums take all of a wave or workgroup)
    for (int64_t row0 = (int64_t)blockIdx.x * Rows::ROWS; row0 < b.rows; row0 += stride, row += stride) {
        read(row, raw);
        const bool is = row < b.rows;
        float v[N], x[N];
        team.widen(raw.branch, is, v);
        team.widen(raw.x, is, x);
        if (b.post) team.norm(b, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float z = 1.0f, rest;
            if constexpr (GATE) gate_of(as_float(raw.gate[i / VEC].v[i % VEC]), z, rest);
            x[i] += factor[i] * z * v[i];
        }
        team.write(out + row * b.dim, is, x);
        if (b.pre) {
            if (!team.whole)
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = team.there[i / VEC] ? x[i] : 0.0f;      // (a gate of the first channels' may be no number)
            team.norm(b, x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] *= pre[i];
            team.write(next + row * b.dim, is, x);
        }
    }
}

// All gradients of a row while it is in registers; norms and gate are computed again.  Every lane adds up its channels' part of the
// weights' gradients over the rows it sees: of scale and post the same sum, of (gradient by out) sigmoid(gate) norm(branch).
// A gradient that is not there is read from x and not used.  A million rows of 128 fp32 channels, 3.07 GB in 611 us (5.0 TB/s); 66600 of 172 bf16,
// 185 MB in 41 us (4.5).  The next row read ahead made it slower (5 %: fewer waves), as did more workgroups.
template <typename T, int VEC, int G, int NV, bool GATE>
__global__ void __launch_bounds__(G > 256 ? G : 256) k_block_grad(const Block<T> b, const T* dout, int64_t ld_dout, const T* dnext, int64_t ld_dnext, T* dx, T* dbranch, T* dgate, float* shares) {
    using Rows = Team<T, VEC, G, NV>;
    constexpr int N = Rows::N;
    const Rows team(b.dim);
    float factor[N], other[N], pre[N], both[N], of_pre[N];
    team.weights(b.scale, factor);
    team.weights(b.post, other);
    team.weights(b.pre, pre);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        factor[i] *= other[i];
        both[i] = of_pre[i] = 0.0f;
    }
    struct Raw {
        Vec<T, VEC> branch[NV], gate[GATE ? NV : 1], x[NV], dout[NV], dnext[NV];
    };
    const T *const from_out = dout ? dout : b.x, *const from_next = dnext ? dnext : b.x;
    const int64_t ld_out = dout ? ld_dout : b.ld_x, ld_next = dnext ? ld_dnext : b.ld_x;
    auto read = [&](int64_t row, Raw& raw) {
        row = min(row, b.rows - 1);
        team.read(b.branch + row * b.ld_branch, raw.branch);
        if constexpr (GATE) team.read(b.gate + row * b.ld_gate, raw.gate);
        team.read(b.x + row * b.ld_x, raw.x);
        team.read(from_out + row * ld_out, raw.dout);
        team.read(from_next + row * ld_next, raw.dnext);
    };
    const int64_t stride = (int64_t)gridDim.x * Rows::ROWS;
    int64_t row = (int64_t)blockIdx.x * Rows::ROWS + threadIdx.x / G;
    Raw raw;
    for (int64_t row0 = (int64_t)blockIdx.x * Rows::ROWS; row0 < b.rows; row0 += stride, row += stride) {
        read(row, raw);
        const bool is = row < b.rows;
        float y[N], z[N], rest[N], g[N], r = 1.0f;
        team.widen(raw.branch, is, y);
        if (b.post) r = team.norm(b, y);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            z[i] = 1.0f;
            rest[i] = 0.0f;
            if constexpr (GATE) {
                gate_of(as_float(raw.gate[i / VEC].v[i % VEC]), z[i], rest[i]);
                z[i] = is && team.there[i / VEC] ? z[i] : 0.0f;
            }
        }
        team.widen(raw.dout, is && dout, g);
        if (dnext) {
            float m[N], d[N];
            team.widen(raw.x, is, m);
            team.widen(raw.dnext, is, d);
#pragma unroll
            for (int i = 0; i < N; ++i) m[i] += factor[i] * z[i] * y[i];
            const float rm = team.norm(b, m);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                of_pre[i] += is ? d[i] * m[i] : 0.0f;      // (a row that is not has a norm of 1 / sqrt(eps))
                d[i] *= pre[i];
            }
            team.through_norm(b, d, m, rm);
#pragma unroll
            for (int i = 0; i < N; ++i) g[i] += d[i];
        }
        team.write(dx + row * b.dim, is, g);
        float to_gate[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            g[i] *= z[i];
            both[i] += is ? g[i] * y[i] : 0.0f;
            g[i] *= factor[i];
            to_gate[i] = g[i] * y[i] * rest[i];
        }
        if constexpr (GATE) team.write(dgate + row * b.dim, is, to_gate);
        if (b.post) team.through_norm(b, g, y, r);
        team.write(dbranch + row * b.dim, is, g);
    }
    if (!shares) return;
    // the workgroup's share
    float* const to = shares + (int64_t)blockIdx.x * 2 * b.dim;
    if constexpr (G <= kWave) {
        __shared__ float s_sum[2][4][G * N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            both[i] = over_strided(both[i], G, Add{});
            of_pre[i] = over_strided(of_pre[i], G, Add{});
        }
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        if (lane < G)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int c = (i / VEC * G + lane) * VEC + i % VEC;
                s_sum[0][wave][c] = both[i];
                s_sum[1][wave][c] = of_pre[i];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < b.dim; c += 256)
#pragma unroll
            for (int k = 0; k < 2; ++k) to[k * b.dim + c] = (s_sum[k][0][c] + s_sum[k][1][c]) + (s_sum[k][2][c] + s_sum[k][3][c]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (team.there[i / VEC]) {
                to[team.at[i / VEC] + i % VEC] = both[i];
                to[b.dim + team.at[i / VEC] + i % VEC] = of_pre[i];
            }
    }
}

// Sums of the workgroups' shares in a fixed order, eight channels a workgroup.
constexpr int kChannels = 8;
__global__ void __launch_bounds__(1024) k_block_sums(const float* shares, int groups, int dim, const float* scale, const float* post, float* dscale, float* dpost, float* dpre) {
    __shared__ float s_sum[2][1024 / kChannels][kChannels];
    const int part = threadIdx.x / kChannels, ch = threadIdx.x % kChannels, c = (int)blockIdx.x * kChannels + ch, at = min(c, dim - 1);
    float a = 0.0f, b = 0.0f;
#pragma unroll 4
    for (int k = part; k < groups; k += 1024 / kChannels) {
        a += shares[(int64_t)k * 2 * dim + at];
        b += shares[(int64_t)k * 2 * dim + dim + at];
    }
    s_sum[0][part][ch] = a;
    s_sum[1][part][ch] = b;
    for (int n = 1024 / kChannels / 2; n; n /= 2) {
        __syncthreads();
        if (part < n) {
            s_sum[0][part][ch] += s_sum[0][part + n][ch];
            s_sum[1][part][ch] += s_sum[1][part + n][ch];
        }
    }
    if (part || c >= dim) return;
    a = s_sum[0][0][ch];
    if (dscale) dscale[c] = post ? post[c] * a : a;
    if (dpost) dpost[c] = scale ? scale[c] * a : a;
    if (dpre) dpre[c] = s_sum[1][0][ch];
}

// ---- host -------------------------------------------------------------------------------------------------

constexpr int kGroups = 2048, kGradGroups = 1024;      // workgroups of a launch, which go round the rows

bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) & (to - 1); }

int check(const tns_block* b) {
    if (!b) return fail(TNS_EINVAL, "null description of the block");
    if (b->rows < 0) return fail(TNS_EINVAL, "negative number of rows");
    if (b->rows > (int64_t)1 << 40) return fail(TNS_ESIZE, "more than 2^40 rows");
    if (b->dim < 1 || b->dim > 8192) return fail(TNS_EINVAL, "dim must be in [1, 8192]");
    if (b->dtype != TNS_F32 && b->dtype != TNS_BF16) return fail(TNS_EINVAL, "unknown dtype");
    if ((b->flags & ~TNS_CENTER) || b->reserved) return fail(TNS_EINVAL, "unknown flag");
    if (b->ld_x < b->dim || b->ld_branch < b->dim || (b->d_gate && b->ld_gate < b->dim)) return fail(TNS_EINVAL, "rows of x, branch or gate overlap");
    if (b->rows > 0 && (!b->d_x || !b->d_branch)) return fail(TNS_EINVAL, "null x or branch");
    if (!(b->eps >= 0) || b->eps > 3e38) return fail(TNS_EINVAL, "eps must be a number from 0 on");
    const size_t size = b->dtype == TNS_F32 ? 4 : 2;
    if (misaligned(b->d_x, size) || misaligned(b->d_branch, size) || misaligned(b->d_gate, size)) return fail(TNS_EINVAL, "x, branch or gate is not aligned to its type");
    return TNS_OK;
}

template <typename T>
Block<T> typed(const tns_block& b) {
    return {b.rows, static_cast<const T*>(b.d_x), static_cast<const T*>(b.d_branch), static_cast<const T*>(b.d_gate), b.ld_x, b.ld_branch, b.ld_gate,
            b.d_scale, b.d_post, b.d_pre, (float)b.eps, 1.0f / (float)b.dim, b.dim, (b.flags & TNS_CENTER) != 0};
}

// Calls `go` with the type, the channels of a vector, the lanes of a row and the vectors of a lane.  A sum over a row takes as many steps as its lanes
// double, whatever they hold, so rows have few lanes of up to kHeld channels before they have more: 66600 rows of 172 bf16 channels in 16 lanes of
// 12 channels, in 32 of 8, in 64 of 4: outputs 29, 28, 33 us, gradients 42, 50, 59.
constexpr int kHeld = 12;
template <typename A, typename F>
void choose(const tns_block& b, const A& fits, const F& go) {
    using std::integral_constant;
    auto teams = [&](auto value, auto vec) {
        constexpr int V = vec();
        const int vectors = (b.dim + V - 1) / V;
        bool done = false;
        auto with = [&](auto lanes, auto many) {
            if constexpr (V * many() <= (lanes() > 64 ? 8 : kHeld)) {
                if (done || vectors > lanes() * many()) return;
                done = true;
                go(value, vec, lanes, many);
            }
        };
        with(integral_constant<int, 8>{}, integral_constant<int, 1>{});
        auto all = [&](auto lanes) {
            with(lanes, integral_constant<int, 1>{});
            with(lanes, integral_constant<int, 2>{});
            with(lanes, integral_constant<int, 3>{});
            with(lanes, integral_constant<int, 4>{});
            if constexpr (V == 1) with(lanes, integral_constant<int, 8>{});
        };
        all(integral_constant<int, 16>{});
        all(integral_constant<int, 32>{});
        all(integral_constant<int, 64>{});
        with(integral_constant<int, 256>{}, integral_constant<int, 8 / V>{});
        with(integral_constant<int, 1024>{}, integral_constant<int, 8 / V>{});
    };
    if (b.dtype == TNS_F32) {
        if (fits(4)) teams(float{}, integral_constant<int, 4>{});
        else teams(float{}, integral_constant<int, 1>{});
    } else {
        if (fits(8)) teams(bf16{}, integral_constant<int, 8>{});
        else if (fits(4)) teams(bf16{}, integral_constant<int, 4>{});
        else teams(bf16{}, integral_constant<int, 1>{});
    }
}
bool fits(const tns_block& b, int n, std::initializer_list<const void*> arrays, int64_t ld_a, int64_t ld_b) {
    if (b.dim % n) return false;
    if (b.rows > 1 && (b.ld_x % n || b.ld_branch % n || (b.d_gate && b.ld_gate % n) || ld_a % n || ld_b % n)) return false;
    const size_t size = b.dtype == TNS_F32 ? 4 : 2;
    for (const void* p : arrays)
        if (misaligned(p, n * size)) return false;
    return true;
}
int groups_of(int64_t rows, int per, int most) { return (int)std::min<int64_t>((rows + per - 1) / per, most); }

int launched(const char* what) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int)TNS_OK : fail_hip(e, what);
}

}  // namespace

extern "C" {

int tns_block_run(const tns_block* b, void* d_out, void* d_next, void* hip_stream) {
    tns::clear_error();
    if (int e = check(b)) return e;
    if (b->rows > 0 && !d_out) return fail(TNS_EINVAL, "null out");
    if (b->rows > 0 && !d_next != !b->d_pre) return fail(TNS_EINVAL, "next and pre come together");
    const size_t size = b->dtype == TNS_F32 ? 4 : 2;
    if (misaligned(d_out, size) || misaligned(d_next, size)) return fail(TNS_EINVAL, "out or next is not aligned to its type");
    if (b->rows == 0) return TNS_OK;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    choose(*b, [&](int n) { return fits(*b, n, {b->d_x, b->d_branch, b->d_gate, d_out, d_next}, 0, 0); }, [&](auto value, auto vec, auto lanes, auto vectors) {
        using T = decltype(value);
        using Rows = Team<T, vec(), lanes(), vectors()>;
        auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(groups_of(b->rows, Rows::ROWS, kGroups)), dim3(Rows::THREADS), 0, stream, typed<T>(*b), static_cast<T*>(d_out), static_cast<T*>(d_next));
        };
        if (b->d_gate) launch(k_block<T, vec(), lanes(), vectors(), true>);
        else launch(k_block<T, vec(), lanes(), vectors(), false>);
    });
    return launched("tns_block_run");
}

int tns_block_workspace(int64_t rows, int32_t dim, size_t* grad_bytes) {
    tns::clear_error();
    if (rows < 0) return fail(TNS_EINVAL, "negative number of rows");
    if (rows > (int64_t)1 << 40) return fail(TNS_ESIZE, "more than 2^40 rows");
    if (dim < 1 || dim > 8192) return fail(TNS_EINVAL, "dim must be in [1, 8192]");
    if (grad_bytes) *grad_bytes = (size_t)std::min<int64_t>(rows, kGradGroups) * 2 * dim * 4;
    return TNS_OK;
}

int tns_block_grad(const tns_block* b, const void* d_dout, int64_t ld_dout, const void* d_dnext, int64_t ld_dnext, void* d_dx, void* d_dbranch, void* d_dgate, float* d_dscale,
                   float* d_dpost, float* d_dpre, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    tns::clear_error();
    if (int e = check(b)) return e;
    if (d_dnext && !b->d_pre) return fail(TNS_EINVAL, "gradient by a next that is not there");
    if ((d_dout && ld_dout < b->dim) || (d_dnext && ld_dnext < b->dim)) return fail(TNS_EINVAL, "rows of dout or dnext overlap");
    if (b->rows > 0 && (!d_dx || !d_dbranch)) return fail(TNS_EINVAL, "null dx or dbranch");
    if (b->rows > 0 && !d_dgate != !b->d_gate) return fail(TNS_EINVAL, "dgate and gate come together");
    if ((d_dscale && !b->d_scale) || (d_dpost && !b->d_post) || (d_dpre && !b->d_pre)) return fail(TNS_EINVAL, "gradient of a weight that is not there");
    const size_t size = b->dtype == TNS_F32 ? 4 : 2;
    for (const void* p : {d_dout, d_dnext, (const void*)d_dx, (const void*)d_dbranch, (const void*)d_dgate})
        if (misaligned(p, size)) return fail(TNS_EINVAL, "a gradient is not aligned to its type");
    size_t need = 0;
    if (int e = tns_block_workspace(b->rows, b->dim, &need)) return e;
    const bool sums = d_dscale || d_dpost || d_dpre;
    if (need && !d_workspace) return fail(TNS_EINVAL, "null workspace");
    if (misaligned(d_workspace, 256)) return fail(TNS_EINVAL, "workspace must be 256-byte aligned");
    if (workspace_bytes < need) return fail(TNS_ESIZE, "workspace smaller than asked for");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    float* const shares = static_cast<float*>(d_workspace);
    int groups = 0;
    if (b->rows > 0)
        choose(*b, [&](int n) { return fits(*b, n, {b->d_x, b->d_branch, b->d_gate, d_dout, d_dnext, d_dx, d_dbranch, d_dgate}, d_dout ? ld_dout : 0, d_dnext ? ld_dnext : 0); },
               [&](auto value, auto vec, auto lanes, auto vectors) {
            using T = decltype(value);
            using Rows = Team<T, vec(), lanes(), vectors()>;
            groups = groups_of(b->rows, Rows::ROWS, kGradGroups);
            auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, dim3(groups), dim3(Rows::THREADS), 0, stream, typed<T>(*b), static_cast<const T*>(d_dout), ld_dout, static_cast<const T*>(d_dnext),
                                   ld_dnext, static_cast<T*>(d_dx), static_cast<T*>(d_dbranch), static_cast<T*>(d_dgate), sums ? shares : nullptr);
            };
            if (b->d_gate) launch(k_block_grad<T, vec(), lanes(), vectors(), true>);
            else launch(k_block_grad<T, vec(), lanes(), vectors(), false>);
        });
    if (sums)
        hipLaunchKernelGGL(k_block_sums, dim3((b->dim + kChannels - 1) / kChannels), dim3(1024), 0, stream, shares, groups, b->dim, b->d_scale, b->d_post, d_dscale, d_dpost, d_dpre);
    return launched("tns_block_grad");
}

}  // extern "C"
