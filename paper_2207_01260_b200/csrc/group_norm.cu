// Group norm with an activation on channels-last tensors, and its gradients.
//
//   y = act(xhat gamma + beta + residual),   xhat = (x - mean) rstd,   rstd = 1 / sqrt(variance + eps)
//
// with the mean and the (biased) variance over the pixels of one image and the channels of one group.  With z what act is taken of and
// dz = dy act'(z):  dbeta = sum dz and dgamma = sum dz xhat over images and pixels, dresidual = dz, and
//   dx = rstd (gamma dz - m1 - xhat m2),   m1 and m2 the group's means of gamma dz and gamma dz xhat.
//
// A block owns whole columns: a thread holds the same 16 bytes of channels (8 bf16, 4 float32; single float32 where rows are not multiples of
// 16 bytes) of every R-th pixel, so that what belongs to a channel stays in its registers, and groups of any number of channels are put
// together from channels.  Two ways through the data:
//   - on chip: one cluster of up to 16 blocks holds the groups of one image, or a range of them, in shared memory; its blocks exchange
//     their sums, and the data is read once.
//   - in three launches (what does not fit): partial sums of chunks of pixels per channel; their combination; a second pass over the data.
// The variance is never a difference of large sums: a thread takes the deviations from its own mean, and means and deviations are put
// together pairwise (Chan, Golub, LeVeque 1979), in float32.
#include <cmath>
#include <type_traits>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace cprune {

// ------------------------------------------------------------------------------------------------ vectors of channels

template <int KIND> struct Lanes;       // 0: 8 bf16, 1: 4 float32, 2: one float32
template <> struct Lanes<0> {
    static constexpr int L = 8;
    using Raw = bf16x8;
    static __device__ __forceinline__ void unpack(const Raw &r, float *f) { unpack8(r, f); }
    static __device__ __forceinline__ Raw pack(const float *f) { return pack8(f); }
};
template <> struct Lanes<1> {
    static constexpr int L = 4;
    using Raw = float4;
    static __device__ __forceinline__ void unpack(const Raw &r, float *f) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
    static __device__ __forceinline__ Raw pack(const float *f) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Lanes<2> {
    static constexpr int L = 1;
    using Raw = float;
    static __device__ __forceinline__ void unpack(const Raw &r, float *f) { f[0] = r; }
    static __device__ __forceinline__ Raw pack(const float *f) { return f[0]; }
};

// An activation that keeps NaN (apply_act's maximum would drop it), and its slope: 0 on the borders of relu and relu6.
__device__ __forceinline__ float norm_act(float z, int act) {
    if (act == CPRUNE_ACT_NONE) return z;
    if (act == CPRUNE_ACT_SILU) return __fdividef(z, 1.f + __expf(-z));
    z = z < 0.f ? 0.f : z;
    return act == CPRUNE_ACT_RELU6 && z > 6.f ? 6.f : z;
}

struct NormParams {
    const void *x, *dy, *res;
    void *out, *dres;                   // y, or dx and dresidual
    const float *gamma, *beta;
    float *stats;                       // [N][G][2]: mean, rstd
    float2 *part;                       // partial results of chunks of pixels, [N][chunks][lanes]
    float2 *means;                      // backward: m1, m2 [N][G]
    float *dgamma, *dbeta;
    int N, HW, C, G, cpg;
    int pv;                             // vectors per pixel
    int sv;                             // columns (vectors) of a block's slice; slices of the last range may reach beyond pv
    int rows;                           // R: pixels that the block's threads hold side by side
    int per;                            // pixels of a block (on chip: of a rank; else: of a chunk)
    int chunks;
    int act;
    float eps;
};

// The side of relu's and relu6's borders on which z lies decides about a whole gradient, so next to a border it is taken in 64 bits.
__device__ __noinline__ float slope_64(float x, float mean, float rstd, float gamma, float beta, float res, int act) {
    const double z = ((double)x - (double)mean) * (double)rstd * (double)gamma + (double)beta + (double)res;
    return z > 0.0 && (act != CPRUNE_ACT_RELU6 || z < 6.0) ? 1.f : (z == z ? 0.f : (float)z);
}

// act'(z)
__device__ __forceinline__ float norm_slope(float x, float mean, float rstd, float gamma, float beta, float res, float xhat, int act) {
    if (act == CPRUNE_ACT_NONE) return 1.f;
    const float t = xhat * gamma, z = t + beta + res;
    if (act == CPRUNE_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-z));
        return s * (1.f + z * (1.f - s));
    }
    // x - mean, its products with rstd and gamma and the two sums are rounded: five times 2^-24 of the largest term bounds the error of z
    const float near = 4e-7f * (fabsf(t) + fabsf(beta) + fabsf(res));
    if (fabsf(z) <= near || (act == CPRUNE_ACT_RELU6 && fabsf(z - 6.f) <= near)) return slope_64(x, mean, rstd, gamma, beta, res, act);
    return z > 0.f && (act != CPRUNE_ACT_RELU6 || z < 6.f) ? 1.f : (z == z ? 0.f : z);
}

// What a thread needs of the channels of its column
template <int L> struct Column {
    float mean[L], rstd[L], gamma[L], beta[L];
    __device__ __forceinline__ void load_affine(const NormParams &p, int c0) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
            const bool in = c0 + l < p.C;
            gamma[l] = in ? (p.gamma ? __ldg(p.gamma + c0 + l) : 1.f) : 0.f;
            beta[l] = in && p.beta ? __ldg(p.beta + c0 + l) : 0.f;
            mean[l] = rstd[l] = 0.f;
        }
    }
};

template <int KIND>
__device__ __forceinline__ void apply_one(const NormParams &p, const Column<Lanes<KIND>::L> &k, int c0, const typename Lanes<KIND>::Raw &x, size_t at) {
    constexpr int L = Lanes<KIND>::L;
    using Raw = typename Lanes<KIND>::Raw;
    float f[L], r[L];
    Lanes<KIND>::unpack(x, f);
    if (p.res) Lanes<KIND>::unpack(((const Raw *)p.res)[at], r);
#pragma unroll
    for (int l = 0; l < L; ++l) {
        float z = (f[l] - k.mean[l]) * k.rstd[l] * k.gamma[l] + k.beta[l];
        if (p.res) z += r[l];
        f[l] = c0 + l < p.C ? norm_act(z, p.act) : 0.f;
    }
    ((Raw *)p.out)[at] = Lanes<KIND>::pack(f);
}

// dz and xhat of a vector
template <int KIND>
__device__ __forceinline__ void gradient_one(const NormParams &p, const Column<Lanes<KIND>::L> &k, const typename Lanes<KIND>::Raw &x,
                                             const typename Lanes<KIND>::Raw &dy, const typename Lanes<KIND>::Raw &res, float *dz, float *xhat) {
    constexpr int L = Lanes<KIND>::L;
    float f[L], r[L];
    Lanes<KIND>::unpack(x, f);
    Lanes<KIND>::unpack(dy, dz);
    if (p.res) Lanes<KIND>::unpack(res, r);
#pragma unroll
    for (int l = 0; l < L; ++l) {
        xhat[l] = (f[l] - k.mean[l]) * k.rstd[l];
        dz[l] *= norm_slope(f[l], k.mean[l], k.rstd[l], k.gamma[l], k.beta[l], p.res ? r[l] : 0.f, xhat[l], p.act);
    }
}

// ---------------------------------------------------------------------------------------------------- three launches

constexpr int NORM_T = 256;
constexpr int NORM_AHEAD = 4;           // vectors of a thread in flight

// Sums over the R rows of a block: v[a][l * T + thread] -> done(column lane, the A sums).  `sub` neighbouring threads share a lane of channels.
template <int L, int A, int T, typename F>
__device__ __forceinline__ void sum_rows(const float *v, int sv, int rows, F done) {
    const int lanes = sv * L;
    int sub = 1;
    while (sub < 32 && lanes * sub * 2 <= T) sub *= 2;
    const int sl = threadIdx.x % sub;
    for (int q0 = 0; q0 < lanes; q0 += T / sub) {
        const int q = q0 + threadIdx.x / sub;
        float s[A];
#pragma unroll
        for (int a = 0; a < A; ++a) s[a] = 0.f;
        if (q < lanes)
            for (int r = sl; r < rows; r += sub)
#pragma unroll
                for (int a = 0; a < A; ++a) s[a] += v[(a * L + q % L) * T + r * sv + q / L];
        for (int o = sub / 2; o > 0; o /= 2)
#pragma unroll
            for (int a = 0; a < A; ++a) s[a] += __shfl_xor_sync(0xffffffffu, s[a], o);
        if (q < lanes && sl == 0) done(q, s);
    }
}

// Number of the pixels r, r + R, ... below n
__device__ __forceinline__ int pixels_of(int n, int r, int rows) { return r < n ? (n - r + rows - 1) / rows : 0; }

// Mean and squared deviations of a chunk of pixels, channel by channel
template <int KIND>
__global__ void __launch_bounds__(NORM_T) norm_partial_kernel(const NormParams p) {
    constexpr int L = Lanes<KIND>::L;
    using Raw = typename Lanes<KIND>::Raw;
    __shared__ float v[2 * L * NORM_T];
    __shared__ float mean_s[L * NORM_T];
    pdl_wait();
    pdl_trigger();
    const int v0 = blockIdx.y * p.sv, sv = min(p.sv, p.pv - v0);
    const int rows = NORM_T / sv, r = threadIdx.x / sv, col = threadIdx.x - r * sv;
    const int p0 = blockIdx.x * p.per, n = min(p.per, p.HW - p0);
    const int cnt = r < rows ? pixels_of(n, r, rows) : 0;
    const size_t base = ((size_t)blockIdx.z * p.HW + p0 + r) * p.pv + v0 + col;
    float mean[L], m2[L];
#pragma unroll
    for (int l = 0; l < L; ++l) mean[l] = m2[l] = 0.f;
    // running mean and deviations of groups of NORM_AHEAD vectors
    for (int i0 = 0; i0 < cnt; i0 += NORM_AHEAD) {
        Raw raw[NORM_AHEAD];
#pragma unroll
        for (int i = 0; i < NORM_AHEAD; ++i)
            if (i0 + i < cnt) raw[i] = ((const Raw *)p.x)[base + (size_t)(i0 + i) * rows * p.pv];
        const float m = (float)min(NORM_AHEAD, cnt - i0), total = i0 + m, share = m / total;
        float f[NORM_AHEAD][L];
#pragma unroll
        for (int i = 0; i < NORM_AHEAD; ++i) Lanes<KIND>::unpack(raw[i], f[i]);
#pragma unroll
        for (int l = 0; l < L; ++l) {
            float s = 0.f, q = 0.f;
#pragma unroll
            for (int i = 0; i < NORM_AHEAD; ++i) s += i0 + i < cnt ? f[i][l] : 0.f;
            s /= m;
#pragma unroll
            for (int i = 0; i < NORM_AHEAD; ++i) {
                const float d = i0 + i < cnt ? f[i][l] - s : 0.f;
                q += d * d;
            }
            const float d = s - mean[l];
            mean[l] += d * share;
            m2[l] += q + d * d * (float)i0 * share;
        }
    }
    if (r < rows) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
            v[l * NORM_T + threadIdx.x] = mean[l] * (float)cnt;
            v[(L + l) * NORM_T + threadIdx.x] = m2[l];
        }
    }
    __syncthreads();
    const float inv = 1.f / (float)n;
    sum_rows<L, 1, NORM_T>(v, sv, rows, [&](int q, const float *s) { mean_s[q] = s[0] * inv; });
    __syncthreads();
    if (r < rows && cnt > 0) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
            const float d = mean[l] - mean_s[col * L + l];
            v[(L + l) * NORM_T + threadIdx.x] += d * d * (float)cnt;
        }
    }
    __syncthreads();
    float2 *part = p.part + ((size_t)blockIdx.z * p.chunks + blockIdx.x) * p.pv * L + v0 * L;
    sum_rows<L, 1, NORM_T>(v + L * NORM_T, sv, rows, [&](int q, const float *s) { part[q] = make_float2(mean_s[q], s[0]); });
}

// Sum over the threads of a team (a warp or a block), the same for all of them and in a fixed order
template <int TEAM>
__device__ __forceinline__ float team_sum(float s, float *scratch) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (TEAM > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int i = 0; i < TEAM / 32; ++i) s += scratch[i];
    }
    return s;
}

// Chunks and channels of a group put together: mean and rstd
template <int TEAM>
__global__ void __launch_bounds__(NORM_T) norm_combine_kernel(const NormParams p, int lanes) {
    __shared__ float scratch[NORM_T / 32];
    pdl_wait();
    pdl_trigger();
    const long long id = (long long)blockIdx.x * (NORM_T / TEAM) + threadIdx.x / TEAM;
    if (id >= (long long)p.N * p.G) return;          // (whole teams)
    const int n = (int)(id / p.G), g = (int)(id - (long long)n * p.G), t = threadIdx.x % TEAM;
    const float2 *part = p.part + (size_t)n * p.chunks * lanes + (size_t)g * p.cpg;
    const int entries = p.chunks * p.cpg;
    float s = 0.f;
    for (int e = t; e < entries; e += TEAM) {
        const int k = e / p.cpg, j = e - k * p.cpg;
        s += __ldcg(part + (size_t)k * lanes + j).x * (float)min(p.per, p.HW - k * p.per);
    }
    const float count = (float)p.HW * (float)p.cpg, mean = team_sum<TEAM>(s, scratch) / count;
    s = 0.f;
    for (int e = t; e < entries; e += TEAM) {
        const int k = e / p.cpg, j = e - k * p.cpg;
        const float2 v = __ldcg(part + (size_t)k * lanes + j);
        const float d = v.x - mean;
        s += v.y + d * d * (float)min(p.per, p.HW - k * p.per);
    }
    const float var = team_sum<TEAM>(s, scratch) / count;
    if (t == 0) ((float2 *)p.stats)[id] = make_float2(mean, 1.f / sqrtf(var + p.eps));
}

template <int L>
__device__ __forceinline__ void load_stats(const NormParams &p, Column<L> &k, int n, int c0) {
    k.load_affine(p, c0);
#pragma unroll
    for (int l = 0; l < L; ++l)
        if (c0 + l < p.C) {
            const float2 s = __ldcg((const float2 *)p.stats + (size_t)n * p.G + (c0 + l) / p.cpg);
            k.mean[l] = s.x;
            k.rstd[l] = s.y;
        }
}

template <int KIND>
__global__ void __launch_bounds__(NORM_T) norm_apply_kernel(const NormParams p) {
    constexpr int L = Lanes<KIND>::L;
    using Raw = typename Lanes<KIND>::Raw;
    pdl_wait();
    pdl_trigger();
    const int v0 = blockIdx.y * p.sv, sv = min(p.sv, p.pv - v0);
    const int rows = NORM_T / sv, r = threadIdx.x / sv, col = threadIdx.x - r * sv;
    const int p0 = blockIdx.x * p.per, n = min(p.per, p.HW - p0);
    if (r >= rows) return;
    const int cnt = pixels_of(n, r, rows), c0 = (v0 + col) * L;
    const size_t base = ((size_t)blockIdx.z * p.HW + p0 + r) * p.pv + v0 + col;
    Column<L> k;
    load_stats<L>(p, k, blockIdx.z, c0);
    for (int i0 = 0; i0 < cnt; i0 += NORM_AHEAD) {
        Raw raw[NORM_AHEAD];
#pragma unroll
        for (int i = 0; i < NORM_AHEAD; ++i)
            if (i0 + i < cnt) raw[i] = ((const Raw *)p.x)[base + (size_t)(i0 + i) * rows * p.pv];
#pragma unroll
        for (int i = 0; i < NORM_AHEAD; ++i)
            if (i0 + i < cnt) apply_one<KIND>(p, k, c0, raw[i], base + (size_t)(i0 + i) * rows * p.pv);
    }
}

// Sums of dz and dz xhat over a chunk of pixels, channel by channel
template <int KIND>
__global__ void __launch_bounds__(NORM_T) norm_grad_partial_kernel(const NormParams p) {
    constexpr int L = Lanes<KIND>::L;
    using Raw = typename Lanes<KIND>::Raw;
    __shared__ float v[2 * L * NORM_T];
    pdl_wait();
    pdl_trigger();
    const int v0 = blockIdx.y * p.sv, sv = min(p.sv, p.pv - v0);
    const int rows = NORM_T / sv, r = threadIdx.x / sv, col = threadIdx.x - r * sv;
    const int p0 = blockIdx.x * p.per, n = min(p.per, p.HW - p0);
    const int cnt = r < rows ? pixels_of(n, r, rows) : 0, c0 = (v0 + col) * L;
    const size_t base = ((size_t)blockIdx.z * p.HW + p0 + r) * p.pv + v0 + col;
    float a[L], b[L];
#pragma unroll
    for (int l = 0; l < L; ++l) a[l] = b[l] = 0.f;
    if (cnt > 0) {
        Column<L> k;
        load_stats<L>(p, k, blockIdx.z, c0);
        for (int i0 = 0; i0 < cnt; i0 += 2) {
            Raw x[2], dy[2], res[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i0 + i < cnt) {
                    const size_t at = base + (size_t)(i0 + i) * rows * p.pv;
                    x[i] = ((const Raw *)p.x)[at];
                    dy[i] = ((const Raw *)p.dy)[at];
                    if (p.res) res[i] = ((const Raw *)p.res)[at];
                }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (i0 + i < cnt) {
                    float dz[L], xhat[L];
                    gradient_one<KIND>(p, k, x[i], dy[i], res[i], dz, xhat);
#pragma unroll
                    for (int l = 0; l < L; ++l) { a[l] += dz[l]; b[l] += dz[l] * xhat[l]; }
                }
        }
    }
    if (r < rows) {
#pragma unroll
        for (int l = 0; l < L; ++l) {
            v[l * NORM_T + threadIdx.x] = a[l];
            v[(L + l) * NORM_T + threadIdx.x] = b[l];
        }
    }
    __syncthreads();
    float2 *part = p.part + ((size_t)blockIdx.z * p.chunks + blockIdx.x) * p.pv * L + v0 * L;
    sum_rows<L, 2, NORM_T>(v, sv, rows, [&](int q, const float *s) { part[q] = make_float2(s[0], s[1]); });
}

template <int TEAM>
__global__ void __launch_bounds__(NORM_T) norm_grad_combine_kernel(const NormParams p, int lanes) {
    __shared__ float scratch[NORM_T / 32];
    pdl_wait();
    pdl_trigger();
    const long long id = (long long)blockIdx.x * (NORM_T / TEAM) + threadIdx.x / TEAM;
    if (id >= (long long)p.N * p.G) return;
    const int n = (int)(id / p.G), g = (int)(id - (long long)n * p.G), t = threadIdx.x % TEAM;
    const float2 *part = p.part + (size_t)n * p.chunks * lanes + (size_t)g * p.cpg;
    const int entries = p.chunks * p.cpg;
    float s1 = 0.f, s2 = 0.f;
    for (int e = t; e < entries; e += TEAM) {
        const int k = e / p.cpg, j = e - k * p.cpg;
        const float2 v = __ldcg(part + (size_t)k * lanes + j);
        const float gamma = p.gamma ? __ldg(p.gamma + g * p.cpg + j) : 1.f;
        s1 += gamma * v.x;
        s2 += gamma * v.y;
    }
    const float count = (float)p.HW * (float)p.cpg;
    s1 = team_sum<TEAM>(s1, scratch);
    s2 = team_sum<TEAM>(s2, scratch);
    if (t == 0) p.means[id] = make_float2(s1 / count, s2 / count);
}

// dgamma and dbeta of 32 channels: the partial sums of all images and chunks, eight at a time, in a fixed order; their total in 64 bits
__device__ __forceinline__ void parameter_gradients(const NormParams &p, int block, int lanes) {
    __shared__ double tot[2][8][33];
    const int cl = threadIdx.x & 31, k = threadIdx.x >> 5, c = block * 32 + cl;
    double a = 0.0, b = 0.0;
    const long long entries = (long long)p.N * p.chunks;
    if (c < p.C)
        for (long long e0 = k; e0 < entries; e0 += 32) {
            float2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = e0 + 8 * i < entries ? __ldcg(p.part + (size_t)(e0 + 8 * i) * lanes + c) : make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) { a += v[i].x; b += v[i].y; }
        }
    tot[0][k][cl] = a;
    tot[1][k][cl] = b;
    __syncthreads();
    if (k < 2 && c < p.C) {
        double s = 0.0;
        for (int i = 0; i < 8; ++i) s += tot[k][i][cl];
        float *to = k ? p.dgamma : p.dbeta;
        if (to) to[c] = (float)s;
    }
}

__global__ void __launch_bounds__(NORM_T) norm_parameter_gradients_kernel(const NormParams p, int lanes) {
    pdl_wait();
    pdl_trigger();
    parameter_gradients(p, blockIdx.x, lanes);
}

template <int KIND>
__device__ __forceinline__ void store_gradient(const NormParams &p, const Column<Lanes<KIND>::L> &k, const float *m1, const float *m2, int c0, const float *dz,
                                               const float *xhat, size_t at) {
    constexpr int L = Lanes<KIND>::L;
    using Raw = typename Lanes<KIND>::Raw;
    float f[L], g[L];
#pragma unroll
    for (int l = 0; l < L; ++l) {
        const bool in = c0 + l < p.C;
        f[l] = in ? k.rstd[l] * (k.gamma[l] * dz[l] - m1[l] - xhat[l] * m2[l]) : 0.f;
        g[l] = in ? dz[l] : 0.f;
    }
    ((Raw *)p.out)[at] = Lanes<KIND>::pack(f);
    if (p.dres) ((Raw *)p.dres)[at] = Lanes<KIND>::pack(g);
}

template <int KIND>
__global__ void __launch_bounds__(NORM_T) norm_grad_apply_kernel(const NormParams p, int lanes) {
    constexpr int L = Lanes<KIND>::L;
    using Raw = typename Lanes<KIND>::Raw;
    pdl_wait();
    pdl_trigger();
    const int v0 = blockIdx.y * p.sv, sv = min(p.sv, p.pv - v0);
    const int rows = NORM_T / sv, r = threadIdx.x / sv, col = threadIdx.x - r * sv;
    const int p0 = blockIdx.x * p.per, n = min(p.per, p.HW - p0);
    if (r >= rows) return;
    const int cnt = pixels_of(n, r, rows), c0 = (v0 + col) * L;
    const size_t base = ((size_t)blockIdx.z * p.HW + p0 + r) * p.pv + v0 + col;
    Column<L> k;
    load_stats<L>(p, k, blockIdx.z, c0);
    float m1[L], m2[L];
#pragma unroll
    for (int l = 0; l < L; ++l) {
        const float2 m = c0 + l < p.C ? __ldcg(p.means + (size_t)blockIdx.z * p.G + (c0 + l) / p.cpg) : make_float2(0.f, 0.f);
        m1[l] = m.x;
        m2[l] = m.y;
    }
    for (int i0 = 0; i0 < cnt; i0 += 2) {
        Raw x[2], dy[2], res[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i0 + i < cnt) {
                const size_t at = base + (size_t)(i0 + i) * rows * p.pv;
                x[i] = ((const Raw *)p.x)[at];
                dy[i] = ((const Raw *)p.dy)[at];
                if (p.res) res[i] = ((const Raw *)p.res)[at];
            }
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (i0 + i < cnt) {
                float dz[L], xhat[L];
                gradient_one<KIND>(p, k, x[i], dy[i], res[i], dz, xhat);
                store_gradient<KIND>(p, k, m1, m2, c0, dz, xhat, base + (size_t)(i0 + i) * rows * p.pv);
            }
    }
}

// ------------------------------------------------------------------------------------------------------------- host

struct NormTiling {
    int lanes;          // per pixel
    int sv, slices, rows, per, chunks;
};

static int norm_kind(int type, int C, uintptr_t addresses) {
    if (type == CPRUNE_TYPE_BF16) return 0;
    return C % 4 == 0 && (addresses & 15) == 0 ? 1 : 2;
}

// Chunks of about `target` vectors, in whole rounds of the block's threads; never more of them than fit a grid's second dimension
static NormTiling norm_tiling(int kind, int HW, int C) {
    NormTiling t;
    const int L = kind == 0 ? 8 : kind == 1 ? 4 : 1;
    t.lanes = kind == 0 ? cprune_padded_channels(C) : C;
    const int pv = t.lanes / L;
    t.slices = (pv + NORM_T - 1) / NORM_T;
    t.sv = (pv + t.slices - 1) / t.slices;
    t.slices = (pv + t.sv - 1) / t.sv;
    t.rows = NORM_T / t.sv;
    const int rounds = 8;
    t.per = t.rows * rounds;
    t.chunks = (HW + t.per - 1) / t.per;
    return t;
}

static size_t norm_part_bytes(int N, int HW, int C, int kind) {
    const NormTiling t = norm_tiling(kind, HW, C);
    return ((size_t)N * t.chunks * t.lanes * sizeof(float2) + 255) / 256 * 256;
}

static cprune_status norm_check(int type, int N, int H, int W, int C, int groups, int act) {
    if ((type != CPRUNE_TYPE_BF16 && type != CPRUNE_TYPE_F32) || N <= 0 || H <= 0 || W <= 0 || C <= 0 || groups <= 0 || C % groups) return CPRUNE_ERR_INVALID_ARG;
    if (act < CPRUNE_ACT_NONE || act > CPRUNE_ACT_SILU) return CPRUNE_ERR_INVALID_ARG;
    const long long hw = (long long)H * W;
    if (C > (1 << 20) || hw * (C + 16LL) > 0x7fffffffLL || N > 65535 || (long long)N * groups > 0x7fffffffLL) return CPRUNE_ERR_UNSUPPORTED;
    return CPRUNE_OK;
}

// Which of the kernels for one, eight or four channels a vector
template <typename F>
static cprune_status by_kind(int kind, F f) {
    switch (kind) {
        case 0: return f(std::integral_constant<int, 0>());
        case 1: return f(std::integral_constant<int, 1>());
        default: return f(std::integral_constant<int, 2>());
    }
}

static NormParams norm_params(int kind, int N, int H, int W, int C, int groups, int act) {
    NormParams p = {};
    p.N = N; p.HW = H * W; p.C = C; p.G = groups; p.cpg = C / groups; p.act = act;
    const NormTiling t = norm_tiling(kind, p.HW, C);
    p.pv = t.lanes / (kind == 0 ? 8 : kind == 1 ? 4 : 1);
    p.sv = t.sv; p.rows = t.rows; p.per = t.per; p.chunks = t.chunks;
    return p;
}

constexpr int NORM_TEAM_ENTRIES = 1024;      // a group of more chunk results than this is put together by a block, not by a warp

}  // namespace cprune

using namespace cprune;

extern "C" {

size_t cprune_group_norm_workspace_bytes(int type, int N, int H, int W, int C, int groups, int backward) {
    if (norm_check(type, N, H, W, C, groups, CPRUNE_ACT_NONE) != CPRUNE_OK) return 0;
    size_t most = 0;
    for (int kind = type == CPRUNE_TYPE_BF16 ? 0 : 1; kind <= (type == CPRUNE_TYPE_BF16 ? 0 : 2); ++kind) {
        if (kind == 1 && C % 4) continue;
        const size_t b = norm_part_bytes(N, H * W, C, kind);
        most = b > most ? b : most;
    }
    return most + (backward ? ((size_t)N * groups * sizeof(float2) + 255) / 256 * 256 : 0);
}

cprune_status cprune_group_norm(const void *x, int type, int N, int H, int W, int C, int groups, const float *gamma, const float *beta, float eps, int act,
                                const void *residual, void *y, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    if (!x || !y || !stats || !(eps > 0.f) || isinf(eps)) return CPRUNE_ERR_INVALID_ARG;
    cprune_status s = norm_check(type, N, H, W, C, groups, act);
    if (s != CPRUNE_OK) return s;
    const uintptr_t tensors = (uintptr_t)x | (uintptr_t)y | (uintptr_t)residual;
    if (tensors & (type == CPRUNE_TYPE_BF16 ? 15 : 3) || ((uintptr_t)gamma | (uintptr_t)beta) & 3 || (uintptr_t)stats & 7 || (uintptr_t)workspace & 15) return CPRUNE_ERR_INVALID_ARG;
    const int kind = norm_kind(type, C, tensors);
    if (workspace_bytes < norm_part_bytes(N, H * W, C, kind) || !workspace) return CPRUNE_ERR_WORKSPACE_TOO_SMALL;
    NormParams p = norm_params(kind, N, H, W, C, groups, act);
    p.x = x; p.res = residual; p.out = y; p.gamma = gamma; p.beta = beta; p.stats = stats; p.eps = eps;
    p.part = (float2 *)workspace;
    const NormTiling t = norm_tiling(kind, p.HW, C);
    cudaStream_t st = (cudaStream_t)stream;
    return by_kind(kind, [&](auto k) -> cprune_status {
        constexpr int K = decltype(k)::value;
        const dim3 grid(t.chunks, t.slices, N);
        ChainScope chain;
        CPRUNE_CUDA_CHECK(launch_chained(norm_partial_kernel<K>, grid, dim3(NORM_T), 0, st, p));
        chain.follow();
        const long long ids = (long long)N * groups;
        if ((long long)t.chunks * p.cpg > NORM_TEAM_ENTRIES) CPRUNE_CUDA_CHECK(launch_chained(norm_combine_kernel<NORM_T>, dim3((unsigned)ids), dim3(NORM_T), 0, st, p, t.lanes));
        else CPRUNE_CUDA_CHECK(launch_chained(norm_combine_kernel<32>, dim3((unsigned)ceil_div(ids, NORM_T / 32)), dim3(NORM_T), 0, st, p, t.lanes));
        CPRUNE_CUDA_CHECK(launch_chained(norm_apply_kernel<K>, grid, dim3(NORM_T), 0, st, p));
        return CPRUNE_OK;
    });
}

cprune_status cprune_group_norm_backward(const void *dy, const void *x, int type, int N, int H, int W, int C, int groups, const float *stats, const float *gamma,
                                         const float *beta, int act, const void *residual, void *dx, float *dgamma, float *dbeta, void *dresidual, void *workspace,
                                         size_t workspace_bytes, void *stream) {
    if (!dy || !x || !stats || !dx || (dresidual && !residual)) return CPRUNE_ERR_INVALID_ARG;
    cprune_status s = norm_check(type, N, H, W, C, groups, act);
    if (s != CPRUNE_OK) return s;
    const uintptr_t tensors = (uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx | (uintptr_t)residual | (uintptr_t)dresidual;
    const uintptr_t floats = (uintptr_t)gamma | (uintptr_t)beta | (uintptr_t)dgamma | (uintptr_t)dbeta;
    if (tensors & (type == CPRUNE_TYPE_BF16 ? 15 : 3) || floats & 3 || (uintptr_t)stats & 7 || (uintptr_t)workspace & 15) return CPRUNE_ERR_INVALID_ARG;
    const int kind = norm_kind(type, C, tensors);
    const size_t part_bytes = norm_part_bytes(N, H * W, C, kind);
    if (workspace_bytes < part_bytes + (size_t)N * groups * sizeof(float2) || !workspace) return CPRUNE_ERR_WORKSPACE_TOO_SMALL;
    NormParams p = norm_params(kind, N, H, W, C, groups, act);
    p.x = x; p.dy = dy; p.res = residual; p.out = dx; p.dres = dresidual; p.gamma = gamma; p.beta = beta; p.stats = const_cast<float *>(stats);
    p.dgamma = dgamma; p.dbeta = dbeta;
    p.part = (float2 *)workspace;
    p.means = (float2 *)((char *)workspace + part_bytes);
    const NormTiling t = norm_tiling(kind, p.HW, C);
    cudaStream_t st = (cudaStream_t)stream;
    return by_kind(kind, [&](auto k) -> cprune_status {
        constexpr int K = decltype(k)::value;
        const dim3 grid(t.chunks, t.slices, N);
        ChainScope chain;
        CPRUNE_CUDA_CHECK(launch_chained(norm_grad_partial_kernel<K>, grid, dim3(NORM_T), 0, st, p));
        chain.follow();
        const long long ids = (long long)N * groups;
        if ((long long)t.chunks * p.cpg > NORM_TEAM_ENTRIES)
            CPRUNE_CUDA_CHECK(launch_chained(norm_grad_combine_kernel<NORM_T>, dim3((unsigned)ids), dim3(NORM_T), 0, st, p, t.lanes));
        else CPRUNE_CUDA_CHECK(launch_chained(norm_grad_combine_kernel<32>, dim3((unsigned)ceil_div(ids, NORM_T / 32)), dim3(NORM_T), 0, st, p, t.lanes));
        if (dgamma || dbeta) CPRUNE_CUDA_CHECK(launch_chained(norm_parameter_gradients_kernel, dim3((C + 31) / 32), dim3(NORM_T), 0, st, p, t.lanes));
        CPRUNE_CUDA_CHECK(launch_chained(norm_grad_apply_kernel<K>, grid, dim3(NORM_T), 0, st, p, t.lanes));
        return CPRUNE_OK;
    });
}

}  // extern "C"
