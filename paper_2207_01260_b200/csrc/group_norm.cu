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
//   - on chip (forward, what fits): one cluster of up to 16 blocks holds the groups of one image, or a range of them, in shared memory; its blocks
//     exchange their sums, and the data is read once.
//   - two passes, a launch each: partial results of chunks of pixels per channel; every block of the second launch puts those of its groups together for
//     itself, in the same order, and goes over the data again, last pixels first, so that part of it still comes from the cache.
// The variance is never a difference of large sums: a thread takes squares of differences from a value near its mean, in runs of a few dozen pixels, and means
// and deviations of threads, chunks and channels are put together pairwise (Chan, Golub, LeVeque 1979), in float32.
// What bounds it (us, with buffers that do not stay in the cache): small images the launch and the exchange, 1 x 7x7x352 4.6, 8 x 28x28x91 float32 6.4; large ones
// the two passes, whose loads, arithmetic and stores wait for one another, 64 x 112x112x44 38.6 (read once and written: 22 at a copy's rate); gradients instructions
// too, 64 x 56x56x108 with silu and a shortcut 66.5 (33), 8 x 14x14x180 7.1; few wide images the number of their blocks (see norm_tiling), 1 x 112x112x512 74 (3.9).
#include <cmath>
#include <mutex>
#include <type_traits>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace cprune {

// ------------------------------------------------------------------------------------------------ vectors of channels

// Two float32 in one register pair: additions and fused multiply-adds of such pairs are one instruction
using f2 = unsigned long long;
__device__ __forceinline__ f2 two(float lo, float hi) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 one_by_one(f2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// L channels of a vector as NP pairs (a single channel: with a zero)
template <int KIND> struct Lanes;       // 0: 8 bf16, 1: 4 float32, 2: one float32
template <> struct Lanes<0> {
    static constexpr int L = 8, NP = 4;
    using Raw = bf16x8;
    static __device__ __forceinline__ void unpack(const Raw &r, f2 *f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = two(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xffff0000u));
    }
    static __device__ __forceinline__ Raw pack(const float *f) { return pack8(f); }
};
template <> struct Lanes<1> {
    static constexpr int L = 4, NP = 2;
    using Raw = float4;
    static __device__ __forceinline__ void unpack(const Raw &r, f2 *f) { f[0] = two(r.x, r.y); f[1] = two(r.z, r.w); }
    static __device__ __forceinline__ Raw pack(const float *f) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Lanes<2> {
    static constexpr int L = 1, NP = 1;
    using Raw = float;
    static __device__ __forceinline__ void unpack(const Raw &r, f2 *f) { f[0] = two(r, 0.f); }
    static __device__ __forceinline__ Raw pack(const float *f) { return f[0]; }
};
template <int KIND>
__device__ __forceinline__ void unpack_floats(const typename Lanes<KIND>::Raw &r, float *f) {
    f2 v[Lanes<KIND>::NP];
    Lanes<KIND>::unpack(r, v);
#pragma unroll
    for (int l = 0; l < Lanes<KIND>::L; ++l) f[l] = l % 2 ? one_by_one(v[l / 2]).y : one_by_one(v[l / 2]).x;
}

constexpr int L_of(int kind) { return kind == 0 ? 8 : kind == 1 ? 4 : 1; }

struct NormParams {
    const void *x, *dy, *res;
    void *out, *dres;                   // y, or dx and dresidual
    const float *gamma, *beta;
    float *stats;                       // [N][G][2]: mean, rstd
    float2 *part;                       // partial results of chunks of pixels, [N][chunks][lanes]
    float *dgamma, *dbeta;
    int N, HW, C, G, cpg;
    int pv;                             // vectors per pixel
    int sv;                             // columns (vectors) of a block's slice; slices of the last range may reach beyond pv
    int rows;                           // R: pixels that the block's threads hold side by side
    int per;                            // on chip: pixels of a rank
    int chunks;                         // two passes: blocks that share an image
    int gs, data_bytes;                 // on chip: groups of a slice, bytes of a tensor's share of a block
    int range, room, ring_bytes;        // two passes: groups that a slice touches at most, channels of these or of the slice (both even), bytes of the ring
    float eps;
};

__device__ __forceinline__ float sigmoid(float z) {
    float e, r;
    asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}

// The activation of a vector, and its form in memory.  relu and relu6 keep a NaN (apply_act's maximum would drop it); 0 and 6 are bf16 values, so that a
// bf16 result is clamped after its rounding, two at a time.
template <int KIND, int ACT>
__device__ __forceinline__ typename Lanes<KIND>::Raw finish(const f2 *z) {
    constexpr int NP = Lanes<KIND>::NP;
    float f[2 * NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const float2 v = one_by_one(z[i]);
        f[2 * i] = v.x;
        f[2 * i + 1] = v.y;
    }
    if (ACT == CPRUNE_ACT_SILU) {
#pragma unroll
        for (int l = 0; l < 2 * NP; ++l) f[l] *= sigmoid(f[l]);
    }
    if (KIND != 0 && (ACT == CPRUNE_ACT_RELU || ACT == CPRUNE_ACT_RELU6)) {
#pragma unroll
        for (int l = 0; l < 2 * NP; ++l) {
            asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(f[l]));
            if (ACT == CPRUNE_ACT_RELU6) asm("min.NaN.f32 %0, %0, 0f40C00000;" : "+f"(f[l]));
        }
    }
    typename Lanes<KIND>::Raw r = Lanes<KIND>::pack(f);
    if constexpr (KIND == 0 && (ACT == CPRUNE_ACT_RELU || ACT == CPRUNE_ACT_RELU6)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(r.w[i]) : "r"(0u));
            if (ACT == CPRUNE_ACT_RELU6) asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(r.w[i]) : "r"(0x40C040C0u));
        }
    }
    return r;
}

// What a thread needs of the channels of its column: z = (x - mean) a + beta with a = rstd gamma.  (x - mean is taken first: multiplied out, a mean far
// from zero would cancel.)  Lanes behind the last channel have zeros everywhere.
template <int NP> struct Column {
    f2 minus_mean[NP], a[NP], beta[NP];
    float most;                         // the largest |beta|
};

// f(l) -> (-mean, rstd gamma, beta) of lane l of the column
template <int KIND, typename F>
__device__ __forceinline__ void fill_column(Column<Lanes<KIND>::NP> &k, F of) {
    constexpr int L = Lanes<KIND>::L;
    float3 v[2 * Lanes<KIND>::NP];
    k.most = 0.f;
#pragma unroll
    for (int l = 0; l < 2 * Lanes<KIND>::NP; ++l) {
        v[l] = l < L ? of(l) : make_float3(0.f, 0.f, 0.f);
        k.most = fmaxf(k.most, fabsf(v[l].z));
    }
#pragma unroll
    for (int i = 0; i < Lanes<KIND>::NP; ++i) {
        k.minus_mean[i] = two(v[2 * i].x, v[2 * i + 1].x);
        k.a[i] = two(v[2 * i].y, v[2 * i + 1].y);
        k.beta[i] = two(v[2 * i].z, v[2 * i + 1].z);
    }
}

// x - mean, and z
template <int KIND, bool RES>
__device__ __forceinline__ void affine(const Column<Lanes<KIND>::NP> &k, const typename Lanes<KIND>::Raw &x, const typename Lanes<KIND>::Raw &res, f2 *d, f2 *z) {
    constexpr int NP = Lanes<KIND>::NP;
    Lanes<KIND>::unpack(x, d);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        d[i] = add2(d[i], k.minus_mean[i]);
        z[i] = fma2(d[i], k.a[i], k.beta[i]);
    }
    if (RES) {
        f2 r[NP];
        Lanes<KIND>::unpack(res, r);
#pragma unroll
        for (int i = 0; i < NP; ++i) z[i] = add2(z[i], r[i]);
    }
}

template <int KIND, int ACT, bool RES>
__device__ __forceinline__ void apply_one(const NormParams &p, const Column<Lanes<KIND>::NP> &k, const typename Lanes<KIND>::Raw &x, const typename Lanes<KIND>::Raw &res, size_t at) {
    f2 d[Lanes<KIND>::NP], z[Lanes<KIND>::NP];
    affine<KIND, RES>(k, x, res, d, z);
    ((typename Lanes<KIND>::Raw *)p.out)[at] = finish<KIND, ACT>(z);
}

// The side of relu's and relu6's borders on which z lies decides about a whole gradient, so next to a border z is taken in 64 bits: a bit
// for each lane of the vector that is inside the borders, from what its z is made of.
template <int KIND>
__device__ __forceinline__ float lane_of(const typename Lanes<KIND>::Raw *v, int l) {
    if constexpr (KIND == 0) return __bfloat162float(((const __nv_bfloat16 *)v)[l]);
    else return ((const float *)v)[l];
}
template <int KIND, int ACT, bool RES>
__device__ __forceinline__ uint32_t inside_64(const NormParams &p, const typename Lanes<KIND>::Raw *x, const typename Lanes<KIND>::Raw *res, int n, int c0) {
    uint32_t inside = 0;
#pragma unroll 1
    for (int l = 0; l < Lanes<KIND>::L && c0 + l < p.C; ++l) {
        const float2 s = __ldcg((const float2 *)p.stats + (size_t)n * p.G + (c0 + l) / p.cpg);
        double z = ((double)lane_of<KIND>(x, l) - (double)s.x) * (double)s.y;
        if (p.gamma) z *= __ldg(p.gamma + c0 + l);
        if (p.beta) z += __ldg(p.beta + c0 + l);
        if (RES) z += lane_of<KIND>(res, l);
        if (z > 0.0 && (ACT != CPRUNE_ACT_RELU6 || z < 6.0)) inside |= 1u << l;
    }
    return inside;
}

// x - mean and dz of a vector of image n (x_at, res_at: where it lies)
template <int KIND, int ACT, bool RES>
__device__ __forceinline__ void gradient_one(const NormParams &p, const Column<Lanes<KIND>::NP> &k, int n, int c0, const typename Lanes<KIND>::Raw &x,
                                             const typename Lanes<KIND>::Raw &dy, const typename Lanes<KIND>::Raw &res, const typename Lanes<KIND>::Raw *x_at,
                                             const typename Lanes<KIND>::Raw *res_at, f2 *d, f2 *dz) {
    constexpr int NP = Lanes<KIND>::NP, L = Lanes<KIND>::L;
    f2 z[NP];
    affine<KIND, RES>(k, x, res, d, z);
    Lanes<KIND>::unpack(dy, dz);
    if constexpr (ACT != CPRUNE_ACT_NONE) {
        float f[2 * NP], g[2 * NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const float2 v = one_by_one(z[i]), w = one_by_one(dz[i]);
            f[2 * i] = v.x; f[2 * i + 1] = v.y;
            g[2 * i] = w.x; g[2 * i + 1] = w.y;
        }
        if (ACT == CPRUNE_ACT_SILU) {
#pragma unroll
            for (int l = 0; l < L; ++l) {
                const float s = sigmoid(f[l]), t = s * f[l];
                g[l] *= fmaf(t, 1.f - s, s);
            }
        } else {
            // Where z is next to 0, |(x - mean) a| is next to |beta + residual|; it is off by two roundings of 2^-24, the sums by one each
            float r[2 * NP];
            if (RES) unpack_floats<KIND>(res, r);
            const float near = 4e-7f * k.most, top = 6.f;
            bool close = false;
#pragma unroll
            for (int l = 0; l < L; ++l) {
                const float e = RES ? fmaf(4e-7f, fabsf(r[l]), near) : near;
                close |= fabsf(f[l]) < e || (ACT == CPRUNE_ACT_RELU6 && fabsf(f[l] - top) < e + 2.4e-6f);
            }
            if (close) {
                const uint32_t inside = inside_64<KIND, ACT, RES>(p, x_at, res_at, n, c0);
#pragma unroll
                for (int l = 0; l < L; ++l) f[l] = inside >> l & 1 ? 1.f : -1.f;
            }
#pragma unroll
            for (int l = 0; l < L; ++l) g[l] = f[l] > 0.f && (ACT != CPRUNE_ACT_RELU6 || f[l] < top) ? g[l] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) dz[i] = two(g[2 * i], g[2 * i + 1]);
    }
}

// dx = a dz + c0 + c1 (x - mean),  c0 = -rstd m1, c1 = -rstd^2 m2
template <int KIND>
__device__ __forceinline__ void store_gradient(const NormParams &p, const Column<Lanes<KIND>::NP> &k, const f2 *k0, const f2 *k1, const f2 *d, const f2 *dz, size_t at) {
    constexpr int NP = Lanes<KIND>::NP;
    float f[2 * NP], g[2 * NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const float2 v = one_by_one(fma2(k.a[i], dz[i], fma2(d[i], k1[i], k0[i]))), w = one_by_one(dz[i]);
        f[2 * i] = v.x; f[2 * i + 1] = v.y;
        g[2 * i] = w.x; g[2 * i + 1] = w.y;
    }
    ((typename Lanes<KIND>::Raw *)p.out)[at] = Lanes<KIND>::pack(f);
    if (p.dres) ((typename Lanes<KIND>::Raw *)p.dres)[at] = Lanes<KIND>::pack(g);
}

// f(l) -> (-rstd m1, -rstd^2 m2) of lane l of the column
template <int KIND, typename F>
__device__ __forceinline__ void fill_means(f2 *k0, f2 *k1, F of) {
    constexpr int NP = Lanes<KIND>::NP;
    float2 v[2 * NP];
#pragma unroll
    for (int l = 0; l < 2 * NP; ++l) v[l] = l < Lanes<KIND>::L ? of(l) : make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NP; ++i) { k0[i] = two(v[2 * i].x, v[2 * i + 1].x); k1[i] = two(v[2 * i].y, v[2 * i + 1].y); }
}

// ---------------------------------------------------------------------------------------------------- sums of a block

constexpr int NORM_T = 256;
constexpr int NORM_PITCH = NORM_T + 4;  // floats between the rows of sums per thread, one row per lane: neighbouring lanes in different banks
constexpr int NORM_AHEAD = 4;           // vectors of a thread in flight

// 1 / n, to one unit in the last place
__device__ __forceinline__ float inverse(int n) {
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"((float)n));
    return r;
}

// 2^k threads share a lane of channels when sums over the R rows of a block are taken
__device__ __forceinline__ int sharers_log2(int lanes) { return lanes > NORM_T ? 0 : min(5, 31 - __clz(NORM_T / lanes)); }
__device__ __forceinline__ float sum_sharers(float s, int log2) {
#pragma unroll
    for (int k = 0; k < 5; ++k)
        if (k < log2) s += __shfl_xor_sync(0xffffffffu, s, 1 << k);
    return s;
}

// A sums over the rows: v[(a L + lane % L) PITCH + thread], handed to done(lane, sums)
template <int L, int A, typename F>
__device__ __forceinline__ void sum_rows(const float *v, int sv, int rows, F done) {
    const int lanes = sv * L, log2 = sharers_log2(lanes), sub = 1 << log2, sl = threadIdx.x & (sub - 1);
    for (int q0 = 0; q0 < lanes; q0 += NORM_T >> log2) {
        const int q = q0 + (threadIdx.x >> log2);
        float s[A];
#pragma unroll
        for (int a = 0; a < A; ++a) s[a] = 0.f;
        const float *w = v + q % L * NORM_PITCH + q / L;
        if (q < lanes)
#pragma unroll 4
            for (int r = sl; r < rows; r += sub)
#pragma unroll
                for (int a = 0; a < A; ++a) s[a] += w[a * L * NORM_PITCH + r * sv];
#pragma unroll
        for (int a = 0; a < A; ++a) s[a] = sum_sharers(s[a], log2);
        if (q < lanes && sl == 0) done(q, s);
    }
}

// Means and squared deviations of the rows' values put together per lane: v holds every thread's mean and its deviations from it over its `few`, or one more, of
// the n pixels.  A sum divided by its number is off by two units of the mean, here and below, so the mean of the differences from it is added, and taken out of
// their squares: equal means stay what they are.  (Without, the variance of two flat channels 1 % apart was off by 2e-5, of equal ones by the square of those units.)
template <int L, typename F>
__device__ __forceinline__ void combine_rows(const float *v, int sv, int rows, int n, int few, F done) {
    const int lanes = sv * L, log2 = sharers_log2(lanes), sub = 1 << log2, sl = threadIdx.x & (sub - 1);
    const int more = n - few * rows;                           // rows below `more` have few + 1 pixels
    const float inv = n > 0 ? inverse(n) : 0.f, count_few = (float)few, count_more = (float)(few + 1);
    const int used = few > 0 ? rows : more;
    for (int q0 = 0; q0 < lanes; q0 += NORM_T >> log2) {
        const int q = q0 + (threadIdx.x >> log2);
        const float *w = v + q % L * NORM_PITCH + q / L;
        float s = 0.f, m2 = 0.f;
        if (q < lanes)
#pragma unroll 4
            for (int r = sl; r < used; r += sub) s += w[r * sv] * (r < more ? count_more : count_few);
        const float about = sum_sharers(s, log2) * inv;
        s = 0.f;
        if (q < lanes)
#pragma unroll 4
            for (int r = sl; r < used; r += sub) {
                const float d = w[r * sv] - about, e = d * (r < more ? count_more : count_few);
                s += e;
                m2 += w[L * NORM_PITCH + r * sv] + d * e;
            }
        s = sum_sharers(s, log2);
        m2 = sum_sharers(m2, log2);
        if (q < lanes && sl == 0) done(q, fmaf(s, inv, about), m2 - s * (s * inv));
    }
}

// A thread's sum and squared deviations, value by value, as differences from a shift that is worth n D^2 in the squares if it lies D from the mean of n values.
// For few values (on chip: 12 at most) the first will do: it has itself D^2 of the deviations and leaves D^2 / (n - 1) to the others, so that n D^2 is at most n - 1
// times what is wanted.
template <int NP> struct Spread {
    f2 minus_shift[NP], s[NP], q[NP];
    __device__ __forceinline__ void begin(const f2 *first) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            minus_shift[i] = two(-one_by_one(first[i]).x, -one_by_one(first[i]).y);
            s[i] = q[i] = 0ull;
        }
    }
    __device__ __forceinline__ void add(const f2 *f) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const f2 d = add2(f[i], minus_shift[i]);
            s[i] = add2(s[i], d);
            q[i] = fma2(d, d, q[i]);
        }
    }
    // means of n values and deviations from them, per lane
    template <int L> __device__ __forceinline__ void store(float *v, int n) const {
        const float inv = n > 0 ? inverse(n) : 0.f;
#pragma unroll
        for (int l = 0; l < L; ++l) {
            const float2 k = one_by_one(minus_shift[l / 2]), a = one_by_one(s[l / 2]), b = one_by_one(q[l / 2]);
            const float shift = l % 2 ? k.y : k.x, sum = l % 2 ? a.y : a.x, square = l % 2 ? b.y : b.x;
            const float dev = square - sum * (sum * inv);
            v[l * NORM_PITCH + threadIdx.x] = n > 0 ? fmaf(sum, inv, -shift) : 0.f;
            v[(L + l) * NORM_PITCH + threadIdx.x] = n > 0 ? (dev < 0.f ? 0.f : dev) : 0.f;         // (a NaN stays one: no maximum)
        }
    }
};

// The same of any number of values, in runs: at the end of one, its squares are taken from the mean of all values so far, which becomes the shift of the next, and
// added to those of the runs before.  The mean of the first four is where it begins (of a single run, the first): with the first of 1568 values as the only shift,
// and that one far from a flat rest (1 x 112x112x1280, a group per channel), 1 / sqrt(variance) was off by 4.5e-3.  A run's squares are then at most twice what
// they add to the deviations (the first run's three times), and runs of about the root of n keep the additions in a row few.
template <int NP> struct LongSpread : Spread<NP> {
    using Spread<NP>::minus_shift;
    using Spread<NP>::s;
    using Spread<NP>::q;
    f2 total[NP];
    // f: the values, n of them (four at most)
    __device__ __forceinline__ void begin(const f2 (*f)[NP], int n) {
        const float part = n > 0 ? -inverse(n) : 0.f;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            f2 sum = f[0][i];
#pragma unroll
            for (int k = 1; k < 4; ++k) sum = add2(sum, f[k][i]);
            minus_shift[i] = fma2(sum, two(part, part), 0ull);
            s[i] = q[i] = total[i] = 0ull;
        }
    }
    // n: values so far
    __device__ __forceinline__ void close(int n) {
        const float inv = -inverse(n);
        const f2 part = two(inv, inv), minus_one = two(-1.f, -1.f), count = two((float)n, (float)n);
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const f2 to = fma2(s[i], part, minus_shift[i]);
            const f2 by = fma2(minus_shift[i], minus_one, to);         // minus the way that the shift goes
            const f2 rest = fma2(count, by, s[i]);                     // the sum of the differences from the new one
            total[i] = add2(total[i], fma2(by, add2(s[i], rest), q[i]));
            minus_shift[i] = to;
            s[i] = rest;
            q[i] = 0ull;
        }
    }
    template <int L> __device__ __forceinline__ void store(float *v, int n) {
#pragma unroll
        for (int i = 0; i < NP; ++i) q[i] = add2(q[i], total[i]);
        Spread<NP>::template store<L>(v, n);
    }
};

__device__ __forceinline__ float sum16(float s) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}
// f(group, thread of its team, team, log2 of it) for `sg` groups (and for numbers behind the last: whole warps go round); 16 or 32 threads a group
template <typename F>
__device__ __forceinline__ void by_group(int sg, int entries, F f) {
    const int log2 = entries <= 16 ? 4 : 5, team = 1 << log2;
    for (int g0 = 0; g0 < sg; g0 += NORM_T >> log2) f(g0 + (int)(threadIdx.x >> log2), (int)(threadIdx.x & (team - 1)), team, log2);
}

// ------------------------------------------------------------------------------------------------------- two passes

// Asynchronous copies of 16 (or 4) bytes into the thread's own places of shared memory: nothing but the thread's own wait orders them
template <typename Raw>
__device__ __forceinline__ void copy_in(Raw *dst, const Raw *src) {
    if constexpr (sizeof(Raw) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// pixels of a thread under way: 48 to 60 KB a block
__host__ __device__ constexpr int ring_of(int tensors) { return tensors == 1 ? 12 : tensors == 2 ? 6 : 5; }

// Chunk k of an image: every chunks-th round of the block's rows, from the k-th on (blocks of an image read neighbouring rows at the same time).  The first
// `last` chunks have a round more, chunk `last` the rows that fill none.
struct Rounds {
    int few, last, rest, rows;
    __device__ __forceinline__ Rounds(const NormParams &p) : rows(p.rows) {
        const int rounds = p.HW / p.rows;
        few = rounds / p.chunks;
        last = rounds - few * p.chunks;
        rest = p.HW - rounds * p.rows;
    }
    __device__ __forceinline__ int full(int k) const { return few + (k < last); }
    __device__ __forceinline__ int pixels(int k) const { return full(k) * rows + (k == last ? rest : 0); }
};

// The pixels and columns of a block
struct Chunk {
    int v0, sv, rows, r, col, n, few, cnt;
    size_t base, step;
    __device__ __forceinline__ Chunk(const NormParams &p) {
        v0 = blockIdx.y * p.sv;
        sv = min(p.sv, p.pv - v0);
        rows = p.rows;
        r = threadIdx.x / sv;
        col = threadIdx.x - r * sv;
        const Rounds rounds(p);
        few = rounds.full(blockIdx.x);
        n = rounds.pixels(blockIdx.x);
        cnt = r < rows ? few + (r < n - few * rows) : 0;
        base = ((size_t)blockIdx.z * p.HW + blockIdx.x * rows + r) * p.pv + v0 + col;
        step = (size_t)p.chunks * rows * p.pv;
    }
    __device__ __forceinline__ size_t at(int i) const { return base + i * step; }
};

// A thread's pixels of T tensors, first to last or last to first, through a ring in shared memory.  (What bounded these loops was their own bookkeeping, 75 of
// 110 instructions a vector, as long as places in the ring and addresses were worked out pixel by pixel: 64 x 112x112x44 42 us, now 38 us.)
template <typename Raw, int T, bool BACK> struct Stream {
    static constexpr int RING = ring_of(T);
    Raw *ring;
    const Raw *from[T];                 // of the next pixel to ask for
    int cnt, left;                      // pixels in all, still to be asked for
    long long step;                     // vectors from one pixel to the next
    size_t at;                          // the first pixel of all
    __device__ __forceinline__ Stream(void *smem, const Chunk &c, const void *a, const void *b = nullptr, const void *d = nullptr) : ring((Raw *)smem + threadIdx.x), cnt(c.cnt), left(c.cnt) {
        at = BACK ? c.at(c.cnt > 0 ? c.cnt - 1 : 0) : c.at(0);
        step = BACK ? -(long long)c.step : (long long)c.step;
        from[0] = (const Raw *)a + at;
        if (T > 1) from[T > 1 ? 1 : 0] = (const Raw *)b + at;
        if (T > 2) from[T > 2 ? 2 : 0] = (const Raw *)d + at;
    }
    __device__ __forceinline__ void issue(int place) {
        if (left > 0) {
#pragma unroll
            for (int k = 0; k < T; ++k) {
                copy_in(ring + (place * T + k) * NORM_T, from[k]);
                from[k] += step;
            }
            --left;
        }
        copy_commit();
    }
    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int i = 0; i < RING - 1; ++i) issue(i);
    }
    // f(where the pixel lies, places of its vectors, NORM_T apart); close(pixels so far) between runs of them: the first has `first` rounds of the ring, the others
    // as many as are next to the root of the number of pixels, and `first` at least
    template <typename F, typename G> __device__ __forceinline__ void run(F f, int first, G close) {
        const int rounds = max(first, __float2int_rn(sqrtf((float)cnt) * (1.f / RING)));
        int run = first;
#pragma unroll 1
        for (int i = cnt; i > 0; i -= RING) {
#pragma unroll
            for (int j = 0; j < RING; ++j) {
                if (j >= i) break;
                copy_wait_but<RING - 2>();
                f(at, ring + j * T * NORM_T);
                at += step;
                issue((j + RING - 1) % RING);
            }
            if (--run == 0 && i > RING) {
                close(cnt - i + RING);
                run = rounds;
            }
        }
        copy_wait();
    }
    template <typename F> __device__ __forceinline__ void run(F f) {
        run(f, 1, [](int) {});
    }
};

// Mean and squared deviations of a chunk of pixels, channel by channel
template <int KIND>
__global__ void __launch_bounds__(NORM_T, 4) norm_partial_kernel(const __grid_constant__ NormParams p) {
    constexpr int L = Lanes<KIND>::L, NP = Lanes<KIND>::NP;
    using Raw = typename Lanes<KIND>::Raw;
    extern __shared__ __align__(16) unsigned char norm_smem[];
    float *v = (float *)norm_smem;      // afterwards
    const Chunk c(p);
    pdl_wait();
    pdl_trigger();
    Stream<Raw, 1, false> x(norm_smem, c, p.x);
    x.begin();
    LongSpread<NP> own;
    {
        f2 f[4][NP];
        const int first = c.cnt > ring_of(1) ? 4 : min(c.cnt, 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) Lanes<KIND>::unpack(i < first ? ((const Raw *)p.x)[c.at(i)] : Raw(), f[i]);
        own.begin(f, first);
    }
    x.run(
        [&](size_t, const Raw *v) {
            f2 f[NP];
            Lanes<KIND>::unpack(*v, f);
            own.add(f);
        },
        1, [&](int n) { own.close(n); });
    __syncthreads();
    if (c.r < c.rows) own.template store<L>(v, c.cnt);
    __syncthreads();
    float2 *part = p.part + ((size_t)blockIdx.z * p.chunks + blockIdx.x) * p.pv * L + c.v0 * L;
    combine_rows<L>(v, c.sv, c.rows, c.n, c.few, [&](int q, float mean, float m2) { part[q] = make_float2(mean, m2); });
}

// The groups that a slice touches
struct GroupRange {
    int g0, n;
    __device__ __forceinline__ GroupRange(const NormParams &p, const Chunk &c, int L) {
        const int first = min(c.v0 * L, p.C - 1), last = min((c.v0 + c.sv) * L, p.C) - 1;
        g0 = first / p.cpg;
        n = max(first, last) / p.cpg - g0 + 1;
    }
};

// Chunks of a channel that a thread of the second pass reads, all at once (a channel has up to 32 threads)
constexpr int CHUNK_BATCH = 8;

// Where a channel's constants lie: lane by lane, so that threads of neighbouring columns read neighbouring ones
template <int L>
__device__ __forceinline__ int slot(int q, int sv) { return q % L * sv + q / L; }

template <int KIND, int ACT, bool RES>
__global__ void __launch_bounds__(NORM_T, 4) norm_apply_kernel(const __grid_constant__ NormParams p, int lanes) {
    constexpr int L = Lanes<KIND>::L, NP = Lanes<KIND>::NP, T = RES ? 2 : 1;
    using Raw = typename Lanes<KIND>::Raw;
    extern __shared__ __align__(16) unsigned char norm_smem[];
    const Chunk c(p);
    const GroupRange range(p, c, L);
    // backwards: what the first pass read last is still in the cache.  (x and the residual are not what the first pass writes.)
    Stream<Raw, T, true> x(norm_smem, c, p.x, p.res);
    x.begin();
    float2 *image = (float2 *)(norm_smem + (size_t)ring_of(T) * T * NORM_T * sizeof(Raw)), *channel = image + p.range;
    float4 *constants = (float4 *)(channel + p.room);
    for (int q = threadIdx.x; q < c.sv * L; q += NORM_T) {
        const int ch = c.v0 * L + q;
        constants[slot<L>(q, c.sv)] = ch < p.C ? make_float4(0.f, p.gamma ? __ldg(p.gamma + ch) : 1.f, p.beta ? __ldg(p.beta + ch) : 0.f, __int_as_float(ch / p.cpg - range.g0))
                                               : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    pdl_wait();
    pdl_trigger();
    // the chunks of every channel of the groups, all read at once
    const float inv_hw = inverse(p.HW), inv_cpg = inverse(p.cpg);
    {
        const Rounds rounds(p);
        const int n = range.n * p.cpg, log2 = sharers_log2(n), sub = 1 << log2, sl = threadIdx.x & (sub - 1);
        const float2 *part = p.part + (size_t)blockIdx.z * p.chunks * lanes + range.g0 * p.cpg;
        for (int q0 = 0; q0 < n; q0 += NORM_T >> log2) {
            const int q = q0 + (threadIdx.x >> log2);
            float2 w[CHUNK_BATCH];
            float pixels[CHUNK_BATCH], s = 0.f, m2 = 0.f;
#pragma unroll
            for (int i = 0; i < CHUNK_BATCH; ++i) {
                const int k = sl + (i << log2);
                pixels[i] = q < n && k < p.chunks ? (float)rounds.pixels(k) : 0.f;
                w[i] = q < n && k < p.chunks ? __ldcg(part + (size_t)k * lanes + q) : make_float2(0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < CHUNK_BATCH; ++i) s += w[i].x * pixels[i];
            const float about = sum_sharers(s, log2) * inv_hw;
            s = 0.f;
#pragma unroll
            for (int i = 0; i < CHUNK_BATCH; ++i) {
                const float d = pixels[i] > 0.f ? w[i].x - about : 0.f, e = d * pixels[i];         // (the square of a mean past 2^64, times no pixels, is no number)
                s += e;
                m2 += w[i].y + d * e;
            }
            s = sum_sharers(s, log2);
            m2 = sum_sharers(m2, log2);
            if (q < n && sl == 0) channel[q] = make_float2(fmaf(s, inv_hw, about), m2 - s * (s * inv_hw));
        }
    }
    __syncthreads();
    by_group(range.n, p.cpg, [&](int g, int i, int team, int log2) {
        const float2 *w = channel + g * p.cpg;
        float a = 0.f, b = 0.f, off = 0.f;
        if (g < range.n)
            for (int j = i; j < p.cpg; j += team) a += w[j].x;
        a = sum_sharers(a, log2) * inv_cpg;
        if (g < range.n)
            for (int j = i; j < p.cpg; j += team) {
                const float d = w[j].x - a;
                off += d;
                b += w[j].y + d * d * (float)p.HW;
            }
        off = sum_sharers(off, log2) * inv_cpg;
        b = fmaf(-off, off, sum_sharers(b, log2) * inv_hw * inv_cpg);
        a += off;
        b = b < 0.f ? 0.f : b;                                 // (a NaN stays one)
        if (g < range.n && i == 0) {
            const float2 result = make_float2(a, 1.f / sqrtf(b + p.eps));
            image[g] = result;
            // (a group of two slices is written by the one in which it begins)
            if (blockIdx.x == 0 && (range.g0 + g) * p.cpg >= c.v0 * L) ((float2 *)p.stats)[(size_t)blockIdx.z * p.G + range.g0 + g] = result;
        }
    });
    __syncthreads();
    for (int q = threadIdx.x; q < c.sv * L; q += NORM_T) {
        float4 &k = constants[slot<L>(q, c.sv)];               // (this thread's own)
        if (c.v0 * L + q < p.C) {
            const float2 w = image[__float_as_int(k.w)];
            k.x = -w.x;
            k.y *= w.y;
        }
    }
    __syncthreads();
    Column<NP> k;
    fill_column<KIND>(k, [&](int l) {
        const float4 w = constants[l * c.sv + c.col];
        return make_float3(w.x, w.y, w.z);
    });
    x.run([&](size_t at, const Raw *v) { apply_one<KIND, ACT, RES>(p, k, v[0], v[RES ? NORM_T : 0], at); });
}

// Sums of dz and dz (x - mean) of a thread.  RUNS: of many pixels, run by run; the sums of the runs before are kept in local memory, for which there are no
// registers left.  In a single run 784 equal values were off by 8e-6 of their sum, 1568 by 1.1e-5.  (us with / without, which is why few pixels do without:
// 64 x 56x56x108 silu and shortcut, 30 pixels a thread, 70.8 / 68.9; 64 x 112x112x44 relu, 50 of them, 71.7 / 70.0; the sums before in registers, with spills, 72.6
// and 73.7.)
constexpr int GRADIENT_RUN = 30, GRADIENT_SINGLE = 64;         // pixels: of a run at least, of a single one at most
template <int NP, bool RUNS> struct GradientSums {
    f2 a[NP], b[NP], *before;
    __device__ __forceinline__ explicit GradientSums(f2 (&place)[2 * NP]) : before(place) {
#pragma unroll
        for (int i = 0; i < NP; ++i) a[i] = b[i] = before[i] = before[NP + i] = 0ull;
        if (RUNS) asm volatile("" ::"l"(before) : "memory");   // (the address is out: the place stays in memory)
    }
    __device__ __forceinline__ void add(const f2 *d, const f2 *dz) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            a[i] = add2(a[i], dz[i]);
            b[i] = fma2(dz[i], d[i], b[i]);
        }
    }
    __device__ __forceinline__ void close() {
#pragma unroll
        for (int i = 0; RUNS && i < NP; ++i) {
            before[i] = add2(before[i], a[i]);
            before[NP + i] = add2(before[NP + i], b[i]);
            a[i] = b[i] = 0ull;
        }
    }
    template <int L> __device__ __forceinline__ void store(float *v) const {
#pragma unroll
        for (int l = 0; l < L; ++l) {
            const float2 s = one_by_one(RUNS ? add2(before[l / 2], a[l / 2]) : a[l / 2]), w = one_by_one(RUNS ? add2(before[NP + l / 2], b[l / 2]) : b[l / 2]);
            v[l * NORM_PITCH + threadIdx.x] = l % 2 ? s.y : s.x;
            v[(L + l) * NORM_PITCH + threadIdx.x] = l % 2 ? w.y : w.x;
        }
    }
};

// Constants of the slice's channels from global memory: -mean, rstd gamma, beta, rstd.  Lanes behind the last channel get z = 1, far from the borders of
// relu and relu6; everything else about them is 0.
template <int L>
__device__ __forceinline__ void fetch_constants(const NormParams &p, const Chunk &c, float4 *constants) {
    const float2 *stats = (const float2 *)p.stats + (size_t)blockIdx.z * p.G;
    for (int q = threadIdx.x; q < c.sv * L; q += NORM_T) {
        const int ch = c.v0 * L + q;
        float4 k = make_float4(0.f, 0.f, 1.f, 0.f);
        if (ch < p.C) {
            const float2 w = __ldcg(stats + ch / p.cpg);
            k = make_float4(-w.x, w.y * (p.gamma ? __ldg(p.gamma + ch) : 1.f), p.beta ? __ldg(p.beta + ch) : 0.f, w.y);
        }
        constants[slot<L>(q, c.sv)] = k;
    }
}

// Sums of dz and dz xhat over a chunk of pixels, channel by channel
template <int KIND, int ACT, bool RES, bool RUNS>
__global__ void __launch_bounds__(NORM_T, 3) norm_grad_partial_kernel(const __grid_constant__ NormParams p) {
    constexpr int L = Lanes<KIND>::L, NP = Lanes<KIND>::NP, T = RES ? 3 : 2;
    using Raw = typename Lanes<KIND>::Raw;
    extern __shared__ __align__(16) unsigned char norm_smem[];
    float *v = (float *)norm_smem;      // afterwards
    float4 *constants = (float4 *)(norm_smem + p.ring_bytes);
    const Chunk c(p);
    const int c0 = (c.v0 + c.col) * L;
    pdl_wait();
    pdl_trigger();
    Stream<Raw, T, false> x(norm_smem, c, p.x, p.dy, p.res);
    x.begin();
    fetch_constants<L>(p, c, constants);
    __syncthreads();
    f2 runs[2 * NP];
    GradientSums<NP, RUNS> sums(runs);
    Column<NP> k;
    fill_column<KIND>(k, [&](int l) {
        const float4 w = constants[l * c.sv + c.col];
        return make_float3(w.x, w.y, w.z);
    });
    x.run(
        [&](size_t, const Raw *v) {
            f2 d[NP], dz[NP];
            const Raw *res = v + (RES ? 2 * NORM_T : 0);
            gradient_one<KIND, ACT, RES>(p, k, blockIdx.z, c0, v[0], v[NORM_T], *res, v, res, d, dz);
            sums.add(d, dz);
        },
        GRADIENT_RUN / Stream<Raw, T, false>::RING, [&](int) { sums.close(); });
    __syncthreads();
    if (c.r < c.rows) sums.template store<L>(v);
    __syncthreads();
    float2 *part = p.part + ((size_t)blockIdx.z * p.chunks + blockIdx.x) * p.pv * L + c.v0 * L;
    sum_rows<L, 2>(v, c.sv, c.rows, [&](int q, const float *s) { part[q] = make_float2(s[0], s[1] * constants[slot<L>(q, c.sv)].w); });
}

// dgamma and dbeta of 32 channels: the partial sums of all images and chunks, eight at a time, in a fixed order; their total in 64 bits
__device__ __forceinline__ void parameter_gradients(const NormParams &p, int lanes, int block, double (*tot)[8][33]) {
    const int cl = threadIdx.x & 31, k = threadIdx.x >> 5, c = block * 32 + cl;
    double a = 0.0, b = 0.0;
    const long long entries = (long long)p.N * p.chunks;
    if (c < p.C)
        for (long long e0 = k; e0 < entries; e0 += 64) {
            float2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = e0 + 8 * i < entries ? __ldcg(p.part + (size_t)(e0 + 8 * i) * lanes + c) : make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) { a += v[i].x; b += v[i].y; }
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
    __syncthreads();
}
// The blocks of image N (grid z) take the parameters' gradients
template <int KIND, int ACT, bool RES>
__global__ void __launch_bounds__(NORM_T, 3) norm_grad_apply_kernel(const __grid_constant__ NormParams p, int lanes) {
    constexpr int L = Lanes<KIND>::L, NP = Lanes<KIND>::NP, T = RES ? 3 : 2;
    using Raw = typename Lanes<KIND>::Raw;
    extern __shared__ __align__(16) unsigned char norm_smem[];
    if (blockIdx.z == p.N) {
        pdl_wait();
        pdl_trigger();
        for (int b = blockIdx.y * gridDim.x + blockIdx.x; b * 32 < p.C; b += gridDim.x * gridDim.y) parameter_gradients(p, lanes, b, (double (*)[8][33])norm_smem);
        return;
    }
    const Chunk c(p);
    const GroupRange range(p, c, L);
    const int c0 = (c.v0 + c.col) * L;
    Stream<Raw, T, true> x(norm_smem, c, p.x, p.dy, p.res);
    x.begin();
    float2 *image = (float2 *)(norm_smem + p.ring_bytes), *channel = image + p.range;
    float4 *constants = (float4 *)(channel + p.room);
    fetch_constants<L>(p, c, constants);
    pdl_wait();
    pdl_trigger();
    {
        const int n = range.n * p.cpg, log2 = sharers_log2(n), sub = 1 << log2, sl = threadIdx.x & (sub - 1), first = range.g0 * p.cpg;
        const float2 *part = p.part + (size_t)blockIdx.z * p.chunks * lanes + first;
        for (int q0 = 0; q0 < n; q0 += NORM_T >> log2) {
            const int q = q0 + (threadIdx.x >> log2);
            const float gamma = p.gamma && q < n ? __ldg(p.gamma + first + q) : 1.f;
            float2 w[CHUNK_BATCH];
#pragma unroll
            for (int i = 0; i < CHUNK_BATCH; ++i) {
                const int k = sl + (i << log2);
                w[i] = q < n && k < p.chunks ? __ldcg(part + (size_t)k * lanes + q) : make_float2(0.f, 0.f);
            }
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < CHUNK_BATCH; ++i) { s1 += w[i].x; s2 += w[i].y; }
            s1 = sum_sharers(s1, log2);
            s2 = sum_sharers(s2, log2);
            if (q < n && sl == 0) channel[q] = make_float2(gamma * s1, gamma * s2);
        }
    }
    __syncthreads();
    by_group(range.n, p.cpg, [&](int g, int i, int team, int log2) {
        const float2 *w = channel + g * p.cpg;
        float s1 = 0.f, s2 = 0.f;
        if (g < range.n)
            for (int j = i; j < p.cpg; j += team) { s1 += w[j].x; s2 += w[j].y; }
        const float inv = 1.f / ((float)p.HW * (float)p.cpg);
        s1 = sum_sharers(s1, log2) * inv;
        s2 = sum_sharers(s2, log2) * inv;
        if (g < range.n && i == 0) image[g] = make_float2(s1, s2);
    });
    __syncthreads();
    float2 *means = channel;            // (their place: sv L of them at most, see the host)
    for (int q = threadIdx.x; q < c.sv * L; q += NORM_T) {
        const int ch = c.v0 * L + q;
        float2 w = make_float2(0.f, 0.f);
        if (ch < p.C) {
            const float2 m = image[ch / p.cpg - range.g0];
            const float rstd = constants[slot<L>(q, c.sv)].w;
            w = make_float2(-rstd * m.x, -rstd * rstd * m.y);
        }
        means[slot<L>(q, c.sv)] = w;
    }
    __syncthreads();
    Column<NP> k;
    f2 k0[NP], k1[NP];
    fill_column<KIND>(k, [&](int l) {
        const float4 w = constants[l * c.sv + c.col];
        return make_float3(w.x, w.y, w.z);
    });
    fill_means<KIND>(k0, k1, [&](int l) { return means[l * c.sv + c.col]; });
    x.run([&](size_t at, const Raw *v) {
        f2 d[NP], dz[NP];
        const Raw *res = v + (RES ? 2 * NORM_T : 0);
        gradient_one<KIND, ACT, RES>(p, k, blockIdx.z, c0, v[0], v[NORM_T], *res, v, res, d, dz);
        store_gradient<KIND>(p, k, k0, k1, d, dz, at);
    });
}

// ------------------------------------------------------------------------------------------------------- on chip

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// writes two floats into the shared memory of a block of the cluster, at the place that `own` has in this one's
__device__ __forceinline__ void push_float2(const float2 *own, int rank, float2 v) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(own)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}
// What a block works on: pixels p0 .. p0 + n of an image, columns v0 .. v0 + sv, groups g0 .. g0 + sg
struct Share {
    int v0, sv, g0, sg, p0, n, rows, r, col, few, cnt;
    size_t base, step;
    __device__ __forceinline__ Share(const NormParams &p, int L, int rank) {
        g0 = blockIdx.y * p.gs;
        sg = min(p.gs, p.G - g0);
        v0 = g0 * p.cpg / L;
        sv = (g0 + sg == p.G ? p.pv : (g0 + sg) * p.cpg / L) - v0;
        p0 = rank * p.per;
        n = max(0, min(p.per, p.HW - p0));
        rows = NORM_T / sv;
        r = threadIdx.x / sv;
        col = threadIdx.x - r * sv;
        few = n / rows;
        cnt = r < rows ? few + (r < n - few * rows) : 0;
        base = ((size_t)blockIdx.z * p.HW + p0 + r) * p.pv + v0 + col;
        step = (size_t)rows * p.pv;
    }
};

// f(group, pair) for the groups of the slice: 16 threads a group, thread i with what rank i sent (zeros from `ranks` on)
template <typename F>
__device__ __forceinline__ void over_ranks(const float2 *inbox, int gs, int sg, int ranks, F f) {
    const int q = threadIdx.x & 15;
    for (int g0 = 0; g0 < sg; g0 += NORM_T / 16) {           // (whole warps go round)
        const int g = g0 + threadIdx.x / 16;
        f(g, g < sg && q < ranks ? inbox[q * gs + g] : make_float2(0.f, 0.f));
    }
}

// Dynamic shared memory: the data ([pixel of a thread][thread] per tensor), sums per thread (afterwards: what a column needs of its channels), what every
// rank sends of its groups, the image's groups, results per channel, scale and shift.  What a channel needs is worked out once for all threads.
__host__ __device__ __forceinline__ size_t norm_sums_bytes(int L, int sv) { return 16 * (size_t)L * (sv > NORM_PITCH / 2 ? sv : NORM_PITCH / 2); }
struct NormSmem {
    unsigned char *data;
    float *v;
    float4 *constants;                  // over v: -mean, rstd gamma, beta
    float2 *inbox, *image, *channel, *affine;
    template <int L> __device__ __forceinline__ NormSmem(unsigned char *base, const NormParams &p, int tensors, std::integral_constant<int, L>) {
        data = base;
        v = (float *)(base + (size_t)p.data_bytes * tensors);
        constants = (float4 *)v;
        inbox = (float2 *)((char *)v + norm_sums_bytes(L, p.sv));
        image = inbox + p.gs * gridDim.x;
        channel = image + p.gs;
        affine = channel + p.sv * L;
    }
};

// scale and shift of the slice's channels: read early, needed late
template <int L>
__device__ __forceinline__ void fetch_affine(const NormParams &p, const Share &s, float2 *to) {
    for (int q = threadIdx.x; q < s.sv * L; q += NORM_T) {
        const int c = s.v0 * L + q;
        const bool in = c < p.C;
        to[q] = make_float2(in ? (p.gamma ? __ldg(p.gamma + c) : 1.f) : 0.f, in && p.beta ? __ldg(p.beta + c) : 0.f);
    }
}

template <int KIND, int ACT, bool RES>
__global__ void __launch_bounds__(NORM_T) norm_cluster_kernel(const __grid_constant__ NormParams p) {
    constexpr int L = Lanes<KIND>::L, NP = Lanes<KIND>::NP;
    using Raw = typename Lanes<KIND>::Raw;
    extern __shared__ __align__(16) unsigned char norm_smem[];
    const int ranks = gridDim.x, rank = (int)cluster_rank(), t = threadIdx.x;
    const Share s(p, L, rank);
    const NormSmem m(norm_smem, p, 1, std::integral_constant<int, L>());
    Raw *data = (Raw *)m.data;
    cluster_arrive();                                          // (waited for before the first write into another block)
    pdl_wait();
    pdl_trigger();
#pragma unroll 4
    for (int i = 0; i < s.cnt; ++i) copy_in(data + i * NORM_T + t, (const Raw *)p.x + s.base + i * s.step);
    fetch_affine<L>(p, s, m.affine);
    copy_wait();
    Spread<NP> own;
    if (s.cnt > 0) {
        f2 f[NP];
        Lanes<KIND>::unpack(data[t], f);
        own.begin(f);
    }
#pragma unroll 4
    for (int i = 1; i < s.cnt; ++i) {
        f2 f[NP];
        Lanes<KIND>::unpack(data[i * NORM_T + t], f);
        own.add(f);
    }
    if (s.r < s.rows) own.template store<L>(m.v, s.cnt);
    __syncthreads();
    combine_rows<L>(m.v, s.sv, s.rows, s.n, s.few, [&](int q, float mean, float m2) { m.channel[q] = make_float2(mean, m2); });
    __syncthreads();
    // channels to groups: 16 or 32 threads a group
    const float inv_cpg = inverse(p.cpg), inv_hw = inverse(p.HW);
    cluster_wait();
    by_group(s.sg, p.cpg, [&](int g, int i, int team, int log2) {
        const float2 *c = m.channel + (s.g0 + g) * p.cpg - s.v0 * L;
        float a = 0.f, b = 0.f, off = 0.f;
        if (g < s.sg)
            for (int j = i; j < p.cpg; j += team) a += c[j].x;
        a = sum_sharers(a, log2) * inv_cpg;
        if (g < s.sg)
            for (int j = i; j < p.cpg; j += team) {
                const float d = c[j].x - a;
                off += d;
                b += c[j].y + d * d * (float)s.n;
            }
        off = sum_sharers(off, log2);
        b = sum_sharers(b, log2) - off * (off * inv_cpg) * (float)s.n;
        a = fmaf(off, inv_cpg, a);
        if (g < s.sg && i < ranks) push_float2(m.inbox + rank * p.gs + g, i, make_float2(a, b));
    });
    cluster_arrive();
    cluster_wait();
    // the ranks' groups to the image's
    const float pixels = (float)max(0, min(p.per, p.HW - (t & 15) * p.per));
    over_ranks(m.inbox, p.gs, s.sg, ranks, [&](int g, float2 w) {
        const float about = sum16(w.x * pixels) * inv_hw, d = pixels > 0.f ? w.x - about : 0.f, e = d * pixels;
        const float off = sum16(e) * inv_hw, mean = about + off;
        const float v = fmaf(-off, off, sum16(w.y + d * e * (float)p.cpg) * inv_hw * inv_cpg);
        if (g < s.sg && (t & 15) == 0) {
            const float2 result = make_float2(mean, 1.f / sqrtf((v < 0.f ? 0.f : v) + p.eps));
            m.image[g] = result;
            if (rank == 0) ((float2 *)p.stats)[(size_t)blockIdx.z * p.G + s.g0 + g] = result;
        }
    });
    __syncthreads();
    for (int q = t; q < s.sv * L; q += NORM_T) {
        const float2 w = s.v0 * L + q < p.C ? m.image[(s.v0 * L + q) / p.cpg - s.g0] : make_float2(0.f, 0.f), k = m.affine[q];
        m.constants[slot<L>(q, s.sv)] = make_float4(-w.x, w.y * k.x, k.y, 0.f);
    }
    __syncthreads();
    if (s.cnt > 0) {
        Column<NP> k;
        fill_column<KIND>(k, [&](int l) {
            const float4 c = m.constants[l * s.sv + s.col];
            return make_float3(c.x, c.y, c.z);
        });
        for (int i0 = 0; i0 < s.cnt; i0 += NORM_AHEAD) {
            Raw raw[NORM_AHEAD], res[NORM_AHEAD];
#pragma unroll
            for (int i = 0; i < NORM_AHEAD; ++i)
                if (i0 + i < s.cnt) {
                    raw[i] = data[(i0 + i) * NORM_T + t];
                    if (RES) res[i] = ((const Raw *)p.res)[s.base + (i0 + i) * s.step];
                }
#pragma unroll
            for (int i = 0; i < NORM_AHEAD; ++i)
                if (i0 + i < s.cnt) apply_one<KIND, ACT, RES>(p, k, raw[i], res[i], s.base + (i0 + i) * s.step);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------- host

// How the on-chip kernel shares out an image; ranks == 0: it does not take it.  It takes what all fits at once, in two blocks to an SM of up to 12 pixels a thread.
// us there / in two passes:  1 x 7x7x352 4.5 / 6.7, 8 x 28x28x128 5.8 / 7.8, 8 x 56x56x64 7.7 / 10.2, 64 x 14x14x360 9.0 / 17.8, 256 x 7x7x352 9.4 / 16.1,
// 1 x 112x112x44 7.1 / 7.1;  with four blocks to an SM and 20 pixels 8 x 28x28x128 7.5, 8 x 56x56x64 9.0, 64 x 14x14x360 11.8.  (Before the means of means were
// corrected, which costs 0.1 us here and up to 0.3 there.)
struct NormCluster {
    int ranks = 0, gs = 0, slices = 0, per = 0, widest = 0;
    size_t data_bytes = 0, smem = 0;
};

constexpr size_t NORM_SMEM = 227 * 1024;
constexpr int NORM_ON_CHIP = 12;          // pixels of a thread

static NormCluster norm_cluster(int kind, int N, int HW, int C, int G) {
    NormCluster best;
    const int L = L_of(kind), pv = (kind == 0 ? cprune_padded_channels(C) : C) / L, cpg = C / G;
    int granule = 1;                       // groups that begin at a vector's boundary
    while ((long long)granule * cpg % L) ++granule;
    double least = 1e30;
    const int most = (G + granule - 1) / granule;
    for (int part = 1; part <= 16 && (part == 1 || part / 2 < most); part *= 2) {
        NormCluster c;
        c.gs = (most + part - 1) / part * granule;
        c.slices = (G + c.gs - 1) / c.gs;
        const int last = pv - (int)((long long)(c.slices - 1) * c.gs * cpg / L), first = c.slices > 1 ? (int)((long long)c.gs * cpg / L) : last;
        c.widest = first > last ? first : last;
        if (c.widest > NORM_T) continue;
        const int rows = NORM_T / c.widest;
        for (c.ranks = 1; c.ranks <= 16; c.ranks *= 2) {
            c.per = (HW + c.ranks - 1) / c.ranks;
            const int pixels = (c.per + rows - 1) / rows;
            const long long blocks = (long long)N * c.slices * c.ranks;
            if (blocks > 2 * 148 && pixels <= NORM_ON_CHIP) break;
            if (pixels > NORM_ON_CHIP || blocks > 2 * 148) continue;
            c.data_bytes = (size_t)pixels * NORM_T * (kind == 2 ? 4 : 16);
            c.smem = c.data_bytes + norm_sums_bytes(L, c.widest) + (size_t)c.gs * 8 * (c.ranks + 1) + (size_t)c.widest * L * 16;
            const double cost = pixels * (1.0 + blocks / 592.0) + 0.05 * c.ranks;
            if (c.smem <= NORM_SMEM / 2 - 1024 && cost < least) {
                least = cost;
                best = c;
            }
        }
    }
    return best;
}

// The limits of a kernel are attributes of a device
template <auto KERNEL>
static cprune_status make_ready(bool cluster) {
    static std::mutex mu;
    static bool ready[64] = {false};
    int dev = 0;
    CPRUNE_CUDA_CHECK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return CPRUNE_ERR_UNSUPPORTED;
    std::lock_guard<std::mutex> lock(mu);
    if (ready[dev]) return CPRUNE_OK;
    CPRUNE_CUDA_CHECK(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)NORM_SMEM));
    if (cluster) CPRUNE_CUDA_CHECK(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
    ready[dev] = true;
    return CPRUNE_OK;
}

// The ring is also the place of the sums
static int norm_ring_bytes(int kind, int tensors) {
    const int ring = ring_of(tensors) * tensors * NORM_T * (kind == 2 ? 4 : 16), sums = 2 * L_of(kind) * NORM_PITCH * 4;
    return ring > sums ? ring : sums;
}
// Behind it: results of the groups that a slice touches and of their channels (or, later, of its own), constants of its channels
static size_t norm_pass_bytes(const NormParams &p, int L) { return (size_t)p.range * 8 + (size_t)p.room * 8 + (size_t)p.sv * L * 16; }

template <auto KERNEL>
static cprune_status launch_pass(dim3 grid, size_t smem, cudaStream_t st, const NormParams &p, int lanes) {
    const cprune_status s = make_ready<KERNEL>(false);
    if (s != CPRUNE_OK) return s;
    if constexpr (std::is_invocable_v<decltype(KERNEL), NormParams, int>) CPRUNE_CUDA_CHECK(launch_chained(KERNEL, grid, dim3(NORM_T), smem, st, p, lanes));
    else CPRUNE_CUDA_CHECK(launch_chained(KERNEL, grid, dim3(NORM_T), smem, st, p));
    return CPRUNE_OK;
}

template <auto KERNEL>
static cprune_status launch_cluster(const NormCluster &c, int N, cudaStream_t st, const NormParams &p) {
    const cprune_status s = make_ready<KERNEL>(true);
    if (s != CPRUNE_OK) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(c.ranks, c.slices, N);
    cfg.blockDim = dim3(NORM_T);
    cfg.dynamicSmemBytes = c.smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = c.ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.numAttrs = 1;
    if (chain_launch_enabled()) {
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.numAttrs = 2;
    }
    CPRUNE_CUDA_CHECK(cudaLaunchKernelEx(&cfg, KERNEL, p));
    return CPRUNE_OK;
}

struct NormTiling {
    int lanes;          // per pixel
    int sv, slices, rows, chunks;
};

static int norm_kind(int type, int C, uintptr_t addresses) {
    if (type == CPRUNE_TYPE_BF16) return 0;
    return C % 4 == 0 && (addresses & 15) == 0 ? 1 : 2;
}

// Chunks of pixels: as many blocks as are resident at a time (four to an SM, the gradients' three), so that none waits for a second round, and at most as many
// an image as the threads of a block of the second pass read at once.  That is 8 where a slice touches more than 128 channels, so that few wide images leave most
// SMs without a block: us 1 x 112x112x512 74, its gradients 191; 1 x 112x112x1280 270 and 735; gradients of 8 x 56x56x256 28, of 8 x 28x28x512 18.5 (floors 3.9, 5.9,
// 9.8, 14.7, 5.9, 2.9)
static NormTiling norm_tiling(int kind, int N, int HW, int C, int G, bool backward) {
    NormTiling t;
    const int L = kind == 0 ? 8 : kind == 1 ? 4 : 1;
    t.lanes = kind == 0 ? cprune_padded_channels(C) : C;
    const int pv = t.lanes / L;
    t.slices = (pv + NORM_T - 1) / NORM_T;
    t.sv = (pv + t.slices - 1) / t.slices;
    t.slices = (pv + t.sv - 1) / t.sv;
    t.rows = NORM_T / t.sv;
    long long chunks = (backward ? 3 : 4) * 148 / ((long long)N * t.slices);
    const long long rounds = (HW + t.rows - 1) / t.rows, most = (rounds + 3) / 4;         // (four rounds of a block's threads at least)
    if (chunks > most) chunks = most;
    int readers = 1;                       // threads to a channel (of the groups that a slice touches)
    const int touched = (t.sv * L + C / G - 1) / (C / G) + 1, channels = (touched < G ? touched : G) * (C / G);
    while (readers < 32 && channels * readers * 2 <= NORM_T) readers *= 2;
    if (chunks > CHUNK_BATCH * readers) chunks = CHUNK_BATCH * readers;
    if (chunks < 1) chunks = 1;
    t.chunks = (int)chunks;
    return t;
}

static size_t norm_part_bytes(int N, int HW, int C, int G, int kind) {
    const NormTiling t = norm_tiling(kind, N, HW, C, G, false);          // (the most of the two)
    return ((size_t)N * t.chunks * t.lanes * sizeof(float2) + 255) / 256 * 256;
}

static size_t norm_bytes(int type, int N, int H, int W, int C) {
    return (size_t)N * H * W * (type == CPRUNE_TYPE_BF16 ? cprune_padded_channels(C) * sizeof(__nv_bfloat16) : C * sizeof(float));
}

constexpr int NORM_GROUP = 8192;          // channels of a group: the second pass holds two groups' results in shared memory

static cprune_status norm_check(int type, int N, int H, int W, int C, int groups, int act) {
    if ((type != CPRUNE_TYPE_BF16 && type != CPRUNE_TYPE_F32) || N <= 0 || H <= 0 || W <= 0 || C <= 0 || groups <= 0 || C % groups) return CPRUNE_ERR_INVALID_ARG;
    if (act < CPRUNE_ACT_NONE || act > CPRUNE_ACT_SILU) return CPRUNE_ERR_INVALID_ARG;
    const long long hw = (long long)H * W;
    if (C > (1 << 20) || C / groups > NORM_GROUP || hw * (C + 16LL) > 0x7fffffffLL || N > 65534 || (long long)N * groups > 0x7fffffffLL) return CPRUNE_ERR_UNSUPPORTED;
    return CPRUNE_OK;
}

// f(kind, activation, whether there is a residual), each as a constant
template <typename F>
static cprune_status by_kind(int kind, int act, bool residual, F f) {
    auto third = [&](auto k, auto a) -> cprune_status { return residual ? f(k, a, std::true_type()) : f(k, a, std::false_type()); };
    auto second = [&](auto k) -> cprune_status {
        switch (act) {
            case CPRUNE_ACT_RELU: return third(k, std::integral_constant<int, CPRUNE_ACT_RELU>());
            case CPRUNE_ACT_RELU6: return third(k, std::integral_constant<int, CPRUNE_ACT_RELU6>());
            case CPRUNE_ACT_SILU: return third(k, std::integral_constant<int, CPRUNE_ACT_SILU>());
            default: return third(k, std::integral_constant<int, CPRUNE_ACT_NONE>());
        }
    };
    return kind == 0 ? second(std::integral_constant<int, 0>()) : kind == 1 ? second(std::integral_constant<int, 1>()) : second(std::integral_constant<int, 2>());
}

static NormParams norm_params(int kind, int N, int H, int W, int C, int groups, bool backward) {
    NormParams p = {};
    p.N = N; p.HW = H * W; p.C = C; p.G = groups; p.cpg = C / groups;
    const NormTiling t = norm_tiling(kind, N, p.HW, C, groups, backward);
    p.pv = t.lanes / (kind == 0 ? 8 : kind == 1 ? 4 : 1);
    p.sv = t.sv; p.rows = t.rows; p.chunks = t.chunks;
    const int touched = (t.sv * L_of(kind) + p.cpg - 1) / p.cpg + 1;
    p.range = round_up(touched < groups ? touched : groups, 2);             // (what lies behind stays on 16 bytes)
    const int channels = (touched < groups ? touched : groups) * p.cpg, own = t.sv * L_of(kind);
    p.room = round_up(channels > own ? channels : own, 2);
    return p;
}

}  // namespace cprune

using namespace cprune;

extern "C" {

size_t cprune_group_norm_workspace_bytes(int type, int N, int H, int W, int C, int groups, int backward) {
    if (norm_check(type, N, H, W, C, groups, CPRUNE_ACT_NONE) != CPRUNE_OK) return 0;
    size_t most = 0;
    for (int kind = type == CPRUNE_TYPE_BF16 ? 0 : 1; kind <= (type == CPRUNE_TYPE_BF16 ? 0 : 2); ++kind) {
        if (kind == 1 && C % 4) continue;
        if (!backward && norm_cluster(kind, N, H * W, C, groups).ranks) continue;
        const size_t b = norm_part_bytes(N, H * W, C, groups, kind);
        most = b > most ? b : most;
    }
    return most;
}

cprune_status cprune_group_norm(const void *x, int type, int N, int H, int W, int C, int groups, const float *gamma, const float *beta, float eps, int act,
                                const void *residual, void *y, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    if (!x || !y || !stats || !(eps > 0.f) || isinf(eps)) return CPRUNE_ERR_INVALID_ARG;
    cprune_status s = norm_check(type, N, H, W, C, groups, act);
    if (s != CPRUNE_OK) return s;
    const uintptr_t tensors = (uintptr_t)x | (uintptr_t)y | (uintptr_t)residual;
    if (tensors & (type == CPRUNE_TYPE_BF16 ? 15 : 3) || ((uintptr_t)gamma | (uintptr_t)beta) & 3 || (uintptr_t)stats & 7 || (uintptr_t)workspace & 15) return CPRUNE_ERR_INVALID_ARG;
    const int kind = norm_kind(type, C, tensors);
    const NormCluster c = norm_cluster(kind, N, H * W, C, groups);
    if (!c.ranks && (workspace_bytes < norm_part_bytes(N, H * W, C, groups, kind) || !workspace)) return CPRUNE_ERR_WORKSPACE_TOO_SMALL;
    const size_t bytes = norm_bytes(type, N, H, W, C), channels = (size_t)C * 4;
    const Buffer bx{x, bytes}, br{residual, bytes}, by{y, bytes}, bg{gamma, channels}, bb{beta, channels}, bs{stats, (size_t)N * groups * 8};
    const Buffer bw{c.ranks ? nullptr : workspace, norm_part_bytes(N, H * W, C, groups, kind)};
    if (!same_or_apart(by, bx) || !same_or_apart(by, br) || !apart_from(by, bg, bb) || !apart_from(bs, bx, br, by, bg, bb) || !apart_from(bw, bx, br, by, bg, bb, bs))
        return CPRUNE_ERR_INVALID_ARG;
    NormParams p = norm_params(kind, N, H, W, C, groups, false);
    p.x = x; p.res = residual; p.out = y; p.gamma = gamma; p.beta = beta; p.stats = stats; p.eps = eps;
    p.part = (float2 *)workspace;
    const NormTiling t = norm_tiling(kind, N, p.HW, C, groups, false);
    cudaStream_t st = (cudaStream_t)stream;
    return by_kind(kind, act, residual != nullptr, [&](auto k, auto a, auto r) -> cprune_status {
        constexpr int K = decltype(k)::value, A = decltype(a)::value;
        constexpr bool R = decltype(r)::value;
        if (c.ranks) {
            p.gs = c.gs; p.sv = c.widest; p.per = c.per; p.data_bytes = (int)c.data_bytes;
            return launch_cluster<norm_cluster_kernel<K, A, R>>(c, N, st, p);
        }
        const dim3 grid(t.chunks, t.slices, N);
        ChainScope chain;
        const cprune_status e = launch_pass<norm_partial_kernel<K>>(grid, norm_ring_bytes(K, 1), st, p, t.lanes);
        if (e != CPRUNE_OK) return e;
        chain.follow();
        p.ring_bytes = ring_of(R + 1) * (R + 1) * NORM_T * (K == 2 ? 4 : 16);
        return launch_pass<norm_apply_kernel<K, A, R>>(grid, p.ring_bytes + norm_pass_bytes(p, L_of(K)), st, p, t.lanes);
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
    const size_t part_bytes = norm_part_bytes(N, H * W, C, groups, kind);
    if (workspace_bytes < part_bytes || !workspace) return CPRUNE_ERR_WORKSPACE_TOO_SMALL;
    const size_t bytes = norm_bytes(type, N, H, W, C), channels = (size_t)C * 4;
    const Buffer bx{x, bytes}, br{residual, bytes}, by{dy, bytes}, bdx{dx, bytes}, bdr{dresidual, bytes}, bw{workspace, part_bytes};
    const Buffer bg{gamma, channels}, bb{beta, channels}, bdg{dgamma, channels}, bdb{dbeta, channels}, bs{stats, (size_t)N * groups * 8};
    for (const Buffer &b : {bdx, bdr})
        if (!same_or_apart(b, bx) || !same_or_apart(b, br) || !same_or_apart(b, by) || !apart_from(b, bg, bb, bs)) return CPRUNE_ERR_INVALID_ARG;
    for (const Buffer &b : {bdg, bdb, bw})
        if (!apart_from(b, bx, br, by, bdx, bdr, bg, bb, bs)) return CPRUNE_ERR_INVALID_ARG;
    if (!apart(bdx, bdr) || !apart(bdg, bdb) || !apart_from(bw, bdg, bdb)) return CPRUNE_ERR_INVALID_ARG;
    NormParams p = norm_params(kind, N, H, W, C, groups, true);
    p.x = x; p.dy = dy; p.res = residual; p.out = dx; p.dres = dresidual; p.gamma = gamma; p.beta = beta; p.stats = const_cast<float *>(stats);
    p.dgamma = dgamma; p.dbeta = dbeta;
    p.part = (float2 *)workspace;
    const NormTiling t = norm_tiling(kind, N, p.HW, C, groups, true);
    cudaStream_t st = (cudaStream_t)stream;
    return by_kind(kind, act, residual != nullptr, [&](auto k, auto a, auto r) -> cprune_status {
        constexpr int K = decltype(k)::value, A = decltype(a)::value;
        constexpr bool R = decltype(r)::value;
        ChainScope chain;
        const dim3 grid(t.chunks, t.slices, N);
        p.ring_bytes = norm_ring_bytes(K, R + 2);
        const size_t smem = p.ring_bytes + (size_t)p.sv * L_of(K) * 16;
        const bool runs = (p.HW / p.rows + p.chunks - 1) / p.chunks >= GRADIENT_SINGLE;           // (and one more pixel behind the last full round)
        const cprune_status e = runs ? launch_pass<norm_grad_partial_kernel<K, A, R, true>>(grid, smem, st, p, t.lanes)
                                     : launch_pass<norm_grad_partial_kernel<K, A, R, false>>(grid, smem, st, p, t.lanes);
        if (e != CPRUNE_OK) return e;
        chain.follow();
        return launch_pass<norm_grad_apply_kernel<K, A, R>>(dim3(t.chunks, t.slices, N + (dgamma || dbeta ? 1 : 0)), p.ring_bytes + norm_pass_bytes(p, L_of(K)), st, p, t.lanes);
    });
}

}  // extern "C"
