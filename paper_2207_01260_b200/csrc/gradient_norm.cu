// Global norm of the gradients of many tensors, and clipping.
//
//   norm = sqrt(sum over all tensors of g^2),   out = g min(1, max_norm / (norm + 1e-6))
//
// Two launches for up to GRAD_TABLE tensors: every block sums the squares of its share of the list, and every block of the second launch
// adds these sums up for itself, in the same order, before it scales its share.  The list travels in the kernels' parameters, so that nothing
// is copied to the device and a captured call keeps it.  The unit of work is a piece of 16 KB, counted in 16-byte vectors from the
// tensor's address rounded down: a tensor may lie at any address of its type, and only its first and last vector are taken value by value.
// Squares and their sums are float64: a float32 square loses gradients below 1e-19 and overflows above 1e19, and the sum runs over
// millions of values.
// What bounds it is memory for large lists, launches for small ones.  62 float32 tensors of 11.7 million values in all 24.7 us (read once and written: 14.3 us at
// a copy's rate; 12.7 of them for the norm alone), of 40 million, which do not stay in the cache, 85 us (read twice and written: 73); 12 small ones 5 us.
// Eight blocks to an SM 24.9 and 84 us (bf16 17.2 us for 16.5), pieces of 32 KB 26.6 and 85; the sums in float32 would save 0.3 and 2 us.
#include <cmath>

#include "common.cuh"

namespace cprune {

constexpr int GRAD_T = 256, GRAD_AHEAD = 4;
constexpr int GRAD_PIECE = GRAD_T * GRAD_AHEAD;     // vectors
constexpr int GRAD_BLOCKS = 148 * 4;
constexpr int GRAD_TABLE_SMALL = 64, GRAD_TABLE = 512;       // (a short list in the small table: 7.1 us a call on the host, in the large one 8.8)

template <int MOST> struct GradTable {
    const void *g[MOST];
    void *out[MOST];
    unsigned long long count[MOST];                 // values; the highest bit: bf16
    unsigned first[MOST + 1];                       // first piece
    int n;
};
constexpr unsigned long long GRAD_BF16 = 1ull << 63;

// A tensor's vectors
struct GradSpan {
    const char *base;                               // the address, rounded down
    int skip;                                       // bytes of the first vector that are before the tensor
    unsigned long long bytes;                       // from base to the tensor's end
    bool bf16;
    __device__ __forceinline__ GradSpan(const void *p, unsigned long long count) {
        bf16 = (count & GRAD_BF16) != 0;
        skip = (int)((uintptr_t)p & 15);
        base = (const char *)p - skip;
        bytes = (count & ~GRAD_BF16) * (bf16 ? 2 : 4) + skip;
    }
    // whether vector v is partly outside
    __device__ __forceinline__ bool edge(unsigned long long v) const { return (v == 0 && skip) || (v + 1) * 16 > bytes; }
    // whether the whole piece that begins at vector v is inside
    __device__ __forceinline__ bool whole(unsigned long long v) const { return (v > 0 || !skip) && (v + GRAD_PIECE) * 16 <= bytes; }
    // its values, 0 in place of those outside
    __device__ __forceinline__ uint4 read(unsigned long long v) const {
        if (!edge(v)) return *(const uint4 *)(base + v * 16);
        uint4 r;
        uint32_t *w = &r.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned long long at = v * 16 + 4 * i;
            w[i] = 0;
            if (bf16) {
                if (at >= skip && at < bytes) w[i] = *(const uint16_t *)(base + at);
                if (at + 2 >= skip && at + 2 < bytes) w[i] |= (uint32_t)*(const uint16_t *)(base + at + 2) << 16;
            } else if (at >= skip && at < bytes) w[i] = *(const uint32_t *)(base + at);
        }
        return r;
    }
};

__device__ __forceinline__ double squares(const uint4 &u, bool bf16) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (bf16) {
            const double a = __uint_as_float(w[i] << 16), b = __uint_as_float(w[i] & 0xffff0000u);
            s = fma(a, a, fma(b, b, s));
        } else {
            const double a = __uint_as_float(w[i]);
            s = fma(a, a, s);
        }
    }
    return s;
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double warps[GRAD_T / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < GRAD_T / 32; ++i) s += warps[i];
    return s;
}

// The pieces of block b of n: contiguous, so that a block walks through the list
__device__ __forceinline__ void share_of(unsigned pieces, unsigned &begin, unsigned &end) {
    begin = (unsigned)((unsigned long long)pieces * blockIdx.x / gridDim.x);
    end = (unsigned)((unsigned long long)pieces * (blockIdx.x + 1) / gridDim.x);
}

// The tensor of a piece: the last one that begins at or before it (tensors without values have no piece)
template <int MOST>
__device__ __forceinline__ int tensor_of(const GradTable<MOST> &t, unsigned piece) {
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.first[mid] <= piece) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// This thread's vectors of a piece, zeros behind the tensor's end.  (Whole pieces without a test per vector: its branches would keep the loads from being under
// way together.)
__device__ __forceinline__ void read_piece(const GradSpan &span, unsigned long long first, uint4 *u) {
    const unsigned long long v0 = first + threadIdx.x;
    if (span.whole(first)) {
#pragma unroll
        for (int i = 0; i < GRAD_AHEAD; ++i) u[i] = *(const uint4 *)(span.base + (v0 + i * GRAD_T) * 16);
    } else {
#pragma unroll
        for (int i = 0; i < GRAD_AHEAD; ++i) u[i] = (v0 + i * GRAD_T) * 16 < span.bytes ? span.read(v0 + i * GRAD_T) : make_uint4(0, 0, 0, 0);
    }
}

template <int MOST>
__global__ void __launch_bounds__(GRAD_T) gradient_squares_kernel(const __grid_constant__ GradTable<MOST> t, double *__restrict__ part) {
    pdl_wait();
    pdl_trigger();
    unsigned piece, end;
    share_of(t.first[t.n], piece, end);
    double s = 0.0;
    if (piece < end) {
        int k = tensor_of(t, piece);
        for (; piece < end; ++piece) {
            while (t.first[k + 1] <= piece) ++k;
            const GradSpan span(t.g[k], t.count[k]);
            uint4 u[GRAD_AHEAD];
            read_piece(span, (unsigned long long)(piece - t.first[k]) * GRAD_PIECE, u);
#pragma unroll
            for (int i = 0; i < GRAD_AHEAD; ++i) s += squares(u[i], span.bf16);
        }
    }
    s = block_sum(s);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double total_norm(const double *part, int parts) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += GRAD_T) s += __ldcg(part + i);
    return sqrt(block_sum(s));
}

__global__ void __launch_bounds__(GRAD_T) gradient_norm_kernel(const double *part, int parts, float *norm) {
    pdl_wait();
    pdl_trigger();
    const double n = total_norm(part, parts);
    if (threadIdx.x == 0) *norm = (float)n;
}

// The values times the factor c, f in float32.  A factor next to or below the smallest normal number has not the digits (or is 0 where the results are not): such
// products are taken in 64 bits.
__device__ __forceinline__ uint4 scaled(const uint4 &u, float f, double c, bool bf16) {
    uint4 r = u;
    uint32_t *w = &r.x;
    if (f < 1e-36f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (bf16) {
                const __nv_bfloat162 b = __floats2bfloat162_rn((float)(__uint_as_float(w[i] << 16) * c), (float)(__uint_as_float(w[i] & 0xffff0000u) * c));
                w[i] = *reinterpret_cast<const uint32_t *>(&b);
            } else w[i] = __float_as_uint((float)(__uint_as_float(w[i]) * c));
        }
        return r;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (bf16) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
            w[i] = *reinterpret_cast<const uint32_t *>(&b);
        } else w[i] = __float_as_uint(__uint_as_float(w[i]) * f);
    }
    return r;
}

// last: this launch is the one that writes the norm
template <int MOST>
__global__ void __launch_bounds__(GRAD_T) gradient_scale_kernel(const __grid_constant__ GradTable<MOST> t, const double *part, int parts, float max_norm, float *norm,
                                                                int last) {
    pdl_wait();
    pdl_trigger();
    const double n = total_norm(part, parts);
    if (last && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
    double c = (double)max_norm / (n + 1e-6);
    c = c > 1.0 ? 1.0 : c;                                 // (a NaN stays one)
    const float f = (float)c;
    unsigned begin, piece;
    share_of(t.first[t.n], begin, piece);
    if (begin >= piece) return;
    // (backwards: what was read last is still in the cache)
    int k = tensor_of(t, piece - 1);
    while (piece-- > begin) {
        while (t.first[k] > piece) --k;
        if (f == 1.f && t.out[k] == t.g[k]) continue;
        const GradSpan span(t.g[k], t.count[k]);
        const bool same = ((uintptr_t)t.out[k] & 15) == (uintptr_t)span.skip;      // vectors of the result are vectors of the gradient
        char *out = (char *)t.out[k] - span.skip;
        const unsigned long long first = (unsigned long long)(piece - t.first[k]) * GRAD_PIECE, v0 = first + threadIdx.x;
        uint4 u[GRAD_AHEAD];
        read_piece(span, first, u);
        if (same && span.whole(first)) {
#pragma unroll
            for (int i = 0; i < GRAD_AHEAD; ++i) *(uint4 *)(out + (v0 + i * GRAD_T) * 16) = scaled(u[i], f, c, span.bf16);
            continue;
        }
#pragma unroll
        for (int i = 0; i < GRAD_AHEAD; ++i) {
            const unsigned long long v = v0 + i * GRAD_T;
            if (v * 16 >= span.bytes) break;
            const uint4 r = scaled(u[i], f, c, span.bf16);
            if (same && !span.edge(v)) {
                *(uint4 *)(out + v * 16) = r;
                continue;
            }
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned long long at = v * 16 + 4 * j;
                if (span.bf16) {
                    if (at >= span.skip && at < span.bytes) *(uint16_t *)(out + at) = (uint16_t)w[j];
                    if (at + 2 >= span.skip && at + 2 < span.bytes) *(uint16_t *)(out + at + 2) = (uint16_t)(w[j] >> 16);
                } else if (at >= span.skip && at < span.bytes) *(uint32_t *)(out + at) = w[j];
            }
        }
    }
}

// Tensors i0 .. of the list into a table; returns the blocks that share its pieces
template <int MOST>
static int fill_table(GradTable<MOST> &t, const void *const *grads, const unsigned long long *counts, const int *types, int n, void *const *out) {
    t.n = n;
    t.first[0] = 0;
    for (int i = 0; i < n; ++i) {
        t.g[i] = grads[i];
        t.out[i] = out ? out[i] : const_cast<void *>(grads[i]);
        const bool bf16 = types[i] == CPRUNE_TYPE_BF16;
        t.count[i] = counts[i] | (bf16 ? GRAD_BF16 : 0);
        const unsigned long long bytes = counts[i] ? counts[i] * (bf16 ? 2 : 4) + ((uintptr_t)grads[i] & 15) : 0;
        t.first[i + 1] = t.first[i] + (unsigned)((bytes + GRAD_PIECE * 16 - 1) / (GRAD_PIECE * 16));
    }
    const unsigned pieces = t.first[n];
    return pieces < 1 ? 1 : pieces < GRAD_BLOCKS ? (int)pieces : GRAD_BLOCKS;
}

static cprune_status check_list(const void *const *grads, const unsigned long long *counts, const int *types, int n, void *const *out, const float *norm,
                                const void *workspace, size_t workspace_bytes) {
    if (n < 0 || (n > 0 && (!grads || !counts || !types)) || !norm || (uintptr_t)norm & 3 || (uintptr_t)workspace & 15) return CPRUNE_ERR_INVALID_ARG;
    unsigned long long pieces = 0;
    for (int i = 0; i < n; ++i) {
        if (types[i] != CPRUNE_TYPE_BF16 && types[i] != CPRUNE_TYPE_F32) return CPRUNE_ERR_INVALID_ARG;
        const uintptr_t odd = types[i] == CPRUNE_TYPE_BF16 ? 1 : 3;
        if (counts[i] >> 44) return CPRUNE_ERR_UNSUPPORTED;
        if (counts[i] && (!grads[i] || (uintptr_t)grads[i] & odd || (out && (!out[i] || (uintptr_t)out[i] & odd)))) return CPRUNE_ERR_INVALID_ARG;
        pieces += counts[i] / (GRAD_PIECE * 4) + 2;
    }
    if (pieces > 0xffffffffull) return CPRUNE_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < cprune_gradient_workspace_bytes(n)) return CPRUNE_ERR_WORKSPACE_TOO_SMALL;
    return CPRUNE_OK;
}

// f(table, its blocks, first tensor) for every part of the list
template <typename F>
static cprune_status by_tables(const void *const *grads, const unsigned long long *counts, const int *types, int n, void *const *out, F f) {
    if (n <= GRAD_TABLE_SMALL) {
        GradTable<GRAD_TABLE_SMALL> t;
        const int blocks = fill_table(t, grads, counts, types, n, out);
        return f(t, blocks, 0);
    }
    for (int i = 0; i < n; i += GRAD_TABLE) {
        GradTable<GRAD_TABLE> t;
        const int blocks = fill_table(t, grads + i, counts + i, types + i, n - i < GRAD_TABLE ? n - i : GRAD_TABLE, out ? out + i : nullptr);
        const cprune_status s = f(t, blocks, i);
        if (s != CPRUNE_OK) return s;
    }
    return CPRUNE_OK;
}

static cprune_status enqueue_squares(const void *const *grads, const unsigned long long *counts, const int *types, int n, double *part, int *parts, ChainScope &chain,
                                     cudaStream_t st) {
    *parts = 0;
    return by_tables(grads, counts, types, n, nullptr, [&](auto &t, int blocks, int) -> cprune_status {
        CPRUNE_CUDA_CHECK(launch_chained(gradient_squares_kernel<sizeof(t.g) / sizeof(t.g[0])>, dim3(blocks), dim3(GRAD_T), 0, st, t, part + *parts));
        *parts += blocks;
        chain.follow();
        return CPRUNE_OK;
    });
}

}  // namespace cprune

using namespace cprune;

extern "C" {

size_t cprune_gradient_workspace_bytes(int n) {
    if (n < 0) return 0;
    return (size_t)(n / GRAD_TABLE + 1) * GRAD_BLOCKS * sizeof(double);
}

cprune_status cprune_gradient_norm(const void *const *grads, const unsigned long long *counts, const int *types, int n, float *norm, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    const cprune_status c = check_list(grads, counts, types, n, nullptr, norm, workspace, workspace_bytes);
    if (c != CPRUNE_OK) return c;
    double *part = (double *)workspace;
    int parts;
    ChainScope chain;
    const cprune_status s = enqueue_squares(grads, counts, types, n, part, &parts, chain, (cudaStream_t)stream);
    if (s != CPRUNE_OK) return s;
    CPRUNE_CUDA_CHECK(launch_chained(gradient_norm_kernel, dim3(1), dim3(GRAD_T), 0, (cudaStream_t)stream, part, parts, norm));
    return CPRUNE_OK;
}

cprune_status cprune_clip_gradients(const void *const *grads, const unsigned long long *counts, const int *types, int n, float max_norm, void *const *out, float *norm,
                                    void *workspace, size_t workspace_bytes, void *stream) {
    if (!(max_norm >= 0.f)) return CPRUNE_ERR_INVALID_ARG;
    const cprune_status c = check_list(grads, counts, types, n, out, norm, workspace, workspace_bytes);
    if (c != CPRUNE_OK) return c;
    double *part = (double *)workspace;
    int parts;
    ChainScope chain;
    const cprune_status s = enqueue_squares(grads, counts, types, n, part, &parts, chain, (cudaStream_t)stream);
    if (s != CPRUNE_OK) return s;
    return by_tables(grads, counts, types, n, out, [&](auto &t, int blocks, int first) -> cprune_status {
        CPRUNE_CUDA_CHECK(launch_chained(gradient_scale_kernel<sizeof(t.g) / sizeof(t.g[0])>, dim3(blocks), dim3(GRAD_T), 0, (cudaStream_t)stream, t, part, parts, max_norm,
                                         norm, first == 0 ? 1 : 0));
        return CPRUNE_OK;
    });
}

}  // extern "C"
