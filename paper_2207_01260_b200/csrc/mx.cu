// Rounding to MXFP4 and back, and the product with weights kept in it.
//
//   rounding   block by block of 32 channels: scale = 2^(floor(log2 max |x|) - 2), code = x / scale to the nearest E2M1 value.
//              Both are exact but for the one rounding: the scale is a power of two.
//   product    y = act(q(x) W^T + b + residual), q the rounding above: 4-bit values on both sides, whose products are exact; float32 sums.
#include <cmath>

#include "common.cuh"
#include "mx.cuh"

namespace cprune {

// ------------------------------------------------------------------------------------------------------- rounding

// The eight values that begin at channel c of a row, at p.  TYPE 0: bf16 rows of c_pad channels; 1: float32 rows on 16-byte boundaries; 2: float32 rows at any
// address.  Channels from C on are zeros.
template <int TYPE> struct Eight {
    float f[8];
    using Value = float;
    __device__ __forceinline__ void read(const Value *p, int c, int C, int) {
        if (TYPE == 1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c + 4 * h < C) v = __ldg((const float4 *)p + h);       // (C is a multiple of 4)
                f[4 * h] = v.x; f[4 * h + 1] = v.y; f[4 * h + 2] = v.z; f[4 * h + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = c + i < C ? __ldg(p + i) : 0.f;
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = 0.f;
    }
    // bits of the largest magnitude
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(f[i]) & 0x7fffffffu);
        return t;
    }
    __device__ __forceinline__ uint32_t codes(uint32_t code) const {
        const float inverse = mx_inverse(code);
        float q[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = f[i] * inverse;
        return code == MX_NAN ? 0u : mx_codes(q);
    }
};
// (two at a time, as bf16: products with a power of two are exact there too, but for what is far under the smallest code)
template <> struct Eight<0> {
    bf16x8 v;
    using Value = __nv_bfloat16;
    __device__ __forceinline__ void read(const Value *p, int c, int C, int pitch) {
        clear();
        if (c >= pitch) return;
        v = ldg8((const bf16x8 *)p);
        if (c + 8 > C) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v.w[i] &= (c + 2 * i < C ? 0xffffu : 0u) | (c + 2 * i + 1 < C ? 0xffff0000u : 0u);
        }
    }
    __device__ __forceinline__ void clear() { v = bf16x8{{0u, 0u, 0u, 0u}}; }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t m = v.w[0] & 0x7fff7fffu;
#pragma unroll
        for (int j = 1; j < 4; ++j) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v.w[j] & 0x7fff7fffu));
        return max(m & 0x7fffu, m >> 16 & 0x7fffu) << 16;
    }
    __device__ __forceinline__ uint32_t codes(uint32_t code) const {
        const uint32_t inverse = (__float_as_uint(mx_inverse(code)) >> 16) * 0x10001u;
        bf16x8 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(q.w[j]) : "r"(v.w[j]), "r"(inverse));
        float f[8];
        unpack8(q, f);
        return code == MX_NAN ? 0u : mx_codes(f);
    }
};

// The exact values of eight codes to p, in the form of x (pad lanes zero)
template <int TYPE>
__device__ __forceinline__ void write_eight(typename Eight<TYPE>::Value *p, int c, int C, int pitch, uint32_t w, uint32_t code) {
    if constexpr (TYPE == 0) {
        if (c >= pitch) return;
        bf16x8 v = mx_values_bf16(w, code);
        if (c + 8 > C) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v.w[i] &= (c + 2 * i < C ? 0xffffu : 0u) | (c + 2 * i + 1 < C ? 0xffff0000u : 0u);
        }
        *(bf16x8 *)p = v;
    } else {
        float f[8];
        mx_values(w, mx_scale(code), f);
        if (TYPE == 1) {
            if (c < C) *(float4 *)p = make_float4(f[0], f[1], f[2], f[3]);
            if (c + 4 < C) *((float4 *)p + 1) = make_float4(f[4], f[5], f[6], f[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < C) p[i] = f[i];
        }
    }
}

constexpr int MX_T = 256, MX_UNIT = 64;      // rows that a block takes at a time

// 16 / E threads take four blocks (128 channels, a tile of scales wide: grid y) of a row, 8 E values each (bf16: sixteen, float32: eight): loads and stores of
// neighbouring threads adjoin, and the four scales are one word of a tile of scales.  What bounds it is the number of instructions, most of them for a block's scale, whatever the values a thread
// has; 200704 x 108 with the values written (98 MB): eight values a thread, one row at a time 36 us, four rows under way and bf16 two at a time 26 us, sixteen
// values 22 us.  Narrow rows leave most of a row's threads without work: a million rows of 16 channels 82 us, 4 million of 3 272 (12.4 and 30 at a copy's
// rate).  FORM 0: codes and scales (either both or neither), values as x; 1: the values in blocks, bf16 [rows][blocks * 32], in the order
// 0 4 1 5 2 6 3 7 of every eight (the order in which mx_pair takes codes apart).
template <int TYPE, int FORM>
__global__ void __launch_bounds__(MX_T) mx_quantize_kernel(const void *__restrict__ x, unsigned long long rows, int C, int pitch, int tiles4, uint32_t *__restrict__ codes,
                                                           uint8_t *__restrict__ scales, void *__restrict__ values) {
    pdl_wait();
    pdl_trigger();
    using Value = typename Eight<TYPE>::Value;
    constexpr int E = TYPE == 0 ? 2 : 1, TEAM = 16 / E, ROWS = MX_T / TEAM, AHEAD = MX_UNIT / ROWS, OF_BLOCK = 4 / E;       // OF_BLOCK: threads of a block of 32
    const int blocks = (C + MX_BLOCK - 1) / MX_BLOCK, sub = threadIdx.x % TEAM, own = threadIdx.x / TEAM, tile = blockIdx.y, c = tile * 128 + sub * 8 * E;
    const int block = tile * 4 + sub / OF_BLOCK;
    const bool mine = block < blocks;
    const int x_step = ROWS * pitch, code_step = ROWS * blocks * 4, value_step = ROWS * blocks * MX_BLOCK;
    // (whole warps go round: the shuffles below need all lanes)
    for (unsigned long long r0 = (unsigned long long)blockIdx.x * MX_UNIT; r0 < rows; r0 += (unsigned long long)gridDim.x * MX_UNIT) {
        const int left = (int)min(rows - r0, (unsigned long long)MX_UNIT);
        const Value *from = (const Value *)x + (r0 + own) * pitch + c;
        Eight<TYPE> f[AHEAD][E];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (mine && k * ROWS + own < left) f[k][e].read(from + k * x_step + 8 * e, c + 8 * e, C, pitch);
                else f[k][e].clear();
            }
        uint32_t *code_to = codes + ((r0 + own) * blocks + block) * 4 + (sub % OF_BLOCK) * E;
        // (64 rows of a tile of scales: words 16 bytes apart, the second 32 rows in the next word)
        uint32_t *scale_to = (uint32_t *)(scales + mx_scale_at((long long)r0, tile * 4, tiles4)) + own * 4;
        Value *value_to = (Value *)values + (FORM == 0 ? (r0 + own) * pitch + c : (r0 + own) * ((size_t)blocks * MX_BLOCK) + c);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (k * ROWS >= left) break;
            const bool in = k * ROWS + own < left;
            uint32_t top = f[k][0].top();
            if (E > 1) top = max(top, f[k][E - 1].top());
#pragma unroll
            for (int o = 1; o < OF_BLOCK; o *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const uint32_t code = mx_scale_code(top);
            uint32_t w[E];
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] = f[k][e].codes(code);
            if (FORM == 0 && codes) {
                uint32_t word = code << (8 * (sub / OF_BLOCK));
                word |= __shfl_xor_sync(0xffffffffu, word, OF_BLOCK);
                word |= __shfl_xor_sync(0xffffffffu, word, 2 * OF_BLOCK);
                if (in && mine) {
                    if constexpr (E == 2) *(uint2 *)(code_to + k * code_step) = make_uint2(w[0], w[1]);
                    else code_to[k * code_step] = w[0];
                }
                if (in && sub == 0) scale_to[k * ROWS % 32 * 4 + k * ROWS / 32] = word;
            }
            if (values && in && mine) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    if constexpr (FORM == 0) write_eight<TYPE>(value_to + k * x_step + 8 * e, c + 8 * e, C, pitch, w[e], code);
                    else {
                        const MxFactors m(code);
                        *(bf16x8 *)(value_to + k * value_step + 8 * e) =
                            bf16x8{{m.value(mx_pair<0>(w[e])), m.value(mx_pair<1>(w[e])), m.value(mx_pair<2>(w[e])), m.value(mx_pair<3>(w[e]))}};
                    }
                }
            }
        }
    }
}

// The grid of the kernel above: tiles of 128 channels by shares of the rows
static dim3 mx_grid(unsigned long long rows, int tiles4) {
    const unsigned long long all = (rows + MX_UNIT - 1) / MX_UNIT, most = 1 << 20;
    return dim3((unsigned)(all < most ? all : most), (unsigned)tiles4);
}

template <int TYPE>
__global__ void __launch_bounds__(MX_T) mx_dequantize_kernel(const uint32_t *__restrict__ codes, const uint8_t *__restrict__ scales, unsigned long long rows, int C, int pitch,
                                                             int tiles4, void *__restrict__ values) {
    pdl_wait();
    pdl_trigger();
    const int eights = TYPE == 0 ? pitch / 8 : (C + 7) / 8, blocks = (C + MX_BLOCK - 1) / MX_BLOCK;
    const unsigned long long total = rows * eights;
    for (unsigned long long e = (unsigned long long)blockIdx.x * MX_T + threadIdx.x; e < total; e += (unsigned long long)gridDim.x * MX_T) {
        const size_t row = e / eights;
        const int c = (int)(e - row * eights) * 8, block = c / MX_BLOCK;
        const uint32_t w = block < blocks ? __ldg(codes + (row * blocks + block) * 4 + (c & 31) / 8) : 0u, code = block < blocks ? __ldg(scales + mx_scale_at((long long)row, block, tiles4)) : 127u;
        write_eight<TYPE>((typename Eight<TYPE>::Value *)values + row * pitch + c, c, C, pitch, w, code);
    }
}

__global__ void mx_pad_bias_kernel(const float *__restrict__ b, int n, int n_pad, float *__restrict__ out) {
    pdl_wait();
    pdl_trigger();
    const int k = blockIdx.x * blockDim.x + threadIdx.x;
    if (k < n_pad) out[k] = (b && k < n) ? b[k] : 0.f;
}

// --------------------------------------------------------------------------------------------- product, few rows

// A block takes 16 rows and 16 features; its eight warps share out the channels, and their sums meet in shared memory.  A thread reads
// a whole block of 32 codes of a feature (16 bytes), makes bf16 values of them, which hold 4-bit values times any power of two exactly, and
// takes the same 32 channels of its two rows: eight MMA steps, in an order of the channels that both sides share.
// The tensor core truncates where it adds to an accumulator; four steps start from zero and are added to the running sum by a rounded
// addition, and the warps' sums meet in float64.
constexpr int MXF_WARPS = 8, MXF_NT = 2, MXF_AHEAD = 2;
constexpr int MXF_BLOCKS = 2 * 148, MXF_IN = 2048;

// (one float32 of y, in its form)
__device__ __forceinline__ void mx_store(const MxProduct &p, unsigned long long n, int o, float v) {
    if (p.out_is_f32) {
        if (o < p.out) ((float *)p.y)[n * p.out + o] = v;
    } else ((__nv_bfloat16 *)p.y)[n * p.out_pad + o] = __float2bfloat16_rn(o < p.out ? v : 0.f);
}

__global__ void __launch_bounds__(MXF_WARPS * 32) mx_few_rows_kernel(const bf16x8 *__restrict__ x, const MxProduct p) {
    __shared__ float part[MXF_WARPS][16][MXF_NT * 8 + 1];
    pdl_trigger();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int o0 = blockIdx.x * (MXF_NT * 8);
    const unsigned long long n0 = (unsigned long long)blockIdx.y * 16;
    const uint4 none = make_uint4(0, 0, 0, 0);
    struct Piece { uint4 w; uint32_t scale; };
    auto load_w = [&](int c, Piece *v) {
        const int b = c * 4 + t;
#pragma unroll
        for (int f = 0; f < MXF_NT; ++f) {
            const int o = o0 + f * 8 + g;
            const bool in = b < p.blocks && o < p.out;
            v[f].w = in ? __ldg(p.codes + (size_t)o * p.blocks + b) : none;
            v[f].scale = in ? __ldg(p.scales + mx_scale_at(o, b, p.tiles4)) : 127;
        }
    };
    const int chunks = (p.blocks + 3) / 4;
    Piece wq[MXF_AHEAD][MXF_NT];
#pragma unroll
    for (int i = 0; i < MXF_AHEAD; ++i) load_w(warp + i * MXF_WARPS, wq[i]);
    pdl_wait();
    float acc[MXF_NT][4];
#pragma unroll
    for (int f = 0; f < MXF_NT; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[f][j] = 0.f;
    const bf16x8 zero = {{0u, 0u, 0u, 0u}};
    for (int c0 = warp; c0 < chunks; c0 += MXF_AHEAD * MXF_WARPS) {
#pragma unroll
        for (int i = 0; i < MXF_AHEAD; ++i) {
            const int c = c0 + i * MXF_WARPS, b = c * 4 + t;
            if (c >= chunks) break;
            bf16x8 xq[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned long long n = n0 + h * 8 + g;
                const bool in = n < p.rows && b < p.blocks;
#pragma unroll
                for (int q = 0; q < 4; ++q) xq[h][q] = in ? ldg8(x + (n * p.blocks + b) * 4 + q) : zero;
            }
#pragma unroll
            for (int f = 0; f < MXF_NT; ++f) {
                const MxFactors m(wq[i][f].scale);
                const uint32_t words[4] = {wq[i][f].w.x, wq[i][f].w.y, wq[i][f].w.z, wq[i][f].w.w};
#pragma unroll
                for (int hh = 0; hh < 2; ++hh) {
                    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q = 2 * hh; q < 2 * hh + 2; ++q) {
                        mma_16816(s, xq[0][q].w[0], xq[1][q].w[0], xq[0][q].w[1], xq[1][q].w[1], m.value(mx_pair<0>(words[q])), m.value(mx_pair<1>(words[q])));
                        mma_16816(s, xq[0][q].w[2], xq[1][q].w[2], xq[0][q].w[3], xq[1][q].w[3], m.value(mx_pair<2>(words[q])), m.value(mx_pair<3>(words[q])));
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[f][j] += s[j];
                }
            }
            load_w(c + MXF_AHEAD * MXF_WARPS, wq[i]);
        }
    }
#pragma unroll
    for (int f = 0; f < MXF_NT; ++f)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[warp][(j >> 1) * 8 + g][f * 8 + t * 2 + (j & 1)] = acc[f][j];
    __syncthreads();
    for (int e = threadIdx.x; e < 16 * MXF_NT * 8; e += MXF_WARPS * 32) {
        const int r = e / (MXF_NT * 8), c = e % (MXF_NT * 8), o = o0 + c;
        const unsigned long long n = n0 + r;
        if (n >= p.rows || o >= p.out_pad) continue;
        double s = 0.0;
#pragma unroll
        for (int q = 0; q < MXF_WARPS; ++q) s += part[q][r][c];
        float v = o < p.out ? (float)(s + (double)p.bias[o]) : 0.f;
        if (p.res && o < p.out) v += __bfloat162float(p.res[n * p.out_pad + o]);
        mx_store(p, n, o, mx_act(v, p.act));
    }
}

static int mx_type(int type, int C, uintptr_t addresses) { return type == CPRUNE_TYPE_BF16 ? 0 : C % 4 == 0 && !(addresses & 15) ? 1 : 2; }

}  // namespace cprune

using namespace cprune;

extern "C" {

int cprune_mx_blocks(int C) { return C > 0 ? mx_blocks(C) : 0; }

size_t cprune_mx_scale_bytes(size_t rows, int C) { return C > 0 ? (rows + 127) / 128 * (size_t)((mx_blocks(C) + 3) / 4) * 512 : 0; }

static cprune_status mx_check(const void *x, int type, size_t rows, int C, const void *codes, const void *scales) {
    if (!x || (type != CPRUNE_TYPE_BF16 && type != CPRUNE_TYPE_F32) || rows == 0 || C <= 0 || !codes != !scales) return CPRUNE_ERR_INVALID_ARG;
    if (((uintptr_t)codes | (uintptr_t)scales) & 15 || (uintptr_t)x & (type == CPRUNE_TYPE_BF16 ? 15 : 3)) return CPRUNE_ERR_INVALID_ARG;
    if (rows >> 40 || C > (1 << 22)) return CPRUNE_ERR_UNSUPPORTED;
    return CPRUNE_OK;
}

static size_t mx_matrix_bytes(int type, size_t rows, int pitch) { return rows * pitch * (type == CPRUNE_TYPE_BF16 ? 2 : 4); }

cprune_status cprune_mx_quantize(const void *x, int type, size_t rows, int C, void *codes, void *scales, void *values, void *stream) {
    const cprune_status c = mx_check(x, type, rows, C, codes, scales);
    if (c != CPRUNE_OK) return c;
    if ((!codes && !values) || (uintptr_t)values & (type == CPRUNE_TYPE_BF16 ? 15 : 3)) return CPRUNE_ERR_INVALID_ARG;
    const int tiles4 = (mx_blocks(C) + 3) / 4, pitch = type == CPRUNE_TYPE_BF16 ? cprune_padded_channels(C) : C;
    const Buffer bx{x, mx_matrix_bytes(type, rows, pitch)}, bv{values, bx.bytes}, bc{codes, rows * mx_blocks(C) * 16}, bs{scales, cprune_mx_scale_bytes(rows, C)};
    if (!same_or_apart(bv, bx) || !apart_from(bc, bx, bv, bs) || !apart_from(bs, bx, bv)) return CPRUNE_ERR_INVALID_ARG;
    const dim3 grid = mx_grid(rows, tiles4);
    auto launch = [&](auto kernel) {
        return launch_chained(kernel, grid, dim3(MX_T), 0, (cudaStream_t)stream, x, (unsigned long long)rows, C, pitch, tiles4, (uint32_t *)codes, (uint8_t *)scales, values);
    };
    switch (mx_type(type, C, (uintptr_t)x | (uintptr_t)values)) {
        case 0: CPRUNE_CUDA_CHECK(launch(mx_quantize_kernel<0, 0>)); break;
        case 1: CPRUNE_CUDA_CHECK(launch(mx_quantize_kernel<1, 0>)); break;
        default: CPRUNE_CUDA_CHECK(launch(mx_quantize_kernel<2, 0>));
    }
    return CPRUNE_OK;
}

cprune_status cprune_mx_dequantize(const void *codes, const void *scales, size_t rows, int C, int type, void *values, void *stream) {
    if (!codes) return CPRUNE_ERR_INVALID_ARG;
    const cprune_status c = mx_check(values, type, rows, C, codes, scales);
    if (c != CPRUNE_OK) return c;
    const int tiles4 = (mx_blocks(C) + 3) / 4, pitch = type == CPRUNE_TYPE_BF16 ? cprune_padded_channels(C) : C;
    if (!apart_from(Buffer{values, mx_matrix_bytes(type, rows, pitch)}, Buffer{codes, rows * mx_blocks(C) * 16}, Buffer{scales, cprune_mx_scale_bytes(rows, C)}))
        return CPRUNE_ERR_INVALID_ARG;
    const unsigned long long all = (rows * ((pitch + 7) / 8) + MX_T - 1) / MX_T;
    const unsigned grid = (unsigned)(all < 148 * 16 ? all : 148 * 16);
    auto launch = [&](auto kernel) {
        return launch_chained(kernel, dim3(grid), dim3(MX_T), 0, (cudaStream_t)stream, (const uint32_t *)codes, (const uint8_t *)scales, (unsigned long long)rows, C, pitch, tiles4,
                              values);
    };
    switch (mx_type(type, C, (uintptr_t)values)) {
        case 0: CPRUNE_CUDA_CHECK(launch(mx_dequantize_kernel<0>)); break;
        case 1: CPRUNE_CUDA_CHECK(launch(mx_dequantize_kernel<1>)); break;
        default: CPRUNE_CUDA_CHECK(launch(mx_dequantize_kernel<2>));
    }
    return CPRUNE_OK;
}

cprune_status cprune_mx_pack(const float *w, const float *b, int out, int in, void *codes, void *scales, float *b_packed, void *stream) {
    if (!codes || !b_packed || out <= 0 || ((uintptr_t)b | (uintptr_t)b_packed) & 3) return CPRUNE_ERR_INVALID_ARG;
    const int out_pad = cprune_padded_channels(out);
    if (in > 0 && !apart_from(Buffer{b_packed, (size_t)out_pad * 4}, Buffer{w, (size_t)out * in * 4}, Buffer{b, (size_t)out * 4}, Buffer{codes, (size_t)out * mx_blocks(in) * 16},
                              Buffer{scales, cprune_mx_scale_bytes(out, in)})) return CPRUNE_ERR_INVALID_ARG;
    for (const Buffer &r : {Buffer{codes, (size_t)out * cprune_mx_blocks(in) * 16}, Buffer{scales, cprune_mx_scale_bytes(out, in)}})
        if (!apart(r, Buffer{b, (size_t)out * 4})) return CPRUNE_ERR_INVALID_ARG;
    ChainScope chain;
    const cprune_status s = cprune_mx_quantize(w, CPRUNE_TYPE_F32, out, in, codes, scales, nullptr, stream);
    if (s != CPRUNE_OK) return s;
    chain.follow();
    CPRUNE_CUDA_CHECK(launch_chained(mx_pad_bias_kernel, dim3((out_pad + 255) / 256), dim3(256), 0, (cudaStream_t)stream, b, out, out_pad, b_packed));
    return CPRUNE_OK;
}

// Whether the kernel for few rows takes a product: where all its blocks run at the same time and none has many channels to go through.  It needs no tensor
// memory, no maps and no third launch.  us there / on the block-scaled path:  1 x 1280 -> 1000 4.4 / 6.4, 64 rows of that 6.9 / 7.7, 96 rows (378 blocks)
// 9.3 / 8.0;  196 x 384 -> 64 4.9 / 7.9;  1568 x 144 -> 24 (196 blocks) 5.4 / 6.4, 3136 rows of that 7.3 / 6.4;  32 x 2048 -> 2048 7.2 / 7.6;
// 64 x 4096 -> 1000 10.9 / 8.5;  8 x 25088 -> 4096 36 / 18.
static MxTiling mx_product_tiling(size_t rows, int in, int out) {
    MxTiling t = {};
    const unsigned long long most = MXF_BLOCKS, wide = ((unsigned long long)out + MXF_NT * 8 - 1) / (MXF_NT * 8);
    return in <= MXF_IN && rows <= most * 16 && (rows + 15) / 16 * wide <= most ? t : mx_tiling(rows, in, out);
}
static size_t mx_codes_bytes(size_t rows, int in) { return (rows * (size_t)mx_blocks(in) * 16 + 255) / 256 * 256; }

size_t cprune_mx_fc_workspace_bytes(size_t rows, int in, int out) {
    if (rows == 0 || in <= 0 || out <= 0) return 0;
    const MxTiling t = mx_product_tiling(rows, in, out);
    if (!t.tensor) return rows * (size_t)mx_blocks(in) * MX_BLOCK * 2;
    return t.round ? 0 : mx_codes_bytes(rows, in) + cprune_mx_scale_bytes(rows, in) + mx_partial_bytes(t, rows, out);
}

cprune_status cprune_mx_fc(const void *x, size_t rows, int in, const void *codes, const void *scales, const float *b_packed, int out, int act, const void *residual,
                           int out_is_f32, void *y, void *workspace, size_t workspace_bytes, void *stream) {
    if (!x || !codes || !scales || !b_packed || !y || rows == 0 || in <= 0 || out <= 0 || act < CPRUNE_ACT_NONE || act > CPRUNE_ACT_RELU6) return CPRUNE_ERR_INVALID_ARG;
    if (((uintptr_t)x | (uintptr_t)codes | (uintptr_t)scales | (uintptr_t)residual | (uintptr_t)workspace) & 15 || (uintptr_t)b_packed & 3) return CPRUNE_ERR_INVALID_ARG;
    if ((uintptr_t)y & (out_is_f32 ? 3 : 15)) return CPRUNE_ERR_INVALID_ARG;
    if (rows >> 31 || in > (1 << 22) || out > (1 << 24)) return CPRUNE_ERR_UNSUPPORTED;
    const size_t need = cprune_mx_fc_workspace_bytes(rows, in, out);
    if (need && (!workspace || workspace_bytes < need)) return CPRUNE_ERR_WORKSPACE_TOO_SMALL;
    const size_t out_bytes = rows * cprune_padded_channels(out) * 2;
    const Buffer bx{x, rows * cprune_padded_channels(in) * 2}, br{residual, out_bytes}, by{y, out_is_f32 ? rows * out * 4 : out_bytes}, bb{b_packed, (size_t)cprune_padded_channels(out) * 4};
    const Buffer bc{codes, (size_t)out * mx_blocks(in) * 16}, bs{scales, cprune_mx_scale_bytes(out, in)}, bw{need ? workspace : nullptr, need};
    if (!(out_is_f32 ? apart(by, br) : same_or_apart(by, br)) || !apart_from(by, bx, bb, bc, bs) || !apart_from(bw, bx, br, by, bb, bc, bs)) return CPRUNE_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    MxProduct p = {};
    p.codes = (const uint4 *)codes; p.scales = (const uint8_t *)scales; p.bias = b_packed; p.res = (const __nv_bfloat16 *)residual; p.y = y; p.rows = rows;
    p.blocks = mx_blocks(in); p.tiles4 = (p.blocks + 3) / 4; p.out = out; p.out_pad = cprune_padded_channels(out); p.act = act; p.out_is_f32 = out_is_f32;
    ChainScope chain;
    const MxTiling t = mx_product_tiling(rows, in, out);
    if (t.tensor && t.round) return launch_mx_product(p, t, x, nullptr, in, nullptr, chain, st);
    if (t.tensor) {
        uint8_t *xscales = (uint8_t *)workspace + mx_codes_bytes(rows, in);
        CPRUNE_CUDA_CHECK(launch_chained(mx_quantize_kernel<0, 0>, mx_grid(rows, p.tiles4), dim3(MX_T), 0, st, x, (unsigned long long)rows, in,
                                         cprune_padded_channels(in), p.tiles4, (uint32_t *)workspace, xscales, (void *)nullptr));
        chain.follow();
        return launch_mx_product(p, t, workspace, xscales, in, (float *)(xscales + cprune_mx_scale_bytes(rows, in)), chain, st);
    }
    CPRUNE_CUDA_CHECK(launch_chained(mx_quantize_kernel<0, 1>, mx_grid(rows, p.tiles4), dim3(MX_T), 0, st, x, (unsigned long long)rows, in,
                                     cprune_padded_channels(in), p.tiles4, (uint32_t *)nullptr, (uint8_t *)nullptr, workspace));
    chain.follow();
    const dim3 grid((p.out_pad + MXF_NT * 8 - 1) / (MXF_NT * 8), (unsigned)((rows + 15) / 16));
    CPRUNE_CUDA_CHECK(launch_chained(mx_few_rows_kernel, grid, dim3(MXF_WARPS * 32), 0, st, (const bf16x8 *)workspace, p));
    return CPRUNE_OK;
}

}  // extern "C"
