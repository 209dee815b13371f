// 4-bit values of the OCP Microscaling formats (MXFP4): E2M1 codes in blocks of 32 along the channels, an E8M0 scale to a block.
#pragma once

#include "common.cuh"

namespace cprune {

constexpr int MX_BLOCK = 32;
constexpr uint32_t MX_NAN = 255;          // the scale of a block without a value

inline int mx_blocks(int C) { return (C + MX_BLOCK - 1) / MX_BLOCK; }

// Where the scale of a row's block lies: tiles of 128 rows by 4 blocks (512 bytes, the order in which the tensor core takes them),
// [rows / 128][blocks / 4][row % 32][row / 32 % 4][block % 4]
__host__ __device__ __forceinline__ size_t mx_scale_at(long long row, int block, int tiles4) {
    return ((size_t)(row >> 7) * tiles4 + (block >> 2)) * 512 + (size_t)((row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3));
}

// The scale's code of a block whose largest magnitude has these bits (of the absolute values: a NaN's are the largest).
// 2^(floor(log2 top) - 2), the two being the exponent of the format's largest value 6; not below 2^-127
__device__ __forceinline__ uint32_t mx_scale_code(uint32_t top) {
    const int e = (int)(top >> 23);
    return e == 255 ? MX_NAN : (uint32_t)max(e - 2, 0);
}
__device__ __forceinline__ float mx_scale(uint32_t code) {
    return __uint_as_float(code == MX_NAN ? 0x7fffffffu : code == 0 ? 0x00400000u : code << 23);
}
// 1 / scale (a power of two: products with it are exact)
__device__ __forceinline__ float mx_inverse(uint32_t code) { return code == MX_NAN ? 0.f : __uint_as_float((254u - code) << 23); }

// Eight values, already divided by the scale, to the nearest codes (ties to the even code, above 6 to 6); value i in bits 4 i
__device__ __forceinline__ uint32_t mx_codes(const float *f) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
    return r;
}

// A code's bits s ee m are those of a bf16 with exponent field ee, which is the code's value times 2^-126 (subnormal codes included).
// Codes i and i + 4 of a word as such bf16:
template <int I>
__device__ __forceinline__ uint32_t mx_pair(uint32_t w) {
    const uint32_t s = I < 3 ? w << (12 - 4 * I) : w >> (4 * I - 12);
    const uint32_t e = I == 0 ? w << 6 : I == 1 ? w << 2 : I == 2 ? w >> 2 : w >> 6;
    return (s & 0x80008000u) | (e & 0x01C001C0u);
}

// The two bf16x2 factors that make values of mx_pair's results: 2^126 and the scale in one, but for scales above 2, whose factor would leave the type
struct MxFactors {
    uint32_t first, second;
    bool two;
    __device__ __forceinline__ explicit MxFactors(uint32_t code) {
        two = code > 128u && code != MX_NAN;
        first = (code == MX_NAN ? 0x7fffu : (min(code, 128u) + 126u) << 7) * 0x10001u;
        second = (two ? (code - 1u) << 7 : 0x3f80u) * 0x10001u;
    }
    __device__ __forceinline__ uint32_t value(uint32_t pair) const {
        uint32_t r;
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(pair), "r"(first));
        if (two) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(r) : "r"(second));
        return r;
    }
};
// Eight codes to bf16 (times the scale), in their order
__device__ __forceinline__ bf16x8 mx_values_bf16(uint32_t w, uint32_t code) {
    const MxFactors m(code);
    const uint32_t a = m.value(mx_pair<0>(w)), b = m.value(mx_pair<1>(w)), c = m.value(mx_pair<2>(w)), d = m.value(mx_pair<3>(w));      // (0, 4), (1, 5), (2, 6), (3, 7)
    return bf16x8{{__byte_perm(a, b, 0x5410), __byte_perm(c, d, 0x5410), __byte_perm(a, b, 0x7632), __byte_perm(c, d, 0x7632)}};
}

// Eight codes to float32 (times the scale)
__device__ __forceinline__ void mx_values(uint32_t w, float scale, float *f) {
    const uint32_t p[4] = {mx_pair<0>(w), mx_pair<1>(w), mx_pair<2>(w), mx_pair<3>(w)};
    const float up = __uint_as_float(253u << 23);      // 2^126
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[i] = __uint_as_float(p[i] << 16) * up * scale;
        f[i + 4] = __uint_as_float(p[i] & 0xffff0000u) * up * scale;
    }
}

struct MxProduct {
    const uint4 *codes;                    // weights [out][blocks] of 16 bytes
    const uint8_t *scales;
    const float *bias;
    const __nv_bfloat16 *res;
    void *y;
    unsigned long long rows;
    int blocks, tiles4, out, out_pad, act, out_is_f32;
};

// relu and relu6 that keep a NaN
__device__ __forceinline__ float mx_act(float v, int act) {
    if (act == CPRUNE_ACT_NONE) return v;
    v = v < 0.f ? 0.f : v;
    return act == CPRUNE_ACT_RELU6 && v > 6.f ? 6.f : v;
}

// How a product is shared out (mx_product.cu); tensor == 0: the kernel for few rows takes it
struct MxTiling {
    int tensor;
    int nt, subs, tiles_n;                 // features of a block, in parts of 128; blocks along the features
    int round;                             // the rows are rounded by the product itself
    int features, splits, per;             // features first: shares of the channels, chunks of a share
};
MxTiling mx_tiling(unsigned long long rows, int in, int out);
size_t mx_partial_bytes(const MxTiling &t, unsigned long long rows, int out);
cprune_status launch_mx_product(const MxProduct &q, const MxTiling &t, const void *x, const uint8_t *xscales, int in, float *partial, ChainScope &chain, cudaStream_t st);

}  // namespace cprune
