// Product of many rows with weights in MXFP4 on the block-scaled tensor core path (kind::mxf4: 4-bit operands from shared memory, a power-of-two
// scale per row and 32 channels from tensor memory, float32 sums).
//
// A block takes 128 rows and up to 384 features (each 128 of them one MMA), and goes through the channels 256 at a time: a row of codes of such a
// chunk is 128 bytes.  The rows come in one of two ways:
//   - rounded here: the bf16 rows arrive by TMA, 128 channels at a time; eight warps round them (a thread 64 channels of a row, so that a block
//     of 32 channels never leaves a thread) and write codes and scales where the tensor core reads them.  x is read once and nothing else
//     is written: taken where one block covers all features.
//   - already rounded (by mx_quantize_kernel) where several blocks share the rows: codes by TMA, scales by bulk copies.
// Scales lie in shared memory in pieces of 512 bytes (128 rows by 4 blocks); tcgen05.cp brings a piece into four columns of tensor memory.
// The accumulator leaves through registers: bias, shortcut and activation on the way.
#include <mutex>

#include "common.cuh"
#include "mx.cuh"
#include "plan.h"
#include "sm100_ptx.cuh"

namespace cprune {

constexpr int MXP_ROWS = 128, MXP_CHUNK = 256;        // rows of a block; channels of a chunk (128 bytes of codes)
constexpr int MXP_WARPS = 8;                          // round and store; two more load and multiply
constexpr int MXP_THREADS = (MXP_WARPS + 2) * 32;
constexpr int MXP_XBYTES = MXP_ROWS * 128 * 2;        // 128 channels of bf16 rows
constexpr int MXP_MOST = 384;                         // features of a block
constexpr int MXP_CTRL = 256;

struct MxpParams {
    MxProduct q;
    int nt, subs, box;               // features of a block, in parts of 128; feature rows of a TMA box
    int chunks, halves;              // of 256 and of 128 channels
    int steps_last;                  // MMA steps (64 channels) of the last chunk
    int stages, xstages;
    int b_bytes, tmem_cols, sf_col;  // bytes of a chunk of weights, columns of tensor memory, where its scales begin
    const uint8_t *xscales;          // of rows that are already rounded
    int tiles_n;
    int *status;
};

__device__ __forceinline__ void umma_mxf4(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "mov.b64 da, {%1, %4};\n\t"
        "mov.b64 db, {%2, %4};\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], da, db, %3, [%6], [%7], p;\n\t}"
        :
        : "r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(DESC_HI_SW128), "r"(accumulate), "r"(sfa), "r"(sfb)
        : "memory");
}
// 32 rows of 16 bytes (8-row groups 128 bytes apart) into four columns, the same for every quarter of the lanes
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint32_t smem) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(smem_desc_interleaved(smem, 128)) : "memory");
}

// 32 bf16 values to codes (16 bytes) and a scale
__device__ __forceinline__ uint4 mx_round_block(const bf16x8 *v, uint32_t &scale) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = __vmaxu2(top, v[i].w[j] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16) << 16;
    scale = mx_scale_code(top);
    const float inverse = mx_inverse(scale);
    const bool none = scale == MX_NAN;
    uint4 r;
    uint32_t *w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f[8];
        unpack8(v[i], f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = f[j] * inverse;
        w[i] = none ? 0u : mx_codes(f);
    }
    return r;
}

template <bool ROUND>
__global__ void __launch_bounds__(MXP_THREADS) mx_product_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ MxpParams p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    // shared memory: codes of the rows, codes of the features, bf16 rows, scales of rows and of features, barriers, bias
    const uint32_t a0 = base, b0 = a0 + p.stages * 16384u, x0 = b0 + (uint32_t)(p.stages * p.b_bytes), sa0 = x0 + (uint32_t)(p.xstages * MXP_XBYTES);
    const uint32_t sb0 = sa0 + p.stages * 1024u, ctrl0 = sb0 + (uint32_t)(p.stages * p.subs) * 1024u;
    uint8_t *ctrl = smem + (ctrl0 - base);
    auto xfull = [&](int s) { return ctrl0 + 8u * s; };
    auto xempty = [&](int s) { return ctrl0 + 32u + 8u * s; };
    auto afull = [&](int s) { return ctrl0 + 64u + 8u * s; };          // rows rounded
    auto bfull = [&](int s) { return ctrl0 + 96u + 8u * s; };          // weights (and rounded rows) here
    auto empty = [&](int s) { return ctrl0 + 128u + 8u * s; };         // the MMAs have read a stage
    const uint32_t done = ctrl0 + 160u;
    uint32_t *tmem_slot = (uint32_t *)(ctrl + 168);
    volatile int *abort_flag = (volatile int *)(ctrl + 172);
    float *bias_s = (float *)(ctrl + MXP_CTRL);

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int tile_n = blockIdx.x % p.tiles_n;
    const long long row0 = (long long)(blockIdx.x / p.tiles_n) * MXP_ROWS;
    const int o0 = tile_n * p.nt;
    if (warp == MXP_WARPS) {
        tmem_alloc(smem_u32(tmem_slot), (uint32_t)p.tmem_cols);
        tmem_relinquish();
        pdl_trigger();
        if (lane == 0) {
            for (int s = 0; s < p.xstages; ++s) { mbar_init(xfull(s), 1); mbar_init(xempty(s), MXP_WARPS); }
            for (int s = 0; s < p.stages; ++s) { mbar_init(afull(s), 2 * MXP_WARPS); mbar_init(bfull(s), 1); mbar_init(empty(s), 1); }
            mbar_init(done, 1);
            *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    } else if (warp < MXP_WARPS) {
        for (int e = threadIdx.x; e < p.nt; e += MXP_WARPS * 32) bias_s[e] = o0 + e < p.q.out ? __ldg(p.q.bias + o0 + e) : 0.f;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    bool ok = true;
    pdl_wait();

    if (warp == MXP_WARPS) {
        // -------------------------------------------------------------------------------------------- loads
        int half = 0;
        auto load_x = [&](int h) {
            const int s = h % p.xstages;
            if (h >= p.xstages) ok = __all_sync(0xffffffffu, mbar_wait(xempty(s), (uint32_t)(h / p.xstages - 1) & 1u, abort_flag, p.status));
            if (ok && elect_one()) {
                mbar_expect_tx(xfull(s), MXP_XBYTES);
                tma_load_2d(x0 + (uint32_t)s * MXP_XBYTES, &tm_x, xfull(s), h * 128, (int)row0);
                tma_load_2d(x0 + (uint32_t)s * MXP_XBYTES + 16384u, &tm_x, xfull(s), h * 128 + 64, (int)row0);
            }
            __syncwarp();
        };
        for (int c = 0; c < p.chunks && ok; ++c) {
            const int s = c % p.stages, tiles = min(2, p.q.tiles4 - 2 * c);
            if (c >= p.stages) ok = __all_sync(0xffffffffu, mbar_wait(empty(s), (uint32_t)(c / p.stages - 1) & 1u, abort_flag, p.status));
            if (ok && elect_one()) {
                const int row_tiles = min(p.subs, (p.q.out + 127) / 128 - o0 / 128);       // tiles of scales that there are
                mbar_expect_tx(bfull(s), (uint32_t)(p.subs * p.box * 128 + row_tiles * tiles * 512 + (ROUND ? 0 : 16384 + tiles * 512)));
                for (int n = 0; n < p.subs; ++n) tma_load_2d(b0 + (uint32_t)(s * p.b_bytes + n * 16384), &tm_w, bfull(s), c * 64, o0 + n * 128);
                for (int n = 0; n < row_tiles; ++n)
                    bulk_load(sb0 + (uint32_t)((s * p.subs + n) * 1024), p.q.scales + ((size_t)(o0 / 128 + n) * p.q.tiles4 + 2 * c) * 512, (uint32_t)tiles * 512u, bfull(s));
                if (!ROUND) {
                    tma_load_2d(a0 + (uint32_t)s * 16384u, &tm_x, bfull(s), c * 64, (int)row0);
                    bulk_load(sa0 + (uint32_t)s * 1024u, p.xscales + ((size_t)(row0 / 128) * p.q.tiles4 + 2 * c) * 512, (uint32_t)tiles * 512u, bfull(s));
                }
            }
            __syncwarp();
            if (ROUND)
                for (; half < p.halves && half < 2 * c + 2 && ok; ++half) load_x(half);
        }
    } else if (warp == MXP_WARPS + 1) {
        // --------------------------------------------------------------------------------------------- MMAs
        // E2M1 operands, scales that are powers of two; 64 channels of every 128 under scales 0 or 2 of a column
        const uint32_t idesc = (1u << 7) | (1u << 10) | (1u << 23) | (1u << 27);
        for (int c = 0; c < p.chunks && ok; ++c) {
            const int s = c % p.stages;
            const uint32_t parity = (uint32_t)(c / p.stages) & 1u;
            ok = __all_sync(0xffffffffu, mbar_wait(bfull(s), parity, abort_flag, p.status));
            if (ROUND) ok = ok && __all_sync(0xffffffffu, mbar_wait(afull(s), parity, abort_flag, p.status));
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                // (features that begin in the middle of a piece of scales: a column has those of 32)
                const uint32_t sfa = tmem_base + (uint32_t)(p.sf_col + s * 8 * (p.subs + 1)), sfb = sfa + 8u, first = (uint32_t)(o0 % 128) / 32u;
                const int steps = c + 1 == p.chunks ? p.steps_last : 4;
                for (int h = 0; 2 * h < steps; ++h) {
                    tmem_copy_scales(sfa + 4u * h, sa0 + (uint32_t)(s * 1024 + h * 512));
                    for (int n = 0; n < p.subs; ++n) tmem_copy_scales(sfb + (uint32_t)(h * p.subs + n) * 4u, sb0 + (uint32_t)((s * p.subs + n) * 1024 + h * 512));
                }
                for (int k = 0; k < steps; ++k) {
                    const uint32_t a = desc_lo(a0 + (uint32_t)s * 16384u) + 2u * k, id = (uint32_t)(k & 1) * 2u;
                    for (int n = 0; n < p.subs; ++n) {
                        const uint32_t b = desc_lo(b0 + (uint32_t)(s * p.b_bytes + n * 16384)) + 2u * k;
                        const int width = min(128, p.nt - n * 128);
                        umma_mxf4(tmem_base + (uint32_t)(n * 128), a, b, idesc | (uint32_t)(width >> 3) << 17 | id << 29 | id << 4, sfa + 4u * (k >> 1),
                                  sfb + (uint32_t)((k >> 1) * p.subs + n) * 4u + first, (c | k) ? 1u : 0u);
                    }
                }
                umma_commit(empty(s));
                if (c + 1 == p.chunks) umma_commit(done);
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------------------------------------ rounding
        const int r = threadIdx.x & 127, box = threadIdx.x >> 7;           // a row, and 64 of a half's 128 channels
        if (ROUND)
            for (int c = 0; c < p.chunks && ok; ++c) {
                const int s = c % p.stages;
                if (c >= p.stages) ok = __all_sync(0xffffffffu, mbar_wait(empty(s), (uint32_t)(c / p.stages - 1) & 1u, abort_flag, p.status));
                for (int part = 0; part < 2 && ok; ++part) {
                    const int h = 2 * c + part;
                    if (h < p.halves) {
                        const int xs = h % p.xstages;
                        ok = __all_sync(0xffffffffu, mbar_wait(xfull(xs), (uint32_t)(h / p.xstages) & 1u, abort_flag, p.status));
                        if (!ok) break;
                        const uint8_t *in = smem + (x0 - base) + xs * MXP_XBYTES + box * 16384;
                        uint8_t *out = smem + (a0 - base) + s * 16384;
                        uint32_t scales = 0;
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            bf16x8 v[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const bf16x8 *>(in + sub_off(r, b * 4 + i));
                            uint32_t code;
                            const uint4 w = mx_round_block(v, code);
                            *reinterpret_cast<uint4 *>(out + sub_off(r, part * 4 + box * 2 + b)) = w;
                            scales |= code << (8 * b);
                        }
                        *reinterpret_cast<uint16_t *>(smem + (sa0 - base) + s * 1024 + part * 512 + (r & 31) * 16 + (r >> 5) * 4 + box * 2) = (uint16_t)scales;
                        fence_async_smem();                // the tensor core reads what was written here
                        __syncwarp();
                        if (lane == 0) mbar_arrive(xempty(xs));
                    }
                    if (lane == 0) mbar_arrive(afull(s));
                }
            }
        // ------------------------------------------------------------------------------------------ epilogue
        ok = ok && __all_sync(0xffffffffu, mbar_wait(done, 0u, abort_flag, p.status));
        if (ok) {
            tc_fence_after();
            const int quarter = warp & 3;
            const long long row = row0 + quarter * 32 + lane;
            const bool in = row < (long long)p.q.rows;
            for (int u = warp >> 2; u * 16 < p.nt; u += 2) {
                const int o = o0 + u * 16;
                if (o >= p.q.out_pad) break;
                bf16x8 rv[2] = {};
                if (p.q.res && in) {
                    rv[0] = *reinterpret_cast<const bf16x8 *>(p.q.res + (size_t)row * p.q.out_pad + o);
                    if (o + 8 < p.q.out_pad) rv[1] = *reinterpret_cast<const bf16x8 *>(p.q.res + (size_t)row * p.q.out_pad + o + 8);
                }
                uint32_t v[16];
                tmem_ld16(tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(u * 16), v);
                tmem_ld_wait();
                float f[16], g[16];
                unpack8(rv[0], g);
                unpack8(rv[1], g + 8);
#pragma unroll
                for (int j = 0; j < 16; ++j) f[j] = o + j < p.q.out ? mx_act(__uint_as_float(v[j]) + bias_s[u * 16 + j] + g[j], p.q.act) : 0.f;
                if (!in) continue;
                if (p.q.out_is_f32) {
                    float *y = (float *)p.q.y + (size_t)row * p.q.out + o;
                    if (((uintptr_t)y & 15) == 0 && o + 16 <= p.q.out) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) reinterpret_cast<float4 *>(y)[j] = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (o + j < p.q.out) y[j] = f[j];
                    }
                } else {
                    __nv_bfloat16 *y = (__nv_bfloat16 *)p.q.y + (size_t)row * p.q.out_pad + o;
                    *reinterpret_cast<bf16x8 *>(y) = pack8(f);
                    if (o + 8 < p.q.out_pad) *reinterpret_cast<bf16x8 *>(y + 8) = pack8(f + 8);
                }
            }
        }
    }

    __syncwarp();
    if (*abort_flag) {
        for (int i = 0; i < 200; ++i) __nanosleep(1000);   // let copies in flight land before the memory goes away
    }
    tc_fence_before();
    __syncthreads();
    if (warp == MXP_WARPS) {
        tc_fence_after();
        tmem_dealloc(tmem_base, (uint32_t)p.tmem_cols);
    }
}

// How a product is shared out
MxTiling mx_tiling(unsigned long long rows, int in, int out) {
    MxTiling t = {};
    const long long tiles_m = (long long)((rows + MXP_ROWS - 1) / MXP_ROWS);
    const int all = round_up(out, 16);
    t.nt = all <= MXP_MOST ? all : 256;
    // fewer features to a block while that leaves SMs without one
    while (t.nt > 64 && tiles_m * ((all + t.nt - 1) / t.nt) * 2 <= 148) t.nt = t.nt > 256 ? 256 : t.nt > 128 ? 128 : 64;
    t.tiles_n = (all + t.nt - 1) / t.nt;
    t.subs = (t.nt + 127) / 128;
    t.round = t.tiles_n == 1;
    t.tensor = 1;
    return t;
}

template <bool ROUND>
static cprune_status launch_product(const CUtensorMap *tm, const MxpParams &p, long long blocks, size_t smem, cudaStream_t st) {
    static std::mutex attr_mu;
    static bool attr_set[64] = {false};    // the shared-memory limit of a kernel is a per-device attribute
    {
        int dev = 0;
        CPRUNE_CUDA_CHECK(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64) return CPRUNE_ERR_UNSUPPORTED;
        std::lock_guard<std::mutex> lock(attr_mu);
        if (!attr_set[dev]) {
            CPRUNE_CUDA_CHECK(cudaFuncSetAttribute(mx_product_kernel<ROUND>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
            attr_set[dev] = true;
        }
    }
    CPRUNE_CUDA_CHECK(launch_chained(mx_product_kernel<ROUND>, dim3((unsigned)blocks), dim3(MXP_THREADS), smem, st, tm[0], tm[1], p));
    return CPRUNE_OK;
}

// x: bf16 rows (t.round), else their codes, with their scales behind them
cprune_status launch_mx_product(const MxProduct &q, const MxTiling &t, const void *x, const uint8_t *xscales, int in, cudaStream_t st) {
    MxpParams p = {};
    p.q = q;
    p.nt = t.nt; p.subs = t.subs; p.tiles_n = t.tiles_n;
    p.box = t.nt < 128 ? t.nt : 128;
    p.chunks = (in + MXP_CHUNK - 1) / MXP_CHUNK;
    p.halves = (in + 127) / 128;
    p.steps_last = (in - (p.chunks - 1) * MXP_CHUNK + 63) / 64;
    p.b_bytes = t.subs * 16384;
    p.xscales = xscales;
    p.status = device_status_word();
    if (!p.status) return cuda_fail(cudaGetLastError(), "status word");
    p.sf_col = t.nt;
    auto bytes = [&](int stages, int xstages) {
        return 1024 + (size_t)stages * (16384 + p.b_bytes + 1024 + t.subs * 1024) + (size_t)xstages * MXP_XBYTES + MXP_CTRL + (size_t)t.nt * 4;
    };
    p.stages = p.chunks < 4 ? p.chunks : 4;
    p.xstages = t.round ? (p.halves < 4 ? p.halves : 4) : 0;
    while (bytes(p.stages, p.xstages) > 113 * 1024 && (p.stages > 2 || p.xstages > 2)) {
        if (p.xstages > 2) --p.xstages;
        else --p.stages;
    }
    while (p.stages > 1 && p.sf_col + p.stages * 8 * (t.subs + 1) > 512) --p.stages;
    const int cols = p.sf_col + p.stages * 8 * (t.subs + 1);
    for (p.tmem_cols = 32; p.tmem_cols < cols;) p.tmem_cols *= 2;
    CUtensorMap tm[2];
    const unsigned long long kb = q.blocks;
    {
        const unsigned long long dims[2] = {t.round ? (unsigned long long)in : kb * 8, q.rows};
        const unsigned long long strides[1] = {t.round ? (unsigned long long)cprune_padded_channels(in) * 2 : kb * 16};
        const unsigned box[2] = {64, MXP_ROWS};
        cprune_status s = encode_tiled_bf16_swz(&tm[0], x, 2, dims, strides, box, 128, true);
        if (s != CPRUNE_OK) return s;
    }
    {
        const unsigned long long dims[2] = {kb * 8, (unsigned long long)q.out};
        const unsigned long long strides[1] = {kb * 16};
        const unsigned box[2] = {64, (unsigned)p.box};
        cprune_status s = encode_tiled_bf16_swz(&tm[1], q.codes, 2, dims, strides, box, 128, true);
        if (s != CPRUNE_OK) return s;
    }
    const long long blocks = (long long)((q.rows + MXP_ROWS - 1) / MXP_ROWS) * t.tiles_n;
    if (blocks > 0x7fffffffLL) return CPRUNE_ERR_UNSUPPORTED;
    const size_t smem = bytes(p.stages, p.xstages);
    return t.round ? launch_product<true>(tm, p, blocks, smem, st) : launch_product<false>(tm, p, blocks, smem, st);
}

}  // namespace cprune
