// Product of many rows with weights in MXFP4 on the block-scaled tensor core path (kind::mxf4: 4-bit operands from shared memory, a power-of-two
// scale per row and 32 channels from tensor memory, float32 sums).
//
// A block takes 128 rows and up to 384 features (each 128 of them one MMA), and goes through the channels 256 at a time: a row of codes of such a
// chunk is 128 bytes.  The rows come in one of two ways:
//   - rounded here: the bf16 rows arrive by TMA, 64 channels at a time; two groups of eight warps round them in turn, a thread a block of 32 channels of a
//     row, and write codes and scales where the tensor core reads them.  x is read once and nothing else is written: taken where one block covers all
//     features.
//   - already rounded (by mx_quantize_kernel) where several blocks share the rows: codes by TMA, scales by bulk copies.
// Up to 128 rows change places with the features: a block takes 128 features and all rows, and a share of the channels (so that enough blocks read the
// weights, which is what such a product consists of); the shares' sums meet in a second kernel, in a fixed order.
// Scales lie in shared memory in pieces of 512 bytes (128 rows by 4 blocks); tcgen05.cp brings a piece into four columns of tensor memory.
// The accumulator leaves through registers: bias, shortcut and activation on the way.  It takes 64 channels a step, and every step truncates: sums of one sign,
// with 129 or more rows, are off by 40 units of 2^-23 after 392 steps (25088 channels), 316 after 2048, 2770 after 16384.  For the networks' layers that is far
// below a bf16 result's half step (32768 units); sums of shares, as of few rows, would cost the shares' way through memory.
// What bounds it: products of a network's 1x1 layers are small, and a block's time is the latency of its parts one after the other.  12544 x 960 -> 320 with
// a shortcut (40 MB, 6.2 us at a copy's rate) takes 15.8 us: 98 blocks for 148 SMs, of 13 us each 2.5 until the first rows are there, 6 for the rows (16 KB every
// 450 ns, six boxes under way) and 4 for the epilogue.  Large images of few channels are bound by the same sequence, once per 128 rows: 200704 x 24 -> 144 43 us and
// 200704 x 144 -> 24 36, where the bf16 layer (cprune_task_run) takes 24.3 and 16.5.  4096 x 4096 -> 4096, with the rounding: 72 us, 1900 TFLOP/s, 1.2 times the rate of bf16 matrix products.
#include <cstring>
#include <mutex>

#include "common.cuh"
#include "mx.cuh"
#include "plan.h"
#include "sm100_ptx.cuh"

namespace cprune {

constexpr int MXP_ROWS = 128, MXP_CHUNK = 256;        // rows of a block; channels of a chunk (128 bytes of codes)
constexpr int MXP_WARPS = 16;                         // round and store; two more load and multiply
constexpr int MXP_THREADS = (MXP_WARPS + 2) * 32;
constexpr int MXP_XBYTES = MXP_ROWS * 64 * 2;         // 64 channels of bf16 rows
constexpr int MXP_MOST = 384;                         // features of a block
constexpr int MXP_CTRL = 512, MXP_FRONT = 2048;       // barriers; with the bias behind them
constexpr int MXP_SF_COLS = 8 + 2 * 12;               // columns of a stage's scales

struct MxpParams {
    MxProduct q;
    int nt, subs, box;               // features of a block, in parts of 128; rows of a TMA box of them
    int chunks, boxes;               // of 256 and of 64 channels
    int steps_last;                  // MMA steps (64 channels) of the last chunk
    int stages, xstages;
    int panels;                      // of 64 features, of a shortcut: they take places in the ring of the rows
    int groups;                      // of four warps that take the panels in turn
    int b_bytes, tmem_cols, sf_col;  // bytes of a chunk of weights, columns of tensor memory, where its scales begin
    const uint8_t *xscales;          // of rows that are already rounded
    float *partial;                  // features first: sums of the shares [splits][rows][out_pad]
    int tiles_n;                     // blocks along the features; features first: shares of the channels
    int per;                         // chunks of a share
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
constexpr uint32_t DESC_HI_SCALES = (128u >> 4) | (1u << 14);
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint32_t desc_lo) {
    asm volatile("{\n\t.reg .b64 d;\n\tmov.b64 d, {%1, %2};\n\ttcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}" ::"r"(taddr), "r"(desc_lo), "r"(DESC_HI_SCALES) : "memory");
}

// 32 bf16 values to codes (16 bytes) and a scale.  The largest magnitude and the division by the scale are taken two values at a time, as bf16: products
// with a power of two are exact there too (what leaves the type below is far under the smallest code).
__device__ __forceinline__ uint4 mx_round_block(const bf16x8 *v, uint32_t &scale) {
    uint32_t m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = v[i].w[0] & 0x7fff7fffu;
#pragma unroll
        for (int j = 1; j < 4; ++j) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m[i]) : "r"(v[i].w[j] & 0x7fff7fffu));
    }
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m[0]) : "r"(m[1]));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m[2]) : "r"(m[3]));
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m[0]) : "r"(m[2]));
    const uint32_t top = max(m[0] & 0x7fffu, m[0] >> 16 & 0x7fffu) << 16;
    scale = mx_scale_code(top);
    const bool none = scale == MX_NAN;
    const uint32_t inverse = (__float_as_uint(mx_inverse(scale)) >> 16) * 0x10001u;
    uint4 r;
    uint32_t *w = &r.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x8 q;
#pragma unroll
        for (int j = 0; j < 4; ++j) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(q.w[j]) : "r"(v[i].w[j]), "r"(inverse));
        float f[8];
        unpack8(q, f);
        w[i] = none ? 0u : mx_codes(f);
    }
    return r;
}

// relu and relu6 of bf16 values, which keep a NaN; 0 and 6 are bf16 values, so that the clamp may follow the rounding
__device__ __forceinline__ bf16x8 mx_clamp8(bf16x8 v, int act) {
    if (act != CPRUNE_ACT_NONE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(v.w[i]) : "r"(0u));
        if (act == CPRUNE_ACT_RELU6) {
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("min.NaN.bf16x2 %0, %0, %1;" : "+r"(v.w[i]) : "r"(0x40C040C0u));
        }
    }
    return v;
}

enum { MXP_ROUND = 0, MXP_CODES = 1, MXP_FEATURES = 2 };        // rows rounded here; rows already rounded; features first

template <int FORM>
__global__ void __launch_bounds__(MXP_THREADS) mx_product_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_y, const __grid_constant__ CUtensorMap tm_res,
                  const __grid_constant__ MxpParams p) {
    constexpr bool ROUND = FORM == MXP_ROUND, FEATURES = FORM == MXP_FEATURES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    // shared memory: barriers, bias, codes of the rows (features first: of the features), codes of the features (of the rows), bf16 rows, scales of rows and of features
    const uint32_t ctrl0 = base, a0 = base + MXP_FRONT, b0 = a0 + p.stages * 16384u, x0 = b0 + (uint32_t)(p.stages * p.b_bytes);
    const uint32_t sa0 = x0 + (uint32_t)(p.xstages * MXP_XBYTES), sb0 = sa0 + p.stages * 1024u;
    uint8_t *ctrl = smem + (ctrl0 - base);
    auto xfull = [&](int s) { return ctrl0 + 8u * s; };
    auto xempty = [&](int s) { return ctrl0 + 64u + 8u * s; };
    auto afull = [&](int s) { return ctrl0 + 128u + 8u * s; };         // rows rounded
    auto bfull = [&](int s) { return ctrl0 + 192u + 8u * s; };         // weights (and rounded rows) here
    auto empty = [&](int s) { return ctrl0 + 256u + 8u * s; };         // the MMAs have read a stage
    const uint32_t done = ctrl0 + 320u;
    uint32_t *tmem_slot = (uint32_t *)(ctrl + 328);
    volatile int *abort_flag = (volatile int *)(ctrl + 332);
    float *bias_s = (float *)(ctrl + MXP_CTRL);

    const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const int tile_n = blockIdx.x % p.tiles_n;
    const long long row0 = (long long)(blockIdx.x / p.tiles_n) * MXP_ROWS;       // (features first: the first feature)
    const int o0 = FEATURES ? 0 : tile_n * p.nt;                                 // (... the first row)
    const int c_begin = FEATURES ? tile_n * p.per : 0, c_end = FEATURES ? min(p.chunks, c_begin + p.per) : p.chunks;
    if (warp == MXP_WARPS) {
        tmem_alloc(smem_u32(tmem_slot), (uint32_t)p.tmem_cols);
        tmem_relinquish();
        pdl_trigger();
        if (lane == 0) {
            for (int s = 0; s < p.xstages; ++s) { mbar_init(xfull(s), 1); mbar_init(xempty(s), MXP_WARPS / 2); }
            for (int s = 0; s < p.stages; ++s) { mbar_init(afull(s), MXP_WARPS); mbar_init(bfull(s), 1); mbar_init(empty(s), 1); }
            mbar_init(done, 1);
            *abort_flag = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
    } else if (warp == MXP_WARPS + 1) {
        if (elect_one()) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_x) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_w) : "memory");
            if (!FEATURES) asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_y) : "memory");
            if (!FEATURES) asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_res) : "memory");
        }
        __syncwarp();
    } else if (!FEATURES) {
        for (int e = threadIdx.x; e < p.nt; e += MXP_WARPS * 32) bias_s[e] = o0 + e < p.q.out ? __ldg(p.q.bias + o0 + e) : 0.f;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    bool ok = true;

    // The weights are nobody's result: those of the first chunks are asked for before the preceding kernel has finished, in the form that rounds by the warp
    // that multiplies, so that the rows' boxes need not queue behind them.
    const uint32_t w0 = FEATURES ? a0 : b0, w_step = FEATURES ? 16384u : (uint32_t)p.b_bytes, ws0 = FEATURES ? sa0 : sb0;
    const int w_first = FEATURES ? (int)row0 : o0, w_box = FEATURES ? MXP_ROWS : p.box, w_rows = FEATURES ? MXP_ROWS : p.nt;
    const int w_parts = FEATURES ? 1 : p.subs, w_tiles = min(w_parts, (p.q.out + 127) / 128 - w_first / 128);         // tiles of scales that there are
    auto scale_tiles = [&](int c) { return min(2, p.q.tiles4 - 2 * c); };
    auto load_w = [&](int c, int s) {
        const int tiles = scale_tiles(c);
        const uint32_t rows = ROUND ? 0u : (uint32_t)((FEATURES ? p.box * 128 : 16384) + tiles * 512);
        mbar_expect_tx(bfull(s), (uint32_t)(w_rows * 128 + w_tiles * tiles * 512) + rows);
        for (int n = 0; n < w_rows; n += w_box) tma_load_2d(w0 + (uint32_t)s * w_step + (uint32_t)n * 128u, &tm_w, bfull(s), c * 64, w_first + n);
        for (int n = 0; n < w_tiles; ++n)
            bulk_load(ws0 + (uint32_t)((s * w_parts + n) * 1024), p.q.scales + ((size_t)(w_first / 128 + n) * p.q.tiles4 + 2 * c) * 512, (uint32_t)tiles * 512u, bfull(s));
    };
    const int ahead = min(p.stages, c_end - c_begin);
    auto load_first = [&]() {
        if (elect_one())
            for (int i = 0; i < ahead; ++i) load_w(c_begin + i, i);
        __syncwarp();
    };

    if (warp == MXP_WARPS) {
        // -------------------------------------------------------------------------------------------- loads
        auto load_rows = [&](int c, int s) {
            if (ROUND) return;
            const int first = FEATURES ? 0 : (int)row0;
            tma_load_2d(FEATURES ? b0 + (uint32_t)(s * p.b_bytes) : a0 + (uint32_t)s * 16384u, &tm_x, bfull(s), c * 64, first);
            bulk_load((FEATURES ? sb0 : sa0) + (uint32_t)s * 1024u, p.xscales + ((size_t)(first / 128) * p.q.tiles4 + 2 * c) * 512, (uint32_t)scale_tiles(c) * 512u, bfull(s));
        };
        auto load_x = [&](int h) {                         // (the shortcut's panels follow the rows' boxes)
            const int s = h % p.xstages;
            if (h >= p.xstages) ok = __all_sync(0xffffffffu, mbar_wait(xempty(s), (uint32_t)(h / p.xstages - 1) & 1u, abort_flag, p.status));
            if (ok && elect_one()) {
                mbar_expect_tx(xfull(s), MXP_XBYTES);
                if (h < p.boxes) tma_load_2d(x0 + (uint32_t)s * MXP_XBYTES, &tm_x, xfull(s), h * 64, (int)row0);
                else tma_load_2d(x0 + (uint32_t)s * MXP_XBYTES, &tm_res, xfull(s), o0 + (h - p.boxes) * 64, (int)row0);
            }
            __syncwarp();
        };
        if (!ROUND) load_first();
        pdl_wait();
        int box = 0;
        for (int i = 0; c_begin + i < c_end && ok; ++i) {
            const int c = c_begin + i, s = i % p.stages;
            // (a chunk's boxes before its weights, which wait for MMAs of boxes that were asked for long ago)
            if (ROUND)
                for (; box < p.boxes && box < 4 * c + 4 && ok; ++box) load_x(box);
            if (i >= p.stages && ok) ok = __all_sync(0xffffffffu, mbar_wait(empty(s), (uint32_t)(i / p.stages - 1) & 1u, abort_flag, p.status));
            if (ok && elect_one()) {
                if (i >= ahead) load_w(c, s);
                load_rows(c, s);
            }
            __syncwarp();
        }
        const int panels = min(p.panels, (p.q.out_pad - o0 + 63) / 64);
        for (box = p.boxes; box < p.boxes + panels && ok; ++box) load_x(box);
    } else if (warp == MXP_WARPS + 1) {
        // --------------------------------------------------------------------------------------------- MMAs
        if (ROUND) load_first();
        // E2M1 operands, scales that are powers of two; 64 channels of every 128 under scales 0 or 2 of a column
        const uint32_t idesc = (1u << 7) | (1u << 10) | (1u << 23) | (1u << 27), idesc_128 = idesc | 16u << 17;
        const uint32_t idesc_last = idesc | (uint32_t)((p.nt - (p.subs - 1) * 128) >> 3) << 17;
        const uint32_t a_lo = desc_lo(a0), b_lo = desc_lo(b0), b_step = (uint32_t)p.b_bytes >> 4, sa_lo = desc_lo(sa0), sb_lo = desc_lo(sb0), cb_step = (uint32_t)p.subs * 64u;
        // a stage's scales: 8 columns of the rows', 2 x 12 of the features' (those that begin in the middle of a piece: a column has those of 32)
        const uint32_t sf_base = tmem_base + (uint32_t)p.sf_col, sf_step = MXP_SF_COLS, first = (uint32_t)(o0 % 128) / 32u;
        for (int i = 0; c_begin + i < c_end && ok; ++i) {
            const int c = c_begin + i, s = i % p.stages;
            const uint32_t parity = (uint32_t)(i / p.stages) & 1u;
            ok = __all_sync(0xffffffffu, mbar_wait(bfull(s), parity, abort_flag, p.status));
            if (ROUND) ok = ok && __all_sync(0xffffffffu, mbar_wait(afull(s), parity, abort_flag, p.status));
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                // (One thread issues all of it, so that every instruction of address arithmetic counts: written out, with additions only.)
                const int steps = c + 1 == p.chunks ? p.steps_last : 4;
                const uint32_t sfa = sf_base + (uint32_t)s * sf_step, a = a_lo + (uint32_t)s * 1024u, b = b_lo + (uint32_t)s * b_step;
                const uint32_t ca = sa_lo + (uint32_t)s * 64u, cb = sb_lo + (uint32_t)s * cb_step;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (2 * h >= steps) break;
                    tmem_copy_scales(sfa + 4u * h, ca + 32u * h);
#pragma unroll
                    for (int n = 0; n < MXP_MOST / 128; ++n)
                        if (n < p.subs) tmem_copy_scales(sfa + 8u + 12u * h + 4u * n, cb + 64u * n + 32u * h);
                }
                const uint32_t sfb = sfa + 8u + first;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k >= steps) break;
#pragma unroll
                    for (int n = 0; n < MXP_MOST / 128; ++n)
                        if (n < p.subs)
                            umma_mxf4(tmem_base + 128u * n, a + 2u * k, b + 1024u * n + 2u * k, (n + 1 < p.subs ? idesc_128 : idesc_last) + (k & 1) * ((2u << 29) | (2u << 4)),
                                      sfa + 4u * (k >> 1), sfb + 12u * (k >> 1) + 4u * n, (i | k) ? 1u : 0u);
                }
                umma_commit(empty(s));
                if (c + 1 == c_end) umma_commit(done);
            }
            __syncwarp();
        }
    } else {
        // ------------------------------------------------------------------------------------------ rounding
        const int r = threadIdx.x & 127, half = (threadIdx.x >> 7) & 1, turn = warp >> 3;          // a row, 32 of a box's 64 channels, every second box
        if (ROUND) {
            const uint8_t *in = smem + (x0 - base);
            uint8_t *out = smem + (a0 - base), *scales = smem + (sa0 - base) + (r & 31) * 16 + (r >> 5) * 4 + half;
            for (int c = 0; c < p.chunks && ok; ++c) {
                const int s = c % p.stages;
                if (c >= p.stages) ok = __all_sync(0xffffffffu, mbar_wait(empty(s), (uint32_t)(c / p.stages - 1) & 1u, abort_flag, p.status));
#pragma unroll 1
                for (int part = turn; part < 4 && 4 * c + part < p.boxes && ok; part += 2) {
                    const int h = 4 * c + part, xs = h % p.xstages;
                    ok = __all_sync(0xffffffffu, mbar_wait(xfull(xs), (uint32_t)(h / p.xstages) & 1u, abort_flag, p.status));
                    if (!ok) break;
                    bf16x8 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const bf16x8 *>(in + xs * MXP_XBYTES + sub_off(r, half * 4 + i));
                    uint32_t code;
                    *reinterpret_cast<uint4 *>(out + s * 16384 + sub_off(r, part * 2 + half)) = mx_round_block(v, code);
                    scales[s * 1024 + (part >> 1) * 512 + (part & 1) * 2] = (uint8_t)code;
                    // (The place is given back once the codes are written, that is, once all values are in registers: given back between the loads and their
                    // first use, the next box overtook loads of warps that had to wait for the scheduler.)
                    __syncwarp();
                    if (lane == 0) mbar_arrive(xempty(xs));
                }
                fence_async_smem();                        // the tensor core reads what was written here
                __syncwarp();
                if (lane == 0) mbar_arrive(afull(s));
            }
        }
        // ------------------------------------------------------------------------------------------ epilogue
        pdl_wait();
        const int quarter = warp & 3;
        const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16);
        if (FEATURES) {
            // a lane has a feature, a column is a row
            ok = __all_sync(0xffffffffu, mbar_wait(done, 0u, abort_flag, p.status));
            if (ok) {
                tc_fence_after();
                const int o = (int)row0 + quarter * 32 + lane;
                for (int u = warp >> 2; u * 16 < p.nt; u += MXP_WARPS / 4) {
                    uint32_t v[16];
                    tmem_ld16(t_lane + (uint32_t)(u * 16), v);
                    tmem_ld_wait();
                    float *to = p.partial + ((size_t)tile_n * p.q.rows + u * 16) * p.q.out_pad + o;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (u * 16 + j < (int)p.q.rows && o < p.q.out) to[(size_t)j * p.q.out_pad] = __uint_as_float(v[j]);
                }
            }
        } else if (!p.q.out_is_f32) {
            // A warp takes 32 rows of 64 features (a panel's quarter, 4 KB) at a time and leaves them to a bulk store: over the shortcut's panel where there is
            // one, else in codes that the MMAs have read.
            const int panels = (min(p.nt, p.q.out_pad - o0) + 63) / 64;
            ok = ok && __all_sync(0xffffffffu, mbar_wait(done, 0u, abort_flag, p.status));
            for (int panel = warp >> 2 < p.groups ? warp >> 2 : panels; panel < panels && ok; panel += p.groups) {
                const int left = min(64, p.nt - panel * 64);                       // (whole sixteens)
                uint32_t from = a0 + (uint32_t)warp * 4096u;
                if (p.panels) {
                    const int h = p.boxes + panel, s = h % p.xstages;
                    ok = __all_sync(0xffffffffu, mbar_wait(xfull(s), (uint32_t)(h / p.xstages) & 1u, abort_flag, p.status));
                    if (!ok) break;
                    from = x0 + (uint32_t)(s * MXP_XBYTES + quarter * 4096);
                } else if (panel >= p.groups) {
                    tma_store_wait_read<0>();              // (by the thread that stored)
                    __syncwarp();
                }
                uint8_t *stage = smem + (from - base);
                tc_fence_after();
                // (a short loop: its instructions come from memory the first time; 12544 x 960 -> 320 written out for 64 features 16.7 us, for 32 16.3, now 15.8)
#pragma unroll 1
                for (int u = 0; u < 4; ++u) {
                    if (u * 16 >= left) break;
                    uint32_t v[16];
                    tmem_ld16(t_lane + (uint32_t)(panel * 64 + u * 16), v);
                    tmem_ld_wait();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        bf16x8 *at = reinterpret_cast<bf16x8 *>(stage + sub_off(lane, u * 2 + h));
                        const int e = panel * 64 + u * 16 + h * 8;
                        const float4 b0v = *reinterpret_cast<const float4 *>(bias_s + e), b1v = *reinterpret_cast<const float4 *>(bias_s + e + 4);
                        float f[8] = {b0v.x, b0v.y, b0v.z, b0v.w, b1v.x, b1v.y, b1v.z, b1v.w};
#pragma unroll
                        for (int j = 0; j < 8; ++j) f[j] += __uint_as_float(v[8 * h + j]);
                        if (p.panels) {
                            float g[8];
                            unpack8(*at, g);
#pragma unroll
                            for (int j = 0; j < 8; ++j) f[j] += g[j];
                        }
                        // (features behind the last have zero weights, but perhaps scales that are no numbers)
                        if (o0 + e + 8 > p.q.out) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) f[j] = o0 + e + j < p.q.out ? f[j] : 0.f;
                        }
                        *at = mx_clamp8(pack8(f), p.q.act);
                    }
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    // (what lies behind the last row, or the last channel in memory, is not stored)
                    if (row0 + quarter * 32 < (long long)p.q.rows) tma_store_2d(&tm_y, from, o0 + panel * 64, (int)row0 + quarter * 32);
                    tma_store_commit();
                    if (p.panels && p.boxes + panel + p.xstages < p.boxes + panels) {
                        tma_store_wait_read<0>();          // the next panel comes into this place
                    }
                }
                __syncwarp();
                if (p.panels && lane == 0) {                      // (four warps, for eight)
                    mbar_arrive(xempty((p.boxes + panel) % p.xstages));
                    mbar_arrive(xempty((p.boxes + panel) % p.xstages));
                }
            }
            if (lane == 0) tma_store_wait_all();
        } else {
            ok = ok && __all_sync(0xffffffffu, mbar_wait(done, 0u, abort_flag, p.status));
            if (ok) {
                tc_fence_after();
                const long long row = row0 + quarter * 32 + lane;
                const bool in = row < (long long)p.q.rows;
                for (int u = warp >> 2; u * 16 < p.nt; u += MXP_WARPS / 4) {
                    const int o = o0 + u * 16;
                    if (o >= p.q.out) break;
                    bf16x8 rv[2] = {};
                    if (p.q.res && in) {
                        rv[0] = *reinterpret_cast<const bf16x8 *>(p.q.res + (size_t)row * p.q.out_pad + o);
                        if (o + 8 < p.q.out_pad) rv[1] = *reinterpret_cast<const bf16x8 *>(p.q.res + (size_t)row * p.q.out_pad + o + 8);
                    }
                    uint32_t v[16];
                    tmem_ld16(t_lane + (uint32_t)(u * 16), v);
                    tmem_ld_wait();
                    float f[16], g[16];
                    unpack8(rv[0], g);
                    unpack8(rv[1], g + 8);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float z = __uint_as_float(v[j]) + bias_s[u * 16 + j];
                        if (p.q.res) z += g[j];
                        f[j] = mx_act(z, p.q.act);
                    }
                    if (!in) continue;
                    float *y = (float *)p.q.y + (size_t)row * p.q.out + o;
                    if (((uintptr_t)y & 15) == 0 && o + 16 <= p.q.out) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) reinterpret_cast<float4 *>(y)[j] = make_float4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (o + j < p.q.out) y[j] = f[j];
                    }
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

// The shares' sums of a product whose features come first, then bias, shortcut and activation: a thread has four features of a row
constexpr int MXP_FINISH = 128;
__global__ void __launch_bounds__(MXP_FINISH) mx_finish_kernel(const float *__restrict__ partial, int splits, const MxProduct q) {
    pdl_wait();
    pdl_trigger();
    const int o = (blockIdx.x * MXP_FINISH + threadIdx.x) * 4;
    const size_t n = blockIdx.y;
    if (o >= q.out_pad) return;
    const size_t step = (size_t)q.rows * q.out_pad;
    const float *from = partial + n * q.out_pad + o;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < splits; k0 += 8) {
        float4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = k0 + k < splits ? __ldcg(reinterpret_cast<const float4 *>(from + (k0 + k) * step)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) { s[0] += v[k].x; s[1] += v[k].y; s[2] += v[k].z; s[3] += v[k].w; }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (o + j < q.out) {
            s[j] += __ldg(q.bias + o + j);
            if (q.res) s[j] += __bfloat162float(q.res[n * q.out_pad + o + j]);
            s[j] = mx_act(s[j], q.act);
        } else s[j] = 0.f;
    }
    if (q.out_is_f32) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (o + j < q.out) ((float *)q.y)[n * q.out + o + j] = s[j];
    } else {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(s[0], s[1]), hi = __floats2bfloat162_rn(s[2], s[3]);
        *reinterpret_cast<uint2 *>((__nv_bfloat16 *)q.y + n * q.out_pad + o) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
    }
}

// How a product is shared out
MxTiling mx_tiling(unsigned long long rows, int in, int out) {
    MxTiling t = {};
    t.tensor = 1;
    if (rows <= MXP_ROWS) {
        t.features = 1;
        t.nt = round_up((int)rows, 16);
        t.subs = 1;
        const int tiles = (out + MXP_ROWS - 1) / MXP_ROWS, chunks = (in + MXP_CHUNK - 1) / MXP_CHUNK;
        // Two blocks to an SM (8 x 25088 -> 4096: 17.6 us, with one 19.0), but three chunks or more to a share and 16 shares or fewer: each has its start to pay
        // for and sums to leave behind (64 x 4096 -> 1000 with a chunk a share 10.3 us, three 8.5; 16 x 16384 -> 512 18.2, three 11.2, four 10.4).
        t.splits = 2 * 148 / tiles;
        t.splits = t.splits < 1 ? 1 : t.splits > 16 ? 16 : t.splits;
        t.per = (chunks + t.splits - 1) / t.splits;
        if (t.per < 3) t.per = 3 < chunks ? 3 : chunks;
        t.splits = (chunks + t.per - 1) / t.per;
        return t;
    }
    const long long tiles_m = (long long)((rows + MXP_ROWS - 1) / MXP_ROWS);
    const int all = round_up(out, 16);
    t.nt = all <= MXP_MOST ? all : 256;
    // (384: rows are rounded here as long as one block covers all features.  12544 x 960 -> 320 16.7 us, already rounded 21.9, already rounded and in parts of 256
    // 26.2; 200704 x 144 -> 24 38 us, already rounded 52.)
    // Fewer features to a block while that leaves half the SMs without one: 784 x 960 -> 320 14.9 -> 7.9 us, 1024 x 4096 -> 1000 18.6 -> 15.1 us.
    while (t.nt > 64 && tiles_m * ((all + t.nt - 1) / t.nt) * 2 <= 148) t.nt = t.nt > 256 ? 256 : t.nt > 128 ? 128 : 64;
    t.tiles_n = (all + t.nt - 1) / t.nt;
    t.subs = (t.nt + 127) / 128;
    t.round = t.tiles_n == 1;
    return t;
}
size_t mx_partial_bytes(const MxTiling &t, unsigned long long rows, int out) {
    return t.features ? (size_t)t.splits * rows * cprune_padded_channels(out) * sizeof(float) : 0;
}

template <int FORM>
static cprune_status launch_product(const CUtensorMap *tm, const MxpParams &p, long long blocks, size_t smem, cudaStream_t st) {
    static std::mutex attr_mu;
    static bool attr_set[64] = {false};    // the shared-memory limit of a kernel is a per-device attribute
    {
        int dev = 0;
        CPRUNE_CUDA_CHECK(cudaGetDevice(&dev));
        if (dev < 0 || dev >= 64) return CPRUNE_ERR_UNSUPPORTED;
        std::lock_guard<std::mutex> lock(attr_mu);
        if (!attr_set[dev]) {
            CPRUNE_CUDA_CHECK(cudaFuncSetAttribute(mx_product_kernel<FORM>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024));
            attr_set[dev] = true;
        }
    }
    CPRUNE_CUDA_CHECK(launch_chained(mx_product_kernel<FORM>, dim3((unsigned)blocks), dim3(MXP_THREADS), smem, st, tm[0], tm[1], tm[2], tm[3], p));
    return CPRUNE_OK;
}

static cprune_status encode_codes(CUtensorMap *map, const void *codes, int blocks, unsigned long long rows, int box_rows) {
    const unsigned long long dims[2] = {(unsigned long long)blocks * 8, rows};           // (in units of two bytes)
    const unsigned long long strides[1] = {(unsigned long long)blocks * 16};
    const unsigned box[2] = {64, (unsigned)box_rows};
    return encode_tiled_bf16_swz(map, codes, 2, dims, strides, box, 128, true);
}

// x: bf16 rows (t.round), else their codes, with their scales
cprune_status launch_mx_product(const MxProduct &q, const MxTiling &t, const void *x, const uint8_t *xscales, int in, float *partial, ChainScope &chain, cudaStream_t st) {
    MxpParams p = {};
    p.q = q;
    p.nt = t.nt; p.subs = t.subs; p.tiles_n = t.features ? t.splits : t.tiles_n; p.per = t.per;
    for (p.box = 128; t.nt % p.box;) p.box /= 2;
    p.chunks = (in + MXP_CHUNK - 1) / MXP_CHUNK;
    p.boxes = t.round ? (in + 63) / 64 : 0;
    p.panels = q.res && !q.out_is_f32 && !t.features ? (t.nt + 63) / 64 : 0;
    p.steps_last = (in - (p.chunks - 1) * MXP_CHUNK + 63) / 64;
    if (t.features) p.box = t.nt;
    p.b_bytes = round_up(t.nt * 128, 1024);
    p.xscales = xscales;
    p.partial = partial;
    p.status = device_status_word();
    if (!p.status) return cuda_fail(cudaGetLastError(), "status word");
    p.sf_col = t.nt;
    const int chunks = t.features ? t.per : p.chunks;
    auto bytes = [&](int stages, int xstages) {
        const size_t s = (size_t)stages * (16384 + p.b_bytes + 1024 + t.subs * 1024) + (size_t)xstages * MXP_XBYTES, y = MXP_WARPS * 4096;
        return 1024 + MXP_FRONT + (s > y ? s : y);          // (the epilogue's place is that of the operands)
    };
    // Two blocks to an SM where that leaves each a pipeline, else one with what there is room for: rows that are rounded here are most of what is
    // read, and need the depth (64 KB or more of them under way); where only weights are read, they do.
    const int most = t.round ? 2 : 6;
    p.stages = chunks < most ? chunks : most;
    p.xstages = p.boxes + p.panels < 8 ? p.boxes + p.panels : 8;
    const size_t half = 113 * 1024, whole = 226 * 1024;
    const int least = p.xstages < 3 ? p.xstages : 3;
    const int two = t.round ? p.stages : chunks < 3 ? chunks : 3;                        // stages that two blocks need each
    const size_t room = bytes(two, t.round ? least : p.xstages < 2 ? p.xstages : 2) <= half ? half : whole;
    while (bytes(p.stages, p.xstages) > room) {
        if (t.round || p.xstages > 2) --p.xstages;
        else --p.stages;
    }
    // A wait tells a phase of a barrier from the one before it, not from the one before that: whoever waits for a place in the ring waits for every box that
    // comes there.  The two groups that round take every second box: an even number of places.  Panels that share a place belong to the same warps.
    if (p.boxes > p.xstages) p.xstages &= ~1;
    if (p.panels > p.xstages && p.xstages > MXP_WARPS / 4) p.xstages = MXP_WARPS / 4;
    p.groups = p.panels && p.xstages < MXP_WARPS / 4 ? p.xstages : MXP_WARPS / 4;
    while (p.stages > 1 && p.sf_col + p.stages * MXP_SF_COLS > 512) --p.stages;
    const int cols = p.sf_col + p.stages * MXP_SF_COLS;
    for (p.tmem_cols = 32; p.tmem_cols < cols;) p.tmem_cols *= 2;
    CUtensorMap tm[4];
    cprune_status s;
    if (t.round) {
        const unsigned long long dims[2] = {(unsigned long long)in, q.rows};
        const unsigned long long strides[1] = {(unsigned long long)cprune_padded_channels(in) * 2};
        const unsigned box[2] = {64, MXP_ROWS};
        s = encode_tiled_bf16_swz(&tm[0], x, 2, dims, strides, box, 128, true);
    } else s = encode_codes(&tm[0], x, q.blocks, q.rows, t.features ? p.box : MXP_ROWS);
    if (s == CPRUNE_OK) s = encode_codes(&tm[1], q.codes, q.blocks, q.out, t.features ? MXP_ROWS : p.box);
    std::memcpy(&tm[2], &tm[1], sizeof(CUtensorMap));         // (of y and the shortcut, where the bulk copies are used)
    std::memcpy(&tm[3], &tm[1], sizeof(CUtensorMap));
    if (!t.features && !q.out_is_f32) {
        const unsigned long long dims[2] = {(unsigned long long)q.out_pad, q.rows};
        const unsigned long long strides[1] = {(unsigned long long)q.out_pad * 2};
        const unsigned box_y[2] = {64, 32}, box_res[2] = {64, MXP_ROWS};
        if (s == CPRUNE_OK) s = encode_tiled_bf16_swz(&tm[2], q.y, 2, dims, strides, box_y, 128, false);
        if (s == CPRUNE_OK && q.res) s = encode_tiled_bf16_swz(&tm[3], q.res, 2, dims, strides, box_res, 128, true);
    }
    if (s != CPRUNE_OK) return s;
    const long long blocks = t.features ? (long long)((q.out + MXP_ROWS - 1) / MXP_ROWS) * t.splits : (long long)((q.rows + MXP_ROWS - 1) / MXP_ROWS) * t.tiles_n;
    if (blocks > 0x7fffffffLL) return CPRUNE_ERR_UNSUPPORTED;
    const size_t smem = bytes(p.stages, p.xstages);
    if (t.round) return launch_product<MXP_ROUND>(tm, p, blocks, smem, st);
    if (!t.features) return launch_product<MXP_CODES>(tm, p, blocks, smem, st);
    s = launch_product<MXP_FEATURES>(tm, p, blocks, smem, st);
    if (s != CPRUNE_OK) return s;
    chain.follow();
    CPRUNE_CUDA_CHECK(launch_chained(mx_finish_kernel, dim3((q.out_pad / 4 + MXP_FINISH - 1) / MXP_FINISH, (unsigned)q.rows), dim3(MXP_FINISH), 0, st, (const float *)partial,
                                     t.splits, q));
    return CPRUNE_OK;
}

}  // namespace cprune
