// Attention of sampled tokens on the cached tree: the wide kernel (up to 128 rows that read the same run of tokens) on tcgen05.
//
// One CTA per (unit, key head), in the roles of the training forward (attn_fwd.cu):
//     S = Q K^T            tcgen05.mma, operands in shared memory, S in tensor memory (two tiles of 64 tokens)
//     P = exp2(S - m)      four warps, one row per thread; P goes back to tensor memory as bf16 over S
//     O += P V             tcgen05.mma with P as the tensor-memory operand
// Pages come by TMA, a box of up to 64 tokens of one page each.  All rows see all tokens of the run; places of a tile ahead of it or behind it
// are taken out of S, and their values (which may be anything) are zeroed, since 0 times an infinity is not 0.
// 8 bits: keys go into the first product as they are.  A query is two 8-bit terms for it (a row brought to 2^7 by a power of two; its 8
// significant bits are 4 and 4, and the second term is off by half of 2^-9 at most, 2^-17 of the row's largest), so S is two products of twice the rate.
// Values become bf16 tiles, exactly, by four more warps: sign, exponent and fraction moved to their places, times 2^120 and the
// token's power of two in one multiplication.  A key's power, times what the scale is beside a power of two, multiplies its scores.
// Bound by the chain S, P, O of a tile, two CTAs an SM: 200,000 shared tokens x 64 branches x 32 heads on 4, bf16, 972 TFLOP/s; runs of a
// thousand tokens with 32 to 128 rows, 8 bits, 1.2 us a tile and SM (NaN bytes, large keys and scores of any size are 2 % of that: 94.1 -> 96.4 us a call).
#include <cuda_fp8.h>

#include <cstddef>

#include "gen_attn.cuh"
#include "kernels.h"

namespace harts {
namespace gen_attn {
namespace {

using namespace tc;

constexpr int NS = 128;                  // softmax threads, thread = row = tensor-memory lane
template <bool F8>
struct Shape {
    static constexpr int NT = NS + 64 + (F8 ? 128 : 0);            // a warp that issues the MMAs, one that asks for pages, four that widen
    static constexpr int CTAS = 2;
    static constexpr int Q_BYTES = WIDE_ROWS * D * 2, KV_BYTES = TILE * D * 2, RAW = F8 ? 2 * TILE * D : 0, RAW_EXP = F8 ? 2 * TILE : 0;
    static constexpr int RAWS = 2, KB = F8 ? 0 : 2 * KV_BYTES;     // stages of 8-bit pages; tiles of bf16 keys
    static constexpr int q = 0, k = Q_BYTES, v = k + KB, raw = v + 2 * KV_BYTES, raw_exp = raw + RAWS * RAW, misc = raw_exp + RAWS * RAW_EXP;
    static constexpr int bytes = misc + (F8 ? 1280 : 256) + 1024;
};
// The exponent byte from which a key's factor, 2^(byte - 127) to twice that, may take a sum of products beyond fp32: those are below 2^24 (256 x 448 x 128,
// and the second terms)
constexpr int LARGE = 127 + 103;
constexpr float UP = 4294967296.f;       // then 2^32 of it goes with the rows' factors: theirs are small, or the scores would not be finite
constexpr int COL_S = 0, COL_O = 128, TMEM_COLS = 256;     // S / P of tile n at COL_S + 64 (n & 1)
struct Misc {
    uint64_t q, k[2], v[2], kfree[2], vfree[2], s[2], p[2], pv, o, exit, kp_full[2];      // 8 bits: k, kfree are those of the stages of pages
    int dead;
    uint32_t tmem;
    float up[2];                                     // 8 bits: what the rows' factors take from those of a tile's keys
    alignas(16) float kp[2][TILE], f[WIDE_ROWS];     // 8 bits: factors of a tile's keys and of the rows, which make a sum of products a score in log2 units
};
static_assert(offsetof(Misc, kp) <= 256 && offsetof(Misc, kp) % 16 == 0 && sizeof(Misc) <= 1280 && Shape<true>::misc % 16 == 0, "misc area");

__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// 16 8-bit values of a token as bf16, times 2^120 and the token's power: f, and f2 where one factor cannot hold both (f2 = 1 elsewhere)
__device__ __forceinline__ uint32_t moved(uint32_t y) { return ((y >> 4) & 0x07f007f0u) | (y & 0x80008000u); }      // from the upper bytes of the halves
__device__ __forceinline__ uint32_t times(uint32_t x, uint32_t f) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(f));
    return r;
}
__device__ __forceinline__ void widen16(const uint4& y, int exp, uint4* z) {
    // 2^(120 + exp - 127) where that is a normal number, else 2^120 first; 255: NaN
    const bool one = exp <= 134;
    const uint32_t f = one ? (uint32_t)(exp + 120) << 7 : 0x7b80u, f2 = f | f << 16;
    const uint32_t w[4] = {y.x, y.y, y.z, y.w};
    uint32_t r[8];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        r[2 * i] = times(moved(__byte_perm(w[i], 0, 0x1404)), f2);
        r[2 * i + 1] = times(moved(__byte_perm(w[i], 0, 0x3424)), f2);
    }
    if (!one) {
        const uint32_t e = exp == 255 ? 0x7fffu : (uint32_t)exp << 7, e2 = e | e << 16;
#pragma unroll
        for (int i = 0; i < 8; i++) r[i] = times(r[i], e2);
    }
    // 0x7f and 0xff are NaN, which moving made 480: the only bytes whose lower seven bits carry into the eighth when 1 is added
    uint32_t nan[4], any = 0;
#pragma unroll
    for (int i = 0; i < 4; i++) any |= nan[i] = (w[i] & 0x7f7f7f7fu) + 0x01010101u;
    if (any & 0x80808080u)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            r[2 * i] |= ((__byte_perm(nan[i], 0, 0x1404) >> 15) & 0x00010001u) * 0x7fffu;
            r[2 * i + 1] |= ((__byte_perm(nan[i], 0, 0x3424) >> 15) & 0x00010001u) * 0x7fffu;
        }
    z[0] = make_uint4(r[0], r[1], r[2], r[3]);
    z[1] = make_uint4(r[4], r[5], r[6], r[7]);
}

__device__ __forceinline__ void mma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
                 "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)accumulate) : "memory");
}
// e4m3 inputs, fp32 sums, both K-major
__host__ __device__ constexpr uint32_t instr_desc_f8(int M, int N) { return (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24); }

// A scale as a power of two and what is left of it, in [1, 2) (below 1 for a subnormal scale).  With a power of two alone, y f - (max y) f is exact whatever the size of the scores; of a
// product with any factor, a multiply-add would see what rounding took from the maximum: 16 at 2^28, beyond exp2's range at 2^32.
__device__ __forceinline__ float power_of(float x) { return __uint_as_float(max(__float_as_uint(x) & 0x7f800000u, 0x00800000u)); }
constexpr float FAR = 268435456.f;       // 2^28

template <bool F8>
__global__ void __launch_bounds__(Shape<F8>::NT, Shape<F8>::CTAS)
wide_kernel(const Tables t, const __nv_bfloat16* __restrict__ q, int64_t ld_q, const __grid_constant__ CUtensorMap map_k,
            const __grid_constant__ CUtensorMap map_v, const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp,
            const int32_t* __restrict__ q_pos, float scale_log2, __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ part_o,
            float* __restrict__ part_lse, int* status) {
    using S = Shape<F8>;
    constexpr int Q_WARPS = F8 ? 8 : 4;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    Misc& m = *reinterpret_cast<Misc*>(smem + S::misc);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    let_next_launch();
    const Unit u = t.units[blockIdx.x / t.Hkv];
    const int h = blockIdx.x % t.Hkv;
    const int tile0 = u.k0 & ~(TILE - 1), n_tiles = (u.k1 - tile0 + TILE - 1) / TILE, active = (u.n + 31) / 32;      // (warps that have rows)
    if (tid == 0) {
        for (int i = 0; i < 2; i++) {
            mbar_init(&m.k[i], 1);
            mbar_init(&m.v[i], F8 ? 4 : 1);
            mbar_init(&m.kfree[i], F8 ? 5 : 1);             // the product that read it, and the warps that widen
            mbar_init(&m.vfree[i], 1);
            mbar_init(&m.s[i], 1);
            mbar_init(&m.p[i], active);
            mbar_init(&m.kp_full[i], 2);
        }
        mbar_init(&m.q, Q_WARPS);
        mbar_init(&m.pv, 1);
        mbar_init(&m.o, 1);
        mbar_init(&m.exit, 1);
        m.dead = 0;
        fence_barrier_init();
    }
    if (warp == 0) tmem_alloc<TMEM_COLS>(&m.tmem);
    PageWalk walk(t, u, tile0, warp == NS / 32 + 1 ? u.k1 : 0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = m.tmem;
    if (warp < NS / 32 || warp >= NS / 32 + 2) {
        // the rows' queries, half a warp a row, while the first pages are on their way
        for (int i = (warp < NS / 32 ? tid : tid - 64) >> 4; i < WIDE_ROWS; i += Q_WARPS * 2) {
            const int ch = tid & 15;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (i < u.n) {
                const int G = t.Hq / t.Hkv, flat = u.flat0 + i;
                x = *reinterpret_cast<const uint4*>(q + (int64_t)t.entries[u.entry + flat / G].row * ld_q + (int64_t)(h * G + flat % G) * D + ch * 8);
            }
            if constexpr (F8) {
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                uint32_t top = 0, hi[2] = {0, 0}, lo[2] = {0, 0};
    #pragma unroll
                for (int e = 0; e < 4; e++) top = __vmaxu2(top, w[e] & 0x7fff7fffu);
                top = max(top & 0xffffu, top >> 16);
    #pragma unroll
                for (int d = 1; d < 16; d <<= 1) top = max(top, __shfl_xor_sync(~0u, top, d));
                const PowerOfTwo f(top, 7);
    #pragma unroll
                for (int e = 0; e < 4; e++) {
                    const float2 y = f.apply(w[e]);
                    const uint32_t y8 = __nv_cvt_float2_to_fp8x2(y, __NV_SATFINITE, __NV_E4M3);
                    const uint32_t y16 = widen(y8);
                    const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&y16));
                    hi[e >> 1] |= y8 << (16 * (e & 1));
                    lo[e >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(y.x - back.x, y.y - back.y), __NV_SATFINITE, __NV_E4M3) << (16 * (e & 1));
                }
                unsigned char* dst = smem + S::q + sw128_chunk(i, ch >> 1) + 8 * (ch & 1);
                *reinterpret_cast<uint2*>(dst) = make_uint2(hi[0], hi[1]);
                *reinterpret_cast<uint2*>(dst + S::Q_BYTES / 2) = make_uint2(lo[0], lo[1]);
                if (ch == 0) m.f[i] = top >= 0x7f80u ? __uint_as_float(0x7fffffffu) : f.undone(power_of(scale_log2));      // infinite or NaN: NaN
            } else {
                *reinterpret_cast<uint4*>(smem + S::q + (ch >> 3) * (S::Q_BYTES / 2) + sw128_chunk(i, ch & 7)) = x;
            }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&m.q);
    }

    if (warp == NS / 32 + 1) {
        // ---- pages ---------------------------------------------------------------------------------------------------------------------
        const int box = 1 << walk.box_shift, per_tile = TILE >> walk.box_shift;
        for (int n = 0; n < n_tiles; n++) {
            const int st = n & 1, ph = ((n >> 1) & 1) ^ 1;
            const int j0 = tile0 + n * TILE, boxes = (min(u.k1 - j0, TILE) + box - 1) >> walk.box_shift;
            int block[4];
#pragma unroll
            for (int b = 0; b < 4; b++) block[b] = b < boxes ? walk.of(n * per_tile + b) * t.Hkv + h : 0;
            auto at = [&](int b) { return (j0 + (b << walk.box_shift)) & (t.page - 1); };
            if constexpr (F8) {
                unsigned char *raw = smem + S::raw + st * S::RAW, *exps = smem + S::raw_exp + st * S::RAW_EXP;
                if (!mbar_wait_warp(&m.kfree[st], ph, status, &m.dead)) break;
                if (lane == 0) {
                    mbar_expect_tx(&m.k[st], boxes * box * (2 * D + 2));
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        if (b >= boxes) break;
                        tma_load_3d(raw + b * box * D, &map_k, 0, at(b), block[b], &m.k[st]);
                        tma_load_3d(raw + TILE * D + b * box * D, &map_v, 0, at(b), block[b], &m.k[st]);
                        bulk_load(exps + b * box, k_exp + (int64_t)block[b] * t.page + at(b), box, &m.k[st]);
                        bulk_load(exps + TILE + b * box, v_exp + (int64_t)block[b] * t.page + at(b), box, &m.k[st]);
                    }
                }
            } else {
                bool alive = true;
#pragma unroll
                for (int is_v = 0; is_v < 2; is_v++) {
                    unsigned char* tile = smem + (is_v ? S::v : S::k) + st * S::KV_BYTES;
                    uint64_t* bar = is_v ? &m.v[st] : &m.k[st];
                    if (!(alive = mbar_wait_warp(is_v ? &m.vfree[st] : &m.kfree[st], ph, status, &m.dead))) break;
                    if (lane == 0) {
                        mbar_expect_tx(bar, boxes * box * 2 * D);
#pragma unroll
                        for (int b = 0; b < 4; b++) {
                            if (b >= boxes) break;
                            for (int p = 0; p < 2; p++)
                                tma_load_3d(tile + p * (S::KV_BYTES / 2) + b * box * 128, is_v ? &map_v : &map_k, p * 64, at(b), block[b], bar);
                        }
                    }
                }
                if (!alive) break;
            }
            __syncwarp();
        }
    } else if (warp == NS / 32) {
        // ---- MMA issue: S as wide as the tile has tokens (steps of 16), P V as deep -----------------------------------------------------------
        constexpr uint32_t I_O = instr_desc(WIDE_ROWS, D, 0, 1);
        const uint64_t dQ = desc_kmajor_base(smem_u32(smem + S::q));
        auto valid = [&](int n) { return min(u.k1 - tile0 - n * TILE, TILE); };
        auto issue_s = [&](int n) {
            const int st = n & 1, width = (valid(n) + 15) & ~15;
            if (!mbar_wait_warp(&m.k[st], (n >> 1) & 1, status, &m.dead)) return false;
            tc_fence_after();
            const uint64_t dK = desc_kmajor_base(smem_u32(smem + (F8 ? S::raw + st * S::RAW : S::k + st * S::KV_BYTES)));
            if (elect_one()) {
#pragma unroll
                for (int ks = 0; ks < 8; ks++) {
                    if constexpr (F8)        // 32 features a step: the first terms of all, then the second
                        mma_f8(tmem + COL_S + st * 64, dQ + kstep_kmajor<WIDE_ROWS>(ks & 3) + (ks >> 2) * (S::Q_BYTES / 2 >> 4), dK + kstep_kmajor<TILE>(ks & 3),
                               instr_desc_f8(WIDE_ROWS, width), ks > 0);
                    else
                        mma_ss(tmem + COL_S + st * 64, dQ + kstep_kmajor<WIDE_ROWS>(ks), dK + kstep_kmajor<TILE>(ks), instr_desc(WIDE_ROWS, width, 0, 0), ks > 0);
                }
                mma_commit(&m.s[st]);
                mma_commit(&m.kfree[st]);
            }
            __syncwarp();
            return true;
        };
        bool alive = mbar_wait_warp(&m.q, 0, status, &m.dead) && issue_s(0);
        for (int n = 0; n < n_tiles && alive; n++) {
            const int st = n & 1, steps = (valid(n) + 15) >> 4;
            // S of tile n + 1 goes to the other buffer and runs under the softmax of tile n (that buffer's P was read by the P V
            // MMAs of tile n - 1, which precede it in the pipe)
            if (n + 1 < n_tiles && !(alive = issue_s(n + 1))) break;
            if (!(alive = mbar_wait_warp(&m.v[st], (n >> 1) & 1, status, &m.dead))) break;
            if (!F8 && (valid(n) < steps * 16 || (n == 0 && tile0 < u.k0))) {      // (8 bits: zeroed where they are widened)
                unsigned char* sv = smem + S::v + st * S::KV_BYTES;
                for (int e = lane; e < TILE * 16; e += 32) {
                    const int key = e >> 4, ch = e & 15;
                    if (tile0 + n * TILE + key < u.k0 || key >= valid(n))
                        *reinterpret_cast<uint4*>(sv + (ch >> 3) * (S::KV_BYTES / 2) + sw128_chunk(key, ch & 7)) = make_uint4(0, 0, 0, 0);
                }
                fence_async_smem();
                __syncwarp();
            }
            if (!(alive = mbar_wait_warp(&m.p[st], (n >> 1) & 1, status, &m.dead))) break;
            tc_fence_after();
            const uint64_t dV = desc_mnmajor_base<TILE>(smem_u32(smem + S::v + st * S::KV_BYTES));
            if (elect_one()) {
#pragma unroll 1
                for (int ks = 0; ks < steps; ks++)
                    mma_ts(tmem + COL_O, tmem + COL_S + st * 64 + ks * 8, dV + kstep_mnmajor(ks), I_O, n > 0 || ks > 0);
                mma_commit(&m.pv);                                    // one phase per tile, in order
                mma_commit(&m.vfree[st]);
                if (n + 1 == n_tiles) mma_commit(&m.o);
            }
            __syncwarp();
        }
    } else if (F8 && warp >= NS / 32 + 2) {
        // ---- 8-bit pages -> tiles ---------------------------------------------------------------------------------------------------------
        // a quarter of a warp stores to eight different places of two keys' rows of 128 bytes
        const int wt = tid - NS - 64, ch0 = wt & 3, key0 = wt >> 2;
        const float rest_of_scale = scale_log2 / power_of(scale_log2);
        for (int n = 0; n < n_tiles; n++) {
            const int st = n & 1, j0 = tile0 + n * TILE;
            if (!mbar_wait_warp(&m.k[st], (n >> 1) & 1, status, &m.dead)) break;
            // (P of two tiles ago has been used: so have its keys' powers)
            if (!mbar_wait_warp(&m.vfree[st], ((n >> 1) & 1) ^ 1, status, &m.dead)) break;
            const unsigned char *raw = smem + S::raw + st * S::RAW + TILE * D, *exps = smem + S::raw_exp + st * S::RAW_EXP;
            if (wt < TILE) {
                const bool large = __any_sync(~0u, max(exps[lane], exps[32 + lane]) >= LARGE);        // (both warps see all keys)
                m.kp[st][wt] = gen_power(exps[wt]) * (large ? rest_of_scale / UP : rest_of_scale);
                if (wt == 0) m.up[st] = large ? UP : 1.f;
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.kp_full[st]);
            }
            unsigned char* tile = smem + S::v + st * S::KV_BYTES;
#pragma unroll 2
            for (int x = 0; x < 4; x++) {                             // 16 features of a token each
                const int key = key0 + 32 * (x >> 1), ch = ch0 + 4 * (x & 1);
                uint4 y = *reinterpret_cast<const uint4*>(raw + sw128_chunk(key, ch)), z[2];
                int exp = exps[TILE + key];
                if (j0 + key < u.k0 || j0 + key >= u.k1) y = make_uint4(0, 0, 0, 0), exp = 127;      // others' may be anything: zeros
                widen16(y, exp, z);
                unsigned char* dst = tile + (ch >> 2) * (S::KV_BYTES / 2);
                *reinterpret_cast<uint4*>(dst + sw128_chunk(key, 2 * ch0)) = z[0];
                *reinterpret_cast<uint4*>(dst + sw128_chunk(key, 2 * ch0 + 1)) = z[1];
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&m.v[st]);
                mbar_arrive(&m.kfree[st]);
            }
        }
    } else if (warp < active) {
        // ---- softmax: a row per thread -----------------------------------------------------------------------------------------------------
        const uint32_t tm_lane = tmem + ((uint32_t)(warp * 32) << 16);
        if (F8) mbar_wait_warp(&m.q, 0, status, &m.dead);         // (the rows' factors are other warps')
        // m_ref: the maximum that p goes by.  bf16: scores of FAR and more differ by 16 at least, so the power of the scale is enough of it to tell the
        // largest; sc and neg_m are what p is made with.
        float m_ref = -INFINITY, l_sum = 0.f, sc = scale_log2, neg_m = 0.f;
        for (int n = 0; n < n_tiles; n++) {
            const int b = n & 1, j0 = tile0 + n * TILE;
            if (!mbar_wait_warp(&m.s[b], (n >> 1) & 1, status, &m.dead)) break;
            if (F8 && !mbar_wait_warp(&m.kp_full[b], (n >> 1) & 1, status, &m.dead)) break;
            tc_fence_after();
            const bool edge = j0 < u.k0 || j0 + TILE > u.k1;
            if constexpr (F8) sc = m.f[tid] * m.up[b];
            float mx = -INFINITY;
            uint32_t x[32];                           // half a row of S at a time, so that two CTAs' registers fit
            auto half = [&](int c) {
                tmem_ld32(tm_lane + COL_S + b * 64 + c * 32, x);
                tmem_ld_wait();
                if constexpr (F8) {
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 kp = *reinterpret_cast<const float4*>(&m.kp[b][c * 32 + e]);
                        float y[4];
                        f2_split(f2_mul(f2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), f2(kp.x, kp.y)), y[0], y[1]);
                        f2_split(f2_mul(f2(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])), f2(kp.z, kp.w)), y[2], y[3]);
#pragma unroll
                        for (int i = 0; i < 4; i++) x[e + i] = __float_as_uint(y[i]);
                    }
                }
                if (edge) {
#pragma unroll
                    for (int e = 0; e < 32; e++)
                        if (j0 + c * 32 + e < u.k0 || j0 + c * 32 + e >= u.k1) x[e] = __float_as_uint(-INFINITY);
                }
            };
#pragma unroll
            for (int c = 1; c >= 0; c--) {
                half(c);
#pragma unroll
                for (int e = 0; e < 32; e += 2) mx = max3(mx, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
            }
            const float top = mx * sc;
            const bool raise = top > RAISE - neg_m || (m_ref == -INFINITY && top > -INFINITY);
            if (__any_sync(~0u, raise)) {
                const float m_new = raise ? F8 ? top : mx * scale_log2 : m_ref;
                if (n > 0) {
                    // O is about to be read and rewritten: the P V MMAs of the tile before must be done (this warp is never more than a phase behind)
                    if (!mbar_wait_warp(&m.pv, (n - 1) & 1, status, &m.dead)) break;
                    tc_fence_after();
                    const float alpha = m_new == -INFINITY ? 1.f : ex2(m_ref - m_new);
                    l_sum *= alpha;
#pragma unroll 1
                    for (int c = 0; c < 8; c++) {
                        uint32_t y[16];
                        tmem_ld16(tm_lane + COL_O + c * 16, y);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; e++) y[e] = __float_as_uint(__uint_as_float(y[e]) * alpha);
                        tmem_st16(tm_lane + COL_O + c * 16, y);
                    }
                }
                if (raise) {
                    m_ref = m_new;
                    if constexpr (!F8) sc = fabsf(m_ref) >= FAR && fabsf(m_ref) < INFINITY ? power_of(scale_log2) : scale_log2;
                    neg_m = F8 ? -m_ref : -(mx * sc);
                }
            }
            const F2 nm = f2(neg_m, neg_m), scale2 = f2(sc, sc);
            F2 part[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
            for (int c = 0; c < 2; c++) {
                if (c == 1) half(1);                      // (the first half is still there)
                uint32_t pk[16];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    float p0, p1;
                    f2_split(f2_fma(f2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), scale2, nm), p0, p1);
                    p0 = ex2(p0);
                    p1 = ex2(p1);
                    part[(e >> 1) & 1] = f2_add(part[(e >> 1) & 1], f2(p0, p1));
                    pk[e >> 1] = pack_bf16(p0, p1);
                }
                tmem_st16(tm_lane + COL_S + b * 64 + c * 16, pk);      // (over what of S has been read: its first half)
            }
            float a0, a1;
            f2_split(f2_add(part[0], part[1]), a0, a1);
            l_sum += a0 + a1;
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.p[b]);
        }
        // ---- O / l, and its place -----------------------------------------------------------------------------------------------------------
        const bool ok = mbar_wait_warp(&m.o, 0, status, &m.dead);
        tc_fence_after();
        const bool mine = ok && tid < u.n;
        const Row r = row_of(t, u, tid, h, q_pos, nullptr);
        const float inv = l_sum == 0.f ? 0.f : 1.f / l_sum;
        const int64_t out = (int64_t)r.row * t.Hq + r.head, part = (int64_t)(u.part0 + u.flat0 + tid) * t.Hkv + h;
        if (mine) {
            const float l2 = m_ref + log2f(l_sum);
            if (r.alone) lse[out] = l2 * LN2;
            else part_lse[part] = l2;
        }
#pragma unroll 1
        for (int c = 0; c < 8; c++) {
            uint32_t x[16];
            tmem_ld16(tm_lane + COL_O + c * 16, x);
            tmem_ld_wait();
            if (mine) {
#pragma unroll
                for (int e = 0; e < 16; e++) x[e] = __float_as_uint(__uint_as_float(x[e]) * inv);
                if (r.alone) {
#pragma unroll
                    for (int e = 0; e < 16; e += 8)
                        *reinterpret_cast<uint4*>(o + out * D + c * 16 + e) =
                            make_uint4(pack_bf16(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), pack_bf16(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])),
                                       pack_bf16(__uint_as_float(x[e + 4]), __uint_as_float(x[e + 5])), pack_bf16(__uint_as_float(x[e + 6]), __uint_as_float(x[e + 7])));
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(part_o + part * D + c * 16 + e) = make_uint4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                }
            }
            __syncwarp();
        }
    }
    __syncwarp();
    if (__syncthreads_or(m.dead)) {               // abandoned: let the loads and MMAs in flight finish (bounded)
        if (warp == NS / 32 && elect_one()) {
            mma_commit(&m.exit);
            mbar_wait_drain(&m.exit, 0);
        }
        drain_delay();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc<TMEM_COLS>(tmem);
}

template <bool F8>
int32_t launch(const Tables& t, int n_units, const Call& a) {
    using S = Shape<F8>;
    static std::atomic<uint64_t> set{0};
    if (!gen_shared_memory(wide_kernel<F8>, S::bytes, set)) return HARTS_ECUDA;
    wide_kernel<F8><<<n_units * t.Hkv, S::NT, S::bytes, a.stream>>>(t, static_cast<const __nv_bfloat16*>(a.q), a.ld_q, a.map_k, a.map_v, a.cache.k_exp,
                                                                  a.cache.v_exp, a.q_pos, a.scale_log2, static_cast<__nv_bfloat16*>(a.o), a.lse, a.part_o,
                                                                  a.part_lse, a.dev_status);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}

}  // namespace

int32_t launch_wide(const Tables& t, int n_units, const Call& a) {
    return a.cache.type == HARTS_E4M3 ? launch<true>(t, n_units, a) : launch<false>(t, n_units, a);
}

}  // namespace gen_attn
}  // namespace harts
