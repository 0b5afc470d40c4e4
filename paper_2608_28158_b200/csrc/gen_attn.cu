// Attention of sampled tokens on the cached tree: the narrow kernel (up to 16 rows -- a query and a head of its group -- that read the
// same run of tokens) and the merge of parts.
//
//     s_j = scale q . k_j    p_j = exp(s_j - m)    o = sum p_j v_j / sum p_j
//
// A CTA works off a list of units for one key head; the lists are of the same length in tiles of 64 tokens, as many as the GPU holds CTAs, and a
// unit that crosses a list's end is cut there.  A warp asks for the pages by TMA, a tile a stage, ahead into the next unit; four warps
// take 16 of a tile's tokens each, so that every key and value is read from shared memory once.  Products are m16n8k16 with tokens (scores) and features (outputs) as m and the rows as n: 8
// or 16 rows cost what they are, and fragments let a warp keep scores, softmax and sums in registers.  At so few rows a token the
// work is far below any tensor path's rate.  A warp has its own running maximum (raised in steps of 2^8 and more), sum and output;
// the four are joined at the unit's end.
// 8-bit values become fp16 by one instruction a pair, exactly, so that the products are fp16 there: a row's queries times a power of two that
// brings the largest to 2^14 (what falls below 2^-24 is 2^-38 of it), p with its token's power of two and a running maximum of
// its own, and 11 bits of it kept instead of bf16's 8.  Which of the 128 features a fragment's place holds is free as long as both
// operands agree, so that a thread takes 32 bytes in a row of a key and 16 of a value.
// Bound by the cache's bytes: 64 sequences x 5,200 tokens x 8 key heads x 4 query heads, bf16, 208 us, as fast as a copy; 3 x 90,000 tokens x 8 x 4, 8 bits,
// 88.0 us, 0.97 of one.
#include <algorithm>

#include "gen_attn.cuh"
#include "kernels.h"

namespace harts {

namespace {

using namespace tc;
using namespace gen_attn;

constexpr int CW = 4, NT = CW * 32 + 32;

template <bool F8, int NR>             // NR: rows, in eights
struct Shape {
    // as many CTAs of an SM as registers allow, and stages for what shared memory is left
    static constexpr int CTAS = NR == 1 ? 3 : 2, STAGES = NR == 1 ? (F8 ? 4 : 2) : (F8 ? 5 : 3);
    static constexpr int KV = TILE * D * (F8 ? 1 : 2), EXP = F8 ? TILE : 0;
    // the exponents of a stage lie behind all tiles (which start on 1,024 bytes), then half of the warps' outputs for eight rows, to be joined
    static constexpr int PITCH = D / 2 + 4;
    static constexpr int exps = STAGES * 2 * KV, joint = exps + STAGES * 2 * EXP, stats = joint + CW * 8 * PITCH * 4, misc = stats + CW * 8 * NR * 16,
                         bytes = misc + 256 + 1024;
    static_assert(CTAS * (bytes + 1024) <= 228 * 1024, "shared memory");
};
struct Misc {
    uint64_t kfull[5], kempty[5], vfull[5], vempty[5];
    int dead, stop;      // latch: a wait ran out; what the four warps have seen of it at a unit's end, all the same
};

template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t saddr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {      // an 8 x 8 matrix of 16-bit elements
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool F8>             // whether any of the values is infinite or NaN (8 bits: 0x7f)
__device__ __forceinline__ bool nonfinite(uint32_t x) {
    if constexpr (F8) return __vcmpeq4(x & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
    return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}

template <bool F8, int NR>
__global__ void __launch_bounds__(NT, (Shape<F8, NR>::CTAS))
narrow_kernel(const Tables t, const __nv_bfloat16* __restrict__ q, int64_t ld_q, const __grid_constant__ CUtensorMap map_k,
              const __grid_constant__ CUtensorMap map_v, const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp,
              const int32_t* __restrict__ q_pos, float scale_log2, __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ part_o,
              float* __restrict__ part_lse, int* status) {
    using S = Shape<F8, NR>;
    constexpr int ROWS = 8 * NR;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    Misc& m = *reinterpret_cast<Misc*>(smem + S::misc);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.x % t.Hkv, first = t.list_ptr[blockIdx.x / t.Hkv], last = t.list_ptr[blockIdx.x / t.Hkv + 1];
    if (tid == 0) {
        for (int i = 0; i < S::STAGES; i++) {
            mbar_init(&m.kfull[i], 1);
            mbar_init(&m.kempty[i], CW);
            mbar_init(&m.vfull[i], 1);
            mbar_init(&m.vempty[i], CW);
        }
        m.dead = 0;
        fence_barrier_init();
    }
    __syncthreads();
    const int g = lane >> 2, c = lane & 3;
    Ring<S::STAGES> rk, rv;                       // the rings of stages run on over the units
    bool alive = true;
#pragma unroll 1
    for (int item = first; item < last && alive; item++) {
    const Unit u = t.units[item];
    const int tile0 = u.k0 & ~(TILE - 1);
    PageWalk walk(t, u, tile0, warp == CW ? u.k1 : 0);
    // what the unit's rows see: lane i has row i; the farthest token that any sees, and the nearest limit
    const Row mine = row_of(t, u, min(lane, ROWS - 1), h, q_pos, tid < ROWS ? status : nullptr);
    int far = lane < u.n ? mine.limit : 0, near = lane < u.n ? mine.limit : INT32_MAX;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        far = max(far, __shfl_xor_sync(~0u, far, x));
        near = min(near, __shfl_xor_sync(~0u, near, x));
    }
    const int k1 = min(u.k1, far), n_tiles = k1 > u.k0 ? (k1 - tile0 + TILE - 1) / TILE : 0;

    if (warp == CW) {
        // ---- pages: a box is up to 64 tokens of one page ----------------------------------------------------------------------------
        const int box = 1 << walk.box_shift, per_tile = TILE >> walk.box_shift;
        for (int n = 0; n < n_tiles; n++) {
            const int j0 = tile0 + n * TILE, boxes = (min(k1 - j0, TILE) + box - 1) >> walk.box_shift;
            int block[4];
#pragma unroll
            for (int b = 0; b < 4; b++) block[b] = b < boxes ? walk.of(n * per_tile + b) * t.Hkv + h : 0;
#pragma unroll
            for (int is_v = 0; is_v < 2; is_v++) {
                Ring<S::STAGES>& r = is_v ? rv : rk;
                if (!(alive = mbar_wait_warp(is_v ? &m.vempty[r.st] : &m.kempty[r.st], r.ph ^ 1, status, &m.dead))) break;
                uint64_t* bar = is_v ? &m.vfull[r.st] : &m.kfull[r.st];
                unsigned char *tile = smem + (2 * r.st + is_v) * S::KV, *se = smem + S::exps + (2 * r.st + is_v) * S::EXP;
                if (lane == 0) {
                    mbar_expect_tx(bar, boxes * box * (F8 ? D + 1 : 2 * D));
#pragma unroll
                    for (int b = 0; b < 4; b++) {
                        if (b >= boxes) break;
                        const int at = (j0 + (b << walk.box_shift)) & (t.page - 1);
                        const CUtensorMap* map = is_v ? &map_v : &map_k;
                        if constexpr (F8) {
                            tma_load_3d(tile + b * box * D, map, 0, at, block[b], bar);
                            bulk_load(se + b * box, (is_v ? v_exp : k_exp) + (int64_t)block[b] * t.page + at, box, bar);
                        } else {
                            for (int p = 0; p < 2; p++) tma_load_3d(tile + p * (S::KV / 2) + b * box * 128, map, p * 64, at, block[b], bar);
                        }
                    }
                }
                r.next();
            }
            if (!alive) break;
            __syncwarp();
        }
    } else {
        // ---- the rows' queries: n = row 8 r + g; scores of rows 8 r + 2 c, 8 r + 2 c + 1 -------------------------------------------------
        uint32_t qb[NR][8][2];
        float f[NR][2];                           // what makes a score log2 units
        int limit[NR][2];
#pragma unroll
        for (int r = 0; r < NR; r++) {
            const int row = __shfl_sync(~0u, mine.row, 8 * r + g), head = __shfl_sync(~0u, mine.head, 8 * r + g);
            const bool there = 8 * r + g < u.n;
            const __nv_bfloat16* src = q + (int64_t)row * ld_q + (int64_t)head * D;
#pragma unroll
            for (int ks = 0; ks < 8; ks++)
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const int d = F8 ? 32 * c + 4 * ks + 2 * x : 16 * ks + 8 * x + 2 * c;
                    qb[r][ks][x] = there ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
                }
            float own = scale_log2;
            if constexpr (F8) {
                uint32_t top = 0;
#pragma unroll
                for (int ks = 0; ks < 8; ks++) top = __vmaxu2(top, __vmaxu2(qb[r][ks][0] & 0x7fff7fffu, qb[r][ks][1] & 0x7fff7fffu));
                top = max(top & 0xffffu, top >> 16);
                top = max(top, __shfl_xor_sync(~0u, top, 1));
                top = max(top, __shfl_xor_sync(~0u, top, 2));
                const PowerOfTwo x(top, 14);         // fp16; what falls below 2^-24 is 2^-38 of the largest
#pragma unroll
                for (int ks = 0; ks < 8; ks++)
#pragma unroll
                    for (int y = 0; y < 2; y++) {
                        const float2 z = x.apply(qb[r][ks][y]);
                        qb[r][ks][y] = pack_f16(z.x, z.y);
                    }
                own = x.undone(scale_log2);
            }
#pragma unroll
            for (int y = 0; y < 2; y++) {
                f[r][y] = __shfl_sync(~0u, own, 4 * (2 * c + y));
                limit[r][y] = __shfl_sync(~0u, mine.limit, 8 * r + 2 * c + y);         // (0 behind the unit's rows)
            }
        }
        // top: of a score.  8 bits: what p goes by is top + ahead, the largest of a score and its value's power; `ahead` for itself, as the sum would
        // round the power off beside a large score.
        float acc[NR][8][4], top[NR][2], ahead[NR][2], sum[NR][2];
#pragma unroll
        for (int r = 0; r < NR; r++) {
#pragma unroll
            for (int j = 0; j < 8; j++) acc[r][j][0] = acc[r][j][1] = acc[r][j][2] = acc[r][j][3] = 0.f;
            top[r][0] = top[r][1] = ahead[r][0] = ahead[r][1] = -INFINITY;
            sum[r][0] = sum[r][1] = 0.f;
        }
        // scores of a tile's tokens 16 warp + g and + 8, in log2 units
        auto scores = [&](auto& s) {
            if (!(alive = mbar_wait_warp(&m.kfull[rk.st], rk.ph, status, &m.dead))) return;
            const unsigned char* sk = smem + 2 * rk.st * S::KV;
            float s2[NR][4];                      // two chains of products
#pragma unroll
            for (int r = 0; r < NR; r++)
#pragma unroll
                for (int x = 0; x < 4; x++) s[r][x] = s2[r][x] = 0.f;
            [[maybe_unused]] float kp[2] = {1.f, 1.f};
            if constexpr (F8) {
                const unsigned char* se = smem + S::exps + 2 * rk.st * S::EXP + 16 * warp;
                kp[0] = gen_power(se[g]);
                kp[1] = gen_power(se[g + 8]);
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const unsigned char* src = sk + sw128_chunk(16 * warp + g, 2 * c + x);
                    const uint4 y = *reinterpret_cast<const uint4*>(src), z = *reinterpret_cast<const uint4*>(src + 8 * 128);
                    const uint32_t w[4] = {y.x, y.y, y.z, y.w}, w8[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const uint32_t a[4] = {widen(w[i]), widen(w8[i]), widen_upper(w[i]), widen_upper(w8[i])};
#pragma unroll
                        for (int r = 0; r < NR; r++) mma16816<true>(x ? s2[r] : s[r], a, qb[r][4 * x + i][0], qb[r][4 * x + i][1]);
                    }
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < 8; ks++) {
                    const int ch = 2 * ks + (lane >> 4);
                    uint32_t a[4];
                    ldmatrix_x4(smem_u32(sk) + (ch >> 3) * (S::KV / 2) + sw128_chunk(16 * warp + (lane & 15), ch & 7), a);
#pragma unroll
                    for (int r = 0; r < NR; r++) mma16816<false>(ks & 1 ? s2[r] : s[r], a, qb[r][ks][0], qb[r][ks][1]);
                }
            }
            fence_async_smem();                   // an arrival alone can pass reads that are still on their way, and the next copy then lands under
            // them: seen beside the wide kernel, whose products keep shared memory busy (1 call in 250)
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.kempty[rk.st]);
            rk.next();
#pragma unroll
            for (int r = 0; r < NR; r++)
#pragma unroll
                for (int x = 0; x < 4; x++) {          // (8 bits: the two factors' product may be beyond fp32 where a score is not)
                    s[r][x] = (s[r][x] + s2[r][x]) * f[r][x & 1];
                    if constexpr (F8) s[r][x] *= kp[x >> 1];
                }
        };
        constexpr bool EARLY = NR == 1;           // (the registers of 16 rows do not allow it)
        float s[NR][4], next[EARLY ? NR : 1][4];
        if constexpr (EARLY)
            if (n_tiles > 0) scores(next);
        for (int n = 0; n < n_tiles && alive; n++) {
            const int j0 = tile0 + n * TILE, key0 = j0 + 16 * warp;
            if constexpr (EARLY) {                // the next tile's products run under this one's softmax
#pragma unroll
                for (int x = 0; x < 4; x++) s[0][x] = next[0][x];
                if (n + 1 < n_tiles) scores(next);
            } else {
                scores(s);
            }
            if (!alive) break;
            if (!(alive = mbar_wait_warp(&m.vfull[rv.st], rv.ph, status, &m.dead))) break;
            unsigned char* sv = smem + (2 * rv.st + 1) * S::KV;
            const bool edge = j0 < u.k0 || j0 + TILE > min(near, u.k1);
            float ve[2] = {0.f, 0.f};
            if constexpr (F8)
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const int e = smem[S::exps + (2 * rv.st + 1) * S::EXP + 16 * warp + g + 8 * y];
                    ve[y] = e == 255 ? __uint_as_float(0x7fffffffu) : (float)(e - 127);
                }
            if (edge)                             // hidden tokens: -inf
#pragma unroll
                for (int r = 0; r < NR; r++)
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const int key = key0 + g + 8 * (x >> 1);
                        if (key < u.k0 || key >= min(limit[r][x & 1], k1)) s[r][x] = -INFINITY;
                    }
            // maxima are looked for only where some score is 2^8 above what its row goes by (or has nothing to go by yet)
            bool over = false;
            auto from = [&](float m) { return m == -INFINITY ? 0.f : m; };         // what is measured from a maximum: of nothing yet, from 0
#pragma unroll
            for (int r = 0; r < NR; r++)
#pragma unroll
                for (int x = 0; x < 4; x++) {
                    over |= s[r][x] > top[r][x & 1] + RAISE;
                    if constexpr (F8) over |= s[r][x] - from(top[r][x & 1]) + ve[x >> 1] > ahead[r][x & 1] + RAISE;
                }
            if (__any_sync(~0u, over)) {
#pragma unroll
                for (int r = 0; r < NR; r++)
#pragma unroll
                    for (int y = 0; y < 2; y++) {
                        float mx = fmaxf(s[r][y], s[r][2 + y]);
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, x));
                        float by = 1.f;           // (from -inf: 0, and all sums are 0)
                        if (mx > top[r][y] + RAISE) {
                            by = ex2(top[r][y] - mx);
                            sum[r][y] *= by;
                            ahead[r][y] += from(top[r][y]) - mx;
                            top[r][y] = mx;
                        }
                        if constexpr (F8) {
                            const float base = from(top[r][y]);
                            float mx2 = fmaxf(s[r][y] - base + ve[0], s[r][2 + y] - base + ve[1]);
#pragma unroll
                            for (int x = 4; x < 32; x <<= 1) mx2 = fmaxf(mx2, __shfl_xor_sync(~0u, mx2, x));
                            by = 1.f;
                            if (mx2 > ahead[r][y] + RAISE) {
                                by = ex2(ahead[r][y] - mx2);
                                ahead[r][y] = mx2;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 8; j++) {
                            acc[r][j][y] *= by;
                            acc[r][j][2 + y] *= by;
                        }
                    }
            }
            uint32_t pb[NR][2];
#pragma unroll
            for (int r = 0; r < NR; r++) {
                float p[4];
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    const float base = from(top[r][y]), base2 = from(ahead[r][y]);
#pragma unroll
                    for (int x = y; x < 4; x += 2) {
                        const float t = s[r][x] - base;
                        p[x] = ex2(t);
                        sum[r][y] += p[x];
                        if constexpr (F8) p[x] = t == -INFINITY ? 0.f : ex2(t + (ve[x >> 1] - base2));      // (a hidden token's power may be anything)
                    }
                }
#pragma unroll
                for (int x = 0; x < 2; x++) pb[r][x] = transposed(F8 ? pack_f16(p[2 * x], p[2 * x + 1]) : pack_bf16(p[2 * x], p[2 * x + 1]));
            }
            bool bad = false;
            if (edge) {
                // Behind the last token that any row sees: zeros (this warp's tokens).
                // Values that some rows see and others do not may be infinite or NaN, and 0 times that is not 0.
                constexpr int CH = F8 ? 8 : 16;           // 16-byte pieces of a token's values
#pragma unroll 1
                for (int e = lane; e < 16 * CH; e += 32) {
                    const int key = key0 + e / CH, ch = e % CH;
                    if (key < k1 && key >= u.k0 && key < near) continue;
                    uint4& y = *reinterpret_cast<uint4*>(sv + (ch >> 3) * (S::KV / 2) + sw128_chunk(16 * warp + e / CH, ch & 7));
                    if (key >= k1) y = make_uint4(0, 0, 0, 0);
                    else bad |= nonfinite<F8>(y.x) || nonfinite<F8>(y.y) || nonfinite<F8>(y.z) || nonfinite<F8>(y.w);
                }
                bad = __any_sync(~0u, bad);
                fence_async_smem();                // (before the next copy into this stage)
                __syncwarp();
            }
            if (bad) {                             // token by token: what a row does not see adds nothing
#pragma unroll 1
                for (int key = 0; key < 16; key++)
#pragma unroll
                    for (int r = 0; r < NR; r++)
#pragma unroll
                        for (int y = 0; y < 2; y++) {
                            // p of (token, row 8 r + 2 c + y): lane 4 (2 c + y) + (key / 2) % 4 has it
                            const uint32_t w = __shfl_sync(~0u, key < 8 ? pb[r][0] : pb[r][1], 4 * (2 * c + y) + ((key & 7) >> 1)) >> (16 * (key & 1));
                            const float p = F8 ? __half2float(__ushort_as_half((unsigned short)w)) : __uint_as_float(w << 16);
                            const bool sees = key0 + key >= u.k0 && key0 + key < min(limit[r][y], k1);
#pragma unroll
                            for (int j = 0; j < 8; j++)
#pragma unroll
                                for (int x = 0; x < 2; x++) {
                                    const int d = F8 ? 16 * g + 2 * j + x : 16 * j + g + 8 * x;
                                    float v;
                                    if constexpr (F8) v = __half2float(__ushort_as_half((unsigned short)widen(sv[sw128_chunk(16 * warp + key, d >> 4) + (d & 15)])));
                                    else v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(sv + (d >> 6) * (S::KV / 2) + sw128(16 * warp + key, d & 63)) << 16);
                                    if (sees) acc[r][j][2 * x + y] += p * v;
                                }
                        }
            } else if constexpr (F8) {
                const unsigned char* v0 = sv + sw128_chunk(16 * warp + 2 * c, g);
                const unsigned char* v1 = sv + sw128_chunk(16 * warp + 2 * c + 1, g);
                const uint4 a = *reinterpret_cast<const uint4*>(v0), b = *reinterpret_cast<const uint4*>(v1);
                const uint4 a8 = *reinterpret_cast<const uint4*>(v0 + 8 * 128), b8 = *reinterpret_cast<const uint4*>(v1 + 8 * 128);
                const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w}, wa8[4] = {a8.x, a8.y, a8.z, a8.w}, wb8[4] = {b8.x, b8.y, b8.z, b8.w};
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int half = 0; half < 2; half++) {
                        const uint32_t y = __byte_perm(wa[i], wb[i], half ? 0x7362 : 0x5140), y8 = __byte_perm(wa8[i], wb8[i], half ? 0x7362 : 0x5140);
                        const uint32_t va[4] = {widen(y), widen_upper(y), widen(y8), widen_upper(y8)};
#pragma unroll
                        for (int r = 0; r < NR; r++) mma16816<true>(acc[r][2 * i + half], va, pb[r][0], pb[r][1]);
                    }
            } else {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const int ch = 2 * j + ((lane >> 3) & 1);
                    uint32_t va[4];
                    ldmatrix_x4_trans(smem_u32(sv) + (ch >> 3) * (S::KV / 2) + sw128_chunk(16 * warp + (lane & 7) + 8 * (lane >> 4), ch & 7), va);
#pragma unroll
                    for (int r = 0; r < NR; r++) mma16816<false>(acc[r][j], va, pb[r][0], pb[r][1]);
                }
            }
            fence_async_smem();                   // (as for the keys)
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.vempty[rv.st]);
            rv.next();
        }
        // ---- the four warps' parts joined -----------------------------------------------------------------------------------------
        float* so = reinterpret_cast<float*>(smem + S::joint);
        float4* stats = reinterpret_cast<float4*>(smem + S::stats);        // [warp][row]{maximum, sum, 8 bits: what outputs go by, from the maximum, -}
        constexpr int PER = CW * 4;                                       // threads a row
#pragma unroll
        for (int r8 = 0; r8 < NR; r8++)
#pragma unroll
            for (int y = 0; y < 2; y++) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) sum[r8][y] += __shfl_xor_sync(~0u, sum[r8][y], x);
                if (g == 0) stats[warp * ROWS + 8 * r8 + 2 * c + y] = make_float4(top[r8][y], sum[r8][y], F8 ? ahead[r8][y] : top[r8][y], 0.f);
            }
#pragma unroll
        for (int r8 = 0; r8 < NR; r8++) {
            if (8 * r8 >= u.n) break;
            const int i = 8 * r8 + tid / PER;
            const Row r = row_of(t, u, i, h, q_pos, nullptr);
            const int64_t out = (int64_t)r.row * t.Hq + r.head, part = (int64_t)(u.part0 + u.flat0 + i) * t.Hkv + h;
            float w[CW], inv = 0.f;
            bool none = true;
#pragma unroll
            for (int half = 0; half < 2; half++) {
#pragma unroll
                for (int y = 0; y < 2; y++) {
                    float* dst = so + (warp * 8 + 2 * c + y) * S::PITCH;
                    if constexpr (F8) {
                        if ((g >> 2) == half)
#pragma unroll
                            for (int j = 0; j < 8; j++)
                                *reinterpret_cast<float2*>(dst + 16 * (g & 3) + 2 * j) = make_float2(acc[r8][j][y], acc[r8][j][2 + y]);
                    } else {
#pragma unroll
                        for (int j = 0; j < 4; j++)
#pragma unroll
                            for (int x = 0; x < 2; x++) dst[16 * j + g + 8 * x] = acc[r8][4 * half + j][2 * x + y];
                    }
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (i < u.n) {
                    if (half == 0) {
                        float M = -INFINITY, L = 0.f;
#pragma unroll
                        for (int x = 0; x < CW; x++) M = fmaxf(M, stats[x * ROWS + i].x);
#pragma unroll
                        for (int x = 0; x < CW; x++) {
                            const float4 y = stats[x * ROWS + i];
                            L += y.x == -INFINITY ? 0.f * y.y : ex2(y.x - M) * y.y;
                            // without a maximum, though the warp has seen something: NaN
                            w[x] = y.y == 0.f ? 0.f : y.z == -INFINITY ? __uint_as_float(0x7fffffffu) : ex2(F8 ? y.x - M + y.z : y.x - M);
                        }
                        none = M == -INFINITY && L == 0.f;
                        inv = none ? 0.f : 1.f / L;
                        if (tid % PER == 0) {
                            const float l2 = none ? -INFINITY : M + log2f(L);
                            if (r.alone) lse[out] = l2 * LN2;
                            else part_lse[part] = l2;
                        }
                    }
                    const int e = tid % PER * 4;
                    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (!none)
#pragma unroll
                        for (int x = 0; x < CW; x++) {
                            if (w[x] == 0.f) continue;
                            const float4 z = *reinterpret_cast<const float4*>(so + (x * 8 + tid / PER) * S::PITCH + e);
                            y.x += w[x] * z.x;
                            y.y += w[x] * z.y;
                            y.z += w[x] * z.z;
                            y.w += w[x] * z.w;
                        }
                    y.x *= inv;
                    y.y *= inv;
                    y.z *= inv;
                    y.w *= inv;
                    if (r.alone) *reinterpret_cast<uint2*>(o + out * D + half * 64 + e) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
                    else *reinterpret_cast<float4*>(part_o + part * D + half * 64 + e) = y;
                }
                if (tid == 0) m.stop = *reinterpret_cast<volatile int*>(&m.dead);
                asm volatile("bar.sync 1, 128;" ::: "memory");           // it has been read
            }
        }
        alive = *reinterpret_cast<volatile int*>(&m.stop) == 0;
    }
    }
    let_next_launch();
    if (__syncthreads_or(m.dead)) drain_delay();          // abandoned: copies in flight must land before the CTA goes
    after_previous();                                     // (the wide kernel ran beside this one; the merge waits for this one only)
}

// A query head's parts joined: W warps, four elements a lane.  Queries of one part have been written by their unit.  One warp a head where
// that gives every scheduler one, else four, a quarter of the parts each (3 x 32 heads of 75 parts 12 -> 9 us; 280 x 16 heads the other way, 17
// against 13).
constexpr int MERGE_WARPS = 4;
template <int W>
__global__ void __launch_bounds__(MERGE_WARPS * 32)
merge_kernel(const Tables t, const float* part_o, const float* part_lse, __nv_bfloat16* __restrict__ o, float* __restrict__ lse) {
    __shared__ float4 so[W][32];
    __shared__ float2 stats[W];
    const int64_t out = (int64_t)blockIdx.x * (MERGE_WARPS / W) + (W == 1 ? threadIdx.x >> 5 : 0);
    if (out >= (int64_t)t.n_q * t.Hq) {           // (a whole warp)
        after_previous();
        return;
    }
    const int warp = W == 1 ? 0 : threadIdx.x >> 5, lane = threadIdx.x & 31, row = (int)(out / t.Hq), head = (int)(out % t.Hq), G = t.Hq / t.Hkv, h = head / G,
              g = head % G;
    // (the index is the call's input: only the parts are the previous kernels')
    const int p0 = t.part_ptr[row], p1 = t.part_ptr[row + 1], n = (p1 - p0 - warp + W - 1) / W;       // this warp's: every W-th
    auto place = [&](int i) { return i < n ? t.part[p0 + warp + W * i] + g : -1; };
    int at = place(lane);
    after_previous();
    if (p1 == p0 + 1) return;
    float M = -INFINITY, L = 0.f;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int b = 0; b < n; b += 32) {             // 32 parts at a time: a lane has a part's place and weight
        if (b > 0) at = place(b + lane);
        const float l = b + lane < n ? part_lse[(int64_t)at * t.Hkv + h] : -INFINITY;
        float m = l;
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, x));
        if (m > M) {
            const float f = ex2(M - m);           // from -inf: 0, and all sums are 0
            L *= f;
            y.x *= f;
            y.y *= f;
            y.z *= f;
            y.w *= f;
            M = m;
        }
        const float w = l != l ? l : M == -INFINITY ? 0.f : ex2(l - M);
        const int here = min(32, n - b);
#pragma unroll 8
        for (int i = 0; i < here; i++) {
            const float wi = __shfl_sync(~0u, w, i);
            const float4 z = *reinterpret_cast<const float4*>(part_o + ((int64_t)__shfl_sync(~0u, at, i) * t.Hkv + h) * D + 4 * lane);
            L += wi;
            if (wi == 0.f) continue;              // (0 times an infinity is not 0)
            y.x += wi * z.x;
            y.y += wi * z.y;
            y.z += wi * z.z;
            y.w += wi * z.w;
        }
    }
    if constexpr (W > 1) {
        so[warp][lane] = y;
        if (lane == 0) stats[warp] = make_float2(M, L);
        __syncthreads();
        if (warp != 0) return;
#pragma unroll
        for (int x = 0; x < W; x++) M = fmaxf(M, stats[x].x);
        L = 0.f;
        y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < W; x++) {
            const float2 part = stats[x];
            if (part.y == 0.f) continue;          // (NaN goes on)
            const float f = part.x == -INFINITY ? 1.f : ex2(part.x - M);
            const float4 z = so[x][lane];
            L += f * part.y;
            y.x += f * z.x;
            y.y += f * z.y;
            y.z += f * z.z;
            y.w += f * z.w;
        }
    }
    const bool none = L == 0.f;
    const float inv = none ? 0.f : 1.f / L;
    *reinterpret_cast<uint2*>(o + out * D + 4 * lane) = make_uint2(pack_bf16(y.x * inv, y.y * inv), pack_bf16(y.z * inv, y.w * inv));
    if (lane == 0) lse[out] = none ? -INFINITY : (M + log2f(L)) * LN2;
}

template <bool F8, int NR>
int32_t launch_narrow(const Tables& t, int n_lists, const Call& a, bool follows) {
    using S = Shape<F8, NR>;
    static std::atomic<uint64_t> set{0};
    if (!gen_shared_memory(narrow_kernel<F8, NR>, S::bytes, set)) return HARTS_ECUDA;
    const auto *q = static_cast<const __nv_bfloat16*>(a.q);
    auto* o = static_cast<__nv_bfloat16*>(a.o);
    if (follows)
        return launch_after(narrow_kernel<F8, NR>, n_lists * t.Hkv, NT, S::bytes, a.stream, t, q, a.ld_q, a.map_k, a.map_v, a.cache.k_exp, a.cache.v_exp,
                            a.q_pos, a.scale_log2, o, a.lse, a.part_o, a.part_lse, a.dev_status) == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
    narrow_kernel<F8, NR><<<n_lists * t.Hkv, NT, S::bytes, a.stream>>>(t, q, a.ld_q, a.map_k, a.map_v, a.cache.k_exp, a.cache.v_exp, a.q_pos, a.scale_log2, o,
                                                                      a.lse, a.part_o, a.part_lse, a.dev_status);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}

}  // namespace

int32_t gen_attn_launch(const int32_t* hi, const int32_t* di, const void* q, int64_t ld_q, const GenCache& c, const int32_t* q_pos, void* o,
                 float* lse, float scale, void* workspace, int32_t* dev_status, cudaStream_t st) {
    Tables t;
    t.entries = reinterpret_cast<const Entry*>(di + hi[ENTRY]);
    t.pages = di + hi[PAGES];
    t.part_ptr = di + hi[PART_PTR];
    t.part = di + hi[PART];
    t.n_q = hi[N_Q];
    t.Hq = hi[HQ];
    t.Hkv = hi[HKV];
    t.page = hi[PAGE];
    float* part_o = static_cast<float*>(workspace);
    float* part_lse = part_o + (size_t)hi[N_PARTS] * t.Hkv * D;
    if ((int64_t)std::max(hi[N_NARROW], hi[N_WIDE]) * t.Hkv > INT32_MAX) return HARTS_EINVAL;
    const bool f8 = c.type == HARTS_E4M3;
    Call a{q, ld_q, {}, {}, c, q_pos, o, lse, part_o, part_lse, scale * LOG2E, dev_status, st};
    int32_t rc;
    if (hi[N_NARROW] > 0 || hi[N_WIDE] > 0) {
        if ((rc = make_cache_map(&a.map_k, c.k, (int64_t)c.n_pages * t.Hkv, t.page, f8)) != HARTS_OK) return rc;
        if ((rc = make_cache_map(&a.map_v, c.v, (int64_t)c.n_pages * t.Hkv, t.page, f8)) != HARTS_OK) return rc;
    }
    if (hi[N_WIDE] > 0) {
        t.units = reinterpret_cast<const Unit*>(di + hi[WIDE]);
        if ((rc = launch_wide(t, hi[N_WIDE], a)) != HARTS_OK) return rc;
    }
    if (hi[N_NARROW] > 0) {
        t.units = reinterpret_cast<const Unit*>(di + hi[NARROW]);
        auto* narrow = hi[NARROW_MAX] <= 8 ? (f8 ? launch_narrow<true, 1> : launch_narrow<false, 1>) : (f8 ? launch_narrow<true, 2> : launch_narrow<false, 2>);
        t.list_ptr = di + hi[LIST_PTR];
        if ((rc = narrow(t, hi[N_LISTS], a, hi[N_WIDE] > 0)) != HARTS_OK) return rc;
    }
    if (hi[MERGED]) {
        const int heads = t.n_q * t.Hq;           // (it fits: the index saw to it)
        const bool few = heads <= 4 * sm_count();
        auto* kernel = few ? merge_kernel<4> : merge_kernel<1>;
        const int grid = few ? heads : (int)(((int64_t)heads + MERGE_WARPS - 1) / MERGE_WARPS);
        if (hi[N_NARROW] == 0 && hi[N_WIDE] == 0) {           // nobody sees anything: this is the call's first kernel, and what ran before may have written the index
            kernel<<<grid, MERGE_WARPS * 32, 0, st>>>(t, part_o, part_lse, static_cast<__nv_bfloat16*>(o), lse);
            return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
        }
        if (launch_after(kernel, grid, MERGE_WARPS * 32, 0, st, t, (const float*)part_o, (const float*)part_lse, (__nv_bfloat16*)o, lse) != cudaSuccess)
            return HARTS_ECUDA;
    }
    return HARTS_OK;
}

}  // namespace harts
