// Attention of sampled tokens on the cached tree: the narrow kernel (up to 16 rows -- a query and a head of its group -- that read the
// same run of tokens) and the merge of parts.
//
//     s_j = scale q . k_j    p_j = exp(s_j - m)    o = sum p_j v_j / sum p_j
//
// One CTA per (unit, key head): a warp asks for the pages by TMA, 64 tokens a stage; four warps take 16 of the 64 tokens each, so that every
// key and value is read from shared memory once.  Products are m16n8k16 with the rows as m: at 16 rows a token the work is far below any
// tensor path's rate, and its fragments let a warp keep scores, softmax and sums in registers.  A warp has its own running
// maximum (raised in steps of 2^8 and more), sum and output; the four are joined at the unit's end.
// 8-bit values become bf16 by moving bits and a multiplication by 2^120 (exact); which of the 128 elements a fragment's place
// holds is free as long as both operands agree, so that a thread takes 32 bytes in a row of a key and 16 of a value.  A key's power of
// two multiplies its score, a value's its p.
// Bound by the cache's bytes.
#include <cuda_bf16.h>

#include "gen.h"
#include "kernels.h"
#include "tc_common.cuh"

namespace harts {

int32_t make_cache_map(CUtensorMap* map, const void* base, int64_t n, int32_t page, bool bytes);
int sm_count();

namespace {

using namespace tc;
using namespace gen_attn;

constexpr int D = 128, TILE = 64, CW = 4, NT = CW * 32 + 32;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float RAISE = 8.f;

struct Tables {
    const Unit* units;
    const Entry* entries;
    const int32_t *pages, *part_ptr, *part;
    int n_q, Hq, Hkv, page;
};
template <bool F8>
struct Shape {
    static constexpr int KV = TILE * D * (F8 ? 1 : 2), EXP = F8 ? TILE : 0, STAGE = 2 * KV + 2 * EXP, STAGES = F8 ? 5 : 3;
    // the exponents of a stage lie behind all tiles (which start on 1,024 bytes)
    static constexpr int exps = STAGES * 2 * KV, misc = exps + STAGES * 2 * EXP, bytes = misc + 256 + 1024;
    static constexpr int PITCH = D + 4;                       // floats of a row of O where the warps' parts are joined
    static_assert(CW * NARROW_ROWS * (PITCH + 2) * 4 <= exps, "room for the parts");
};
struct Misc {
    uint64_t full[5], empty[5];
    int dead;
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t saddr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
// Two 8-bit values in the upper bytes of the halves of y, as bf16: sign | exponent and fraction four places down, times 2^120.
__device__ __forceinline__ uint32_t widen(uint32_t y) {
    const uint32_t x = ((y >> 4) & 0x07f007f0u) | (y & 0x80008000u);
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(0x7b807b80u));
    return r;
}
__device__ __forceinline__ bool nonfinite(uint32_t x) { return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u; }

// Row i of a unit: its query and the query head; what it sees ends at `limit`.
struct Row {
    int row, head, limit;
    bool alone;                     // the query has no other part
};
__device__ __forceinline__ Row row_of(const Tables& t, const Unit& u, int i, int h, const int32_t* q_pos, int32_t* status) {
    const int G = t.Hq / t.Hkv, flat = u.flat0 + min(i, u.n - 1);
    const Entry e = t.entries[u.entry + flat / G];
    Row r;
    r.row = e.row;
    r.head = h * G + flat % G;
    r.alone = e.most < 0;
    r.limit = e.limit;
    if (e.limit < 0) {
        const int most = e.most < 0 ? -e.most - 1 : e.most, pos = q_pos[e.row];
        r.limit = pos < e.least ? (pos + 1 < e.least ? e.least : pos + 1) : pos >= most ? most : pos + 1;
        if (status && (pos + 1 < e.least || pos >= most)) gen_report(status, e.row);
    }
    if (i >= u.n) r.limit = 0;
    return r;
}

template <bool F8>
__global__ void __launch_bounds__(NT, 2)
narrow_kernel(const Tables t, const __nv_bfloat16* __restrict__ q, int64_t ld_q, const __grid_constant__ CUtensorMap map_k,
              const __grid_constant__ CUtensorMap map_v, const uint8_t* __restrict__ k_exp, const uint8_t* __restrict__ v_exp,
              const int32_t* __restrict__ q_pos, float scale_log2, __nv_bfloat16* __restrict__ o, float* __restrict__ lse, float* __restrict__ part_o,
              float* __restrict__ part_lse, int* status) {
    using S = Shape<F8>;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    Misc& m = *reinterpret_cast<Misc*>(smem + S::misc);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const Unit u = t.units[blockIdx.x / t.Hkv];
    const int h = blockIdx.x % t.Hkv;
    if (tid == 0) {
        for (int i = 0; i < S::STAGES; i++) {
            mbar_init(&m.full[i], 1);
            mbar_init(&m.empty[i], CW);
        }
        m.dead = 0;
        fence_barrier_init();
    }
    // rows g and g + 8 of this thread; the farthest token that any row sees, and the nearest limit
    const int g = lane >> 2, c = lane & 3;
    Row row[2];
    int far = 0, near = INT32_MAX;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        row[i] = row_of(t, u, g + 8 * i, h, q_pos, tid < 32 && c == 0 ? status : nullptr);
        if (g + 8 * i < u.n) {
            far = max(far, row[i].limit);
            near = min(near, row[i].limit);
        }
    }
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) {
        far = max(far, __shfl_xor_sync(~0u, far, x));
        near = min(near, __shfl_xor_sync(~0u, near, x));
    }
    const int k1 = min(u.k1, far), tile0 = u.k0 & ~(TILE - 1), n_tiles = k1 > u.k0 ? (k1 - tile0 + TILE - 1) / TILE : 0;
    __syncthreads();

    if (warp == CW) {
        // ---- pages: a box is up to 64 tokens of one page ----------------------------------------------------------------------------
        if (lane == 0) {
            const int box = min(t.page, TILE), box_shift = 31 - __clz(box), page_shift = 31 - __clz(t.page);
            for (int n = 0; n < n_tiles; n++) {
                const int st = n % S::STAGES;
                if (!mbar_wait(&m.empty[st], ((n / S::STAGES) & 1) ^ 1, status, &m.dead)) break;
                const int j0 = tile0 + n * TILE, boxes = (min(k1 - j0, TILE) + box - 1) >> box_shift;
                unsigned char *sk = smem + st * 2 * S::KV, *sv = sk + S::KV, *se = smem + S::exps + st * 2 * S::EXP;
                mbar_expect_tx(&m.full[st], boxes * box * (F8 ? 2 * D + 2 : 4 * D));
                for (int b = 0; b < boxes; b++) {
                    const int j = j0 + (b << box_shift), at = j & (t.page - 1);
                    const int64_t block = (int64_t)t.pages[u.page0 + (j >> page_shift)] * t.Hkv + h;
                    if constexpr (F8) {
                        tma_load_3d(sk + b * box * D, &map_k, 0, at, (int)block, &m.full[st]);
                        tma_load_3d(sv + b * box * D, &map_v, 0, at, (int)block, &m.full[st]);
                        bulk_load(se + b * box, k_exp + block * t.page + at, box, &m.full[st]);
                        bulk_load(se + TILE + b * box, v_exp + block * t.page + at, box, &m.full[st]);
                    } else {
                        for (int p = 0; p < 2; p++) {
                            tma_load_3d(sk + p * (S::KV / 2) + b * box * 128, &map_k, p * 64, at, (int)block, &m.full[st]);
                            tma_load_3d(sv + p * (S::KV / 2) + b * box * 128, &map_v, p * 64, at, (int)block, &m.full[st]);
                        }
                    }
                }
            }
        }
        __syncwarp();
    } else {
        uint32_t qa[8][4];                        // the rows' fragments
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const bool there = g + 8 * i < u.n;
            const __nv_bfloat16* src = q + (int64_t)row[i].row * ld_q + (int64_t)row[i].head * D;
#pragma unroll
            for (int ks = 0; ks < 8; ks++)
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    const int d = F8 ? 32 * c + 4 * ks + 2 * x : 16 * ks + 8 * x + 2 * c;
                    qa[ks][2 * x + i] = there ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
                }
        }
        float acc[16][4];
#pragma unroll
        for (int j = 0; j < 16; j++) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
        float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
        for (int n = 0; n < n_tiles; n++) {
            const int st = n % S::STAGES, j0 = tile0 + n * TILE, key0 = j0 + 16 * warp;
            if (!mbar_wait_warp(&m.full[st], (n / S::STAGES) & 1, status, &m.dead)) break;
            const unsigned char *sk = smem + st * 2 * S::KV, *sv = sk + S::KV, *se = smem + S::exps + st * 2 * S::EXP;
            float s[2][4] = {};
            if constexpr (F8) {
#pragma unroll
                for (int nt = 0; nt < 2; nt++) {
                    const int key = 16 * warp + 8 * nt + g;
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        const uint4 y = *reinterpret_cast<const uint4*>(sk + sw128_chunk(key, 2 * c + x));
                        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                        for (int i = 0; i < 4; i++)
                            mma16816(s[nt], qa[4 * x + i], widen(__byte_perm(w[i], 0, 0x1404)), widen(__byte_perm(w[i], 0, 0x3424)));
                    }
                }
            } else {
#pragma unroll
                for (int k2 = 0; k2 < 4; k2++)
#pragma unroll
                    for (int nt = 0; nt < 2; nt++) {
                        const int key = 16 * warp + 8 * nt + (lane & 7), ch = 4 * k2 + (lane >> 3);
                        uint32_t b[4];
                        ldmatrix_x4(smem_u32(sk) + (ch >> 3) * (S::KV / 2) + sw128_chunk(key, ch & 7), b);
                        mma16816(s[nt], qa[2 * k2], b[0], b[1]);
                        mma16816(s[nt], qa[2 * k2 + 1], b[2], b[3]);
                    }
            }
            // scores in log2 units; hidden tokens -inf
            float vp[2][2];
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int x = 0; x < 2; x++) {
                    float f = scale_log2;
                    if constexpr (F8) {
                        const int at = 16 * warp + 8 * nt + 2 * c + x;
                        f *= gen_power(se[at]);
                        vp[nt][x] = gen_power(se[TILE + at]);
                    }
                    s[nt][x] *= f;
                    s[nt][2 + x] *= f;
                }
            const bool edge = j0 < u.k0 || j0 + TILE > min(near, u.k1);
            if (edge)
#pragma unroll
                for (int nt = 0; nt < 2; nt++)
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const int key = key0 + 8 * nt + 2 * c + (x & 1);
                        if (key < u.k0 || key >= min(row[x >> 1].limit, k1)) s[nt][x] = -INFINITY;
                    }
            bool raise[2];
            float mx[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                mx[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(~0u, mx[i], 1));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(~0u, mx[i], 2));
                raise[i] = mx[i] > top[i] + RAISE || (top[i] == -INFINITY && mx[i] > -INFINITY);
            }
            if (__any_sync(~0u, raise[0] || raise[1])) {
                float f[2];
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    f[i] = raise[i] ? ex2(top[i] - mx[i]) : 1.f;          // from -inf: 0, and all sums are 0
                    if (raise[i]) top[i] = mx[i];
                    sum[i] *= f[i];
                }
#pragma unroll
                for (int j = 0; j < 16; j++) {
                    acc[j][0] *= f[0];
                    acc[j][1] *= f[0];
                    acc[j][2] *= f[1];
                    acc[j][3] *= f[1];
                }
            }
            uint32_t pa[4];
            const float base[2] = {top[0] == -INFINITY ? 0.f : top[0], top[1] == -INFINITY ? 0.f : top[1]};
#pragma unroll
            for (int nt = 0; nt < 2; nt++)
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    float p0 = ex2(s[nt][2 * i] - base[i]), p1 = ex2(s[nt][2 * i + 1] - base[i]);
                    sum[i] += p0 + p1;
                    if constexpr (F8) {           // (a hidden token's power may be anything)
                        p0 = p0 == 0.f ? 0.f : p0 * vp[nt][0];
                        p1 = p1 == 0.f ? 0.f : p1 * vp[nt][1];
                    }
                    pa[2 * nt + i] = pack_bf16(p0, p1);
                }
            if constexpr (F8) {
                const unsigned char* v0 = sv + sw128_chunk(16 * warp + 2 * c, g);
                const unsigned char* v1 = sv + sw128_chunk(16 * warp + 2 * c + 1, g);
                const uint4 a = *reinterpret_cast<const uint4*>(v0), b = *reinterpret_cast<const uint4*>(v1);
                const uint4 a8 = *reinterpret_cast<const uint4*>(v0 + 8 * 128), b8 = *reinterpret_cast<const uint4*>(v1 + 8 * 128);
                const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w}, wa8[4] = {a8.x, a8.y, a8.z, a8.w}, wb8[4] = {b8.x, b8.y, b8.z, b8.w};
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    mma16816(acc[4 * i], pa, widen(__byte_perm(wa[i], wb[i], 0x4000)), widen(__byte_perm(wa8[i], wb8[i], 0x4000)));
                    mma16816(acc[4 * i + 1], pa, widen(__byte_perm(wa[i], wb[i], 0x5010)), widen(__byte_perm(wa8[i], wb8[i], 0x5010)));
                    mma16816(acc[4 * i + 2], pa, widen(__byte_perm(wa[i], wb[i], 0x6020)), widen(__byte_perm(wa8[i], wb8[i], 0x6020)));
                    mma16816(acc[4 * i + 3], pa, widen(__byte_perm(wa[i], wb[i], 0x7030)), widen(__byte_perm(wa8[i], wb8[i], 0x7030)));
                }
            } else {
                bool bad = false;
                if (edge) {
                    // Behind the last token that any row sees: zeros (this warp's tokens; it is the last tile, nothing is loaded over them).
                    // Values that some rows see and others do not may be infinite or NaN, and 0 times that is not 0.
                    if (key0 + 16 > k1) {
#pragma unroll 1
                        for (int e = lane + 16 * max(k1 - key0, 0); e < 256; e += 32)
                            *reinterpret_cast<uint4*>(smem + st * 2 * S::KV + S::KV + ((e & 15) >> 3) * (S::KV / 2) + sw128_chunk(16 * warp + (e >> 4), e & 7)) =
                                make_uint4(0, 0, 0, 0);
                        __syncwarp();
                    }
#pragma unroll
                    for (int x = 0; x < 2; x++) {
                        const int key = key0 + 2 * c + 8 * x;
                        uint32_t any = 0;
#pragma unroll 1
                        for (int e = 0; e < 2; e++) {
                            if (key + e >= k1 || (key + e >= u.k0 && key + e < near)) continue;
#pragma unroll 1
                            for (int ch = g; ch < 16; ch += 8) {
                                const uint4 y = *reinterpret_cast<const uint4*>(sv + (ch >> 3) * (S::KV / 2) + sw128_chunk(key + e - j0, ch & 7));
                                any |= nonfinite(y.x) || nonfinite(y.y) || nonfinite(y.z) || nonfinite(y.w);
                            }
                        }
                        bad |= any != 0;
                    }
                    bad = __any_sync(~0u, bad);
                }
                if (!bad) {
#pragma unroll
                    for (int j2 = 0; j2 < 8; j2++) {
                        const int key = 16 * warp + (lane & 15), ch = 2 * j2 + (lane >> 4);
                        uint32_t b[4];
                        ldmatrix_x4_trans(smem_u32(sv) + (ch >> 3) * (S::KV / 2) + sw128_chunk(key, ch & 7), b);
                        mma16816(acc[2 * j2], pa, b[0], b[1]);
                        mma16816(acc[2 * j2 + 1], pa, b[2], b[3]);
                    }
                } else {                           // row by row: what a row does not see adds nothing
#pragma unroll 1
                    for (int key = 0; key < 16; key++) {
                        const int from = (lane & ~3) | ((key & 7) >> 1);
                        float p[2];
#pragma unroll
                        for (int i = 0; i < 2; i++) {
                            const uint32_t y = __shfl_sync(~0u, key < 8 ? pa[i] : pa[2 + i], from);
                            p[i] = __uint_as_float((key & 1) ? y & 0xffff0000u : y << 16);
                        }
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            const uint32_t y = *reinterpret_cast<const uint32_t*>(sv + (j >> 3) * (S::KV / 2) + sw128_chunk(16 * warp + key, j & 7) + 4 * c);
                            const float v0 = __uint_as_float(y << 16), v1 = __uint_as_float(y & 0xffff0000u);
#pragma unroll
                            for (int i = 0; i < 2; i++)
                                if (key0 + key >= u.k0 && key0 + key < min(row[i].limit, k1)) {
                                    acc[j][2 * i] += p[i] * v0;
                                    acc[j][2 * i + 1] += p[i] * v1;
                                }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.empty[st]);
        }
        // ---- the four warps' parts joined -----------------------------------------------------------------------------------------
#pragma unroll
        for (int i = 0; i < 2; i++) {
            sum[i] += __shfl_xor_sync(~0u, sum[i], 1);
            sum[i] += __shfl_xor_sync(~0u, sum[i], 2);
        }
        float* so = reinterpret_cast<float*>(smem);
        float* stats = so + CW * NARROW_ROWS * S::PITCH;                   // [warp][row]{maximum, sum}
        asm volatile("bar.sync 1, 128;" ::: "memory");                   // all warps have read all stages
#pragma unroll
        for (int i = 0; i < 2; i++) {
            float* dst = so + (warp * NARROW_ROWS + g + 8 * i) * S::PITCH;
#pragma unroll
            for (int j = 0; j < 16; j++) {
                if constexpr (F8) {
                    dst[32 * c + j] = acc[j][2 * i];
                    dst[32 * c + 16 + j] = acc[j][2 * i + 1];
                } else {
                    *reinterpret_cast<float2*>(dst + 8 * j + 2 * c) = make_float2(acc[j][2 * i], acc[j][2 * i + 1]);
                }
            }
            if (c == 0) *reinterpret_cast<float2*>(stats + 2 * (warp * NARROW_ROWS + g + 8 * i)) = make_float2(top[i], sum[i]);
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const int i = tid >> 3, e0 = (tid & 7) * 4;                       // row, and every 32nd element group of four
        if (i < u.n) {
            float w[CW], M = -INFINITY, L = 0.f;
#pragma unroll
            for (int x = 0; x < CW; x++) M = fmaxf(M, stats[2 * (x * NARROW_ROWS + i)]);
#pragma unroll
            for (int x = 0; x < CW; x++) {
                const float2 y = *reinterpret_cast<const float2*>(stats + 2 * (x * NARROW_ROWS + i));
                w[x] = y.x == -INFINITY ? 0.f : ex2(y.x - M);
                L += w[x] * y.y;
            }
            const bool none = M == -INFINITY && !(L != L);
            const float inv = none ? 0.f : 1.f / L;
            const Row r = row_of(t, u, i, h, q_pos, nullptr);
            const int64_t out = (int64_t)r.row * t.Hq + r.head, part = (int64_t)(u.part0 + u.flat0 + i) * t.Hkv + h;
#pragma unroll
            for (int b = 0; b < 4; b++) {
                const int e = e0 + 32 * b;
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
                if (!none)
#pragma unroll
                    for (int x = 0; x < CW; x++) {
                        if (w[x] == 0.f) continue;
                        const float4 z = *reinterpret_cast<const float4*>(so + (x * NARROW_ROWS + i) * S::PITCH + e);
                        y.x += w[x] * z.x;
                        y.y += w[x] * z.y;
                        y.z += w[x] * z.z;
                        y.w += w[x] * z.w;
                    }
                y.x *= inv;
                y.y *= inv;
                y.z *= inv;
                y.w *= inv;
                if (r.alone) *reinterpret_cast<uint2*>(o + out * D + e) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
                else *reinterpret_cast<float4*>(part_o + part * D + e) = y;
            }
            if (e0 == 0) {
                const float l2 = none ? -INFINITY : M + log2f(L);
                if (r.alone) lse[out] = l2 * LN2;
                else part_lse[part] = l2;
            }
        }
    }
    if (__syncthreads_or(m.dead)) drain_delay();          // abandoned: copies in flight must land before the CTA goes
}

// A query head's parts joined: one warp each, four elements a lane.  Queries of one part have been written by their unit.
constexpr int MERGE_WARPS = 4;
__global__ void __launch_bounds__(MERGE_WARPS * 32)
merge_kernel(const Tables t, const float* __restrict__ part_o, const float* __restrict__ part_lse, __nv_bfloat16* __restrict__ o, float* __restrict__ lse) {
    after_previous();
    const int64_t out = (int64_t)blockIdx.x * MERGE_WARPS + (threadIdx.x >> 5);
    if (out >= (int64_t)t.n_q * t.Hq) return;
    const int lane = threadIdx.x & 31, row = (int)(out / t.Hq), head = (int)(out % t.Hq), G = t.Hq / t.Hkv, h = head / G, g = head % G;
    const int p0 = t.part_ptr[row], p1 = t.part_ptr[row + 1];
    if (p1 == p0 + 1) return;
    float M = -INFINITY, L = 0.f;
    bool nan = false;
    for (int p = p0 + lane; p < p1; p += 32) {
        const float y = part_lse[(int64_t)(t.part[p] + g) * t.Hkv + h];
        M = fmaxf(M, y);
        nan |= y != y;
    }
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) M = fmaxf(M, __shfl_xor_sync(~0u, M, x));
    nan = __any_sync(~0u, nan);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (M > -INFINITY || nan) {
#pragma unroll 4
        for (int p = p0; p < p1; p++) {
            const int64_t at = (int64_t)(t.part[p] + g) * t.Hkv + h;
            const float w = ex2(part_lse[at] - M);
            const float4 z = *reinterpret_cast<const float4*>(part_o + at * D + 4 * lane);
            if (w == 0.f) continue;
            L += w;
            y.x += w * z.x;
            y.y += w * z.y;
            y.z += w * z.z;
            y.w += w * z.w;
        }
        const float inv = 1.f / L;
        y.x *= inv;
        y.y *= inv;
        y.z *= inv;
        y.w *= inv;
    }
    *reinterpret_cast<uint2*>(o + out * D + 4 * lane) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    if (lane == 0) lse[out] = M == -INFINITY && !nan ? -INFINITY : (M + log2f(L)) * LN2;
}

template <bool F8>
int32_t launch_narrow(const Tables& t, int n_units, const void* q, int64_t ld_q, const CUtensorMap& mk, const CUtensorMap& mv, const GenCache& c,
                      const int32_t* q_pos, void* o, float* lse, float scale, float* part_o, float* part_lse, int32_t* dev_status, cudaStream_t st) {
    using S = Shape<F8>;
    if (cudaFuncSetAttribute(narrow_kernel<F8>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::bytes) != cudaSuccess) return HARTS_ECUDA;
    narrow_kernel<F8><<<n_units * t.Hkv, NT, S::bytes, st>>>(t, (const __nv_bfloat16*)q, ld_q, mk, mv, c.k_exp, c.v_exp, q_pos, scale * LOG2E,
                                                           (__nv_bfloat16*)o, lse, part_o, part_lse, dev_status);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}

}  // namespace

int32_t gen_attn_launch(const int32_t* hi, const int32_t* di, const void* q, int64_t ld_q, const GenCache& c, const int32_t* q_pos, void* o,
                 float* lse, float scale, void* workspace, int32_t* dev_status, cudaStream_t st) {
    Tables t;
    t.units = reinterpret_cast<const Unit*>(di + hi[NARROW]);
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
    if (hi[N_NARROW] > 0) {
        if ((int64_t)hi[N_NARROW] * t.Hkv > INT32_MAX) return HARTS_EINVAL;
        CUtensorMap mk, mv;
        int32_t rc;
        const bool f8 = c.type == HARTS_E4M3;
        if ((rc = make_cache_map(&mk, c.k, (int64_t)c.n_pages * t.Hkv, t.page, f8)) != HARTS_OK) return rc;
        if ((rc = make_cache_map(&mv, c.v, (int64_t)c.n_pages * t.Hkv, t.page, f8)) != HARTS_OK) return rc;
        rc = f8 ? launch_narrow<true>(t, hi[N_NARROW], q, ld_q, mk, mv, c, q_pos, o, lse, scale, part_o, part_lse, dev_status, st)
                : launch_narrow<false>(t, hi[N_NARROW], q, ld_q, mk, mv, c, q_pos, o, lse, scale, part_o, part_lse, dev_status, st);
        if (rc != HARTS_OK) return rc;
    }
    if (hi[MERGED]) {
        const int64_t blocks = ((int64_t)t.n_q * t.Hq + MERGE_WARPS - 1) / MERGE_WARPS;
        if (blocks > INT32_MAX) return HARTS_EINVAL;
        if (launch_after(merge_kernel, (int)blocks, MERGE_WARPS * 32, 0, st, t, (const float*)part_o, (const float*)part_lse, (__nv_bfloat16*)o, lse) != cudaSuccess)
            return HARTS_ECUDA;
    }
    return HARTS_OK;
}

}  // namespace harts
