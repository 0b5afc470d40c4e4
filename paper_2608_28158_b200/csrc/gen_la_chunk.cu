// Linear attention from and into kept states in chunks (bf16, d = 128): the work table, and what lets several CTAs share one long
// sequence.
//
// The walk itself is pipe_fwd_kernel (la_pipe_fwd.cu): 2.2 us a chunk and head where a chain of chunks is all that an SM has, 3 in a mix.  A sequence that
// is long beside what every SM has to do is cut into segments of L chunks, whose start states are found first:
//     U_i = sum over segment i of e^{B_end - B_j} k_j^T v_j,   S_{i+1} = e^{B_i} S_i + U_i
// The sums do not depend on each other (one product of k~^T v with the tokens as its inner dimension, left in tensor memory until the
// segment's end); the recurrence over segments is a multiply-add per element.  That reads k and v twice, and 192 KB a segment and head.
#include <algorithm>

#include "gen.h"
#include "kernels.h"
#include "tc_common.cuh"

namespace harts {

int32_t make_row_map_ld(CUtensorMap* map, const void* base, int64_t rows, int32_t H, int64_t ld);
int sm_count();

namespace {

using namespace tc;

constexpr int BT = 64, D = 128;
constexpr int MIN_L = 4, MAX_L = 48;          // chunks of a segment (its weights stay in shared memory)
constexpr float LOG2E = 1.4426950408889634f;

struct Sizes {
    int64_t max_items;
    int least;                                // chunks of the shortest segments that the device may choose, 0: sequences are not cut
    size_t items, follows, chains, gamma, starts, total;
};
Sizes sizes_of(const GenLaArgs& a) {
    Sizes z;
    const int64_t longest = ((int64_t)a.max_len + BT - 1) / BT;
    int64_t chunks = a.n_rows / BT + a.n_seq;                       // there are at most that many
    if (chunks > longest * a.n_seq) chunks = longest * a.n_seq;
    const int64_t share = (chunks * a.H + sm_count() - 1) / sm_count(), room = sm_count() / a.H - a.n_seq;
    z.least = 0;
    if (longest > 8 && 2 * longest > 3 * share) {
        const int64_t L = room > 0 ? (chunks + room - 1) / room : (share + 1) / 2;
        // By the bounds: whether the passes that a cut needs are launched at all, which costs the time of some six chunks (16 sequences of 16 chunks
        // x 4 heads: in segments of 13 70 us, whole 45).  How long the segments are is chosen on the device, where the lengths are.
        if (4 * longest > 7 * (L > MAX_L ? MAX_L : L) + 24) {
            const int64_t least = share / 2 < 2 * L / 3 ? share / 2 : 2 * L / 3;
            z.least = (int)(least < MIN_L ? MIN_L : least > MAX_L ? MAX_L : least);
        }
    }
    z.max_items = a.n_seq + (z.least ? chunks / z.least : 0);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    z.items = 256;
    z.follows = up(z.items + (size_t)z.max_items * sizeof(int4));
    z.chains = up(z.follows + (size_t)z.max_items * sizeof(int));
    z.gamma = up(z.chains + (size_t)a.n_seq * sizeof(int4));
    z.starts = up(z.gamma + (z.least ? (size_t)z.max_items * a.H * sizeof(float) : 0));
    z.total = z.starts + (z.least ? (size_t)z.max_items * a.H * D * D * sizeof(float) : 0);
    return z;
}

constexpr int WHOLE = 2, CUT = 3;             // places behind the number of items: whole segments, sequences of several items
constexpr int PLAN_THREADS = 512, PLAN_WARPS = PLAN_THREADS / 32, CHOICES = 3 * PLAN_WARPS;
static_assert(CHOICES > MAX_L - MIN_L + 1, "a place for every length, and for no cut");

// How long segments are, in rows, for the sequences' lengths (len_of(i), -1: no item): every warp weighs three lengths, from `least` chunks on, the
// last place is no cut at all.  The time of a choice, in microseconds: the sums, an SM each in rounds, the recurrence over the longest
// sequence's segments, then the walk, whose items take an SM 6.8 and 3 a chunk: whole segments in rounds, or the SMs filled with the rest.  6 % off the
// measured ones (25 shapes x 27 lengths), and the choice 2 % from the best length; weighing takes 1 us.  Against one length from the bounds alone:
// 2 sequences of 15,000 and 1 tokens x 32 heads 298 -> 216 us, 1 of 31,017 x 16 327 -> 220, 3 of up to 20,000 x 16 200 -> 160, 1 of 31,017 x 4
// 81 -> 77 (with the sums' pipeline, which is 8 of each).
template <class LEN>
__device__ __forceinline__ int choose_rows(LEN len_of, int n_seq, int H, int least, int sms) {
    __shared__ float time[CHOICES];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto rows_of = [&](int i) { return i == CHOICES - 1 ? INT32_MAX : min(least + i, MAX_L) * BT; };
    struct Sum {
        int whole, sums, rests, chunks, most, longest;        // segments; those that are summed; rests, their chunks; the largest rest; a sequence's items
    } sum[3] = {};
    for (int i = lane; i < n_seq; i += 32) {
        const int len = len_of(i);
        if (len < 0) continue;
#pragma unroll
        for (int c = 0; c < 3; c++) {
            const int rows = rows_of(warp + PLAN_WARPS * c), whole = (int)((unsigned)len / (unsigned)rows), left = len - whole * rows, rest = len == 0 || left > 0,
                      chunks = (left + BT - 1) / BT;
            sum[c].whole += whole;
            sum[c].sums += max(whole + rest - 1, 0);
            sum[c].rests += rest;
            sum[c].chunks += chunks;
            sum[c].most = max(sum[c].most, chunks);
            sum[c].longest = max(sum[c].longest, whole + rest);
        }
    }
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 3; c++) {
        const int rows = rows_of(warp + PLAN_WARPS * c), whole = __reduce_add_sync(~0u, sum[c].whole) * H, sums = __reduce_add_sync(~0u, sum[c].sums) * H,
                  rests = __reduce_add_sync(~0u, sum[c].rests) * H, chunks = __reduce_add_sync(~0u, sum[c].chunks), most = __reduce_max_sync(~0u, sum[c].most),
                  longest = __reduce_max_sync(~0u, sum[c].longest);
        const unsigned rounds = (unsigned)(whole + sms - 1) / (unsigned)sms, sum_rounds = (unsigned)(sums + sms - 1) / (unsigned)sms;
        const float L = (float)(rows / BT), seg = whole > 0 ? 6.8f + 3.f * L : 0.f, last = rests > 0 ? 6.8f + 3.f * most : 0.f;
        float y = whole + rests <= sms ? fmaxf(seg, last)
                                       : fmaxf(fmaxf(rounds * seg, (whole * seg + rests * 6.8f + (float)chunks * H * 3.f) / sms + 0.5f * last), last);
        if (sums > 0) y += 0.2f * longest + sum_rounds * (4.f + 0.3f * L);
        if (lane == 0) time[warp + PLAN_WARPS * c] = y;
    }
    __syncthreads();
    float y = time[lane];
    int at = lane;
    auto take = [&](float y2, int at2) {
        if (y2 < y || (y2 == y && at2 < at)) {
            y = y2;
            at = at2;
        }
    };
    if (lane + 32 < CHOICES) take(time[lane + 32], lane + 32);
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        const float y2 = __shfl_xor_sync(~0u, y, x);
        take(y2, __shfl_xor_sync(~0u, at, x));
    }
    return rows_of(at);
}

// The items: whole segments first, in the order of the sequences, then what is left of each (the walk's CTAs draw them from a counter, so the
// short ones fill the gaps).  chains: of each sequence of several items, in any order, {first whole segment, items, start state, item of the rest or -1}.
__global__ void __launch_bounds__(PLAN_THREADS)
plan_kernel(const GenLaArgs a, int least, int sms, int max_items, int* count, int4* items, int* follows, int4* chains) {
    __shared__ int2 warp_sum[PLAN_WARPS];
    __shared__ int64_t warp_used[PLAN_WARPS];
    __shared__ int cut;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    let_next_launch();
    auto look_up = [&](int i, GenSeq& s, bool report) {           // its length, or -1: nothing to do
        if (i >= a.n_seq) return -1;
        if (!gen_seq(a, i, s)) {
            if (report) gen_report(a.dev_status, i);
            return -1;
        }
        return s.out < 0 && !(a.o && s.len > 0) ? -1 : s.len;
    };
    GenSeq s, s0;
    const int len0 = look_up(tid, s0, true);      // (kept: there are seldom more sequences than threads)
    const int rows = least ? choose_rows([&](int i) { return i == tid ? len0 : look_up(i, s, false); }, a.n_seq, a.H, least, sms) : INT32_MAX;
    auto parts = [&](int len) { return len < 0 ? make_int2(0, 0) : make_int2(len / rows, len == 0 || len % rows != 0); };        // {whole segments, rest}
    const int2 n0 = parts(len0);
    int2 all = n0;
    int64_t used = max(len0, 0);
    for (int i0 = PLAN_THREADS; i0 < a.n_seq; i0 += PLAN_THREADS) {
        const int len = look_up(i0 + tid, s, true);
        const int2 n = parts(len);
        all.x += n.x;
        all.y += n.y;
        used += max(len, 0);
    }
    for (int d = 16; d > 0; d >>= 1) {
        all.x += __shfl_xor_sync(~0u, all.x, d);
        all.y += __shfl_xor_sync(~0u, all.y, d);
        used += __shfl_xor_sync(~0u, used, d);
    }
    if (lane == 0) {
        warp_sum[warp] = all;
        warp_used[warp] = used;
    }
    __syncthreads();
    all = make_int2(0, 0);
    used = 0;
    for (int w = 0; w < PLAN_WARPS; w++) {
        all.x += warp_sum[w].x;
        all.y += warp_sum[w].y;
        used += warp_used[w];
    }
    __syncthreads();
    const int whole = all.x;
    // sequences that share rows could have more segments than the rows allow: none of them is done then
    const bool fits = whole + all.y <= max_items && (least == 0 || used <= a.n_rows);
    if (tid == 0) {
        if (!fits) gen_report(a.dev_status, 0);
        count[0] = fits ? whole + all.y : 0;
        count[1] = 0;                             // the walk's counter
        count[WHOLE] = fits ? whole : 0;
        cut = 0;
    }
    __syncthreads();
    int2 base = make_int2(0, whole);
    for (int i0 = 0; i0 < a.n_seq; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        const int2 n = i0 == 0 ? n0 : parts(look_up(i, s, false));
        if (i0 == 0) s = s0;
        int2 upto = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int x = __shfl_up_sync(~0u, upto.x, d), y = __shfl_up_sync(~0u, upto.y, d);
            if (lane >= d) {
                upto.x += x;
                upto.y += y;
            }
        }
        if (lane == 31) warp_sum[warp] = upto;
        __syncthreads();
        int2 at = make_int2(base.x + upto.x - n.x, base.y + upto.y - n.y);
        for (int w = 0; w < PLAN_WARPS; w++) {
            if (w < warp) {
                at.x += warp_sum[w].x;
                at.y += warp_sum[w].y;
            }
            base.x += warp_sum[w].x;
            base.y += warp_sum[w].y;
        }
        const int items_here = n.x + n.y;
        if (i < a.n_seq && fits) {
            for (int j = 0; j < items_here; j++) {
                const int item = j < n.x ? at.x + j : at.y;
                const bool last = j + 1 == items_here;
                items[item] = make_int4(s.begin + j * rows, j < n.x ? rows : s.len - j * rows, items_here > 1 ? -2 - item : s.in, last ? s.out : -1);
                follows[item] = !last;
            }
            if (items_here > 1) chains[atomicAdd(&cut, 1)] = make_int4(at.x, items_here, s.in, n.y ? at.y : -1);
        }
        __syncthreads();
    }
    if (tid == 0) count[CUT] = cut;
}

// ---- sums of segments --------------------------------------------------------------------------------------------------------
// A CTA an SM works off (segment, head) after (segment, head).  A chunk's keys are weighed by 16 warps, the first term in place, the others in one of two
// pairs of tiles, while the products of the chunk before run.
constexpr int PANEL = BT * 128, TILE = 2 * PANEL, STAGE = 2 * TILE, STAGES = 4, SUM_WARPS = 16, SUM_THREADS = SUM_WARPS * 32 + 64, WEIGHING = SUM_WARPS * 32;
struct SumMisc {
    float w[(MAX_L * BT + WEIGHING - 1) / WEIGHING * WEIGHING];
    float warp_sum[SUM_WARPS];
    uint64_t full[STAGES], ready[STAGES], done[STAGES];
    uint32_t tmem;
    int dead, stop;      // latch: a wait ran out; what the weighing warps have seen of it at a segment's end, all the same
};
// stages of k, v, then two times the second and third terms of weighted keys
constexpr int SUM_REST = STAGES * STAGE, SUM_MISC = SUM_REST + 4 * TILE, SUM_BYTES = SUM_MISC + sizeof(SumMisc) + 1024;
static_assert(SUM_BYTES <= 227 * 1024, "shared memory");

// (What the kernel ahead writes is not __restrict__ here and below: loads of what never changes could be moved ahead of the wait for it.)
__global__ void __launch_bounds__(SUM_THREADS, 1)
sum_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const float* __restrict__ g, int H,
           const GenItems gen, const int* follows, float* __restrict__ gamma, int* status) {
    let_next_launch();
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    SumMisc& m = *reinterpret_cast<SumMisc*>(smem + SUM_MISC);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < STAGES; i++) {
            mbar_init(&m.full[i], 1);
            mbar_init(&m.ready[i], SUM_WARPS);
            mbar_init(&m.done[i], 1);
        }
        m.dead = 0;
        fence_barrier_init();
    }
    if (warp == 0) {
        __syncwarp();
        tmem_alloc<128>(&m.tmem);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = m.tmem;
    after_previous();
    const int units = gen.count[WHOLE] * H;       // only whole segments are followed by another one
    // the CTA's next (segment, head) from `unit` on: its first row and chunks
    struct Segment {
        int item, h, begin, len, n_chunks;
    };
    auto take = [&](int& unit, Segment& x) {
        for (; unit < units; unit += gridDim.x) {
            x.item = unit / H;
            if (!follows[x.item]) continue;
            const int4 it = gen.items[x.item];
            x.h = unit - x.item * H;
            x.begin = it.x;
            x.len = it.y;
            x.n_chunks = it.y / BT;
            unit += gridDim.x;
            return true;
        }
        return false;
    };
    Segment x;
    int n = 0, unit = blockIdx.x;                 // n: chunks so far
    if (warp == SUM_WARPS) {
        // ---- loads -------------------------------------------------------------------------------------------------------------
        bool alive = true;
        while (alive && take(unit, x))
            for (int c = 0; c < x.n_chunks; c++, n++) {
                const int st = n % STAGES;
                if (n >= STAGES && !(alive = mbar_wait_warp(&m.done[st], ((n / STAGES) - 1) & 1, status, &m.dead))) break;
                if (lane == 0) {
                    unsigned char* tile = smem + st * STAGE;
                    mbar_expect_tx(&m.full[st], 2 * TILE);
                    for (int p = 0; p < 2; p++) {
                        tma_load_3d(tile + p * PANEL, &map_k, p * 64, x.h, x.begin + c * BT, &m.full[st]);
                        tma_load_3d(tile + TILE + p * PANEL, &map_v, p * 64, x.h, x.begin + c * BT, &m.full[st]);
                    }
                }
                __syncwarp();
            }
    } else if (warp == SUM_WARPS + 1) {
        // ---- products ----------------------------------------------------------------------------------------------------------
        constexpr uint32_t IDESC = instr_desc(128, 128, 1, 1);
        bool alive = true;
        while (alive && take(unit, x))
            for (int c = 0; c < x.n_chunks; c++, n++) {
                const int st = n % STAGES;
                if (!(alive = mbar_wait_warp(&m.ready[st], (n / STAGES) & 1, status, &m.dead))) break;
                tc_fence_after();
                const uint32_t tile = smem_u32(smem + st * STAGE), rest = smem_u32(smem + SUM_REST + (n & 1) * 2 * TILE);
                if (elect_one()) {
#pragma unroll
                    for (int term = 0; term < 3; term++)
#pragma unroll
                        for (int ks = 0; ks < 4; ks++)
                            mma_ss(tmem, desc_mnmajor<BT>(term == 0 ? tile : rest + (term - 1) * TILE, ks), desc_mnmajor<BT>(tile + TILE, ks), IDESC, c > 0 || term > 0 || ks > 0);
                    mma_commit(&m.done[st]);
                }
                __syncwarp();
            }
    } else {
        while (take(unit, x)) {
            // ---- weights e^{B_end - B_j}: some tokens in a row per thread, summed from the end ----------------------------------------
            const int per = (x.len + WEIGHING - 1) / WEIGHING;         // (behind the segment: nothing decays)
            for (int e = tid; e < per * WEIGHING; e += WEIGHING) m.w[e] = e < x.len ? g[(size_t)(x.begin + e) * H + x.h] * LOG2E : 0.f;
            asm volatile("bar.sync 1, %0;" ::"n"(WEIGHING) : "memory");
            float own = 0.f;
            for (int e = 0; e < per; e++) own += m.w[tid * per + e];
            float behind = own;                   // of this thread and the ones behind it in the warp
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const float y = __shfl_down_sync(~0u, behind, d);
                if (lane + d < 32) behind += y;
            }
            if (lane == 0) m.warp_sum[warp] = behind;
            asm volatile("bar.sync 1, %0;" ::"n"(WEIGHING) : "memory");
            float after = __shfl_down_sync(~0u, behind, 1), total = 0.f;
            if (lane == 31) after = 0.f;
            for (int w = SUM_WARPS - 1; w >= 0; w--) {
                if (w > warp) after += m.warp_sum[w];
                total += m.warp_sum[w];
            }
            for (int e = per - 1; e >= 0; e--) {
                const float y = m.w[tid * per + e];
                m.w[tid * per + e] = ex2(after);
                after += y;
            }
            if (tid == 0) gamma[(size_t)x.item * H + x.h] = ex2(total);
            asm volatile("bar.sync 1, %0;" ::"n"(WEIGHING) : "memory");
            bool alive = true;
            for (int c = 0; c < x.n_chunks; c++, n++) {
                const int st = n % STAGES;
                if (!(alive = mbar_wait_warp(&m.full[st], (n / STAGES) & 1, status, &m.dead))) break;
                // the tiles of second and third terms: the products of two chunks ago are done
                if (n >= 2 && !(alive = mbar_wait_warp(&m.done[(n - 2) % STAGES], ((n - 2) / STAGES) & 1, status, &m.dead))) break;
                unsigned char *tile = smem + st * STAGE, *rest = smem + SUM_REST + (n & 1) * 2 * TILE;
#pragma unroll
                for (int u = 0; u < 2 * PANEL / 16 / WEIGHING; u++) {
                    const int e = tid + u * WEIGHING, t = (e >> 3) & (BT - 1), off = (e >> 9) * PANEL + sw128_chunk(t, e & 7);
                    const float w = m.w[c * BT + t];
                    uint4 y = *reinterpret_cast<const uint4*>(tile + off), z, z2;
                    three_terms(y.x, z.x, z2.x, f2(w, w));
                    three_terms(y.y, z.y, z2.y, f2(w, w));
                    three_terms(y.z, z.z, z2.z, f2(w, w));
                    three_terms(y.w, z.w, z2.w, f2(w, w));
                    *reinterpret_cast<uint4*>(tile + off) = y;
                    *reinterpret_cast<uint4*>(rest + off) = z;
                    *reinterpret_cast<uint4*>(rest + TILE + off) = z2;
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.ready[st]);
            }
            if (alive && mbar_wait_warp(&m.done[(n - 1) % STAGES], ((n - 1) / STAGES) & 1, status, &m.dead)) {
                tc_fence_after();
                const int quarter = warp & 3, col = (warp >> 2) * 32;
                float* dst = gen.starts + ((size_t)x.item * H + x.h) * (D * D) + (size_t)(quarter * 32 + lane) * D + col;
                uint32_t y[32];
                tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + col, y);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; e++) *reinterpret_cast<uint4*>(dst + 4 * e) = make_uint4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
            }
            tc_fence_before();                    // (the next segment's first product is behind these warps' arrivals)
            asm volatile("bar.sync 1, %0;" ::"n"(WEIGHING) : "memory");
            if (tid == 0) m.stop = m.dead;
            asm volatile("bar.sync 1, %0;" ::"n"(WEIGHING) : "memory");
            if (m.stop) break;                    // (all of them: they meet at these barriers)
        }
    }
    __syncwarp();
    if (__syncthreads_or(m.dead)) drain_delay();          // abandoned: copies and MMAs in flight must land before the CTA goes
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc<128>(tmem);
}

// ---- start states of segments: starts[i] holds U_i on entry and S_i afterwards; four elements a thread -------------------------------
constexpr int BATCH = 8, BLOCKS = D * D / 1024;
// CTAs that fit take (sequence of several items, head, part of a state) in turn: a CTA for each, of all sequences, took 23 x 16 of 1 to 6,000 tokens
// 160 us instead of 157.
__global__ void __launch_bounds__(256)
scan_kernel(const float* __restrict__ states, float* starts, const int* count, const int4* chains, const float* gamma, int H) {
    let_next_launch();
    after_previous();
    int4 chain = chains[blockIdx.x / (H * BLOCKS)];           // (there are not more CTAs than these would do; read beside the count)
    const int units = count[CUT] * H * BLOCKS;
    for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
        if (unit != blockIdx.x) chain = chains[unit / (H * BLOCKS)];
        const int h = unit / BLOCKS % H;
        const size_t off = (size_t)(unit % BLOCKS * 256 + threadIdx.x) * 4;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (chain.z >= 0) s = *reinterpret_cast<const float4*>(states + ((size_t)chain.z * H + h) * (D * D) + off);
        auto item = [&](int j) { return j + 1 == chain.y && chain.w >= 0 ? chain.w : chain.x + j; };
        auto at = [&](int j) { return reinterpret_cast<float4*>(starts + ((size_t)item(j) * H + h) * (D * D) + off); };
        for (int j0 = 0; j0 < chain.y; j0 += BATCH) {
            float4 u[BATCH];
            float e[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; j++)
                if (j0 + j + 1 < chain.y) {
                    u[j] = *at(j0 + j);
                    e[j] = gamma[(size_t)item(j0 + j) * H + h];
                }
#pragma unroll
            for (int j = 0; j < BATCH; j++)
                if (j0 + j < chain.y) {
                    *at(j0 + j) = s;
                    if (j0 + j + 1 < chain.y) {
                        s.x = fmaf(e[j], s.x, u[j].x);
                        s.y = fmaf(e[j], s.y, u[j].y);
                        s.z = fmaf(e[j], s.z, u[j].z);
                        s.w = fmaf(e[j], s.w, u[j].w);
                    }
                }
        }
    }
}

}  // namespace

// Tokens one by one or chunks, tokens a sequence: a walk costs about a microsecond a token where states wait for a free SM, a chunk the same
// for 1 to 64.  200 branches x 32 heads: 12 tokens 292 us, 14 339, a chunk 311; 64 x 16: 61 at 14, 65 at 16, a chunk 64.  Where every state has an SM
// (8 x 16), 14.6 at 16 and a chunk 18.5.
bool gen_la_chunked(const GenLaArgs& a) {
    return a.dtype == HARTS_BF16 && a.d == 128 && a.max_len > ((int64_t)a.n_seq * a.H > 2 * sm_count() ? 12 : 20);
}

size_t gen_la_chunk_bytes(const GenLaArgs& a) { return sizes_of(a).total; }

int32_t gen_la_chunks(const GenLaArgs& a) {
    const Sizes z = sizes_of(a);
    char* ws = static_cast<char*>(a.workspace);
    if (z.max_items * a.H * 2 > INT32_MAX) return HARTS_EINVAL;
    int* count = reinterpret_cast<int*>(ws);
    int4 *items = reinterpret_cast<int4*>(ws + z.items), *chains = reinterpret_cast<int4*>(ws + z.chains);
    int* follows = reinterpret_cast<int*>(ws + z.follows);
    float *gamma = reinterpret_cast<float*>(ws + z.gamma), *starts = reinterpret_cast<float*>(ws + z.starts);
    plan_kernel<<<1, PLAN_THREADS, 0, a.stream>>>(a, z.least, sm_count(), (int)z.max_items, count, items, follows, chains);
    if (cudaGetLastError() != cudaSuccess) return HARTS_ECUDA;
    const GenItems gen{count, count + 1, items, starts};
    if (z.least) {
        CUtensorMap mk, mv;
        int32_t rc;
        if ((rc = make_row_map_ld(&mk, a.k, a.n_rows, a.H, a.ld_k)) != HARTS_OK) return rc;
        if ((rc = make_row_map_ld(&mv, a.v, a.n_rows, a.H, a.ld_v)) != HARTS_OK) return rc;
        static std::atomic<uint64_t> set{0};
        if (!gen_shared_memory(sum_kernel, SUM_BYTES, set)) return HARTS_ECUDA;
        if (launch_after(sum_kernel, (int)std::min<int64_t>(z.max_items * a.H, sm_count()), SUM_THREADS, SUM_BYTES, a.stream, mk, mv, a.g, a.H, gen, (const int*)follows, gamma,
                         a.dev_status) != cudaSuccess)
            return HARTS_ECUDA;
        if (launch_after(scan_kernel, (int)std::min<int64_t>((int64_t)a.n_seq * a.H * BLOCKS, 3 * sm_count()), 256, 0, a.stream, (const float*)a.states, starts, (const int*)count,
                         (const int4*)chains, (const float*)gamma, (int)a.H) != cudaSuccess)
            return HARTS_ECUDA;
    }
    return pipe_gen(a, gen, z.max_items);
}

}  // namespace harts
