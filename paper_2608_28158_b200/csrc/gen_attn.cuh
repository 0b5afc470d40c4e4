// Shared by the kernels of harts_gen_attn: the device view of the index, a unit's rows, 8-bit values as fp16.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gen.h"
#include "tc_common.cuh"

namespace harts {

int32_t make_cache_map(CUtensorMap* map, const void* base, int64_t n, int32_t page, bool bytes);
int sm_count();

namespace gen_attn {

constexpr int D = 128, TILE = 64;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float RAISE = 8.f;            // a running maximum follows in steps of at least 2^8

struct Tables {
    const Unit* units;
    const Entry* entries;
    const int32_t *pages, *part_ptr, *part, *list_ptr;
    int n_q, Hq, Hkv, page;
};
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

// two 8-bit values, the lower halves of x, as fp16
__device__ __forceinline__ uint32_t widen(uint32_t x) {
    uint32_t y;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t widen_upper(uint32_t x) {
    uint32_t y;
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// Position in a ring of N stages, and the parity of its barriers in this lap.
template <int N>
struct Ring {
    int st = 0;
    uint32_t ph = 0;
    __device__ __forceinline__ void next() {
        if (++st == N) {
            st = 0;
            ph ^= 1;
        }
    }
};

// The pages of a unit's boxes (up to 64 tokens of one page), asked for 32 at a time by a whole warp and a batch ahead of their use, so that
// copies do not wait for table entries.
struct PageWalk {
    const int32_t* pages;
    int tile0, end, box_shift, page_shift, lane, batch = -1, now = 0, next = 0;
    __device__ PageWalk(const Tables& t, const Unit& u, int tile0_, int end_) : pages(t.pages + u.page0), tile0(tile0_), end(end_), lane(threadIdx.x & 31) {
        box_shift = 31 - __clz(min(t.page, TILE));
        page_shift = 31 - __clz(t.page);
        next = ask(0);
    }
    __device__ int ask(int i) const {            // batch i
        const int j = tile0 + ((32 * i + lane) << box_shift);
        return j < end ? pages[j >> page_shift] : 0;
    }
    __device__ int of(int box) {                 // boxes in order; the whole warp
        if (box >> 5 != batch) {
            batch = box >> 5;
            now = next;
            next = ask(batch + 1);
        }
        return __shfl_sync(~0u, now, box & 31);
    }
};

// What brings a row of bf16 queries to 2^to: 2^x with x = to less the largest exponent (top: bits of the largest magnitude);
// infinities and NaN as they are.  Applied in two steps, as 2^x may be beyond fp32's powers.
struct PowerOfTwo {
    float f1, f2;
    int x1, x2;
    __device__ __forceinline__ PowerOfTwo(uint32_t top, int to) {
        const int e = (int)(top >> 7), x = e == 255 ? 0 : to + 127 - max(e, 1);        // (subnormal rows: as the smallest normal ones)
        x1 = x / 2;
        x2 = x - x1;
        f1 = __uint_as_float((uint32_t)(127 + x1) << 23);
        f2 = __uint_as_float((uint32_t)(127 + x2) << 23);
    }
    __device__ __forceinline__ float2 apply(uint32_t pair) const {
        return make_float2(__uint_as_float(pair << 16) * f1 * f2, __uint_as_float(pair & 0xffff0000u) * f1 * f2);
    }
    __device__ __forceinline__ float undone(float scale) const {
        return scale * __uint_as_float((uint32_t)(127 - x1) << 23) * __uint_as_float((uint32_t)(127 - x2) << 23);
    }
};

struct Call {                           // what the kernels are launched with
    const void* q;
    int64_t ld_q;
    CUtensorMap map_k, map_v;
    GenCache cache;
    const int32_t* q_pos;
    void* o;
    float *lse, *part_o, *part_lse;
    float scale_log2;
    int32_t* dev_status;
    cudaStream_t stream;
};
int32_t launch_wide(const Tables& t, int n_units, const Call& a);       // gen_attn_wide.cu

}  // namespace gen_attn
}  // namespace harts
