// Keys and values into the pages of a cache and back (harts_gen_cache_write / _read), bf16 or 8 bits with a power of two a row.
//
// Eight lanes a row of 128: each has 16 values, so that a row is read by eight 32-byte pieces and written as 8-bit values by eight
// 16-byte ones.  The scale being a power of two, x 2^-e is exact and rounding is that of the significand alone (values far below the
// row's largest lose bits as subnormals do).  Bound by the traffic, 512 + 258 bytes a (token, head)
// either way: 16,385 tokens x 8 heads written in 21.3 us (4.7 TB/s), 24,000 x 4 read in 16.1 (4.6); kernels alone, inputs larger than the L2.
// bf16, call and launch: 16,385 x 8 in 25.0 either way (0.82 of a copy), 24,000 x 4 in 20.5 (0.74).
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "gen.h"

namespace harts {
namespace {

constexpr int D = 128, LANES = 8, NT = 256;

// largest of 16 values' magnitudes, as bits
__device__ __forceinline__ uint32_t top_of(const uint4 (&x)[2]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        m = __vmaxu2(m, x[i].x & 0x7fff7fffu);
        m = __vmaxu2(m, x[i].y & 0x7fff7fffu);
        m = __vmaxu2(m, x[i].z & 0x7fff7fffu);
        m = __vmaxu2(m, x[i].w & 0x7fff7fffu);
    }
    return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ uint32_t two_e4m3(uint32_t x, float f) {
    return __nv_cvt_float2_to_fp8x2(make_float2(__uint_as_float(x << 16) * f, __uint_as_float(x & 0xffff0000u) * f), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ uint32_t two_bf16(uint32_t y, float f) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(y & 0xffffu), __NV_E4M3);
    const float2 x = __half22float2(__half2(h));
    const __nv_bfloat162 b = __floats2bfloat162_rn(x.x * f, x.y * f);
    return *reinterpret_cast<const uint32_t*>(&b);
}
// where (token, head) is in the cache, in rows; pages are 16, 32, 64 or 128 tokens
__device__ __forceinline__ int64_t row_at(const GenCache& c, int slot, int h) {
    const int shift = 31 - __clz(c.page);
    return ((int64_t)(slot >> shift) * c.Hkv + h) * c.page + (slot & (c.page - 1));
}
// A CTA has 32 rows of k or of v in their own order, (token, head), so that what it reads (or writes) of them is in one piece; one row a
// thread.  A CTA for one head of 64 tokens, whose pages' rows follow each other instead: 16,385 tokens x 8 heads written in 24.8 us instead
// of 22.8, 24,000 x 4 read in 20.7 instead of 18.7.  Two rows a thread: 22.7 and 21.2.
constexpr int ROWS = NT / LANES;
struct Place {
    int64_t token;
    int h;
};
__device__ __forceinline__ Place place_of(const GenCache& c) {
    const int64_t id = (int64_t)blockIdx.x * ROWS + threadIdx.x / LANES;
    if (id <= UINT32_MAX) return {(uint32_t)id / (uint32_t)c.Hkv, (int)((uint32_t)id % (uint32_t)c.Hkv)};
    return {id / c.Hkv, (int)(id % c.Hkv)};
}
// The slot of a token, -1: none.  The first lane of the token's first head reports one beyond the cache.
__device__ __forceinline__ int slot_of(const GenCache& c, const GenRows& r, int64_t token, bool report) {
    if (token >= r.n) return -1;
    const int slot = r.slot[token];
    if (slot < 0) return -1;
    if (slot >> (31 - __clz(c.page)) < c.n_pages) return slot;
    if (report) gen_report(r.dev_status, (int)token);
    return -1;
}

template <bool F8>
__global__ void __launch_bounds__(NT) write_kernel(const GenCache c, const GenRows r) {
    const int lane = threadIdx.x % LANES;
    const bool is_v = blockIdx.y != 0;
    const Place at = place_of(c);
    const int slot = slot_of(c, r, at.token, lane == 0 && at.h == 0 && !is_v);
    uint4 x[2] = {};
    if (slot >= 0) {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_v ? r.v : r.k) + at.token * (is_v ? r.ld_v : r.ld_k) + (int64_t)at.h * D + lane * 16;
        x[0] = *reinterpret_cast<const uint4*>(src);
        x[1] = *reinterpret_cast<const uint4*>(src + 8);
    }
    const int64_t row = slot >= 0 ? row_at(c, slot, at.h) : 0;
    if constexpr (!F8) {
        if (slot < 0) return;
        uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(is_v ? c.v : c.k) + row * D + lane * 16);
        dst[0] = x[0];
        dst[1] = x[1];
    } else {
        uint32_t top = top_of(x);                          // bits of bf16 magnitudes are in the order of the magnitudes
#pragma unroll
        for (int m = 1; m < LANES; m <<= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
        if (slot < 0) return;
        // 448 = 1.75 2^8: the power goes one up where the significand is above 1.75
        const int exp = top >= 0x7f80u ? 255 : max((int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u), 1);
        uint4 y = make_uint4(0, 0, 0, 0);
        if (exp != 255) {
            uint32_t w[8] = {x[0].x, x[0].y, x[0].z, x[0].w, x[1].x, x[1].y, x[1].z, x[1].w};
            if (exp == 247) {                              // 256 2^120 would not be a number any more: the next one below it is taken
#pragma unroll
                for (int e = 0; e < 8; e++) w[e] = (w[e] & 0x80008000u) | __vminu2(w[e] & 0x7fff7fffu, 0x7f707f70u);
            }
            const float f = __uint_as_float((uint32_t)(254 - exp) << 23);
            y.x = two_e4m3(w[0], f) | two_e4m3(w[1], f) << 16;
            y.y = two_e4m3(w[2], f) | two_e4m3(w[3], f) << 16;
            y.z = two_e4m3(w[4], f) | two_e4m3(w[5], f) << 16;
            y.w = two_e4m3(w[6], f) | two_e4m3(w[7], f) << 16;
        }
        *reinterpret_cast<uint4*>(static_cast<uint8_t*>(is_v ? c.v : c.k) + row * D + lane * 16) = y;
        if (lane == 0) (is_v ? c.v_exp : c.k_exp)[row] = (uint8_t)exp;
    }
}

template <bool F8>
__global__ void __launch_bounds__(NT) read_kernel(const GenCache c, const GenRows r) {
    const int lane = threadIdx.x % LANES;
    const bool is_v = blockIdx.y != 0;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(is_v ? r.v : r.k);
    if (!out) return;
    const Place at = place_of(c);
    if (at.token >= r.n) return;
    const int slot = slot_of(c, r, at.token, lane == 0 && at.h == 0);
    uint4 x[2] = {};
    if (slot >= 0) {
        const int64_t row = row_at(c, slot, at.h);
        if constexpr (F8) {
            const uint4 y = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(is_v ? c.v : c.k) + row * D + lane * 16);
            const float f = gen_power((is_v ? c.v_exp : c.k_exp)[row]);
            x[0] = make_uint4(two_bf16(y.x, f), two_bf16(y.x >> 16, f), two_bf16(y.y, f), two_bf16(y.y >> 16, f));
            x[1] = make_uint4(two_bf16(y.z, f), two_bf16(y.z >> 16, f), two_bf16(y.w, f), two_bf16(y.w >> 16, f));
        } else {
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(is_v ? c.v : c.k) + row * D + lane * 16);
            x[0] = src[0];
            x[1] = src[1];
        }
    }
    uint4* dst = reinterpret_cast<uint4*>(out + (at.token * c.Hkv + at.h) * D + lane * 16);
    dst[0] = x[0];
    dst[1] = x[1];
}

int32_t grid_of(const GenCache& c, const GenRows& r, dim3& grid) {
    const int64_t blocks = (r.n * c.Hkv + ROWS - 1) / ROWS;
    grid = dim3((unsigned)blocks, 2);
    return blocks <= INT32_MAX ? HARTS_OK : HARTS_EINVAL;
}

}  // namespace

int32_t gen_cache_write(const GenCache& c, const GenRows& r) {
    dim3 grid;
    if (grid_of(c, r, grid) != HARTS_OK) return HARTS_EINVAL;
    if (c.type == HARTS_E4M3) write_kernel<true><<<grid, NT, 0, r.stream>>>(c, r);
    else write_kernel<false><<<grid, NT, 0, r.stream>>>(c, r);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}
int32_t gen_cache_read(const GenCache& c, const GenRows& r) {
    dim3 grid;
    if (grid_of(c, r, grid) != HARTS_OK) return HARTS_EINVAL;
    if (c.type == HARTS_E4M3) read_kernel<true><<<grid, NT, 0, r.stream>>>(c, r);
    else read_kernel<false><<<grid, NT, 0, r.stream>>>(c, r);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}

}  // namespace harts
