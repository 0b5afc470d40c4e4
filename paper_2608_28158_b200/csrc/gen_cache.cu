// Keys and values into the pages of a cache and back (harts_gen_cache_write / _read), bf16 or 8 bits with a power of two a row.
//
// Eight lanes a row of 128: each has 16 values, so that a row is read by eight 32-byte pieces and written as 8-bit values by eight
// 16-byte ones.  The scale being a power of two, x 2^-e is exact and rounding is that of the significand alone (values far below the
// row's largest lose bits as subnormals do).  Bound by the traffic: 512 + 258 bytes a (token, head) written, 258 + 512 read.
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
// where (token, head) is in the cache, in rows
__device__ __forceinline__ int64_t row_at(const GenCache& c, int slot, int h) {
    return ((int64_t)(slot / c.page) * c.Hkv + h) * c.page + slot % c.page;
}

template <bool F8>
__global__ void __launch_bounds__(NT) write_kernel(const GenCache c, const GenRows r) {
    const int64_t id = ((int64_t)blockIdx.x * NT + threadIdx.x) / LANES;          // (token, head)
    const int lane = threadIdx.x % LANES, h = (int)(id % c.Hkv);
    const int64_t token = id / c.Hkv;
    int slot = -1;
    if (token < r.n) {
        slot = r.slot[token];
        if (slot >= 0 && slot / c.page >= c.n_pages) {
            if (lane == 0 && h == 0 && blockIdx.y == 0) gen_report(r.dev_status, (int)token);
            slot = -1;
        }
    }
    const bool is_v = blockIdx.y != 0;
    uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (slot >= 0) {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_v ? r.v : r.k) + token * (is_v ? r.ld_v : r.ld_k) + h * D + lane * 16;
        x[0] = *reinterpret_cast<const uint4*>(src);
        x[1] = *reinterpret_cast<const uint4*>(src + 8);
    }
    const int64_t row = slot >= 0 ? row_at(c, slot, h) : 0;
    if constexpr (!F8) {
        if (slot < 0) return;
        uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(is_v ? c.v : c.k) + row * D + lane * 16);
        dst[0] = x[0];
        dst[1] = x[1];
        return;
    }
    uint32_t top = top_of(x);                      // bits of bf16 magnitudes are in the order of the magnitudes
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
    if (slot < 0) return;
    // 448 = 1.75 2^8: the power goes one up where the significand is above 1.75
    const int exp = top >= 0x7f80u ? 255 : max((int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u), 1);
    uint4 y = make_uint4(0, 0, 0, 0);
    if (exp != 255) {
        if (exp == 247) {                          // 256 2^120 would not be a number any more: the next one below it is taken
            uint32_t* w = reinterpret_cast<uint32_t*>(x);
#pragma unroll
            for (int i = 0; i < 8; i++) w[i] = (w[i] & 0x80008000u) | __vminu2(w[i] & 0x7fff7fffu, 0x7f707f70u);
        }
        const float f = __uint_as_float((uint32_t)(254 - exp) << 23);
        y.x = two_e4m3(x[0].x, f) | two_e4m3(x[0].y, f) << 16;
        y.y = two_e4m3(x[0].z, f) | two_e4m3(x[0].w, f) << 16;
        y.z = two_e4m3(x[1].x, f) | two_e4m3(x[1].y, f) << 16;
        y.w = two_e4m3(x[1].z, f) | two_e4m3(x[1].w, f) << 16;
    }
    *reinterpret_cast<uint4*>(static_cast<uint8_t*>(is_v ? c.v : c.k) + row * D + lane * 16) = y;
    if (lane == 0) (is_v ? c.v_exp : c.k_exp)[row] = (uint8_t)exp;
}

template <bool F8>
__global__ void __launch_bounds__(NT) read_kernel(const GenCache c, const GenRows r) {
    const int64_t id = ((int64_t)blockIdx.x * NT + threadIdx.x) / LANES;
    const int lane = threadIdx.x % LANES, h = (int)(id % c.Hkv);
    const int64_t token = id / c.Hkv;
    const bool is_v = blockIdx.y != 0;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(is_v ? r.v : r.k);
    if (token >= r.n || !out) return;
    int slot = r.slot[token];
    if (slot >= 0 && slot / c.page >= c.n_pages) {
        if (lane == 0 && h == 0) gen_report(r.dev_status, (int)token);
        slot = -1;
    }
    uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (slot >= 0) {
        const int64_t row = row_at(c, slot, h);
        if constexpr (F8) {
            const uint4 y = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(is_v ? c.v : c.k) + row * D + lane * 16);
            const int exp = (is_v ? c.v_exp : c.k_exp)[row];
            const float f = gen_power(exp);
            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
            uint32_t z[8];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                z[2 * i] = two_bf16(w[i], f);
                z[2 * i + 1] = two_bf16(w[i] >> 16, f);
            }
            x[0] = make_uint4(z[0], z[1], z[2], z[3]);
            x[1] = make_uint4(z[4], z[5], z[6], z[7]);
        } else {
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(is_v ? c.v : c.k) + row * D + lane * 16);
            x[0] = src[0];
            x[1] = src[1];
        }
    }
    uint4* dst = reinterpret_cast<uint4*>(out + (token * c.Hkv + h) * D + lane * 16);
    dst[0] = x[0];
    dst[1] = x[1];
}

int32_t grid_of(const GenCache& c, const GenRows& r, dim3& grid) {
    const int64_t blocks = (r.n * c.Hkv * LANES + NT - 1) / NT;
    if (blocks > INT32_MAX) return HARTS_EINVAL;
    grid = dim3((unsigned)blocks, 2);
    return HARTS_OK;
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
