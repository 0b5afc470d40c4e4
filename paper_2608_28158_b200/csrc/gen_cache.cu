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
// where (token, head) is in the cache, in rows; pages are 16, 32, 64 or 128 tokens
__device__ __forceinline__ int64_t row_at(const GenCache& c, int slot, int h) {
    const int shift = 31 - __clz(c.page);
    return ((int64_t)(slot >> shift) * c.Hkv + h) * c.page + (slot & (c.page - 1));
}
// A CTA has PER * 32 tokens of one head (of k or of v), so that rows of a page that follow each other are written by one CTA; a thread has PER
// rows, whose loads are on their way together.
constexpr int PER = 2, TOKENS = PER * NT / LANES;
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
    const int lane = threadIdx.x % LANES, h = blockIdx.y;
    const bool is_v = blockIdx.z != 0;
    int slot[PER];
    uint4 x[PER][2];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int64_t token = (int64_t)blockIdx.x * TOKENS + i * (NT / LANES) + threadIdx.x / LANES;
        slot[i] = slot_of(c, r, token, lane == 0 && h == 0 && !is_v);
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        if (slot[i] >= 0) {
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(is_v ? r.v : r.k) + token * (is_v ? r.ld_v : r.ld_k) + h * D + lane * 16;
            x[i][0] = *reinterpret_cast<const uint4*>(src);
            x[i][1] = *reinterpret_cast<const uint4*>(src + 8);
        }
    }
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const int64_t row = slot[i] >= 0 ? row_at(c, slot[i], h) : 0;
        if constexpr (!F8) {
            if (slot[i] < 0) continue;
            uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(is_v ? c.v : c.k) + row * D + lane * 16);
            dst[0] = x[i][0];
            dst[1] = x[i][1];
        } else {
            uint32_t top = top_of(x[i]);                   // bits of bf16 magnitudes are in the order of the magnitudes
#pragma unroll
            for (int m = 1; m < LANES; m <<= 1) top = max(top, __shfl_xor_sync(~0u, top, m));
            if (slot[i] < 0) continue;
            // 448 = 1.75 2^8: the power goes one up where the significand is above 1.75
            const int exp = top >= 0x7f80u ? 255 : max((int)(top >> 7) - 8 + ((top & 0x7fu) > 0x60u), 1);
            uint4 y = make_uint4(0, 0, 0, 0);
            if (exp != 255) {
                uint32_t w[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
                if (exp == 247) {                          // 256 2^120 would not be a number any more: the next one below it is taken
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
}

template <bool F8>
__global__ void __launch_bounds__(NT) read_kernel(const GenCache c, const GenRows r) {
    const int lane = threadIdx.x % LANES, h = blockIdx.y;
    const bool is_v = blockIdx.z != 0;
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(is_v ? r.v : r.k);
    if (!out) return;
    int64_t token[PER];
    int exp[PER];
    uint4 x[PER][2];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        token[i] = (int64_t)blockIdx.x * TOKENS + i * (NT / LANES) + threadIdx.x / LANES;
        const int slot = slot_of(c, r, token[i], lane == 0 && h == 0);
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        exp[i] = 127;
        if (slot >= 0) {
            const int64_t row = row_at(c, slot, h);
            if constexpr (F8) {
                x[i][0] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(is_v ? c.v : c.k) + row * D + lane * 16);
                exp[i] = (is_v ? c.v_exp : c.k_exp)[row];
            } else {
                const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(is_v ? c.v : c.k) + row * D + lane * 16);
                x[i][0] = src[0];
                x[i][1] = src[1];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if (token[i] >= r.n) continue;
        if constexpr (F8) {
            const float f = gen_power(exp[i]);
            const uint32_t w[4] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w};
            uint32_t z[8];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                z[2 * e] = two_bf16(w[e], f);
                z[2 * e + 1] = two_bf16(w[e] >> 16, f);
            }
            x[i][0] = make_uint4(z[0], z[1], z[2], z[3]);
            x[i][1] = make_uint4(z[4], z[5], z[6], z[7]);
        }
        uint4* dst = reinterpret_cast<uint4*>(out + (token[i] * c.Hkv + h) * D + lane * 16);
        dst[0] = x[i][0];
        dst[1] = x[i][1];
    }
}

dim3 grid_of(const GenCache& c, const GenRows& r) { return dim3((unsigned)((r.n + TOKENS - 1) / TOKENS), (unsigned)c.Hkv, 2); }

}  // namespace

int32_t gen_cache_write(const GenCache& c, const GenRows& r) {
    if (c.type == HARTS_E4M3) write_kernel<true><<<grid_of(c, r), NT, 0, r.stream>>>(c, r);
    else write_kernel<false><<<grid_of(c, r), NT, 0, r.stream>>>(c, r);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}
int32_t gen_cache_read(const GenCache& c, const GenRows& r) {
    if (c.type == HARTS_E4M3) read_kernel<true><<<grid_of(c, r), NT, 0, r.stream>>>(c, r);
    else read_kernel<false><<<grid_of(c, r), NT, 0, r.stream>>>(c, r);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}

}  // namespace harts
