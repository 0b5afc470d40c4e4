// Linear attention from and into kept states, token by token: S_t = e^{g_t} S_{t-1} + k_t^T v_t, o_t = q_t S_t.
//
// One CTA holds NV columns of one (sequence, head)'s state in registers (columns do not interact) and walks the tokens: read the
// state once, write it once.  A thread has R rows x 4 columns, so that a warp's loads are whole rows of the slice; the sums over the
// rows of q_t S_t are finished over the warps in shared memory, TT tokens at a time.  All in fp32.
// Bound by the states' traffic (128 KB an item at d = 128 against 1 KB of rows): 201 sequences x 32 heads, one token, bf16: 138 us, 6.16 TB/s,
// 0.95 of a copy.
#include <cuda_bf16.h>

#include "gen.h"
#include "tc_common.cuh"

namespace harts {

int sm_count();

namespace {

using tc::F2;
using tc::f2;
using tc::f2_fma;
using tc::f2_mul;
using tc::f2_split;

constexpr int TT = 8;          // tokens staged at a time

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float& y, float x) { y = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

template <class T, int D, int NV, int NT>
__global__ void __launch_bounds__(NT)
walk_kernel(const GenLaArgs a) {
    constexpr int LANES = NV / 4, GROUPS = 32 / LANES, WARPS = NT / 32, STEP = WARPS * GROUPS, R = D / STEP, SLICES = D / NV;
    static_assert(R * STEP == D && LANES <= 32, "layout");
    __shared__ float sq[TT][D], sk[TT][D], sv[TT][NV], sg[TT];
    __shared__ float part[TT][WARPS][NV];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int slice = blockIdx.x % SLICES, h = blockIdx.x / SLICES % a.H, seq = blockIdx.x / SLICES / a.H;
    GenSeq s;
    if (!gen_seq(a, seq, s)) {
        if (tid == 0 && h == 0 && slice == 0) gen_report(a.dev_status, seq);
        return;
    }
    if (s.out < 0 && (!a.o || s.len == 0)) return;
    // row of element r: r * STEP + row0, so that a warp's GROUPS rows follow each other
    const int row0 = warp * GROUPS + lane / LANES, col = lane % LANES * 4;
    F2 x[R][2];
    if (s.in >= 0) {
        const float* src = a.states + ((size_t)s.in * a.H + h) * (D * D) + slice * NV + col;
#pragma unroll
        for (int r = 0; r < R; r++) {
            const float4 y = *reinterpret_cast<const float4*>(src + (size_t)(r * STEP + row0) * D);
            x[r][0] = f2(y.x, y.y);
            x[r][1] = f2(y.z, y.w);
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; r++) x[r][0] = x[r][1] = f2(0.f, 0.f);
    }
    const T *q = static_cast<const T*>(a.q), *k = static_cast<const T*>(a.k), *v = static_cast<const T*>(a.v);
    const bool outputs = a.o != nullptr;
    for (int t0 = 0; t0 < s.len; t0 += TT) {
        const int n = min(TT, s.len - t0);
        const int64_t first = (int64_t)s.begin + t0;
        for (int e = tid; e < n * D; e += NT) {
            const int t = e / D, i = e % D;
            sk[t][i] = to_float(k[(first + t) * a.ld_k + (size_t)h * D + i]);
            if (outputs) sq[t][i] = to_float(q[(first + t) * a.ld_q + (size_t)h * D + i]);
        }
        for (int e = tid; e < n * NV; e += NT) {
            const int t = e / NV, i = e % NV;
            sv[t][i] = to_float(v[(first + t) * a.ld_v + (size_t)h * D + slice * NV + i]);
        }
        if (tid < n) sg[tid] = expf(a.g[(first + tid) * a.H + h]);
        __syncthreads();
#pragma unroll 1
        for (int t = 0; t < n; t++) {
            const F2 gamma = f2(sg[t], sg[t]);
            const float4 vv = *reinterpret_cast<const float4*>(&sv[t][col]);
            const F2 v0 = f2(vv.x, vv.y), v1 = f2(vv.z, vv.w);
            F2 y0 = f2(0.f, 0.f), y1 = y0;
#pragma unroll
            for (int r = 0; r < R; r++) {
                const float kk = sk[t][r * STEP + row0];
                const F2 k2 = f2(kk, kk);
                x[r][0] = f2_fma(gamma, x[r][0], f2_mul(k2, v0));
                x[r][1] = f2_fma(gamma, x[r][1], f2_mul(k2, v1));
            }
            if (outputs) {
#pragma unroll
                for (int r = 0; r < R; r++) {
                    const float qq = sq[t][r * STEP + row0];
                    y0 = f2_fma(f2(qq, qq), x[r][0], y0);
                    y1 = f2_fma(f2(qq, qq), x[r][1], y1);
                }
                float4 y;
                f2_split(y0, y.x, y.y);
                f2_split(y1, y.z, y.w);
#pragma unroll
                for (int m = LANES; m < 32; m <<= 1) {
                    y.x += __shfl_xor_sync(~0u, y.x, m);
                    y.y += __shfl_xor_sync(~0u, y.y, m);
                    y.z += __shfl_xor_sync(~0u, y.z, m);
                    y.w += __shfl_xor_sync(~0u, y.w, m);
                }
                if (lane < LANES) *reinterpret_cast<float4*>(&part[t][warp][col]) = y;
            }
        }
        __syncthreads();
        if (outputs) {
            for (int e = tid; e < n * NV; e += NT) {
                const int t = e / NV, i = e % NV;
                float y = 0.f;
#pragma unroll
                for (int w = 0; w < WARPS; w++) y += part[t][w][i];
                from_float(static_cast<T*>(a.o)[((first + t) * a.H + h) * D + slice * NV + i], y);
            }
        }
    }
    if (s.out >= 0) {
        float* dst = a.states + ((size_t)s.out * a.H + h) * (D * D) + slice * NV + col;
#pragma unroll
        for (int r = 0; r < R; r++) {
            float4 y;
            f2_split(x[r][0], y.x, y.y);
            f2_split(x[r][1], y.z, y.w);
            *reinterpret_cast<float4*>(dst + (size_t)(r * STEP + row0) * D) = y;
        }
    }
}

template <class T, int D, int NV, int NT>
int32_t launch(const GenLaArgs& a) {
    const int64_t n = (int64_t)a.n_seq * a.H * (D / NV);
    if (n > INT32_MAX) return HARTS_EINVAL;
    walk_kernel<T, D, NV, NT><<<(int)n, NT, 0, a.stream>>>(a);
    return cudaGetLastError() == cudaSuccess ? HARTS_OK : HARTS_ECUDA;
}
template <class T>
int32_t by_size(const GenLaArgs& a) {
    // With few states narrow slices of their columns give every SM some of the work; else a thread's 64 values, whose loads are on their way
    // together, and small CTAs, whose loads and stores overlap with each other's (201 branches x 32 heads of 128: 256 threads and all columns
    // 149 us, 128 threads and half of them 138, 0.95 of the copy bandwidth)
    const bool few = (int64_t)a.n_seq * a.H <= sm_count();
    if (a.d == 128) return few ? launch<T, 128, 32, 256>(a) : launch<T, 128, 64, 128>(a);
    return few ? launch<T, 64, 16, 128>(a) : launch<T, 64, 64, 128>(a);
}

}  // namespace

int32_t gen_la_walk(const GenLaArgs& a) { return a.dtype == HARTS_FP32 ? by_size<float>(a) : by_size<__nv_bfloat16>(a); }

}  // namespace harts
