// 8-bit checkpoints of q, k and v: packed for the backward, and unpacked.  Format: include/rib_attn.h.
//
// A (tensor, unit, token) row of d values becomes dp = 16 ceil(d / 16) codes and an exponent byte e: value = (code - 128) 2^(e - 127), e
// the smallest for which the row's largest fits 127 steps.  Codes lie in the units' own token order, so what the backward
// reads of a unit is contiguous.  Codes under a power of two are exact in either storage type.
// Bound by memory: q, k, v read once and a little over half of that (bf16; a quarter, fp32) written.
#include "rpb_common.h"

namespace rib {
namespace rpb {
namespace {

__device__ __forceinline__ float load(const float *p) { return *p; }
__device__ __forceinline__ float load(const bf16_t *p) { return widen(*p); }

// 16 lanes a row, 4 values each.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(Geo g, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                                                   uint8_t *__restrict__ ckpt)
{
    const int64_t rows = g.units * g.N, row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    if (row >= rows) return;
    const int dp = ckpt_row(g.d), c = 4 * (threadIdx.x & 15), which = blockIdx.y;
    // rows in the order token, head: neighbours share a pixel
    const int64_t wt = row / g.heads;
    const int hd = (int)(row - wt * g.heads), w = (int)(wt / g.N), n = (int)(wt - (int64_t)w * g.N);
    const T *src = (which == 0 ? q : which == 1 ? k : v) + grid_token(g, w, n) * g.tstride + (int64_t)hd * g.d;
    const int64_t to = ((int64_t)w * g.heads + hd) * g.N + n + which * rows;
    float x[4];
    uint32_t big = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = c + i < g.d ? load(src + c + i) : 0.f;
        const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
        big = a > big ? a : big;
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)big, m);
        big = o > big ? o : big;
    }
    // big = 1.f 2^(E - 127): 127 steps of 2^(E - 127 - 6) hold it unless its fraction is above 127/64 - 1
    int e = 0;
    if (big >= 0x7f800000u) e = 255;                        // not finite: the row stands for NaN
    else if (big != 0u) {
        e = (int)(big >> 23) - 6 + ((big & 0x7fffffu) > 0x7e0000u ? 1 : 0);
        if (e < 1) e = 1;
    }
    uint32_t codes = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int s = e == 0 || e == 255 ? 0 : (int)rintf(ldexpf(x[i], 127 - e));
        codes |= (uint32_t)(s + 128) << (8 * i);
    }
    if (c < dp) *(uint32_t *)(ckpt + to * dp + c) = codes;
    if (c == 0) (ckpt + 3 * rows * dp)[to] = (uint8_t)e;
}

template <class T>
__global__ __launch_bounds__(256) void unpack_kernel(Geo g, const uint8_t *__restrict__ ckpt, T *__restrict__ q, T *__restrict__ k, T *__restrict__ v)
{
    const int64_t rows = g.units * g.N, row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    if (row >= rows) return;
    const int dp = ckpt_row(g.d), c = 4 * (threadIdx.x & 15), which = blockIdx.y;
    const int64_t wt = row / g.heads;
    const int hd = (int)(row - wt * g.heads), w = (int)(wt / g.N), n = (int)(wt - (int64_t)w * g.N);
    T *dst = (which == 0 ? q : which == 1 ? k : v) + grid_token(g, w, n) * g.tstride + (int64_t)hd * g.d;
    const int64_t from = ((int64_t)w * g.heads + hd) * g.N + n + which * rows;
    const float s = __uint_as_float((uint32_t)(ckpt + 3 * rows * dp)[from] << 23), z = -128.f * s;
    if (c >= g.d) return;
    const uint32_t codes = *(const uint32_t *)(ckpt + from * dp + c);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < g.d) store_as(dst + c + i, fmaf((float)((codes >> (8 * i)) & 255u), s, z));
}

}  // namespace

hipError_t launch_pack(const Geo &g, int dtype, const void *q, const void *k, const void *v, uint8_t *ckpt, hipStream_t st)
{
    const dim3 grid((unsigned)((g.units * g.N + 15) / 16), 3);
    if (dtype == RIB_BF16)
        hipLaunchKernelGGL(pack_kernel<bf16_t>, grid, dim3(256), 0, st, g, (const bf16_t *)q, (const bf16_t *)k, (const bf16_t *)v, ckpt);
    else hipLaunchKernelGGL(pack_kernel<float>, grid, dim3(256), 0, st, g, (const float *)q, (const float *)k, (const float *)v, ckpt);
    return hipGetLastError();
}
hipError_t launch_unpack(const Geo &g, int dtype, const uint8_t *ckpt, void *q, void *k, void *v, hipStream_t st)
{
    const dim3 grid((unsigned)((g.units * g.N + 15) / 16), 3);
    if (dtype == RIB_BF16) hipLaunchKernelGGL(unpack_kernel<bf16_t>, grid, dim3(256), 0, st, g, ckpt, (bf16_t *)q, (bf16_t *)k, (bf16_t *)v);
    else hipLaunchKernelGGL(unpack_kernel<float>, grid, dim3(256), 0, st, g, ckpt, (float *)q, (float *)k, (float *)v);
    return hipGetLastError();
}

}  // namespace rpb
}  // namespace rib
