// 8-bit checkpoints of q, k and v: packed for the backward, and unpacked.  Format: include/rib_attn.h.
//
// A (tensor, unit, token) row of d values becomes dp = 16 ceil(d / 16) codes and an exponent byte e: value = (code - 128) 2^(e - 127), e
// the smallest for which the row's largest fits 127 steps (248 at most: above 127 * 2^121 codes stay at 127).  Codes lie in the units' own token order, so what the backward
// reads of a unit is contiguous.  Codes under a power of two are exact in either storage type.
// Bound by memory: q, k, v read once and a little over half of that (bf16; a quarter, fp32) written.  16 images of 96 x 96, 6 heads of 30, bf16:
// pack 78 us, 247 MB, 3.2 TB/s of the 5.1 a copy reaches (a head at a time, rows in 16 lanes 256 us, in 4 lanes 90); unpack 100 us: it stores value by value,
// and is for users of other backward passes, since the one here reads codes.
#include "rpb_common.h"

namespace rib {
namespace rpb {
namespace {

// A workgroup takes 32 tokens of a window, all heads of one after the other, LP lanes a row and 8 values a lane: a wave reads whole pixels.
constexpr int kTokens = 32;
struct __attribute__((packed, aligned(4))) words4 {
    uint32_t w[4];
};
struct Slot {
    int hd, n, c;           // head, token of the window (-1: none), first value
    int64_t row, at;        // row of the checkpoint within a tensor; element of the grid
};
// The workgroup's window and first token (all of it uniform).
struct Corner {
    int w, n0, y0, x0;
    int64_t img;
};
__device__ __forceinline__ Corner corner_of(const Geo &g)
{
    Corner c;
    const int chunks = (g.N + kTokens - 1) / kTokens;
    c.w = blockIdx.x / chunks, c.n0 = (blockIdx.x - c.w * chunks) * kTokens;
    const int wx = c.w % g.nwx, t = c.w / g.nwx, wy = t % g.nwy;
    c.y0 = wy * g.M + g.s, c.x0 = wx * g.M + g.s, c.img = (int64_t)(t / g.nwy) * g.H * g.W;
    return c;
}
template <int LP>
__device__ __forceinline__ Slot slot_of(const Geo &g, const Corner &k, int slot)
{
    Slot s;
    const int r = slot / LP, tk = r / g.heads, n = k.n0 + tk, iy = row_of(n, g.inv_m);
    s.hd = r - tk * g.heads, s.n = n < g.N ? n : -1, s.c = 8 * (slot % LP);
    s.row = ((int64_t)k.w * g.heads + s.hd) * g.N + n;
    int y = k.y0 + iy, x = k.x0 + n - iy * g.M;
    if (y >= g.H) y -= g.H;
    if (x >= g.W) x -= g.W;
    s.at = s.n < 0 ? 0 : (k.img + (int64_t)y * g.W + x) * g.tstride + s.hd * g.d;
    return s;
}
// Values c .. c+7 of a row, zeros past its end.
template <bool PAIRS>
__device__ __forceinline__ void load8(const bf16_t *p, int c, int d, float (&x)[8])
{
    if (PAIRS && c + 8 <= d) {
        const words4 v = *(const words4 *)(p + c);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(i & 1 ? v.w[i >> 1] & 0xffff0000u : v.w[i >> 1] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < d ? widen(p[c + i]) : 0.f;
    }
}
template <bool PAIRS>
__device__ __forceinline__ void load8(const float *p, int c, int d, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c + i < d ? p[c + i] : 0.f;
}

template <class T, int LP, bool PAIRS>
__global__ __launch_bounds__(256) void pack_kernel(Geo g, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                                                   uint8_t *__restrict__ ckpt)
{
    const int dp = ckpt_row(g.d), which = blockIdx.y;
    const int64_t rows = ckpt_rows(g);
    const T *src = which == 0 ? q : which == 1 ? k : v;
    const Corner corner = corner_of(g);
    for (int slot = threadIdx.x; slot < kTokens * LP * g.heads; slot += 256) {      // (the lanes of a row stay together)
        const Slot s = slot_of<LP>(g, corner, slot);
        float x[8];
        uint32_t big = 0u;
        if (s.n >= 0) load8<PAIRS>(src + s.at, s.c, g.d, x);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
            big = a > big ? a : big;
        }
#pragma unroll
        for (int m = 1; m < LP; m <<= 1) {
            const uint32_t o = (uint32_t)__shfl_xor((int)big, m);
            big = o > big ? o : big;
        }
        // big = 1.f 2^(E - 127): 127 steps of 2^(E - 127 - 6) hold it unless its fraction is above 127/64 - 1
        int e = 0;
        if (big >= 0x7f800000u) e = 255;                        // not finite: the row stands for NaN
        else if (big != 0u) {
            e = (int)(big >> 23) - 6 + ((big & 0x7fffffu) > 0x7e0000u ? 1 : 0);
            e = e < 1 ? 1 : e > 248 ? 248 : e;                  // (64 steps of 2^122 would be beyond either type)
        }
        const float per = e == 0 || e == 255 ? 0.f : __uint_as_float((uint32_t)(254 - e) << 23);
        uint32_t codes[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < 8; ++i) codes[i >> 2] |= (uint32_t)((e == 255 ? 0 : (int)fminf(fmaxf(rintf(x[i] * per), -127.f), 127.f)) + 128) << (8 * (i & 3));
        if (s.n < 0) continue;
        const int64_t to = s.row + which * rows;
        if (s.c < dp) *(uint2 *)(ckpt + to * dp + s.c) = uint2{codes[0], codes[1]};
        if (s.c == 0) (ckpt + 3 * rows * dp)[to] = (uint8_t)e;
    }
}

template <class T, int LP>
__global__ __launch_bounds__(256) void unpack_kernel(Geo g, const uint8_t *__restrict__ ckpt, T *__restrict__ q, T *__restrict__ k, T *__restrict__ v)
{
    const int dp = ckpt_row(g.d), which = blockIdx.y;
    const int64_t rows = ckpt_rows(g);
    T *dst = which == 0 ? q : which == 1 ? k : v;
    const Corner corner = corner_of(g);
    for (int slot = threadIdx.x; slot < kTokens * LP * g.heads; slot += 256) {
        const Slot s = slot_of<LP>(g, corner, slot);
        if (s.n < 0 || s.c >= g.d) continue;
        const int64_t from = s.row + which * rows;
        const float sc = code_step((ckpt + 3 * rows * dp)[from]);
        const uint2 codes = *(const uint2 *)(ckpt + from * dp + s.c);
        T *p = dst + s.at + s.c;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (s.c + i < g.d) store_as(p + i, code_value(((i < 4 ? codes.x : codes.y) >> (8 * (i & 3))) & 255u, sc));
    }
}

}  // namespace

template <class T, int LP>
hipError_t pack_width(const Geo &g, bool pairs, const void *q, const void *k, const void *v, uint8_t *ckpt, hipStream_t st)
{
    const dim3 grid((unsigned)(g.units / g.heads * ((g.N + kTokens - 1) / kTokens)), 3);
    if (pairs) hipLaunchKernelGGL((pack_kernel<T, LP, true>), grid, dim3(256), 0, st, g, (const T *)q, (const T *)k, (const T *)v, ckpt);
    else hipLaunchKernelGGL((pack_kernel<T, LP, false>), grid, dim3(256), 0, st, g, (const T *)q, (const T *)k, (const T *)v, ckpt);
    return hipGetLastError();
}
template <class T>
hipError_t unpack_type(const Geo &g, const uint8_t *ckpt, void *q, void *k, void *v, hipStream_t st)
{
    const dim3 grid((unsigned)(g.units / g.heads * ((g.N + kTokens - 1) / kTokens)), 3);
    if (g.d <= 32) hipLaunchKernelGGL((unpack_kernel<T, 4>), grid, dim3(256), 0, st, g, ckpt, (T *)q, (T *)k, (T *)v);
    else hipLaunchKernelGGL((unpack_kernel<T, 8>), grid, dim3(256), 0, st, g, ckpt, (T *)q, (T *)k, (T *)v);
    return hipGetLastError();
}

hipError_t launch_pack(const Geo &g, int dtype, const void *q, const void *k, const void *v, uint8_t *ckpt, hipStream_t st)
{
    if (dtype != RIB_BF16)
        return g.d <= 32 ? pack_width<float, 4>(g, false, q, k, v, ckpt, st) : pack_width<float, 8>(g, false, q, k, v, ckpt, st);
    const bool pairs = !(g.d & 1) && !(g.tstride & 1) && (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v) & 3) == 0;
    return g.d <= 32 ? pack_width<bf16_t, 4>(g, pairs, q, k, v, ckpt, st) : pack_width<bf16_t, 8>(g, pairs, q, k, v, ckpt, st);
}
hipError_t launch_unpack(const Geo &g, int dtype, const uint8_t *ckpt, void *q, void *k, void *v, hipStream_t st)
{
    return dtype == RIB_BF16 ? unpack_type<bf16_t>(g, ckpt, q, k, v, st) : unpack_type<float>(g, ckpt, q, k, v, st);
}

}  // namespace rpb
}  // namespace rib
