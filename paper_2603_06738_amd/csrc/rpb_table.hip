// The learned relative position bias itself: offsets from buckets, the sum of the attention backward's partial gradients, and
// the buckets' gradient.  Operators: include/rib_attn.h.
#include "rpb_common.h"

namespace rib {
namespace rpb {
namespace {

// bias[head][o] = table[head][index[o]].  Bound by memory, and by its launch at most sizes.
template <class T>
__global__ __launch_bounds__(256) void table_fwd_kernel(int L, int buckets, const T *__restrict__ table, const int32_t *__restrict__ index,
                                                        float *__restrict__ bias)
{
    const int o = blockIdx.x * 256 + threadIdx.x, hd = blockIdx.y;
    if (o >= L) return;
    const int i = index[o];
    float x = -INFINITY;
    if ((uint32_t)i < (uint32_t)buckets) {
        x = widen(table[(int64_t)hd * buckets + i]);
        if (x <= kExcluded) x = -INFINITY;
    }
    bias[(int64_t)hd * L + o] = x;
}

// dtable[head][b] = sum of dbias[head][o] over the offsets of bucket b.
//
// Many offsets share a bucket, so their values are added in LDS, as 64-bit whole numbers: such sums do not depend on the order of
// the additions.  A bucket's unit is the power of two above its largest value over 2^(62 - bits of the number of offsets): sums cannot overflow, and
// a term is off by 2^-44 of its bucket's largest at most (256 x 256 windows: 18 bits).  Values that are not finite are noted by kind beside the sums.
constexpr int kBuckets = 2048;          // buckets a workgroup at most
// Every workgroup of a head reads all offsets and adds those of its `chunk` buckets: the conversions, not the reads, are what costs
// (36481 offsets in 625 buckets, us: 36 in one workgroup a head, 15 in 16).
template <class T>
__global__ __launch_bounds__(1024) void table_bwd_kernel(int L, int buckets, int chunk, int bits, const float *__restrict__ dbias,
                                                         const int32_t *__restrict__ index, T *__restrict__ dtable)
{
    __shared__ unsigned long long sum[kBuckets];
    __shared__ uint32_t odd[kBuckets], top[kBuckets];
    const int hd = blockIdx.y, b0 = blockIdx.x * chunk, tid = threadIdx.x;
    const float *x = dbias + (int64_t)hd * L;
    for (int i = tid; i < chunk; i += 1024) sum[i] = 0ull, odd[i] = top[i] = 0u;
    __syncthreads();
    // f(bucket of this workgroup, value) for all offsets (eight loads in flight)
    auto each = [&](auto f) {
        for (int o0 = tid; o0 < L; o0 += 8 * 1024) {
            int at[8];
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int o = o0 + j * 1024 < L ? o0 + j * 1024 : L - 1;
                at[j] = o0 + j * 1024 < L ? index[o] : -1, v[j] = x[o];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = at[j] - b0;
                if ((uint32_t)at[j] < (uint32_t)buckets && (uint32_t)i < (uint32_t)chunk) f(i, v[j]);
            }
        }
    };
    each([&](int i, float v) {
        const uint32_t a = __float_as_uint(v) & 0x7fffffffu;
        if (a >= 0x7f800000u) atomicOr(&odd[i], v != v ? 4u : v > 0.f ? 1u : 2u);
        else atomicMax(&top[i], a);
    });
    __syncthreads();
    // 2^k of a bucket's unit: its largest is below 2^(k + 62 - bits)
    auto unit = [&](int i) { return (int)(top[i] >> 23 > 0u ? top[i] >> 23 : 1u) - 126 + bits - 62; };
    auto power = [](int k) { return __longlong_as_double((long long)(1023 + k) << 52); };
    each([&](int i, float v) {
        if ((__float_as_uint(v) & 0x7f800000u) != 0x7f800000u) atomicAdd(&sum[i], (unsigned long long)llrint((double)v * power(-unit(i))));
    });
    __syncthreads();
    for (int i = tid; i < chunk && b0 + i < buckets; i += 1024) {
        float v = (float)((double)(long long)sum[i] * power(unit(i)));
        if (odd[i] != 0u) v = odd[i] == 1u ? INFINITY : odd[i] == 2u ? -INFINITY : NAN;
        store_as(dtable + (int64_t)hd * buckets + b0 + i, v);
    }
}

// dbias[head][o] = sum over windows and their workgroups of the workgroups' sums.  64 offsets a workgroup, 16 threads an offset: up to 16 runs
// of windows, the rest of the 16 over a window's workgroups, then the 16 in a fixed order.  Bound by memory: every partial sum is read once.
__global__ __launch_bounds__(1024) void reduce_kernel(Geo g, Bias bi, int windows, int runs, int nblk, int group, const float *__restrict__ part,
                                                      float *__restrict__ dbias)
{
    __shared__ float run[16][64];
    const int L = bi.w2 * bi.w2, hd = blockIdx.y, strips = bi.sh < 0 ? 1 : g.M >> bi.sh, size = strips * bi.prows * bi.ws;
    const int lane = threadIdx.x & 63, r = threadIdx.x >> 6, o = blockIdx.x * 64 + lane, rw = r % runs;
    const int per = (windows + runs - 1) / runs, w0 = rw * per, w1 = w0 + per < windows ? w0 + per : windows;
    const int64_t step = (int64_t)g.heads * nblk * size;
    // from stationary to streamed, a query to a key, is minus the offset
    const int oy = o / bi.w2, dy = g.M - 1 - oy, dx = g.M - 1 - (o - oy * bi.w2);
    float sum = 0.f;
    if (o < L)
        for (int blk = r / runs; blk < nblk; blk += 16 / runs) {
            const int first = blk * group, last = first + group < g.N ? first + group - 1 : g.N - 1;
            const Span v = bi.sh >= 0 ? span_of<true>(g, bi, first, last) : span_of<false>(g, bi, first, last);
            const int row = dy + v.y1;
            if (row < 0 || row >= g.M + v.y1 - v.y0) continue;
            for (int s = 0; s < strips; ++s) {
                const int c = dx + v.x0 - s * bi.sw + bi.sw - 1;
                if (c < 0 || c >= bi.ws) continue;
                const float *p = part + sums_at(g, bi, (int64_t)w0 * g.heads + hd, nblk, blk, bi.prows, s * bi.sw) + row * bi.ws + c;
#pragma unroll 8
                for (int w = w0; w < w1; ++w, p += step) sum += *p;
            }
        }
    run[r][lane] = sum;
    __syncthreads();
    if (r == 0 && o < L) {
        for (int i = 1; i < 16; ++i) sum += run[i][lane];
        dbias[(int64_t)hd * L + o] = sum;
    }
}

}  // namespace

hipError_t launch_reduce(const Geo &g, int dtype, const Ws &w, const float *part, float *dbias, hipStream_t st)
{
    const int L = (2 * g.M - 1) * (2 * g.M - 1);
    Bias bi{};
    plan_order(g, dtype, &bi, w.strips);
    bi.prows = g.M - 1 + most_rows(w.group, g, bi);
    const int windows = w.shares;
    int runs = 16;
    while (runs > 1 && (runs > windows || (runs / 2 >= windows && w.nblk > 1))) runs /= 2;
    hipLaunchKernelGGL(reduce_kernel, dim3((L + 63) / 64, g.heads), dim3(1024), 0, st, g, bi, windows, runs, w.nblk,
                       w.group, part, dbias);
    return hipGetLastError();
}
hipError_t launch_table_fwd(int M, int heads, int buckets, int dtype, const void *table, const int32_t *index, float *bias, hipStream_t st)
{
    const int L = (2 * M - 1) * (2 * M - 1);
    const dim3 grid((L + 255) / 256, heads);
    if (dtype == RIB_BF16) hipLaunchKernelGGL(table_fwd_kernel<bf16_t>, grid, dim3(256), 0, st, L, buckets, (const bf16_t *)table, index, bias);
    else hipLaunchKernelGGL(table_fwd_kernel<float>, grid, dim3(256), 0, st, L, buckets, (const float *)table, index, bias);
    return hipGetLastError();
}
hipError_t launch_table_bwd(int M, int heads, int buckets, int dtype, const float *dbias, const int32_t *index, void *dtable, hipStream_t st)
{
    const int L = (2 * M - 1) * (2 * M - 1);
    int bits = 1;
    while ((1 << bits) < L) ++bits;
    int chunk = (buckets + 15) / 16;
    chunk = chunk < 32 ? 32 : chunk > kBuckets ? kBuckets : chunk;
    const dim3 grid((buckets + chunk - 1) / chunk, heads);
    if (dtype == RIB_BF16) hipLaunchKernelGGL(table_bwd_kernel<bf16_t>, grid, dim3(1024), 0, st, L, buckets, chunk, bits, dbias, index, (bf16_t *)dtable);
    else hipLaunchKernelGGL(table_bwd_kernel<float>, grid, dim3(1024), 0, st, L, buckets, chunk, bits, dbias, index, (float *)dtable);
    return hipGetLastError();
}

}  // namespace rpb
}  // namespace rib
