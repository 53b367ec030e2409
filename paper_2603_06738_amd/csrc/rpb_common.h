// Window attention with a learned relative position bias: what its kernels share.  Operators and layouts:
// include/rib_attn.h.
//
// The pairs of a unit are walked as 32x32 blocks of STATIONARY tokens (a workgroup's own, in registers) against
// STREAMED ones (in LDS, tiles of 64).  The bias of a pair depends on its relative offset alone, and with
//     lin(n) = (2M-1) * (n / M) + n % M
// the offset is linear in lin(streamed) - lin(stationary).  So a workgroup keeps the offsets' rows it needs in LDS
// such that a lane's 16 values of a block lie at   lin(streamed) - lin(stationary) + c0,   four neighbours at a time.
// Where all rows would not fit, the walk is cut into chunks of tiles, each with its own rows.
#pragma once

#include "rib_rows.h"

namespace rib {
namespace rpb {

constexpr int kTile = 64;               // streamed tokens a tile
constexpr float kExcluded = -1e30f;     // a bias at or below this excludes the pair

// Problem of one attention call beside Geo.
struct Bias {
    const float *bias;      // [heads][(2M-1)^2]
    int w2;                 // 2M - 1
    int chunk;              // tiles a chunk
    int rows;               // bias rows in LDS at most
    int hrows;              // rows of a wave's histogram at most
    // Logits in the products' own unit, q.k + bias / scale: `qs` is what q is multiplied by first (1: as it is), `bs` the
    // bias, and `c` brings a sum to base 2.  `ks`: what dS q is multiplied by.
    float qs, bs, c, ks;
};
// Scales that are no ordinary positive number go into q (rounded to its type), so that neither bias / scale nor
// an excluded pair's minus infinity comes out wrong.
inline void plan_scale(const Geo &g, Bias *b)
{
    const bool plain = g.scale_c >= 0x1p-40f && g.scale_c <= 0x1p40f;
    b->qs = plain ? 1.f : g.scale_c;
    b->bs = plain ? 1.f / g.scale_c : 1.f;
    b->c = plain ? g.scale_c * rows::kLog2e : rows::kLog2e;
    b->ks = plain ? g.scale_c : 1.f;
}

// The most window rows that `len` tokens from a multiple of `len` on touch.
inline int most_rows(int len, int N, int M)
{
    if (len >= N) return M;
    const int rows = len % M == 0 ? len / M : M % len == 0 ? 1 : (len + M - 2) / M + 1;
    return rows < M ? rows : M;
}

// The bias rows of one chunk: window rows [sy0, sy1] stationary, [ty0, ty1] streamed.
struct Chunk {
    int ty0, ty1, c0, count;            // `count`: offsets
};
__device__ __forceinline__ int row_of(int n, uint32_t inv_m) { return (int)__umulhi((uint32_t)n, inv_m); }
__device__ __forceinline__ Chunk chunk_of(const Geo &g, const Bias &b, int t0, int t1, int sy0, int sy1)
{
    Chunk c;
    const int e = t1 * kTile < g.N ? t1 * kTile : g.N;
    c.ty0 = row_of(t0 * kTile, g.inv_m);
    c.ty1 = row_of(e - 1, g.inv_m);
    c.c0 = (sy1 - c.ty0) * b.w2 + g.M - 1;
    c.count = (c.ty1 - c.ty0 + sy1 - sy0 + 1) * b.w2;
    return c;
}
__device__ __forceinline__ int lin(const Geo &g, int n) { return n + row_of(n, g.inv_m) * (g.M - 1); }

// Whether some key is not excluded for query n; asked by whole waves.
__device__ __forceinline__ bool has_key(const Geo &g, const Bias &b, int hd, int n)
{
    const float *row = b.bias + (int64_t)hd * b.w2 * b.w2 + 2 * g.M * (g.M - 1) + lin(g, n);
    for (int j0 = 0; j0 < g.N; j0 += 64) {
        const int j = j0 + (threadIdx.x & 63);
        if (__any(j < g.N && !(row[-lin(g, j < g.N ? j : 0)] <= kExcluded))) return true;
    }
    return false;
}
// Whether a wave's walk without a running maximum has to be done again: a denominator that left [2^-60, 2^60], other than
// zeros of rows without a key.  `n`: the lane's row, the same in both halves.
__device__ __forceinline__ bool bad_rows(const Geo &g, const Bias &b, int hd, int n, float sum)
{
    if (__any(!(sum >= 0x1p-60f && sum <= 0x1p60f) && sum != 0.f)) return true;
    for (uint32_t zeros = (uint32_t)__ballot(sum == 0.f && n < g.N); zeros != 0u; zeros &= zeros - 1u)
        if (has_key(g, b, hd, __shfl(n, __ffs((int)zeros) - 1))) return true;
    return false;
}

// Copies a chunk's bias rows to LDS, times `scale`; excluded pairs as minus infinity.  SGN = -1: the streamed tokens are the keys
// (offset = query - key falls as the key rises), +1: the queries.
template <int SGN>
__device__ __forceinline__ void stage_bias(const Geo &g, const Bias &b, const Chunk &c, int hd, float scale, float *lds, int nt)
{
    const float *src = b.bias + (int64_t)hd * b.w2 * b.w2;
    const int at = 2 * g.M * (g.M - 1) - SGN * c.c0;
    for (int l = threadIdx.x; l < c.count; l += nt) {
        const float x = src[at + SGN * l];
        lds[l] = x <= kExcluded ? -INFINITY : x * scale;
    }
}

// Adds the waves' histograms of a chunk (dS summed by offset, `hsize` values a wave, WT stationary tokens each) in their order, writes
// them to the workgroup's sums `dst` (from the chunk's first row on) and clears them.  `before`: the last streamed row of the chunk
// before (-1: none); rows which that one touched are added to.
template <int W, int WT>
__device__ __forceinline__ void flush(const Geo &g, const Bias &b, const Chunk &ch, double *H, int hsize, int first, int sy0, int sy1, int before, float *dst)
{
    const int old = before < 0 ? 0 : (before - ch.ty0 + sy1 - sy0 + 1) * b.w2;
    for (int e = threadIdx.x; e < ch.count; e += 64 * W) {
        double sum = 0.;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int f = first + w * WT, l = f + WT < g.N ? f + WT - 1 : g.N - 1;
            if (f >= g.N) break;
            const int y0 = row_of(f, g.inv_m), y1 = row_of(l, g.inv_m), at = e - (sy1 - y1) * b.w2;
            if (at >= 0 && at < (ch.ty1 - ch.ty0 + y1 - y0 + 1) * b.w2) {
                sum += H[w * hsize + at];
                H[w * hsize + at] = 0.;
            }
        }
        dst[e] = (float)(e < old ? sum + dst[e] : sum);
    }
}

// ---- sources of rows ---------------------------------------------------------------------------------------------

// kFast: grid tensors, rows of 8 or more values, everything on 4-byte boundaries.  kAny: grid tensors, value by value.
// kCkpt: rows of an 8-bit checkpoint.
enum Source { kFast = 0, kAny = 1, kCkpt = 2 };

// Checkpoint (include/rib_attn.h): for q, k and v in turn [units][N][dp] codes; then for each [units][N] exponent bytes.
__host__ __device__ inline int ckpt_row(int d) { return (d + 15) & ~15; }
__host__ __device__ inline int64_t ckpt_rows(const Geo &g) { return g.units * g.N; }

// Launchers.
struct FwdArgs {
    const void *q, *k, *v;
    const float *bias;
    void *out;
    float *lse;
    int force_max;
    hipStream_t st;
};
struct BwdArgs {
    const void *q, *k, *v;          // null with a checkpoint
    const uint8_t *ckpt;            // null with grid tensors
    const float *bias;
    const void *out, *dout;
    const float *lse;
    void *dq, *dk, *dv;
    float *dbias;                   // may be null
    void *ws;
    hipStream_t st;
};
hipError_t launch_fwd_bf16(const Geo &g, const FwdArgs &a);
hipError_t launch_bwd_bf16(const Geo &g, const BwdArgs &a);
hipError_t launch_fwd_f32(const Geo &g, const FwdArgs &a);
hipError_t launch_bwd_f32(const Geo &g, const BwdArgs &a);

hipError_t launch_table_fwd(int M, int heads, int buckets, int dtype, const void *table, const int32_t *index, float *bias, hipStream_t st);
hipError_t launch_table_bwd(int M, int heads, int buckets, int dtype, const float *dbias, const int32_t *index, void *dtable, hipStream_t st);
hipError_t launch_pack(const Geo &g, int dtype, const void *q, const void *k, const void *v, uint8_t *ckpt, hipStream_t st);
hipError_t launch_unpack(const Geo &g, int dtype, const uint8_t *ckpt, void *q, void *k, void *v, hipStream_t st);

// Backward scratch: per token and head the two values that the second kernel streams beside Q and dO; then, per workgroup of
// the first kernel, sums of dS by offset.
struct Ws {
    size_t ext, part, total;
    int nblk;                           // workgroups a unit
    int prows;                          // rows of a workgroup's sums
    int shares;                         // sums a head: of windows, or of the runs of windows a wave takes
};
// Stationary tokens of a wave, and of a workgroup.
constexpr int wave_tokens(int dtype) { return dtype == RIB_BF16 ? 64 : 32; }
constexpr int group_tokens(int dtype, int N) { return N <= wave_tokens(dtype) ? wave_tokens(dtype) : 4 * wave_tokens(dtype); }
inline Ws ws_layout(const Geo &g, int dtype)
{
    Ws w;
    const int sb = group_tokens(dtype, g.N);
    w.nblk = (g.N + sb - 1) / sb;
    w.prows = g.M - 1 + most_rows(sb, g.N, g.M);
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    w.shares = (int)(g.units / g.heads);
    w.ext = 0;
    w.part = up((size_t)g.units * g.N * 8);
    w.total = w.part + up((size_t)g.units * w.nblk * w.prows * (2 * g.M - 1) * sizeof(float));
    return w;
}
// dbias[head][offset] from the workgroups' sums: windows and workgroups in a fixed order.
hipError_t launch_reduce(const Geo &g, int dtype, const Ws &w, const float *part, float *dbias, hipStream_t st);

// Tiles a chunk and the rows that go with it: as many tiles as fit `bias_bytes` of bias and (hist) `hist_bytes` a wave.
inline void plan_chunks(const Geo &g, int dtype, Bias *b, bool hist, size_t bias_bytes, size_t hist_bytes)
{
    const int sb = group_tokens(dtype, g.N), ntiles = (g.N + kTile - 1) / kTile;
    const int srows = most_rows(sb, g.N, g.M), wrows = most_rows(wave_tokens(dtype), g.N, g.M);
    b->w2 = 2 * g.M - 1;
    int tiles = ntiles;
    for (;; tiles = tiles > 8 ? tiles - tiles / 8 : tiles - 1) {
        const int trows = most_rows(tiles * kTile, g.N, g.M);
        b->chunk = tiles;
        b->rows = trows + srows - 1;
        b->hrows = hist ? trows + wrows - 1 : 0;
        const bool fits = (size_t)b->rows * b->w2 * 4 <= bias_bytes && (size_t)b->hrows * b->w2 * 8 <= hist_bytes;
        if (fits || tiles == 1) return;
    }
}

}  // namespace rpb
}  // namespace rib
