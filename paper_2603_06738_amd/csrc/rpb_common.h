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

#include <cmath>

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
    int prows;              // rows of a workgroup's sums at most
    // Logits in the products' own unit, q.k + bias / scale: `qs` is what q is multiplied by first (1: as it is; -1, 0 or a power of two else), `bs` the
    // bias, and `c` brings a sum to base 2.  `ks`: what dS q is multiplied by.
    float qs, bs, c, ks;
    // Strips: 2^sh columns, `strip` tokens each (a multiple of 64); sh < 0: rows of the whole window.
    int sh, strip;
    int sw, ws;             // columns of a strip, offsets of a row in LDS: 2 sw - 1
    uint32_t inv_strip, inv_ws;     // n / strip == mulhi(n, inv_strip)
};
// Waves a workgroup: 4, or 3 or 2 where that leaves fewer of them idle at a window's end; 1 where one holds the window.
constexpr int kSplitGroups = 160;
constexpr int wave_tokens(int dtype) { return dtype == RIB_BF16 ? 64 : 32; }
constexpr int group_waves(int dtype, int N)
{
    const int nb = (N + wave_tokens(dtype) - 1) / wave_tokens(dtype);
    if (nb == 1) return 1;
    if (dtype != RIB_BF16) return 4;
    return nb == 2 ? 2 : (nb + 2) / 3 * 3 < (nb + 3) / 4 * 4 ? 3 : 4;
}
// Whether four waves share 64 stationary tokens (bf16): four times as many workgroups, for grids that would leave most of the chip's 256 compute
// units without one.  By sizes alone (workgroups of 4 x 64 tokens: us of a forward, forward + backward with its bias gradient, unsplit /
// split): 32 x 32 windows, 4: 23 / 14, 105 / 67; 96: 24 / 20, 110 / 90; 120: 24 / 19, 111 / 91; 240: 26 / 27, 117 / 139; 64 x 64 windows, 32: 75 /
// 41, 338 / 192; 192: 80 / 71, 360 / 361; one 96 x 96 window of 6 heads, 216: 176 / 214, 773 / 974.
inline bool splits(const Geo &g, int dtype)
{
    const int sb = group_waves(dtype, g.N) * wave_tokens(dtype);
    return dtype == RIB_BF16 && g.N > 64 && g.units * ((g.N + sb - 1) / sb) <= kSplitGroups;
}
// Stationary tokens a workgroup.
inline int group_tokens(const Geo &g, int dtype) { return splits(g, dtype) ? 64 : group_waves(dtype, g.N) * wave_tokens(dtype); }
// Whether windows of this side are walked in strips, and of how many columns (a power of two): where workgroups do not cross them.
inline int strip_shift(int dtype, int M)
{
    const int sh = M % 32 == 0 ? 5 : M % 16 == 0 ? 4 : M % 8 == 0 ? 3 : -1;
    return sh >= 0 && (M << sh == M * M || (M << sh) % (group_waves(dtype, M * M) * wave_tokens(dtype)) == 0) ? sh : -1;
}
inline void plan_order(const Geo &g, int dtype, Bias *b, bool strips)
{
    auto inverse = [](int n) { return n > 1 ? (uint32_t)((((uint64_t)1 << 32) + n - 1) / n) : 0xffffffffu; };
    b->w2 = 2 * g.M - 1;
    b->sh = strips ? strip_shift(dtype, g.M) : -1;
    b->sw = b->sh < 0 ? g.M : 1 << b->sh;
    b->strip = g.M * b->sw;
    b->ws = 2 * b->sw - 1;
    b->inv_strip = inverse(b->strip), b->inv_ws = inverse(b->ws);
}
// What the products cannot carry of the scale goes into q: its sign, and a power of two where it is outside [2^-20, 2^21) (so that neither bias / scale
// nor the sums overflow; 0 is 0 times 1).  Both leave q's digits as they are.
inline void plan_scale(const Geo &g, Bias *b)
{
    float rest = 1.f;
    b->qs = 0.f;
    if (g.scale_c != 0.f) {
        const int e = std::ilogb(g.scale_c), k = e < -20 ? e + 20 : e > 20 ? e - 20 : 0;
        rest = std::ldexp(std::fabs(g.scale_c), -k);
        b->qs = std::copysign(std::ldexp(1.f, k), g.scale_c);
    }
    b->bs = 1.f / rest;
    b->c = rest * rows::kLog2e;
    b->ks = rest;
}

// The most window rows that `len` tokens from a multiple of `len` on touch.
inline int most_rows(int len, const Geo &g, const Bias &b)
{
    if (len >= g.N) return g.M;
    if (b.sh >= 0) return b.strip % len == 0 ? len >> b.sh : g.M;
    const int rows = len % g.M == 0 ? len / g.M : g.M % len == 0 ? 1 : (len + g.M - 2) / g.M + 1;
    return rows < g.M ? rows : g.M;
}

// A probability made again from LSE, 2^x: at most 1.  (A row whose logits all lie near -1e9, say, has an LSE that fp32 rounds by tens; without the bound,
// which is a bit of the instruction, such a row's gradients would overflow and take its window's with them.)
__device__ __forceinline__ float prob(float x) { return __builtin_amdgcn_fmed3f(__builtin_amdgcn_exp2f(x), 0.f, 1.f); }

__device__ __forceinline__ int row_of(int n, uint32_t inv_m) { return (int)__umulhi((uint32_t)n, inv_m); }
// The n-th token of the walk: its row and column.
struct Cell {
    int y, x, xl;           // (xl: column in its strip)
    __device__ __forceinline__ int lin(const Bias &b) const { return y * b.ws + xl; }
    __device__ __forceinline__ int index(const Geo &g) const { return y * g.M + x; }       // its number in the window, as lse has it
};
template <bool STRIPS>
__device__ __forceinline__ Cell cell_of(const Geo &g, const Bias &b, int n)
{
    Cell c;
    if (STRIPS) {
        const int s = (int)__umulhi((uint32_t)n, b.inv_strip), r = n - s * b.strip;
        c.y = r >> b.sh, c.xl = r & (b.sw - 1), c.x = (s << b.sh) + c.xl;
    } else {
        c.y = row_of(n, g.inv_m), c.x = c.xl = n - c.y * g.M;
    }
    return c;
}
// The window rows of tokens [first, last] of one strip, and the strip's first column.
struct Span {
    int y0, y1, x0;
};
template <bool STRIPS>
__device__ __forceinline__ Span span_of(const Geo &g, const Bias &b, int first, int last)
{
    const Cell c = cell_of<STRIPS>(g, b, first);
    return Span{c.y, cell_of<STRIPS>(g, b, last).y, c.x - c.xl};
}

// The offsets of one chunk: rows `s` stationary, `t` streamed.
struct Chunk {
    Span s, t;
    int c0, count;          // `count`: offsets
    int t0;                 // first token of the streamed strip
};
template <bool STRIPS>
__device__ __forceinline__ Chunk chunk_of(const Geo &g, const Bias &b, int t0, int t1, const Span &s)
{
    Chunk c;
    const int e = t1 * kTile < g.N ? t1 * kTile : g.N;
    c.s = s, c.t = span_of<STRIPS>(g, b, t0 * kTile, e - 1);
    c.c0 = (s.y1 - c.t.y0) * b.ws + b.sw - 1;
    c.count = (c.t.y1 - c.t.y0 + s.y1 - s.y0 + 1) * b.ws;
    c.t0 = STRIPS ? c.t.x0 * g.M : 0;
    return c;
}

__device__ __forceinline__ int lin(const Geo &g, int n) { return n + row_of(n, g.inv_m) * (g.M - 1); }

// Whether some key is not excluded for query n (numbered as in lse); asked by whole waves.
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
    // word (row, column) is row + t.y0 - s.y1 rows and column + t.x0 - s.x0 - (sw - 1) columns from stationary to streamed
    const int at = 2 * g.M * (g.M - 1) + SGN * ((c.t.y0 - c.s.y1) * b.w2 + c.t.x0 - c.s.x0 - (b.sw - 1));
    for (int l = threadIdx.x; l < c.count; l += nt) {
        const int r = (int)__umulhi((uint32_t)l, b.inv_ws);
        const float x = src[at + SGN * (l + r * (b.w2 - b.ws))];
        lds[l] = x <= kExcluded ? -INFINITY : x * scale;
    }
}

// Adds the waves' histograms of a chunk (dS summed by offset, `hsize` values a wave, WT stationary tokens each, STEP from one wave's to the next's) in their order, writes
// them to the workgroup's sums `dst` (of this streamed strip, from the chunk's first row on) and clears them.  `before`: the last row of
// the strip's chunk before (-1: none); what that one touched is added to.
template <bool STRIPS, int W, int STEP, int WT>
__device__ __forceinline__ void flush(const Geo &g, const Bias &b, const Chunk &ch, double *H, int hsize, int first, int before, float *dst)
{
    const int old = before < 0 ? 0 : (before - ch.t.y0 + ch.s.y1 - ch.s.y0 + 1) * b.ws;
    for (int e = threadIdx.x; e < ch.count; e += 64 * W) {
        double sum = 0.;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const int f = first + w * STEP;
            if (f >= g.N) break;
            const Span v = span_of<STRIPS>(g, b, f, f + WT < g.N ? f + WT - 1 : g.N - 1);
            const int at = e - (ch.s.y1 - v.y1) * b.ws;
            if (at >= 0 && at < (ch.t.y1 - ch.t.y0 + v.y1 - v.y0 + 1) * b.ws) {
                sum += H[w * hsize + at];
                H[w * hsize + at] = 0.;
            }
        }
        dst[e] = (float)(e < old ? sum + dst[e] : sum);
    }
}
// The place of a workgroup's sums: [unit][workgroup][streamed strip][prows][ws].
__device__ __forceinline__ int64_t sums_at(const Geo &g, const Bias &b, int64_t u, int nblk, int blk, int prows, int x0)
{
    const int n = b.sh < 0 ? 1 : g.M >> b.sh;
    return (((u * nblk + blk) * n + (b.sh < 0 ? 0 : x0 >> b.sh)) * prows) * b.ws;
}

// ---- sources of rows ---------------------------------------------------------------------------------------------

// kFast: grid tensors, rows of 8 or more values, everything on 4-byte boundaries.  kAny: grid tensors, value by value.
// kCkpt: rows of an 8-bit checkpoint.
enum Source { kFast = 0, kAny = 1, kCkpt = 2 };

// Checkpoint (include/rib_attn.h): for q, k and v in turn [units][N][dp] codes; then for each [units][N] exponent bytes.
__host__ __device__ inline int ckpt_row(int d) { return (d + 15) & ~15; }
__host__ __device__ inline int64_t ckpt_rows(const Geo &g) { return g.units * g.N; }
// The step of exponent byte `e`, and what code `c` stands for under it.  (Exact: 128 is taken off first, since 128 steps may pass the largest number.)
__device__ __forceinline__ float code_step(uint32_t e) { return __uint_as_float(e << 23); }
__device__ __forceinline__ float code_value(uint32_t c, float step) { return ((float)c - 128.f) * step; }

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
    int group, nblk;                    // stationary tokens a workgroup, workgroups a unit
    int words;                          // of a workgroup's sums at most
    bool strips;                        // how the first kernel walked the windows
    int shares;                         // sums a head: of windows, or of the runs of windows a wave takes
};
inline Ws ws_layout(const Geo &g, int dtype)
{
    Ws w;
    const int sb = group_tokens(g, dtype);
    w.group = sb;
    w.nblk = (g.N + sb - 1) / sb;
    w.words = 0;
    for (int strips = 0; strips < 2; ++strips) {        // (which way depends on the tensors' alignment too)
        Bias b{};
        plan_order(g, dtype, &b, strips != 0);
        const int prows = g.M - 1 + most_rows(sb, g, b), words = (b.sh < 0 ? 1 : g.M >> b.sh) * prows * b.ws;
        if (words > w.words) w.words = words;
    }
    w.strips = false;
    w.shares = (int)(g.units / g.heads);
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    w.ext = 0;
    w.part = up((size_t)g.units * g.N * 8);
    w.total = w.part + up((size_t)g.units * w.nblk * w.words * sizeof(float));
    return w;
}
// dbias[head][offset] from the workgroups' sums: windows and workgroups in a fixed order.
hipError_t launch_reduce(const Geo &g, int dtype, const Ws &w, const float *part, float *dbias, hipStream_t st);

// Tiles a chunk and the rows that go with it: as many tiles as fit `bias_bytes` of bias and (hist) `hist_bytes` a wave, of one strip.
inline void plan_chunks(const Geo &g, int dtype, Bias *b, bool strips, int sb, bool hist, size_t bias_bytes, size_t hist_bytes)
{
    plan_order(g, dtype, b, strips);
    const int ntiles = (b->strip + kTile - 1) / kTile;
    const int srows = most_rows(sb, g, *b), wrows = most_rows(wave_tokens(dtype), g, *b);
    b->prows = g.M - 1 + srows;
    for (int tiles = ntiles;; tiles = tiles > 8 ? tiles - tiles / 8 : tiles - 1) {
        // (a strip's chunks start at multiples of `tiles` from its start)
        const int trows = b->sh >= 0 ? tiles * kTile >> b->sh : most_rows(tiles * kTile, g, *b);
        b->chunk = tiles;
        b->rows = trows + srows - 1;
        b->hrows = hist ? trows + wrows - 1 : 0;
        const bool fits = (size_t)b->rows * b->ws * 4 <= bias_bytes && (size_t)b->hrows * b->ws * 8 <= hist_bytes;
        if (fits || tiles == 1) return;
    }
}

}  // namespace rpb
}  // namespace rib
