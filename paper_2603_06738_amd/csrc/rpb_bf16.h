// Window attention with a learned relative position bias on the bf16 matrix cores: forward, and the backward pair (dq with
// the bias's gradient, then dkv).  Operator: include/rib_attn.h; the walk and the bias in LDS: rpb_common.h.
//
// A wave owns 64 stationary tokens as MFMA B operands, a workgroup W waves; the other side of the unit streams through LDS in
// tiles of 64 token rows, two stages in turn.  (SPLIT, for grids that would leave most of the chip idle: four waves share 64 stationary
// tokens, two blocks of them by two of every tile's; the sums of a block's two waves are added through LDS at the end.)  Scores are
// 32x32 blocks with the streamed tokens as rows, so a lane owns one stationary token and 16 streamed ones; their bias is the C operand
// of the score product.  What is packed to bf16 there
// (P, dS) is the B operand of the product that contracts over the streamed tokens, whose A operand is read transposed from
// the same rows.  Products of q and k are exact in fp32 and scaled there: rounding a scaled q to bf16 would save 16 of some 100 vector
// instructions a block, and cost as much accuracy as the rounding of P (2-norm errors of a training step 2.5e-3 so, 3.4e-3 with it; forward 8 %,
// whole step 5 % slower).
//
// LSE and delta stay in fp32: the lane's own in dq, in LDS beside the streamed rows in dkv, where -delta is the C operand of dP's product.  (As
// bf16 pairs in two more columns of the rows they were 4 % of dkv cheaper up to 30 channels and dearer from 32 on, and lost 2^-17 of LSE, which is an exponent.)
//
// What bounds it, by counters (16 images of 96 x 96, 32 x 32 windows, 6 heads of 30; forward with LSE / dq / dkv 207 / 374 / 312 us, forward without
// LSE 188): the vector issue is busy 81 / 57 / 60 % of the time and the matrix pipe 26 / 21 / 35 %, and the two hardly overlap.  A block of the forward has 60
// vector instructions in its loop, 40 of them exp2, scale and pack, and 17 more with LSE.  Parts taken out (of kernels without LSE's sum, with the pairs), us: staging -20 /
// -32 / -39, the barriers too -22 / -43 / -46, the bias -18 / -17 / -14.  Three waves a SIMD (168 registers) in the forward up to 32 channels, two
// elsewhere, one in the backward of wide heads (below).  Tiles of 128 tokens (half the barriers): forward the same, dq 5 % slower.
#pragma once

#include "rpb_common.h"

namespace rib {
namespace rpb {
namespace bf {

using namespace rows;

constexpr float kNoRow = 1e30f;         // in place of LSE where a row has no key: every probability is zero

// LDS image of a tile: X and Y rows, a streamed token's lin() and (EXT) -LSE in base 2 and -delta.  K: columns of the contracted width.
template <int KX, int KY, bool EXT = false>
struct Img {
    static constexpr int XS = KX + 8, YS = KY + 8;
    static constexpr int YR = kTile * XS, LT = YR + kTile * YS, EX = LT + 2 * kTile;
    static constexpr int STAGE = EX + (EXT ? 4 * kTile : 0);    // bf16 elements
    static constexpr int TOTAL = 2 * STAGE + 32;                // (transposed reads of the last row may run over its end)
};

// ---- rows: request, commit ---------------------------------------------------------------------------------------

struct Rows {
    const char *base;       // grid: this image's and head's slice; checkpoint: this unit's codes
    int64_t stride;         // bytes between tokens
    const uint8_t *exps;    // checkpoint: this unit's exponent bytes
};
struct Raw {
    uint32_t w[4];
};
struct __attribute__((packed, aligned(4))) u128a4 {
    uint32_t x, y, z, w;
};
template <int SRC>
__device__ __forceinline__ int piece_col(int j, int d)
{
    if (SRC == kAny) return 8 * j;
    const int n = SRC == kCkpt ? ckpt_row(d) : d;
    return 8 * j < n - 8 ? 8 * j : n - 8;
}
// Piece j (8 values) of token n, which is pixel `t`.
template <int SRC>
__device__ __forceinline__ Raw get_piece(const Rows &s, uint32_t t, int n, int j, int d)
{
    Raw r;
    const int c = piece_col<SRC>(j, d);
    if constexpr (SRC == kCkpt) {
        const uint2 w = *(const uint2 *)(s.base + (int64_t)n * s.stride + c);
        r.w[0] = w.x, r.w[1] = w.y, r.w[2] = s.exps[n], r.w[3] = 0u;
    } else if constexpr (SRC == kFast) {
        const u128a4 w = *(const u128a4 *)(s.base + (int64_t)t * s.stride + 2 * c);
        r.w[0] = w.x, r.w[1] = w.y, r.w[2] = w.z, r.w[3] = w.w;
    } else {
        const bf16_t *p = (const bf16_t *)(s.base + (int64_t)t * s.stride);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = c + 2 * i < d ? p[c + 2 * i] : 0u, hi = c + 2 * i + 1 < d ? p[c + 2 * i + 1] : 0u;
            r.w[i] = lo | hi << 16;
        }
    }
    return r;
}
// The bf16 pairs of a piece.  A checkpoint's values are exact in bf16: 7 bits under a power of two.
template <int SRC>
__device__ __forceinline__ Raw widen_piece(const Raw &r)
{
    if constexpr (SRC != kCkpt) return r;
    const float s = code_step(r.w[2]);
    Raw o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = r.w[i >> 1] >> (16 * (i & 1));
        o.w[i] = trunc_pack(code_value(w & 255u, s), code_value((w >> 8) & 255u, s));
    }
    return o;
}
template <int SRC>
__device__ __forceinline__ void put_piece(bf16_t *row, const Raw &r, int j, int d)
{
    const int c = piece_col<SRC>(j, d);
    if (SRC == kAny && c >= d) return;
    *(u128a4 *)(row + c) = u128a4{r.w[0], r.w[1], r.w[2], r.w[3]};
}
__device__ __forceinline__ Raw scaled(Raw r, float s)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = scale_pair(r.w[i], s);
    return r;
}

// A token as a pixel of its image.
__device__ __forceinline__ uint32_t pixel(const Win &w, const Cell &c) { return (uint32_t)(w.rowb[c.y] + w.colo[c.x]); }

// What a thread moves of a tile: LP lanes a token, P passes of nt lanes.
template <int LP, int W, int SX, int SY, bool EXT, bool ALN>
struct Mover {
    static constexpr int NT = 64 * W, P = (kTile * LP + NT - 1) / NT;
    Raw x[P], y[P];
    float2 e[EXT ? P : 1];

    __device__ __forceinline__ void request(const Geo &g, const Bias &bi, const Win &win, const Rows &xs, const Rows &ys, const float2 *ext, int tile)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int slot = p * NT + threadIdx.x, row = slot / LP, j = slot % LP;
            if (NT * P != kTile * LP && slot >= kTile * LP) break;
            const int n0 = tile * kTile + row, n = n0 < g.N ? n0 : g.N - 1;
            const Cell c = cell_of<ALN>(g, bi, n);
            const uint32_t t = SX == kCkpt && SY == kCkpt ? 0u : pixel(win, c);
            x[p] = get_piece<SX>(xs, t, c.index(g), j, g.d);
            y[p] = get_piece<SY>(ys, t, c.index(g), j, g.d);
            if (EXT) e[p] = ext[n];
        }
    }
    // KX, KY: the images' widths.
    template <int KX, int KY>
    __device__ __forceinline__ void commit(const Geo &g, const Bias &bi, bf16_t *S, int tile, float scale)
    {
        using I = Img<KX, KY, EXT>;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int slot = p * NT + threadIdx.x, row = slot / LP, j = slot % LP;
            if (NT * P != kTile * LP && slot >= kTile * LP) break;
            const int n = tile * kTile + row;
            const bool in = ALN || n < g.N;
            bf16_t *xr = S + row * I::XS, *yr = S + I::YR + row * I::YS;
            Raw a = widen_piece<SX>(x[p]), b = widen_piece<SY>(y[p]);
            if (EXT && scale != 1.f) a = scaled(a, scale);
            if (!in) b.w[0] = b.w[1] = b.w[2] = b.w[3] = 0u;    // (an infinity in the repeated last token must not meet P = 0)
            put_piece<SX>(xr, a, j, g.d);
            put_piece<SY>(yr, b, j, g.d);
            if (EXT && j == 0) {
                ((float *)(S + I::EX))[row] = in ? e[p].x : -kNoRow;
                ((float *)(S + I::EX))[kTile + row] = in ? e[p].y : 0.f;
            }
            if (!ALN && j == 0) ((int *)(S + I::LT))[row] = cell_of<false>(g, bi, in ? n : g.N - 1).lin(bi);
        }
    }
};
// Columns that no commit writes, once for both stages (beside the first commit: what both write is the same).  `one`: a one in Y's last.
template <int KX, int KY, bool EXT = false>
__device__ __forceinline__ void init_cols(const Geo &g, bf16_t *S, bool one, int nt)
{
    using I = Img<KX, KY, EXT>;
    for (int e = threadIdx.x; e < 2 * kTile; e += nt) {
        bf16_t *xr = S + (e / kTile) * I::STAGE + (e % kTile) * I::XS, *yr = S + (e / kTile) * I::STAGE + I::YR + (e % kTile) * I::YS;
        for (int c = g.d; c < KX; ++c) xr[c] = 0;
        for (int c = g.d; c < KY; ++c) yr[c] = one && c == KY - 1 ? 0x3f80 : 0;
    }
}

// A wave's 64 stationary rows of a tensor, LP lanes a row.  Asked for at a workgroup's very start, together with whatever else it needs
// first, so that it waits for memory once.
template <int LP>
struct Held {
    Raw r[LP];
};
template <int LP, int SRC, bool ALN>
__device__ __forceinline__ void hold(Held<LP> &h, const Geo &g, const Bias &bi, const Win &win, const Rows &s, int n0)
{
    const int lane = threadIdx.x & 63, l = lane / LP, j = lane % LP;
#pragma unroll
    for (int p = 0; p < LP; ++p) {
        const int n = n0 + p * (64 / LP) + l;
        const Cell c = cell_of<ALN>(g, bi, n < g.N ? n : g.N - 1);
        h.r[p] = get_piece<SRC>(s, SRC == kCkpt ? 0u : pixel(win, c), c.index(g), j, g.d);
    }
}
// QB blocks of the rows, from block `sel` on, as B operands, times `s`, through `area` (64 rows of K + 8 columns, the wave's own).
template <int K, int LP, int SRC, int QB>
__device__ __forceinline__ void operands(const Held<LP> &h, const Geo &g, bf16_t *area, bf16x8 (&B)[QB][K / 16], int sel, float s)
{
    constexpr int STR = K + 8;
    const int lane = threadIdx.x & 63, l = lane / LP, j = lane % LP;
    {
        bf16_t *xr = area + lane * STR;
        for (int c = g.d; c < K; ++c) xr[c] = 0;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int p = 0; p < LP; ++p) {
        const Raw r = widen_piece<SRC>(h.r[p]);
        put_piece<SRC>(area + (p * (64 / LP) + l) * STR, s != 1.f ? scaled(r, s) : r, j, g.d);
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int b = 0; b < QB; ++b) read_rows<K / 16>(B[b], area + ((sel + b) * 32 + (lane & 31)) * STR + 8 * (lane >> 5));
    __builtin_amdgcn_wave_barrier();
}

// ---- blocks ------------------------------------------------------------------------------------------------------

// LDS words of a lane's 16 streamed tokens of block `kb` of a tile, relative to the lane's own word (c0 - lin(stationary)).
// Tokens 8a + 4 hf + 0..3: four neighbours each in strips (ALN), else from the tile's table.
template <bool ALN>
struct Words16 {
    int at[ALN ? 4 : 16];
    __device__ __forceinline__ int operator()(int i) const { return ALN ? at[i >> 2] + (i & 3) : at[ALN ? 0 : i]; }
};
template <bool ALN>
__device__ __forceinline__ Words16<ALN> words_of(const Bias &bi, const Chunk &ch, const int *table, int tile, int kb, int hf)
{
    Words16<ALN> w;
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        if constexpr (ALN) {
            const int r = tile * kTile + kb * 32 + 8 * a - ch.t0;       // (all but 4 hf uniform)
            w.at[a] = (r >> bi.sh) * bi.ws + (r & (bi.sw - 1)) + 4 * hf;
        } else {
            const int4 t = *(const int4 *)(table + kb * 32 + 8 * a + 4 * hf);
            w.at[4 * a] = t.x, w.at[4 * a + 1] = t.y, w.at[4 * a + 2] = t.z, w.at[4 * a + 3] = t.w;
        }
    }
    return w;
}
template <bool ALN>
__device__ __forceinline__ f32x16 bias_block(const float *mine, const Words16<ALN> &w)
{
    f32x16 c;
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = mine[w(i)];
    return c;
}

// Adds a block of dS to the wave's sums by offset, in 64 bits (LDS adds doubles 20 times as fast as floats: 55 and 1290 ns for a wave's 16).
// The sums are the wave's own and its additions happen in its order, so they do not depend on what other waves do.
template <bool ALN>
__device__ __forceinline__ void add_offsets(double *mine, const Words16<ALN> &w, const f32x16 &v)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) __hip_atomic_fetch_add(mine + w(i), (double)v[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}

// Channels 8 (i / 4) + 4 hf .. + 3 of block `db` of a token's row, times `s`.
template <int SRC>
__device__ __forceinline__ void store_row(bf16_t *row, const f32x16 &v, int db, int d, int hf, float s)
{
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int c = 32 * db + 8 * a + 4 * hf, left = d - c;
        if (left <= 0) continue;
        const uint32_t w0 = pack_bf16(v[4 * a] * s, v[4 * a + 1] * s), w1 = pack_bf16(v[4 * a + 2] * s, v[4 * a + 3] * s);
        if (SRC == kAny) {
            row[c] = (bf16_t)w0;
            if (left > 1) row[c + 1] = (bf16_t)(w0 >> 16);
            if (left > 2) row[c + 2] = (bf16_t)w1;
            if (left > 3) row[c + 3] = (bf16_t)(w1 >> 16);
        } else {
            put8(row + c, dword2{w0, w1}, left < 4);
        }
    }
}

// Where a workgroup works: its unit, its block of stationary tokens, the window's map (in `map`, 2 M ints).
struct Place {
    int u, blk, w, hd, b;
    Win win;
    int64_t img;        // first pixel of the image
};
__device__ __forceinline__ Place place_of(const Geo &g, int nblk, int nt, int *map)
{
    Place p;
    int64_t u;
    block_coords(nblk, u, p.blk);
    p.u = (int)u, p.w = p.u / g.heads, p.hd = p.u - p.w * g.heads;
    p.win = window_of<false>(g, p.w, nt, map, p.b);
    p.img = (int64_t)p.b * g.H * g.W;
    return p;
}
__device__ __forceinline__ Rows grid_rows(const Geo &g, const Place &p, const void *x, int64_t stride)
{
    return Rows{(const char *)x + (p.img * stride + p.hd * g.d) * 2, stride * 2, nullptr};
}
// Tensor `which` (0 q, 1 k, 2 v) of a unit in a checkpoint.
__device__ __forceinline__ Rows ckpt_rows_of(const Geo &g, const Place &p, const uint8_t *c, int which)
{
    const int dp = ckpt_row(g.d);
    const int64_t rows = ckpt_rows(g), first = (int64_t)p.u * g.N + which * rows;
    return Rows{(const char *)c + first * dp, dp, c + 3 * rows * dp + first};
}

template <int KX, int KY, int W, bool EXT = false>
constexpr size_t stage_bytes()
{
    using I = Img<KX, KY, EXT>;
    const size_t tiles = (size_t)I::TOTAL * 2, stat = (size_t)W * 64 * (KX + 8) * 2;
    return ((tiles > stat ? tiles : stat) + 15) & ~(size_t)15;
}

// Adds the odd waves' sums to their even neighbours', through `lds` (16 * 64 floats a block and pair of waves).
template <int DB>
__device__ __forceinline__ void join(f32x16 (&v)[DB], float *lds, bool odd)
{
    float *const part = lds + (threadIdx.x >> 7) * DB * 16 * 64 + (threadIdx.x & 63);
    __syncthreads();
    if (odd)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) part[(16 * db + i) * 64] = v[db][i];
    __syncthreads();
    if (!odd)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) v[db][i] += part[(16 * db + i) * 64];
}

// ---- forward -----------------------------------------------------------------------------------------------------

// Two denominators of a row.  O's weights are P as rounded, so O is divided by the sum of those: a row of one key gives its v.  LSE wants P before it is rounded (with
// few keys the other sum would move it by up to 2^-8).  The first is a column of ones in V where V's block has one to spare, else (SUM)
// one instruction for two values of P; the second 16 additions a block, made only where LSE is asked for (forward of 32 x 32 windows, 6 heads of 30,
// 16 images: 188 us without, 207 with).
__device__ __forceinline__ float add_pair(float sum, uint32_t pair)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
}
struct Sums {
    float rounded, exact;
};

// One walk over the keys; `mv` holds the first tile.  MAX: with the running maximum of every row (`top`, in the products' unit).
template <bool MAX, int KX, int DB, bool SUM, bool LSE, int SRC, bool ALN, bool SPLIT, int W>
__device__ __forceinline__ void fwd_walk(const Geo &g, const Bias &bi, const Place &pl, const Rows &ks, const Rows &vs, bf16_t *S, float *B,
                                         const bf16x8 (&Q)[SPLIT ? 1 : 2][KX / 16], f32x16 (&O)[SPLIT ? 1 : 2][DB], Sums (&sum)[SPLIT ? 1 : 2], float (&top)[SPLIT ? 1 : 2], const Span &span,
                                         const int (&mylin)[SPLIT ? 1 : 2], bool active, Mover<KX <= 32 ? 4 : 8, W, SRC, SRC, false, ALN> &mv)
{
    constexpr int KY = 32 * DB, NT = 64 * W, QB = SPLIT ? 1 : 2;
    constexpr bool CARRY = ALN && !SPLIT;
    using I = Img<KX, KY>;
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 1;
    const int ntiles = (g.N + kTile - 1) / kTile, strip_tiles = ALN ? bi.strip / kTile : ntiles;
    const int tro = tr_lane_offset<I::YS>(lane), ako = col * I::XS + 8 * hf;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) O[qb][db][i] = 0.f;
        sum[qb] = Sums{0.f, 0.f}, top[qb] = MAX ? -INFINITY : 0.f;
    }
    mv.template commit<KX, KY>(g, bi, S, 0, 1.f);
    mv.request(g, bi, pl.win, ks, vs, nullptr, ntiles > 1 ? 1 : 0);
    f32x16 next;            // (CARRY) the bias of block (1, the coming one)
    for (int t0 = 0, t1, end = strip_tiles; t0 < ntiles; t0 = t1) {
        t1 = t0 + bi.chunk < end ? t0 + bi.chunk : end;
        const Chunk ch = chunk_of<ALN>(g, bi, t0, t1, span);
        stage_bias<-1>(g, bi, ch, pl.hd, bi.bs, B, NT);
        __syncthreads();
        if (CARRY && t0 * kTile == ch.t0 && active) next = bias_block<ALN>(B + ch.c0 - mylin[QB - 1], words_of<ALN>(bi, ch, nullptr, t0, 0, hf));
        for (int tile = t0; tile < t1; ++tile) {
            const bf16_t *cur = S + (tile & 1) * I::STAGE;
            if (tile + 1 < ntiles) {
                mv.template commit<KX, KY>(g, bi, S + ((tile + 1) & 1) * I::STAGE, tile + 1, 1.f);
                mv.request(g, bi, pl.win, ks, vs, nullptr, tile + 2 < ntiles ? tile + 2 : ntiles - 1);
            }
            if (active) {
#pragma unroll
                for (int kx = 0; kx < (SPLIT ? 1 : 2); ++kx) {
                    const int kb = SPLIT ? half : kx, key0 = tile * kTile + kb * 32;
                    if (!ALN && key0 >= g.N) break;
                    const Words16<ALN> wd = words_of<ALN>(bi, ch, (const int *)(cur + I::LT), tile, kb, hf);
                    bf16x8 Ak[KX / 16], At[DB][2];
                    read_rows<KX / 16>(Ak, cur + kb * 32 * I::XS + ako);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 2; ++i) At[db][i] = read_tr<I::YS>(cur + I::YR + (kb * 32 + 16 * i) * I::YS, tro, 32 * db);
#pragma unroll
                    for (int qx = 0; qx < QB; ++qx) {
                        const int qb = QB - 1 - qx;
                        f32x16 s = CARRY && qb == 1 ? next : bias_block<ALN>(B + ch.c0 - mylin[qb], wd);
                        if (CARRY && qb == 0) next = s;
#pragma unroll
                        for (int i = 0; i < KX / 16; ++i) s = mfma(Ak[i], Q[qb][i], s);
                        if (!ALN) mask_rows(s, key0, g.N, hf);
                        if (MAX) {
                            float m = s[0];
#pragma unroll
                            for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
                            m = fmaxf(top[qb], fmaxf(m, __shfl_xor(m, 32)));
                            // (a row of minus infinities so far: any finite stabiliser does)
                            const float ms = m == -INFINITY ? 0.f : m, alpha = __builtin_amdgcn_exp2f((top[qb] - ms) * bi.c);
                            top[qb] = m;
                            sum[qb].rounded *= alpha, sum[qb].exact *= alpha;
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] -= ms;            // (before the scale: the other way round a fused difference keeps the product's rounding)
#pragma unroll
                            for (int db = 0; db < DB; ++db)
#pragma unroll
                                for (int i = 0; i < 16; ++i) O[qb][db][i] *= alpha;
                        }
                        uint32_t P[8];
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * bi.c);
#pragma unroll
                        for (int i = 0; i < 8; ++i) P[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
                        if (LSE) {
                            float a = 0.f, b = 0.f;
#pragma unroll
                            for (int i = 0; i < 8; ++i) a += s[2 * i], b += s[2 * i + 1];
                            sum[qb].exact += a + b;
                        }
                        if (SUM) {
                            float a = 0.f, b = 0.f;
#pragma unroll
                            for (int i = 0; i < 4; ++i) a = add_pair(a, P[2 * i]), b = add_pair(b, P[2 * i + 1]);
                            sum[qb].rounded += a + b;
                        }
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            O[qb][db] = mfma(At[db][0], as_bf16x8(P[0], P[1], P[2], P[3]), O[qb][db]);
                            O[qb][db] = mfma(At[db][1], as_bf16x8(P[4], P[5], P[6], P[7]), O[qb][db]);
                        }
                    }
                }
            }
            __syncthreads();
        }
        if (t1 == end) end += strip_tiles;
    }
    if constexpr (SPLIT) {
        // the two halves' sums; with maxima of their own they are first brought to the larger one
        float *const part = (float *)S + (threadIdx.x >> 7) * (16 * DB + 3) * 64 + lane;
        if (half) {
            part[0] = top[0], part[64] = sum[0].rounded, part[128] = sum[0].exact;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) part[(3 + 16 * db + i) * 64] = O[0][db][i];
        }
        __syncthreads();
        if (!half) {
            float a = 1.f, b = 1.f;
            if (MAX) {
                const float m = fmaxf(top[0], part[0]), ms = m == -INFINITY ? 0.f : m;
                a = __builtin_amdgcn_exp2f((top[0] - ms) * bi.c), b = __builtin_amdgcn_exp2f((part[0] - ms) * bi.c);
                top[0] = m;
            }
            sum[0].rounded = sum[0].rounded * a + part[64] * b, sum[0].exact = sum[0].exact * a + part[128] * b;
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[0][db][i] = O[0][db][i] * a + part[(3 + 16 * db + i) * 64] * b;
        }
        __syncthreads();
    }
    // (the column of ones: the last row of O^T is register 15 of the upper lane half)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float mine = SUM ? sum[qb].rounded : O[qb][DB - 1][15], other = __shfl_xor(mine, 32);
        sum[qb].rounded = SUM ? mine + other : hf ? mine : other;
        if (LSE) sum[qb].exact += __shfl_xor(sum[qb].exact, 32);
    }
}

template <int KX, int DB, bool SUM, bool LSE, int SRC, bool ALN, bool SPLIT, int W>
__global__ __launch_bounds__(W * 64, DB == 1 ? 3 : 2) void fwd_kernel(Geo g, Bias bi, int nblk, int force_max, const bf16_t *__restrict__ q,
                                                        const bf16_t *__restrict__ k, const bf16_t *__restrict__ v,
                                                        bf16_t *__restrict__ out, float *__restrict__ lse)
{
    constexpr int LP = KX <= 32 ? 4 : 8, NT = 64 * W, QB = SPLIT ? 1 : 2, GT = SPLIT ? 64 : NT;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *S = (bf16_t *)smem;
    int *map = (int *)(smem + stage_bytes<KX, 32 * DB, W>());
    float *B = (float *)(map + 2 * g.M);
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(g, nblk, NT, map);
    __syncthreads();
    const int first = pl.blk * GT, last = first + GT < g.N ? first + GT - 1 : g.N - 1, n0 = first + (SPLIT ? 0 : wave * 64), sel = SPLIT ? wave >> 1 : 0, half = wave & 1;
    const Span span = span_of<ALN>(g, bi, first, last);
    const bool active = n0 < g.N;
    const Rows ks = grid_rows(g, pl, k, g.tstride), vs = grid_rows(g, pl, v, g.tstride);
    bf16x8 Q[QB][KX / 16];
    Mover<LP, W, SRC, SRC, false, ALN> mv;
    {
        Held<LP> hq;
        hold<LP, SRC, ALN>(hq, g, bi, pl.win, grid_rows(g, pl, q, g.tstride), n0);
        mv.request(g, bi, pl.win, ks, vs, nullptr, 0);
        operands<KX, LP, SRC, QB>(hq, g, S + wave * 64 * (KX + 8), Q, sel, bi.qs);
    }
    int mylin[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int n = n0 + (sel + qb) * 32 + col;
        mylin[qb] = cell_of<ALN>(g, bi, n < g.N ? n : g.N - 1).lin(bi);
    }
    __syncthreads();
    init_cols<KX, 32 * DB>(g, S, !SUM, NT);
    f32x16 O[QB][DB];
    Sums sum[QB];
    float top[QB];
    // First without a running maximum: exp2 of a logit is a normal number far beyond what bounded logits need.  A row whose
    // denominator leaves [2^-60, 2^60], and not for want of keys, sends the workgroup on a second walk, with one.
    bool bad = true;
    if (!force_max) {
        fwd_walk<false, KX, DB, SUM, LSE, SRC, ALN, SPLIT, W>(g, bi, pl, ks, vs, S, B, Q, O, sum, top, span, mylin, active, mv);
        bad = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb)
            if (active && !(SPLIT && half) && bad_rows(g, bi, pl.hd, n0 + (sel + qb) * 32 + col < g.N ? cell_of<ALN>(g, bi, n0 + (sel + qb) * 32 + col).index(g) : g.N, sum[qb].rounded)) bad = true;
    }
    if (__syncthreads_or(bad)) {
        mv.request(g, bi, pl.win, ks, vs, nullptr, 0);
        if (SPLIT) init_cols<KX, 32 * DB>(g, S, !SUM, NT);       // (the first walk's sums went through the tiles)
        fwd_walk<true, KX, DB, SUM, LSE, SRC, ALN, SPLIT, W>(g, bi, pl, ks, vs, S, B, Q, O, sum, top, span, mylin, active, mv);
    }
    if (SPLIT && half) return;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int n = n0 + (sel + qb) * 32 + col;
        if (n >= g.N) continue;
        const Cell c = cell_of<ALN>(g, bi, n);
        const bool none = sum[qb].rounded == 0.f;
        const float inv = none ? 0.f : 1.f / sum[qb].rounded;           // (a row without a key: zeros)
        // (asked of the pointer, which is null without LSE: where `top` goes unused the compiler spills up to 181 registers)
        if (lse != nullptr && hf == 0) lse[(int64_t)pl.u * g.N + c.index(g)] = none ? -INFINITY : (top[qb] * bi.c + __builtin_amdgcn_logf(LSE ? sum[qb].exact : sum[qb].rounded)) * kLn2;
        bf16_t *row = out + (pl.img + pixel(pl.win, c)) * g.C + pl.hd * g.d;
#pragma unroll
        for (int db = 0; db < DB; ++db) store_row<SRC>(row, O[qb][db], db, g.d, hf, inv);
    }
}

// ---- backward: dq and the bias's gradient -------------------------------------------------------------------------

// Two blocks of channels are more than 256 registers hold.  One wave a SIMD has 512 and spills nothing; whether that beats two that spill is measured (8 images
// of 96 x 96, 4 heads; us, two waves / one): dkv, 32 x 32 windows of 64 channels 1145 / 282, 24 x 24 of 48 673 / 182, 12 x 12 of 64 320 / 117: one
// throughout; dq, in strips, 64 columns 437 / 323, 48 columns 201 / 226, without strips 12 x 12 of 64 135 / 143, 20 x 20 of 40 170 / 246: one in the first.
template <int K, int DB, int SRC, int SG, bool ALN, bool SPLIT, int W, bool HIST>
__global__ __launch_bounds__(W * 64, DB == 2 && K == 64 && ALN && !SPLIT ? 1 : 2) void dq_kernel(Geo g, Bias bi, int nblk, const bf16_t *__restrict__ q,
                                                       const bf16_t *__restrict__ k, const bf16_t *__restrict__ v,
                                                       const uint8_t *__restrict__ ckpt, const bf16_t *__restrict__ out,
                                                       const bf16_t *__restrict__ dout, const float *__restrict__ lse,
                                                       bf16_t *__restrict__ dq, float2 *__restrict__ ext, float *__restrict__ part)
{
    constexpr int LP = DB == 1 ? 4 : 8, NT = 64 * W, QB = SPLIT ? 1 : 2, GT = SPLIT ? 64 : NT;      // (GT: the workgroup's stationary tokens)
    constexpr bool CARRY = ALN && !SPLIT;
    using I = Img<K, K>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *S = (bf16_t *)smem;
    int *map = (int *)(smem + stage_bytes<K, K, W>());
    float *B = (float *)(map + 2 * g.M);
    double *H = (double *)(B + ((bi.rows * bi.ws + 1) & ~1));           // [wave][hrows * w2]
    const int hsize = bi.hrows * bi.ws;
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(g, nblk, NT, map);
    if (HIST)
        for (int e = threadIdx.x; e < W * hsize; e += NT) H[e] = 0.;
    __syncthreads();
    const int first = pl.blk * GT, last = first + GT < g.N ? first + GT - 1 : g.N - 1, n0 = first + (SPLIT ? 0 : wave * 64), sel = SPLIT ? wave >> 1 : 0, half = wave & 1;
    const Span span = span_of<ALN>(g, bi, first, last);
    const Span own = span_of<ALN>(g, bi, n0 < g.N ? n0 : g.N - 1, n0 + 63 < g.N ? n0 + 63 : g.N - 1);      // the wave's own rows
    const bool active = n0 < g.N;
    const Rows ks = SRC == kCkpt ? ckpt_rows_of(g, pl, ckpt, 1) : grid_rows(g, pl, k, g.tstride);
    const Rows vs = SRC == kCkpt ? ckpt_rows_of(g, pl, ckpt, 2) : grid_rows(g, pl, v, g.tstride);
    bf16x8 Q[QB][K / 16], D[QB][K / 16];
    Mover<LP, W, SRC, SRC, false, ALN> mv;
    float L, delta = 0.f;       // LSE in base 2 and delta of row `lane`
    {
        Held<LP> hq, hd, ho;
        hold<LP, SG, ALN>(hd, g, bi, pl.win, grid_rows(g, pl, dout, g.C), n0);
        hold<LP, SG, ALN>(ho, g, bi, pl.win, grid_rows(g, pl, out, g.C), n0);
        const int n = n0 + lane, nc = n < g.N ? n : g.N - 1;
        const float e = lse[(int64_t)pl.u * g.N + cell_of<ALN>(g, bi, nc).index(g)];
        hold<LP, SRC, ALN>(hq, g, bi, pl.win, SRC == kCkpt ? ckpt_rows_of(g, pl, ckpt, 0) : grid_rows(g, pl, q, g.tstride), n0);
        mv.request(g, bi, pl.win, ks, vs, nullptr, 0);
        // delta of the wave's rows: LP lanes share one
        const int j = lane % LP, c = piece_col<SG>(j, g.d);
        // (row `lane` belongs to pass lane / (64 / LP), lanes (lane % (64 / LP)) * LP ..)
#pragma unroll
        for (int p = 0; p < LP; ++p) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {       // (a piece that slid back holds a neighbour's values first)
                const uint32_t a = ho.r[p].w[i >> 1], b = hd.r[p].w[i >> 1];
                const float x = i & 1 ? hi_bf16(a) * hi_bf16(b) : lo_bf16(a) * lo_bf16(b);
                s += SG == kAny || c + i >= 8 * j ? x : 0.f;
            }
#pragma unroll
            for (int m = 1; m < LP; m <<= 1) s += __shfl_xor(s, m);
            const float x = __shfl(s, (lane % (64 / LP)) * LP);
            if (lane / (64 / LP) == p) delta = x;
        }
        const bool none = n >= g.N || e == -INFINITY;
        L = none ? kNoRow : e * kLog2e;
        if (n < g.N) ext[(int64_t)pl.u * g.N + n] = float2{-L, -delta};
        bf16_t *area = S + wave * 64 * (K + 8);
        operands<K, LP, SRC, QB>(hq, g, area, Q, sel, bi.qs);
        operands<K, LP, SG, QB>(hd, g, area, D, sel, 1.f);
    }
    int mylin[QB];
    float mylse[QB], mydelta[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int n = n0 + (sel + qb) * 32 + col;
        mylin[qb] = cell_of<ALN>(g, bi, n < g.N ? n : g.N - 1).lin(bi);
        mylse[qb] = __shfl(L, (sel + qb) * 32 + col), mydelta[qb] = __shfl(delta, (sel + qb) * 32 + col);
    }
    __syncthreads();
    init_cols<K, K>(g, S, false, NT);
    f32x16 A[QB][DB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) A[qb][db][i] = 0.f;
    const int ntiles = (g.N + kTile - 1) / kTile, strip_tiles = ALN ? bi.strip / kTile : ntiles;
    const int tro = tr_lane_offset<I::XS>(lane), ako = col * I::XS + 8 * hf;
    const f32x16 z = {0};
    // -delta as the C operand of dP's product, held (the compiler would make it again for every product), where there are registers for it: up to 32
    // channels (dq of 32 x 32 windows, 6 heads of 30: 413 us with the subtraction, 386 so)
    constexpr bool MINUS = DB == 1;
    f32x16 minus[QB];
    if (MINUS)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
            for (int i = 0; i < 16; ++i) minus[qb][i] = -mydelta[qb];
            asm volatile("" : "+v"(minus[qb]));
        }
    mv.template commit<K, K>(g, bi, S, 0, 1.f);
    mv.request(g, bi, pl.win, ks, vs, nullptr, ntiles > 1 ? 1 : 0);
    f32x16 next, held;      // (CARRY) the bias of block (1, the coming one); dS of block (0, the last one)
    if (CARRY && HIST) held = z;
    int before = -1;            // last streamed row of the strip's chunk before
    for (int t0 = 0, t1, end = strip_tiles; t0 < ntiles; t0 = t1) {
        t1 = t0 + bi.chunk < end ? t0 + bi.chunk : end;
        const Chunk ch = chunk_of<ALN>(g, bi, t0, t1, span);
        stage_bias<-1>(g, bi, ch, pl.hd, bi.bs, B, NT);
        double *const mine = H + wave * hsize + ch.c0 - (span.y1 - own.y1) * bi.ws;
        __syncthreads();
        if (CARRY && t0 * kTile == ch.t0 && active) next = bias_block<ALN>(B + ch.c0 - mylin[QB - 1], words_of<ALN>(bi, ch, nullptr, t0, 0, hf));
        for (int tile = t0; tile < t1; ++tile) {
            const bf16_t *cur = S + (tile & 1) * I::STAGE;
            if (tile + 1 < ntiles) {
                mv.template commit<K, K>(g, bi, S + ((tile + 1) & 1) * I::STAGE, tile + 1, 1.f);
                mv.request(g, bi, pl.win, ks, vs, nullptr, tile + 2 < ntiles ? tile + 2 : ntiles - 1);
            }
            if (active) {
#pragma unroll
                for (int kx = 0; kx < (SPLIT ? 1 : 2); ++kx) {
                    const int kb = SPLIT ? half : kx, key0 = tile * kTile + kb * 32;
                    if (!ALN && key0 >= g.N) break;
                    const Words16<ALN> wd = words_of<ALN>(bi, ch, (const int *)(cur + I::LT), tile, kb, hf);
                    bf16x8 Ak[K / 16], Av[K / 16], At[DB][2];
                    read_rows<K / 16>(Ak, cur + kb * 32 * I::XS + ako);
                    read_rows<K / 16>(Av, cur + I::YR + kb * 32 * I::YS + ako);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 2; ++i) At[db][i] = read_tr<I::XS>(cur + (kb * 32 + 16 * i) * I::XS, tro, 32 * db);
#pragma unroll
                    for (int qx = 0; qx < QB; ++qx) {
                        const int qb = QB - 1 - qx;
                        f32x16 s = CARRY && qb == 1 ? next : bias_block<ALN>(B + ch.c0 - mylin[qb], wd), p = MINUS ? minus[qb] : z;
                        if (CARRY && qb == 0) next = s;
#pragma unroll
                        for (int i = 0; i < K / 16; ++i) s = mfma(Ak[i], Q[qb][i], s);
#pragma unroll
                        for (int i = 0; i < K / 16; ++i) p = mfma(Av[i], D[qb][i], p);
                        if (!ALN) mask_rows(s, key0, g.N, hf);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = prob(fmaf(s[i], bi.c, -mylse[qb])) * (MINUS ? p[i] : p[i] - mydelta[qb]);
                        if (HIST && CARRY && qb == 1) add_offsets<ALN>(mine - mylin[QB - 1], wd, s + held);
                        else if (HIST && CARRY) held = s;
                        else if (HIST && (ALN || n0 + (sel + qb) * 32 + col < g.N)) add_offsets<ALN>(mine - mylin[qb], wd, s);     // (many lanes at one word are slow)
                        uint32_t P[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) P[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            A[qb][db] = mfma(At[db][0], as_bf16x8(P[0], P[1], P[2], P[3]), A[qb][db]);
                            A[qb][db] = mfma(At[db][1], as_bf16x8(P[4], P[5], P[6], P[7]), A[qb][db]);
                        }
                    }
                }
            }
            __syncthreads();
        }
        if (HIST) {
            if (CARRY && t1 == end) {
                if (active) add_offsets<ALN>(mine - mylin[0], words_of<ALN>(bi, ch, nullptr, t1 - 1, 1, hf), held);
                held = z;
                __syncthreads();
            }
            flush<ALN, W, SPLIT ? 0 : 64, 64>(g, bi, ch, H, hsize, first, before,
                              part + sums_at(g, bi, pl.u, nblk, pl.blk, bi.prows, ch.t.x0) + ch.t.y0 * bi.ws);
            before = t1 == end ? -1 : ch.t.y1;
        }
        if (t1 == end) end += strip_tiles;
    }
    if constexpr (SPLIT) {
        join<DB>(A[0], (float *)S, half);
        if (half) return;
    }
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int n = n0 + (sel + qb) * 32 + col;
        if (n >= g.N) continue;
        bf16_t *row = dq + (pl.img + pixel(pl.win, cell_of<ALN>(g, bi, n))) * g.C + pl.hd * g.d;
#pragma unroll
        for (int db = 0; db < DB; ++db) store_row<SG>(row, A[qb][db], db, g.d, hf, g.scale_c);
    }
}

// ---- backward: dk, dv --------------------------------------------------------------------------------------------

template <int K, int DB, int SRC, int SG, bool ALN, bool SPLIT, int W>
__global__ __launch_bounds__(W * 64, DB == 1 || SPLIT ? 2 : 1) void dkv_kernel(Geo g, Bias bi, int nblk, const bf16_t *__restrict__ q,
                                                        const bf16_t *__restrict__ k, const bf16_t *__restrict__ v,
                                                        const uint8_t *__restrict__ ckpt, const bf16_t *__restrict__ dout,
                                                        const float2 *__restrict__ ext, bf16_t *__restrict__ dk, bf16_t *__restrict__ dv)
{
    constexpr int LP = DB == 1 ? 4 : 8, NT = 64 * W, QB = SPLIT ? 1 : 2, GT = SPLIT ? 64 : NT;      // (GT: the workgroup's stationary tokens)
    constexpr bool CARRY = ALN && !SPLIT;
    using I = Img<K, K, true>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *S = (bf16_t *)smem;
    int *map = (int *)(smem + stage_bytes<K, K, W, true>());
    float *B = (float *)(map + 2 * g.M);
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(g, nblk, NT, map);
    __syncthreads();
    const int first = pl.blk * GT, last = first + GT < g.N ? first + GT - 1 : g.N - 1, n0 = first + (SPLIT ? 0 : wave * 64), sel = SPLIT ? wave >> 1 : 0, half = wave & 1;
    const Span span = span_of<ALN>(g, bi, first, last);
    const bool active = n0 < g.N;
    const Rows qs = SRC == kCkpt ? ckpt_rows_of(g, pl, ckpt, 0) : grid_rows(g, pl, q, g.tstride), ds = grid_rows(g, pl, dout, g.C);
    const float2 *const ex = ext + (int64_t)pl.u * g.N;
    bf16x8 Kb[QB][K / 16], Vb[QB][K / 16];
    Mover<LP, W, SRC, SG, true, ALN> mv;
    {
        Held<LP> hk, hv;
        hold<LP, SRC, ALN>(hk, g, bi, pl.win, SRC == kCkpt ? ckpt_rows_of(g, pl, ckpt, 1) : grid_rows(g, pl, k, g.tstride), n0);
        hold<LP, SRC, ALN>(hv, g, bi, pl.win, SRC == kCkpt ? ckpt_rows_of(g, pl, ckpt, 2) : grid_rows(g, pl, v, g.tstride), n0);
        mv.request(g, bi, pl.win, qs, ds, ex, 0);
        bf16_t *area = S + wave * 64 * (K + 8);
        operands<K, LP, SRC, QB>(hk, g, area, Kb, sel, 1.f);
        operands<K, LP, SRC, QB>(hv, g, area, Vb, sel, 1.f);
    }
    int mylin[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int n = n0 + (sel + b) * 32 + col;
        mylin[b] = cell_of<ALN>(g, bi, n < g.N ? n : g.N - 1).lin(bi);
    }
    __syncthreads();
    init_cols<K, K, true>(g, S, false, NT);
    f32x16 Ak[QB][DB], Av[QB][DB];
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) Ak[b][db][i] = 0.f, Av[b][db][i] = 0.f;
    const int ntiles = (g.N + kTile - 1) / kTile, strip_tiles = ALN ? bi.strip / kTile : ntiles;
    const int tro = tr_lane_offset<I::XS>(lane), ako = col * I::XS + 8 * hf;
    const float scale = bi.qs;
    f32x16 next;            // (CARRY) the bias of block (1, the coming one)
    mv.template commit<K, K>(g, bi, S, 0, scale);
    mv.request(g, bi, pl.win, qs, ds, ex, ntiles > 1 ? 1 : 0);
    for (int t0 = 0, t1, end = strip_tiles; t0 < ntiles; t0 = t1) {
        t1 = t0 + bi.chunk < end ? t0 + bi.chunk : end;
        const Chunk ch = chunk_of<ALN>(g, bi, t0, t1, span);
        stage_bias<1>(g, bi, ch, pl.hd, bi.bs, B, NT);
        __syncthreads();
        if (CARRY && t0 * kTile == ch.t0 && active) next = bias_block<ALN>(B + ch.c0 - mylin[QB - 1], words_of<ALN>(bi, ch, nullptr, t0, 0, hf));
        for (int tile = t0; tile < t1; ++tile) {
            const bf16_t *cur = S + (tile & 1) * I::STAGE;
            if (tile + 1 < ntiles) {
                mv.template commit<K, K>(g, bi, S + ((tile + 1) & 1) * I::STAGE, tile + 1, scale);
                mv.request(g, bi, pl.win, qs, ds, ex, tile + 2 < ntiles ? tile + 2 : ntiles - 1);
            }
            if (active) {
#pragma unroll
                for (int qx = 0; qx < (SPLIT ? 1 : 2); ++qx) {
                    const int qb = SPLIT ? half : qx;
                    if (!ALN && tile * kTile + qb * 32 >= g.N) break;
                    const Words16<ALN> wd = words_of<ALN>(bi, ch, (const int *)(cur + I::LT), tile, qb, hf);
                    bf16x8 Aq[K / 16], Ad[K / 16], Tq[DB][2], Td[DB][2];
                    float4 l[4];            // -LSE in base 2 of the lane's 16 queries, and their -delta
                    f32x16 dl;
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const float *const e = (const float *)(cur + I::EX) + qb * 32 + 8 * a + 4 * hf;
                        const float4 x = *(const float4 *)(e + kTile);
                        l[a] = *(const float4 *)e;
                        dl[4 * a] = x.x, dl[4 * a + 1] = x.y, dl[4 * a + 2] = x.z, dl[4 * a + 3] = x.w;
                    }
                    read_rows<K / 16>(Aq, cur + qb * 32 * I::XS + ako);
                    read_rows<K / 16>(Ad, cur + I::YR + qb * 32 * I::YS + ako);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            Tq[db][i] = read_tr<I::XS>(cur + (qb * 32 + 16 * i) * I::XS, tro, 32 * db);
                            Td[db][i] = read_tr<I::YS>(cur + I::YR + (qb * 32 + 16 * i) * I::YS, tro, 32 * db);
                        }
#pragma unroll
                    for (int bx = 0; bx < QB; ++bx) {
                        const int b = QB - 1 - bx;
                        f32x16 s = CARRY && b == 1 ? next : bias_block<ALN>(B + ch.c0 - mylin[b], wd), p = dl;
                        if (CARRY && b == 0) next = s;
#pragma unroll
                        for (int i = 0; i < K / 16; ++i) s = mfma(Aq[i], Kb[b][i], s);
#pragma unroll
                        for (int i = 0; i < K / 16; ++i) p = mfma(Ad[i], Vb[b][i], p);
                        uint32_t P[8], G[8];
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] = prob(fmaf(s[i], bi.c, ((const float *)&l[i >> 2])[i & 3]));
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            P[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
                            G[i] = pack_bf16(s[2 * i] * p[2 * i], s[2 * i + 1] * p[2 * i + 1]);
                        }
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            Av[b][db] = mfma(Td[db][0], as_bf16x8(P[0], P[1], P[2], P[3]), Av[b][db]);
                            Av[b][db] = mfma(Td[db][1], as_bf16x8(P[4], P[5], P[6], P[7]), Av[b][db]);
                            Ak[b][db] = mfma(Tq[db][0], as_bf16x8(G[0], G[1], G[2], G[3]), Ak[b][db]);
                            Ak[b][db] = mfma(Tq[db][1], as_bf16x8(G[4], G[5], G[6], G[7]), Ak[b][db]);
                        }
                    }
                }
            }
            __syncthreads();
        }
        if (t1 == end) end += strip_tiles;
    }
    if constexpr (SPLIT) {
        join<DB>(Ak[0], (float *)S, half);
        join<DB>(Av[0], (float *)S, half);
        if (half) return;
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int n = n0 + (sel + b) * 32 + col;
        if (n >= g.N) continue;
        const int64_t at = (pl.img + pixel(pl.win, cell_of<ALN>(g, bi, n))) * g.C + pl.hd * g.d;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            store_row<SG>(dk + at, Ak[b][db], db, g.d, hf, bi.ks);
            store_row<SG>(dv + at, Av[b][db], db, g.d, hf, 1.f);
        }
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------

constexpr size_t kBiasBytes = 36 * 1024, kHistBytes = 9 * 1024;

template <int KX, int DB, bool SUM, bool LSE, int SRC, bool ALN, bool SPLIT, int W>
hipError_t launch_fwd_lse(const Geo &g, const FwdArgs &a)
{
    Bias bi{a.bias};
    plan_scale(g, &bi);
    plan_chunks(g, RIB_BF16, &bi, ALN, SPLIT ? 64 : 64 * W, false, kBiasBytes, 0);
    const int nblk = (g.N + (SPLIT ? 64 : 64 * W) - 1) / (SPLIT ? 64 : 64 * W);
    const size_t smem = stage_bytes<KX, 32 * DB, W>() + 8 * (size_t)g.M + (size_t)bi.rows * bi.ws * 4;
    if (smem > (size_t)kMaxDynLds) return hipErrorInvalidValue;
    auto kern = fwd_kernel<KX, DB, SUM, LSE, SRC, ALN, SPLIT, W>;
    const hipError_t e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.units * nblk)), dim3(64 * W), smem, a.st, g, bi, nblk, a.force_max, (const bf16_t *)a.q,
                       (const bf16_t *)a.k, (const bf16_t *)a.v, (bf16_t *)a.out, a.lse);
    return hipGetLastError();
}
template <int KX, int DB, bool SUM, int SRC, bool ALN, bool SPLIT, int W>
hipError_t launch_fwd_one(const Geo &g, const FwdArgs &a)
{
    return a.lse != nullptr ? launch_fwd_lse<KX, DB, SUM, true, SRC, ALN, SPLIT, W>(g, a) : launch_fwd_lse<KX, DB, SUM, false, SRC, ALN, SPLIT, W>(g, a);
}
template <int K, int DB, int SRC, int SG, bool ALN, bool SPLIT, int W, bool HIST>
hipError_t launch_dq_one(const Geo &g, const BwdArgs &a, const Ws &ws)
{
    Bias bi{a.bias};
    plan_scale(g, &bi);
    plan_chunks(g, RIB_BF16, &bi, ALN, SPLIT ? 64 : 64 * W, HIST, kBiasBytes, kHistBytes);
    const size_t smem = stage_bytes<K, K, W>() + 8 * (size_t)g.M + ((size_t)bi.rows * bi.ws + 1) / 2 * 8 + (size_t)W * bi.hrows * bi.ws * 8;
    if (smem > (size_t)kMaxDynLds) return hipErrorInvalidValue;
    auto kern = dq_kernel<K, DB, SRC, SG, ALN, SPLIT, W, HIST>;
    const hipError_t e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.units * ws.nblk)), dim3(64 * W), smem, a.st, g, bi, ws.nblk, (const bf16_t *)a.q,
                       (const bf16_t *)a.k, (const bf16_t *)a.v, a.ckpt, (const bf16_t *)a.out, (const bf16_t *)a.dout, a.lse,
                       (bf16_t *)a.dq, (float2 *)((char *)a.ws + ws.ext), (float *)((char *)a.ws + ws.part));
    return hipGetLastError();
}
template <int K, int DB, int SRC, int SG, bool ALN, bool SPLIT, int W>
hipError_t launch_pair(const Geo &g, const BwdArgs &a, Ws &ws)
{
    ws.strips = ALN;
    if (ws.group != (SPLIT ? 64 : 64 * W)) return hipErrorInvalidValue;
    hipError_t e = a.dbias != nullptr ? launch_dq_one<K, DB, SRC, SG, ALN, SPLIT, W, true>(g, a, ws) : launch_dq_one<K, DB, SRC, SG, ALN, SPLIT, W, false>(g, a, ws);
    if (e != hipSuccess) return e;
    Bias bi{a.bias};
    plan_scale(g, &bi);
    plan_chunks(g, RIB_BF16, &bi, ALN, SPLIT ? 64 : 64 * W, false, kBiasBytes, 0);
    const size_t smem = stage_bytes<K, K, W, true>() + 8 * (size_t)g.M + (size_t)bi.rows * bi.ws * 4;
    if (smem > (size_t)kMaxDynLds) return hipErrorInvalidValue;
    auto kern = dkv_kernel<K, DB, SRC, SG, ALN, SPLIT, W>;
    e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.units * ws.nblk)), dim3(64 * W), smem, a.st, g, bi, ws.nblk, (const bf16_t *)a.q,
                       (const bf16_t *)a.k, (const bf16_t *)a.v, a.ckpt, (const bf16_t *)a.dout, (const float2 *)((const char *)a.ws + ws.ext),
                       (bf16_t *)a.dk, (bf16_t *)a.dv);
    return hipGetLastError();
}
}  // namespace bf
}  // namespace rpb
}  // namespace rib
