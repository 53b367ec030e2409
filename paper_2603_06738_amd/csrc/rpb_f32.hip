// Window attention with a learned relative position bias, fp32 storage, on the fp32 matrix instruction (32x32x2): products,
// sums and softmax state in fp32.  Operator: include/rib_attn.h; the walk and the bias in LDS: rpb_common.h.
//
// A wave owns 32 stationary tokens, a workgroup W waves; the other side streams through LDS in tiles of 64 token rows, two
// stages in turn.  Scores have the streamed tokens as rows: a lane owns one stationary token and 16 streamed ones, and its
// P and dS are, register by register, the B operands of the product that contracts over the streamed tokens (k = 0 and 1 of
// an instruction are the two lane halves).  What bounds it is that instruction: a 32x32 block at 32 channels is 16 of them
// a product (64 clk each), the exponentials beside it a tenth.  By counters (4 images of 96 x 96, 32 x 32 windows, 6 heads of 30; forward / dq / dkv
// 318 / 504 / 515 us) it is busy 65 / 59 / 76 % of the time; the rest is starts, ends and barriers.
#include "rpb_bf16.h"

namespace rib {
namespace rpb {
namespace fp {

using namespace rows;
using bf::bias_block;
using bf::Place;
using bf::place_of;
using bf::pixel;
using bf::Words16;
using bf::words_of;

__device__ __forceinline__ f32x16 mfma2(float a, float b, const f32x16 &c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

template <int DB>
struct Img {
    static constexpr int STR = 32 * DB + 4;                     // floats: an odd number of 16 bytes
    static constexpr int YR = kTile * STR, LT = 2 * YR, EX = LT + kTile;
    static constexpr int STAGE = EX + 2 * kTile;
};

struct Rows {
    const char *base;
    int64_t stride;         // bytes between tokens
    const uint8_t *exps;
};
__device__ __forceinline__ Rows rows_of_grid(const Geo &g, const Place &p, const void *x, int64_t stride)
{
    return Rows{(const char *)x + (p.img * stride + p.hd * g.d) * 4, stride * 4, nullptr};
}
// Values c .. c+3 of a token's row (zeros past the head).  With a checkpoint a raw word of codes and the exponent.
struct Raw {
    float x, y, z, w;
};
template <bool CKPT>
__device__ __forceinline__ Raw get4(const Rows &s, uint32_t t, int n, int c, int d)
{
    if constexpr (CKPT) {
        const int dp = ckpt_row(d);
        const uint32_t w = c < dp ? *(const uint32_t *)(s.base + (int64_t)n * s.stride + c) : 0x80808080u;
        const float sc = code_step(s.exps[n]);
        return Raw{code_value(w & 255u, sc), code_value((w >> 8) & 255u, sc), code_value((w >> 16) & 255u, sc), code_value(w >> 24, sc)};
    } else {
        const float *p = (const float *)(s.base + (int64_t)t * s.stride) + c;
        if (c + 4 <= d) {
            const float4u v = *(const float4u *)p;
            return Raw{v.x, v.y, v.z, v.w};
        }
        return Raw{c < d ? p[0] : 0.f, c + 1 < d ? p[1] : 0.f, c + 2 < d ? p[2] : 0.f, 0.f};
    }
}

template <int DB, int W, bool CX, bool CY, bool EXT, bool ALN>
struct Mover {
    static constexpr int LP = 8 * DB, NT = 64 * W, P = (kTile * LP + NT - 1) / NT;
    Raw x[P], y[P];
    float2 e;

    __device__ __forceinline__ void request(const Geo &g, const Bias &bi, const Win &win, const Rows &xs, const Rows &ys, const float2 *ext, int tile)
    {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int slot = p * NT + threadIdx.x, row = slot / LP, j = slot % LP;
            const int n0 = tile * kTile + row, n = n0 < g.N ? n0 : g.N - 1;
            const Cell c = cell_of<ALN>(g, bi, n);
            const uint32_t t = CX && CY ? 0u : pixel(win, c);
            x[p] = get4<CX>(xs, t, c.index(g), 4 * j, g.d);
            y[p] = get4<CY>(ys, t, c.index(g), 4 * j, g.d);
        }
        if (EXT && threadIdx.x < kTile) {
            const int n = tile * kTile + threadIdx.x;
            e = n < g.N ? ext[n] : float2{-bf::kNoRow, 0.f};
        }
    }
    __device__ __forceinline__ void commit(const Geo &g, const Bias &bi, float *S, int tile, float scale)
    {
        using I = Img<DB>;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int slot = p * NT + threadIdx.x, row = slot / LP, j = slot % LP;
            Raw a = x[p], b = y[p];
            if (EXT) a.x *= scale, a.y *= scale, a.z *= scale, a.w *= scale;
            if (tile * kTile + row >= g.N) b.x = b.y = b.z = b.w = 0.f;     // (an infinity in the repeated last token must not meet P = 0)
            *(Raw *)(S + row * I::STR + 4 * j) = a;
            *(Raw *)(S + I::YR + row * I::STR + 4 * j) = b;
        }
        if (threadIdx.x < kTile) {
            const int n = tile * kTile + threadIdx.x;
            if (!ALN) ((int *)(S + I::LT))[threadIdx.x] = cell_of<false>(g, bi, n < g.N ? n : g.N - 1).lin(bi);
            if (EXT) S[I::EX + threadIdx.x] = e.x, S[I::EX + kTile + threadIdx.x] = e.y;
        }
    }
};

// A lane's B operands of its stationary token: channels 8 s + 4 hf .. + 3 of step s.
template <int DB, bool CKPT>
__device__ __forceinline__ void operand(const Geo &g, const Place &pl, const Rows &s, const Cell &c, float scale, Raw (&B)[4 * DB])
{
    const int hf = (threadIdx.x & 63) >> 5;
    const uint32_t t = CKPT ? 0u : pixel(pl.win, c);
#pragma unroll
    for (int k = 0; k < 4 * DB; ++k) {
        B[k] = get4<CKPT>(s, t, c.index(g), 8 * k + 4 * hf, g.d);
        B[k].x *= scale, B[k].y *= scale, B[k].z *= scale, B[k].w *= scale;
    }
}
// 32 streamed rows against the lane's operands: `row` is this lane's streamed row (+ 4 hf).
template <int DB>
__device__ __forceinline__ f32x16 scores(const float *row, const Raw (&B)[4 * DB], f32x16 c, int d)
{
#pragma unroll
    for (int k = 0; k < 4 * DB; ++k) {
        if (8 * k >= d) break;
        const Raw a = *(const Raw *)(row + 8 * k);
        c = mfma2(a.x, B[k].x, c);
        c = mfma2(a.y, B[k].y, c);
        c = mfma2(a.z, B[k].z, c);
        c = mfma2(a.w, B[k].w, c);
    }
    return c;
}
// acc^T += rows^T p: `col` is the block's first streamed row + 4 hf rows + this lane's channel.
template <int DB>
__device__ __forceinline__ void contract(f32x16 (&acc)[DB], const float *col, const f32x16 &p)
{
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = mfma2(col[(8 * (i >> 2) + (i & 3)) * Img<DB>::STR + 32 * db], p[i], acc[db]);
}
template <int DB>
__device__ __forceinline__ void store_row(float *row, const f32x16 (&v)[DB], int d, int hf, float s)
{
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int c = 32 * db + 8 * a + 4 * hf;
            if (c + 4 <= d) *(float4u *)(row + c) = float4u{v[db][4 * a] * s, v[db][4 * a + 1] * s, v[db][4 * a + 2] * s, v[db][4 * a + 3] * s};
            else
#pragma unroll
                for (int r = 0; r < 3; ++r)
                    if (c + r < d) row[c + r] = v[db][4 * a + r] * s;
        }
}
template <int DB>
constexpr size_t stage_bytes()
{
    return (size_t)2 * Img<DB>::STAGE * 4;
}
__device__ __forceinline__ Rows rows_of_ckpt(const Geo &g, const Place &p, const uint8_t *c, int which)
{
    const bf::Rows r = bf::ckpt_rows_of(g, p, c, which);
    return Rows{r.base, r.stride, r.exps};
}

template <bool MAX, int DB, bool ALN, int W>
__device__ __forceinline__ void fwd_walk(const Geo &g, const Bias &bi, const Place &pl, const Rows &ks, const Rows &vs, float *S, float *B,
                                         const Raw (&Q)[4 * DB], f32x16 (&O)[DB], float &sum, float &top, const Span &span, int mylin, bool active)
{
    using I = Img<DB>;
    constexpr int NT = 64 * W;
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5;
    const int ntiles = (g.N + kTile - 1) / kTile, strip_tiles = ALN ? bi.strip / kTile : ntiles;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) O[db][i] = 0.f;
    sum = 0.f, top = MAX ? -INFINITY : 0.f;
    Mover<DB, W, false, false, false, ALN> mv;
    mv.request(g, bi, pl.win, ks, vs, nullptr, 0);
    mv.commit(g, bi, S, 0, 1.f);
    mv.request(g, bi, pl.win, ks, vs, nullptr, ntiles > 1 ? 1 : 0);
    for (int t0 = 0, t1, end = strip_tiles; t0 < ntiles; t0 = t1) {
        t1 = t0 + bi.chunk < end ? t0 + bi.chunk : end;
        const Chunk ch = chunk_of<ALN>(g, bi, t0, t1, span);
        stage_bias<-1>(g, bi, ch, pl.hd, 1.f, B, NT);
        __syncthreads();
        for (int tile = t0; tile < t1; ++tile) {
            const float *cur = S + (tile & 1) * I::STAGE;
            if (tile + 1 < ntiles) {
                mv.commit(g, bi, S + ((tile + 1) & 1) * I::STAGE, tile + 1, 1.f);
                mv.request(g, bi, pl.win, ks, vs, nullptr, tile + 2 < ntiles ? tile + 2 : ntiles - 1);
            }
            if (active) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const int key0 = tile * kTile + kb * 32;
                    if (!ALN && key0 >= g.N) break;
                    const Words16<ALN> wd = words_of<ALN>(bi, ch, (const int *)(cur + I::LT), tile, kb, hf);
                    f32x16 s = scores<DB>(cur + (kb * 32 + col) * I::STR + 4 * hf, Q, bias_block<ALN>(B + ch.c0 - mylin, wd), g.d);
                    if (!ALN) mask_rows(s, key0, g.N, hf);
                    if (MAX) {
                        float m = s[0];
#pragma unroll
                        for (int i = 1; i < 16; ++i) m = fmaxf(m, s[i]);
                        m = fmaxf(top, fmaxf(m, __shfl_xor(m, 32)));
                        // (a row of minus infinities so far: any finite stabiliser does)
                        const float ms = m == -INFINITY ? 0.f : m, alpha = __builtin_amdgcn_exp2f((top - ms) * kLog2e);
                        top = m;
                        sum *= alpha;
#pragma unroll
                        for (int i = 0; i < 16; ++i) s[i] -= ms;
#pragma unroll
                        for (int db = 0; db < DB; ++db)
#pragma unroll
                            for (int i = 0; i < 16; ++i) O[db][i] *= alpha;
                    }
                    float a = 0.f, b = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * kLog2e);
#pragma unroll
                    for (int i = 0; i < 8; ++i) a += s[2 * i], b += s[2 * i + 1];
                    sum += a + b;
                    contract<DB>(O, cur + I::YR + (kb * 32 + 4 * hf) * I::STR + col, s);
                }
            }
            __syncthreads();
        }
        if (t1 == end) end += strip_tiles;
    }
    sum += __shfl_xor(sum, 32);
}

template <int DB, bool ALN, int W>
__global__ __launch_bounds__(W * 64, W == 1 ? 1 : 2) void fwd_kernel(Geo g, Bias bi, int nblk, int force_max, const float *__restrict__ q,
                                                        const float *__restrict__ k, const float *__restrict__ v, float *__restrict__ out,
                                                        float *__restrict__ lse)
{
    constexpr int NT = 64 * W, SB = 32 * W;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *S = (float *)smem;
    int *map = (int *)(smem + stage_bytes<DB>());
    float *B = (float *)(map + 2 * g.M);
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(g, nblk, NT, map);
    __syncthreads();
    const int first = pl.blk * SB, last = first + SB < g.N ? first + SB - 1 : g.N - 1, n0 = first + wave * 32, n = n0 + col;
    const Span span = span_of<ALN>(g, bi, first, last);
    const int nc = n < g.N ? n : g.N - 1;
    const Cell cell = cell_of<ALN>(g, bi, nc);
    const bool active = n0 < g.N;
    Raw Q[4 * DB];
    operand<DB, false>(g, pl, rows_of_grid(g, pl, q, g.tstride), cell, g.scale_c, Q);
    const Rows ks = rows_of_grid(g, pl, k, g.tstride), vs = rows_of_grid(g, pl, v, g.tstride);
    f32x16 O[DB];
    float sum, top;
    // First without a running maximum; a denominator outside [2^-60, 2^60], and not for want of keys, sends the
    // workgroup on a second walk, with one.
    bool bad = true;
    if (!force_max) {
        fwd_walk<false, DB, ALN, W>(g, bi, pl, ks, vs, S, B, Q, O, sum, top, span, cell.lin(bi), active);
        bad = active && bad_rows(g, bi, pl.hd, n < g.N ? cell.index(g) : g.N, sum);
    }
    if (__syncthreads_or(bad)) fwd_walk<true, DB, ALN, W>(g, bi, pl, ks, vs, S, B, Q, O, sum, top, span, cell.lin(bi), active);
    if (n >= g.N) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;         // (a row without a key: zeros)
    if (lse != nullptr && hf == 0) lse[(int64_t)pl.u * g.N + cell.index(g)] = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum) * kLn2;
    store_row<DB>(out + (pl.img + pixel(pl.win, cell)) * g.C + pl.hd * g.d, O, g.d, hf, inv);
}

// dq and the bias's gradient; the second kernel's -LSE and -delta of every row.
template <int DB, bool CKPT, bool ALN, int W, bool HIST>
__global__ __launch_bounds__(W * 64, W == 1 ? 1 : 2) void dq_kernel(Geo g, Bias bi, int nblk, const float *__restrict__ q,
                                                       const float *__restrict__ k, const float *__restrict__ v,
                                                       const uint8_t *__restrict__ ckpt, const float *__restrict__ out,
                                                       const float *__restrict__ dout, const float *__restrict__ lse,
                                                       float *__restrict__ dq, float2 *__restrict__ ext, float *__restrict__ part)
{
    constexpr int NT = 64 * W, SB = 32 * W;
    using I = Img<DB>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *S = (float *)smem;
    int *map = (int *)(smem + stage_bytes<DB>());
    float *B = (float *)(map + 2 * g.M);
    double *H = (double *)(B + ((bi.rows * bi.ws + 1) & ~1));
    const int hsize = bi.hrows * bi.ws;
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(g, nblk, NT, map);
    if (HIST)
        for (int e = threadIdx.x; e < W * hsize; e += NT) H[e] = 0.;
    __syncthreads();
    const int first = pl.blk * SB, last = first + SB < g.N ? first + SB - 1 : g.N - 1, n0 = first + wave * 32, n = n0 + col;
    const Span span = span_of<ALN>(g, bi, first, last);
    const int nc = n < g.N ? n : g.N - 1;
    const Cell cell = cell_of<ALN>(g, bi, nc);
    const bool active = n0 < g.N;
    Raw Q[4 * DB], D[4 * DB];
    operand<DB, false>(g, pl, rows_of_grid(g, pl, dout, g.C), cell, 1.f, D);
    float delta = 0.f;
    {
        Raw O[4 * DB];
        operand<DB, false>(g, pl, rows_of_grid(g, pl, out, g.C), cell, 1.f, O);
#pragma unroll
        for (int i = 0; i < 4 * DB; ++i) delta += (O[i].x * D[i].x + O[i].y * D[i].y) + (O[i].z * D[i].z + O[i].w * D[i].w);
        delta += __shfl_xor(delta, 32);
    }
    operand<DB, CKPT>(g, pl, CKPT ? rows_of_ckpt(g, pl, ckpt, 0) : rows_of_grid(g, pl, q, g.tstride), cell, g.scale_c, Q);
    const float e0 = lse[(int64_t)pl.u * g.N + cell.index(g)], L = n >= g.N || e0 == -INFINITY ? bf::kNoRow : e0;
    if (n < g.N && hf == 0) ext[(int64_t)pl.u * g.N + n] = float2{-L, -delta};
    const int mylin = cell.lin(bi), wsy1 = span_of<ALN>(g, bi, n0 < g.N ? n0 : g.N - 1, n0 + 31 < g.N ? n0 + 31 : g.N - 1).y1;
    const Rows ks = CKPT ? rows_of_ckpt(g, pl, ckpt, 1) : rows_of_grid(g, pl, k, g.tstride);
    const Rows vs = CKPT ? rows_of_ckpt(g, pl, ckpt, 2) : rows_of_grid(g, pl, v, g.tstride);
    f32x16 A[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) A[db][i] = 0.f;
    const int ntiles = (g.N + kTile - 1) / kTile, strip_tiles = ALN ? bi.strip / kTile : ntiles;
    const f32x16 z = {0};
    Mover<DB, W, CKPT, CKPT, false, ALN> mv;
    mv.request(g, bi, pl.win, ks, vs, nullptr, 0);
    mv.commit(g, bi, S, 0, 1.f);
    mv.request(g, bi, pl.win, ks, vs, nullptr, ntiles > 1 ? 1 : 0);
    int before = -1;
    for (int t0 = 0, t1, end = strip_tiles; t0 < ntiles; t0 = t1) {
        t1 = t0 + bi.chunk < end ? t0 + bi.chunk : end;
        const Chunk ch = chunk_of<ALN>(g, bi, t0, t1, span);
        stage_bias<-1>(g, bi, ch, pl.hd, 1.f, B, NT);
        double *const mine = H + wave * hsize + ch.c0 - (span.y1 - wsy1) * bi.ws - mylin;
        __syncthreads();
        for (int tile = t0; tile < t1; ++tile) {
            const float *cur = S + (tile & 1) * I::STAGE;
            if (tile + 1 < ntiles) {
                mv.commit(g, bi, S + ((tile + 1) & 1) * I::STAGE, tile + 1, 1.f);
                mv.request(g, bi, pl.win, ks, vs, nullptr, tile + 2 < ntiles ? tile + 2 : ntiles - 1);
            }
            if (active) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    const int key0 = tile * kTile + kb * 32;
                    if (!ALN && key0 >= g.N) break;
                    const Words16<ALN> wd = words_of<ALN>(bi, ch, (const int *)(cur + I::LT), tile, kb, hf);
                    const float *row = cur + (kb * 32 + col) * I::STR + 4 * hf;
                    f32x16 s = scores<DB>(row, Q, bias_block<ALN>(B + ch.c0 - mylin, wd), g.d);
                    const f32x16 p = scores<DB>(row + I::YR, D, z, g.d);
                    if (!ALN) mask_rows(s, key0, g.N, hf);
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = prob((s[i] - L) * kLog2e) * (p[i] - delta);
                    if (HIST && (ALN || n < g.N)) {         // (many lanes at one word are slow)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            __hip_atomic_fetch_add(mine + wd(i), (double)s[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    }
                    contract<DB>(A, cur + (kb * 32 + 4 * hf) * I::STR + col, s);
                }
            }
            __syncthreads();
        }
        if (HIST) {
            flush<ALN, W, 32, 32>(g, bi, ch, H, hsize, first, before,
                              part + sums_at(g, bi, pl.u, nblk, pl.blk, bi.prows, ch.t.x0) + ch.t.y0 * bi.ws);
            before = t1 == end ? -1 : ch.t.y1;
        }
        if (t1 == end) end += strip_tiles;
    }
    if (n >= g.N) return;
    store_row<DB>(dq + (pl.img + pixel(pl.win, cell)) * g.C + pl.hd * g.d, A, g.d, hf, g.scale_c);
}

template <int DB, bool CKPT, bool ALN, int W>
__global__ __launch_bounds__(W * 64, W == 1 ? 1 : 2) void dkv_kernel(Geo g, Bias bi, int nblk, const float *__restrict__ q, const float *__restrict__ k,
                                                        const float *__restrict__ v, const uint8_t *__restrict__ ckpt,
                                                        const float *__restrict__ dout, const float2 *__restrict__ ext,
                                                        float *__restrict__ dk, float *__restrict__ dv)
{
    constexpr int NT = 64 * W, SB = 32 * W;
    using I = Img<DB>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float *S = (float *)smem;
    int *map = (int *)(smem + stage_bytes<DB>());
    float *B = (float *)(map + 2 * g.M);
    const int lane = threadIdx.x & 63, col = lane & 31, hf = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Place pl = place_of(g, nblk, NT, map);
    __syncthreads();
    const int first = pl.blk * SB, last = first + SB < g.N ? first + SB - 1 : g.N - 1, n0 = first + wave * 32, n = n0 + col;
    const Span span = span_of<ALN>(g, bi, first, last);
    const int nc = n < g.N ? n : g.N - 1;
    const Cell cell = cell_of<ALN>(g, bi, nc);
    const bool active = n0 < g.N;
    Raw Kb[4 * DB], Vb[4 * DB];
    operand<DB, CKPT>(g, pl, CKPT ? rows_of_ckpt(g, pl, ckpt, 1) : rows_of_grid(g, pl, k, g.tstride), cell, 1.f, Kb);
    operand<DB, CKPT>(g, pl, CKPT ? rows_of_ckpt(g, pl, ckpt, 2) : rows_of_grid(g, pl, v, g.tstride), cell, 1.f, Vb);
    const int mylin = cell.lin(bi);
    const Rows qs = CKPT ? rows_of_ckpt(g, pl, ckpt, 0) : rows_of_grid(g, pl, q, g.tstride), ds = rows_of_grid(g, pl, dout, g.C);
    const float2 *const ex = ext + (int64_t)pl.u * g.N;
    f32x16 Ak[DB], Av[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) Ak[db][i] = 0.f, Av[db][i] = 0.f;
    const int ntiles = (g.N + kTile - 1) / kTile, strip_tiles = ALN ? bi.strip / kTile : ntiles;
    const float scale = g.scale_c;
    const f32x16 z = {0};
    Mover<DB, W, CKPT, false, true, ALN> mv;
    mv.request(g, bi, pl.win, qs, ds, ex, 0);
    mv.commit(g, bi, S, 0, scale);
    mv.request(g, bi, pl.win, qs, ds, ex, ntiles > 1 ? 1 : 0);
    for (int t0 = 0, t1, end = strip_tiles; t0 < ntiles; t0 = t1) {
        t1 = t0 + bi.chunk < end ? t0 + bi.chunk : end;
        const Chunk ch = chunk_of<ALN>(g, bi, t0, t1, span);
        stage_bias<1>(g, bi, ch, pl.hd, 1.f, B, NT);
        __syncthreads();
        for (int tile = t0; tile < t1; ++tile) {
            const float *cur = S + (tile & 1) * I::STAGE;
            if (tile + 1 < ntiles) {
                mv.commit(g, bi, S + ((tile + 1) & 1) * I::STAGE, tile + 1, scale);
                mv.request(g, bi, pl.win, qs, ds, ex, tile + 2 < ntiles ? tile + 2 : ntiles - 1);
            }
            if (active) {
#pragma unroll
                for (int qb = 0; qb < 2; ++qb) {
                    if (!ALN && tile * kTile + qb * 32 >= g.N) break;
                    const Words16<ALN> wd = words_of<ALN>(bi, ch, (const int *)(cur + I::LT), tile, qb, hf);
                    const float *row = cur + (qb * 32 + col) * I::STR + 4 * hf;
                    f32x16 s = scores<DB>(row, Kb, bias_block<ALN>(B + ch.c0 - mylin, wd), g.d), p = scores<DB>(row + I::YR, Vb, z, g.d);
                    // (LSE and delta only then: sums that start from them would round at their size)
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const float4 l = *(const float4 *)(cur + I::EX + qb * 32 + 8 * a + 4 * hf), dl = *(const float4 *)(cur + I::EX + kTile + qb * 32 + 8 * a + 4 * hf);
                        const float lr[4] = {l.x, l.y, l.z, l.w}, dr[4] = {dl.x, dl.y, dl.z, dl.w};
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[4 * a + r] = prob((s[4 * a + r] + lr[r]) * kLog2e);
                            p[4 * a + r] = (p[4 * a + r] + dr[r]) * s[4 * a + r];
                        }
                    }
                    contract<DB>(Av, cur + I::YR + (qb * 32 + 4 * hf) * I::STR + col, s);
                    contract<DB>(Ak, cur + (qb * 32 + 4 * hf) * I::STR + col, p);
                }
            }
            __syncthreads();
        }
        if (t1 == end) end += strip_tiles;
    }
    if (n >= g.N) return;
    const int64_t at = (pl.img + pixel(pl.win, cell)) * g.C + pl.hd * g.d;
    store_row<DB>(dk + at, Ak, g.d, hf, 1.f);           // (Q carries the scale)
    store_row<DB>(dv + at, Av, g.d, hf, 1.f);
}

constexpr size_t kBiasBytes = 36 * 1024, kHistBytes = 9 * 1024;

template <int DB, bool ALN, int W>
hipError_t launch_fwd_one(const Geo &g, const FwdArgs &a)
{
    Bias bi{a.bias};
    plan_chunks(g, RIB_F32, &bi, ALN, 32 * W, false, kBiasBytes, 0);
    const int nblk = (g.N + 32 * W - 1) / (32 * W);
    const size_t smem = stage_bytes<DB>() + 8 * (size_t)g.M + (size_t)bi.rows * bi.ws * 4;
    if (smem > (size_t)kMaxDynLds) return hipErrorInvalidValue;
    auto kern = fwd_kernel<DB, ALN, W>;
    const hipError_t e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.units * nblk)), dim3(64 * W), smem, a.st, g, bi, nblk, a.force_max, (const float *)a.q,
                       (const float *)a.k, (const float *)a.v, (float *)a.out, a.lse);
    return hipGetLastError();
}
template <int DB>
hipError_t launch_fwd_width(const Geo &g, const FwdArgs &a)
{
    if (g.N <= 32) return launch_fwd_one<DB, false, 1>(g, a);
    return strip_shift(RIB_F32, g.M) >= 0 ? launch_fwd_one<DB, true, 4>(g, a) : launch_fwd_one<DB, false, 4>(g, a);
}

template <int DB, bool CKPT, bool ALN, int W, bool HIST>
hipError_t launch_dq_one(const Geo &g, const BwdArgs &a, const Ws &ws)
{
    Bias bi{a.bias};
    plan_chunks(g, RIB_F32, &bi, ALN, 32 * W, HIST, kBiasBytes, kHistBytes);
    const size_t smem = stage_bytes<DB>() + 8 * (size_t)g.M + ((size_t)bi.rows * bi.ws + 1) / 2 * 8 + (size_t)W * bi.hrows * bi.ws * 8;
    if (smem > (size_t)kMaxDynLds) return hipErrorInvalidValue;
    auto kern = dq_kernel<DB, CKPT, ALN, W, HIST>;
    const hipError_t e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.units * ws.nblk)), dim3(64 * W), smem, a.st, g, bi, ws.nblk, (const float *)a.q,
                       (const float *)a.k, (const float *)a.v, a.ckpt, (const float *)a.out, (const float *)a.dout, a.lse, (float *)a.dq,
                       (float2 *)((char *)a.ws + ws.ext), (float *)((char *)a.ws + ws.part));
    return hipGetLastError();
}
template <int DB, bool CKPT, bool ALN, int W>
hipError_t launch_pair(const Geo &g, const BwdArgs &a, Ws &ws)
{
    ws.strips = ALN;
    hipError_t e = a.dbias != nullptr ? launch_dq_one<DB, CKPT, ALN, W, true>(g, a, ws) : launch_dq_one<DB, CKPT, ALN, W, false>(g, a, ws);
    if (e != hipSuccess) return e;
    Bias bi{a.bias};
    plan_chunks(g, RIB_F32, &bi, ALN, 32 * W, false, kBiasBytes, 0);
    const size_t smem = stage_bytes<DB>() + 8 * (size_t)g.M + (size_t)bi.rows * bi.ws * 4;
    if (smem > (size_t)kMaxDynLds) return hipErrorInvalidValue;
    auto kern = dkv_kernel<DB, CKPT, ALN, W>;
    e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.units * ws.nblk)), dim3(64 * W), smem, a.st, g, bi, ws.nblk, (const float *)a.q,
                       (const float *)a.k, (const float *)a.v, a.ckpt, (const float *)a.dout, (const float2 *)((const char *)a.ws + ws.ext),
                       (float *)a.dk, (float *)a.dv);
    return hipGetLastError();
}
template <int DB, bool CKPT>
hipError_t launch_bwd_src(const Geo &g, const BwdArgs &a, Ws &ws)
{
    if (g.N <= 32) return launch_pair<DB, CKPT, false, 1>(g, a, ws);
    return strip_shift(RIB_F32, g.M) >= 0 ? launch_pair<DB, CKPT, true, 4>(g, a, ws) : launch_pair<DB, CKPT, false, 4>(g, a, ws);
}
template <int DB>
hipError_t launch_bwd_width(const Geo &g, const BwdArgs &a, Ws &ws)
{
    return a.ckpt != nullptr ? launch_bwd_src<DB, true>(g, a, ws) : launch_bwd_src<DB, false>(g, a, ws);
}

}  // namespace fp

hipError_t launch_fwd_f32(const Geo &g, const FwdArgs &a)
{
    return g.d <= 32 ? fp::launch_fwd_width<1>(g, a) : fp::launch_fwd_width<2>(g, a);
}

hipError_t launch_bwd_f32(const Geo &g, const BwdArgs &a)
{
    Ws ws = ws_layout(g, RIB_F32);
    const hipError_t e = g.d <= 32 ? fp::launch_bwd_width<1>(g, a, ws) : fp::launch_bwd_width<2>(g, a, ws);
    if (e != hipSuccess || a.dbias == nullptr) return e;
    return launch_reduce(g, RIB_F32, ws, (const float *)((const char *)a.ws + ws.part), a.dbias, a.st);
}

}  // namespace rpb
}  // namespace rib
