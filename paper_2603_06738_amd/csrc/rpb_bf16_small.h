// Window attention with a learned relative position bias, bf16, windows of up to 64 tokens (a side of 8 and less): a wave takes a whole
// (window, head) unit, and several windows of its head in turn.
//
// At this size a unit is two blocks of 32 by two, and what counts is how often its rows are fetched and how many units are in
// flight.  So the backward is one kernel: Q, K, V and dO are fetched once, and lie in LDS two at a time, K and V for dq, Q and dO for dk
// and dv, whose other sides wait in registers; scores and exponentials are made in both layouts, which is cheaper than turning them in LDS.  Nothing
// is shared between waves, so nothing waits for another; bias and histogram stay in LDS over the wave's windows.
// Forward + backward of 32 images of 56 x 56, 7 x 7 windows, 3 heads of 32, us, as two tiled kernels and a forward in single-wave
// workgroups / here: kernels 180 / 102 (both with the bias's gradient).  P as two bf16 parts would bring O to its own rounding (2-norm error 2.2e-3 to 1.7e-3) for a
// forward of 37 us instead of 31.
#pragma once

#include "rpb_bf16.h"

namespace rib {
namespace rpb {
namespace bf {

// The windows of one head that a wave works on.
struct Share {
    int hd, w0, w1, part;       // head, windows [w0, w1), which of the head's shares
};
__device__ __forceinline__ Share share_of(const Geo &g, int windows, int per)
{
    int64_t u;
    int b;
    block_coords(1, u, b);      // neighbours on one XCD: the heads of a window share its lines
    Share s;
    s.hd = (int)u % g.heads, s.part = (int)u / g.heads;
    s.w0 = s.part * per, s.w1 = s.w0 + per < windows ? s.w0 + per : windows;
    return s;
}
// A window's place in the grid, and its tokens' pixels.
struct Spot {
    int y0, x0;
    int64_t img;
    __device__ __forceinline__ uint32_t pixel(const Geo &g, int n) const
    {
        const int iy = row_of(n, g.inv_m);
        int y = y0 + iy, x = x0 + n - iy * g.M;
        if (y >= g.H) y -= g.H;
        if (x >= g.W) x -= g.W;
        return (uint32_t)(y * g.W + x);
    }
};
__device__ __forceinline__ Spot spot_of(const Geo &g, int w)
{
    Spot s;
    const int wx = w % g.nwx, t = w / g.nwx;
    s.y0 = (t % g.nwy) * g.M + g.s, s.x0 = wx * g.M + g.s, s.img = (int64_t)(t / g.nwy) * g.H * g.W;
    return s;
}
__device__ __forceinline__ Rows rows_at(const Geo &g, const Spot &s, int hd, const void *x, int64_t stride)
{
    return Rows{(const char *)x + (s.img * stride + hd * g.d) * 2, stride * 2, nullptr};
}

// A window's rows of a tensor, by their pixels `t`.
template <int LP, int SRC>
__device__ __forceinline__ void hold(Held<LP> &h, const Geo &g, const Rows &s, const uint32_t (&t)[LP])
{
    const int l = threadIdx.x / LP, j = threadIdx.x % LP;
#pragma unroll
    for (int p = 0; p < LP; ++p) {
        const int n = p * (64 / LP) + l;
        if (n < g.N) h.r[p] = get_piece<SRC>(s, t[p], n, j, g.d);
    }
}
// (Rows past the window are zero.)
template <int LP, int SRC, int K>
__device__ __forceinline__ void lay(const Held<LP> &h, const Geo &g, bf16_t *image, float scale)
{
    const int l = threadIdx.x / LP, j = threadIdx.x % LP;
#pragma unroll
    for (int p = 0; p < LP; ++p) {
        const int n = p * (64 / LP) + l;
        if (n >= g.N) continue;
        Raw a = widen_piece<SRC>(h.r[p]);
        if (scale != 1.f) a = scaled(a, scale);
        put_piece<SRC>(image + n * (K + 8), a, j, g.d);
    }
}
// Everything of an image that lay() does not write: padding columns, rows past the window.
template <int K>
__device__ __forceinline__ void clear_image(const Geo &g, bf16_t *image)
{
    const int n = threadIdx.x;
    for (int c = n < g.N ? g.d : 0; c < K; ++c) image[n * (K + 8) + c] = 0;
}

template <int KX, int DB, bool SUM, bool LSE, int SRC>
__global__ __launch_bounds__(64, DB == 1 ? 3 : 2) void fwd_small_kernel(Geo g, Bias bi, int windows, int per, int force_max, const bf16_t *__restrict__ q,
                                                          const bf16_t *__restrict__ k, const bf16_t *__restrict__ v, bf16_t *__restrict__ out,
                                                          float *__restrict__ lse)
{
    constexpr int LP = KX <= 32 ? 4 : 8, KY = 32 * DB;
    using I = Img<KX, KY>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *X = (bf16_t *)smem, *Y = X + I::YR;
    int *table = (int *)(X + I::LT);
    float *B = (float *)(smem + I::STAGE * 2 + 64);
    const int lane = threadIdx.x, col = lane & 31, hf = lane >> 5, nb = (g.N + 31) / 32;
    const Share sh = share_of(g, windows, per);
    const Chunk ch = chunk_of<false>(g, bi, 0, 1, Span{0, g.M - 1, 0});
    stage_bias<-1>(g, bi, ch, sh.hd, bi.bs, B, 64);
    clear_image<KX>(g, X);
    clear_image<KY>(g, Y);
    if (!SUM) Y[lane * I::YS + KY - 1] = 0x3f80;
    table[lane] = lin(g, lane < g.N ? lane : g.N - 1);
    __syncthreads();
    int mylin[2];
#pragma unroll
    for (int qb = 0; qb < 2; ++qb) mylin[qb] = lin(g, qb * 32 + col < g.N ? qb * 32 + col : g.N - 1);
    const int tro = tr_lane_offset<I::YS>(lane), ako = col * I::XS + 8 * hf;

    Held<LP> hq, hk, hv;
    auto request = [&](int w) {
        const Spot s = spot_of(g, w);
        uint32_t t[LP];
#pragma unroll
        for (int p = 0; p < LP; ++p) {
            const int n = p * (64 / LP) + lane / LP;
            t[p] = s.pixel(g, n < g.N ? n : g.N - 1);
        }
        hold<LP, SRC>(hq, g, rows_at(g, s, sh.hd, q, g.tstride), t);
        hold<LP, SRC>(hk, g, rows_at(g, s, sh.hd, k, g.tstride), t);
        hold<LP, SRC>(hv, g, rows_at(g, s, sh.hd, v, g.tstride), t);
    };
    request(sh.w0);
    for (int w = sh.w0; w < sh.w1; ++w) {
        bf16x8 Q[2][KX / 16];
        lay<LP, SRC, KX>(hq, g, X, bi.qs);
#pragma unroll
        for (int b = 0; b < 2; ++b) read_rows<KX / 16>(Q[b], X + b * 32 * I::XS + ako);
        lay<LP, SRC, KX>(hk, g, X, 1.f);
        lay<LP, SRC, KY>(hv, g, Y, 1.f);
        if (w + 1 < sh.w1) request(w + 1);
        f32x16 O[2][DB];
        Sums sum[2];
        float top[2] = {0.f, 0.f};
        // all keys of a block of queries at once: scores first, so that their maximum is at hand where it is wanted
        auto walk = [&](bool max) {
#pragma unroll
            for (int qb = 0; qb < 2; ++qb) {
                if (qb >= nb) break;
                f32x16 s[2];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    if (kb >= nb) break;
                    bf16x8 A[KX / 16];
                    read_rows<KX / 16>(A, X + kb * 32 * I::XS + ako);
                    s[kb] = bias_block<false>(B + ch.c0 - mylin[qb], words_of<false>(bi, ch, table, 0, kb, hf));
#pragma unroll
                    for (int i = 0; i < KX / 16; ++i) s[kb] = mfma(A[i], Q[qb][i], s[kb]);
                    if (kb == nb - 1) mask_rows(s[kb], kb * 32, g.N, hf);
                }
                top[qb] = 0.f;
                if (max) {
                    float m = s[0][0];
#pragma unroll
                    for (int i = 1; i < 16; ++i) m = fmaxf(m, s[0][i]);
                    if (nb > 1)
#pragma unroll
                        for (int i = 0; i < 16; ++i) m = fmaxf(m, s[1][i]);
                    m = fmaxf(m, __shfl_xor(m, 32));
                    top[qb] = m == -INFINITY ? 0.f : m;         // (a row without a key: any finite stabiliser does)
                }
                sum[qb] = Sums{0.f, 0.f};
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) O[qb][db][i] = 0.f;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
                    if (kb >= nb) break;
                    uint32_t P[8];
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[kb][i] = __builtin_amdgcn_exp2f((s[kb][i] - top[qb]) * bi.c);
#pragma unroll
                    for (int i = 0; i < 8; ++i) P[i] = pack_bf16(s[kb][2 * i], s[kb][2 * i + 1]);
                    if (LSE) {
                        float a = 0.f, b = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) a += s[kb][2 * i], b += s[kb][2 * i + 1];
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
                        O[qb][db] = mfma(read_tr<I::YS>(Y + kb * 32 * I::YS, tro, 32 * db), as_bf16x8(P[0], P[1], P[2], P[3]), O[qb][db]);
                        O[qb][db] = mfma(read_tr<I::YS>(Y + (kb * 32 + 16) * I::YS, tro, 32 * db), as_bf16x8(P[4], P[5], P[6], P[7]), O[qb][db]);
                    }
                }
                if (LSE) sum[qb].exact += __shfl_xor(sum[qb].exact, 32);
                const float mine = SUM ? sum[qb].rounded : O[qb][DB - 1][15], other = __shfl_xor(mine, 32);
                sum[qb].rounded = SUM ? mine + other : hf ? mine : other;
            }
        };
        bool bad = force_max != 0;
        if (!bad) {
            walk(false);
#pragma unroll
            for (int qb = 0; qb < 2; ++qb)
                if (qb < nb && bad_rows(g, bi, sh.hd, qb * 32 + col, qb * 32 + col < g.N ? sum[qb].rounded : 1.f)) bad = true;
        }
        if (bad) walk(true);
        const Spot s = spot_of(g, w);
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            const int n = qb * 32 + col;
            if (n >= g.N) continue;
            const bool none = sum[qb].rounded == 0.f;
            const float inv = none ? 0.f : 1.f / sum[qb].rounded;
            if (LSE && hf == 0)
                lse[((int64_t)w * g.heads + sh.hd) * g.N + n] = none ? -INFINITY : (top[qb] * bi.c + __builtin_amdgcn_logf(sum[qb].exact)) * kLn2;
            bf16_t *row = out + (s.img + s.pixel(g, n)) * g.C + sh.hd * g.d;
#pragma unroll
            for (int db = 0; db < DB; ++db) store_row<SRC>(row, O[qb][db], db, g.d, hf, inv);
        }
    }
}

// (Two blocks of channels: one wave a SIMD, whose 512 registers hold them.  8 x 8 windows, 4 heads of 64, 8 images of 96 x 96: 242 us with two waves, 150 so.)
template <int K, int DB, int SRC, int SG, bool HIST>
__global__ __launch_bounds__(64, DB == 1 ? 2 : 1) void bwd_small_kernel(Geo g, Bias bi, int windows, int per, const bf16_t *__restrict__ q, const bf16_t *__restrict__ k,
                                                          const bf16_t *__restrict__ v, const uint8_t *__restrict__ ckpt, const bf16_t *__restrict__ out,
                                                          const bf16_t *__restrict__ dout, const float *__restrict__ lse, bf16_t *__restrict__ dq,
                                                          bf16_t *__restrict__ dk, bf16_t *__restrict__ dv, float *__restrict__ part)
{
    constexpr int LP = DB == 1 ? 4 : 8, XS = K + 8, IM = 64 * XS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    bf16_t *X = (bf16_t *)smem, *Y = X + IM;                    // q and dO, or k and v
    int *table = (int *)(Y + IM + 32);                          // (transposed reads of the last row may run over its end)
    float *E = (float *)(table + 64);                           // -LSE in base 2, then -delta
    double *H = (double *)(E + 128);
    const int count = bi.w2 * bi.w2;
    float *B = (float *)(H + (HIST ? count : 0));
    const int lane = threadIdx.x, col = lane & 31, hf = lane >> 5, nb = (g.N + 31) / 32;
    const int l = lane / LP, j = lane % LP;
    const Share sh = share_of(g, windows, per);
    const Chunk ch = chunk_of<false>(g, bi, 0, 1, Span{0, g.M - 1, 0});
    stage_bias<-1>(g, bi, ch, sh.hd, bi.bs, B, 64);
    if (HIST)
        for (int e = lane; e < count; e += 64) H[e] = 0.;
    clear_image<K>(g, X);
    clear_image<K>(g, Y);
    table[lane] = lin(g, lane < g.N ? lane : g.N - 1);
    __syncthreads();
    int mylin[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) mylin[b] = lin(g, b * 32 + col < g.N ? b * 32 + col : g.N - 1);
    const int tro = tr_lane_offset<XS>(lane), ako = col * XS + 8 * hf;
    const f32x16 z = {0};
    for (int w = sh.w0; w < sh.w1; ++w) {
        const Spot sp = spot_of(g, w);
        const int64_t u = (int64_t)w * g.heads + sh.hd;
        Held<LP> hq, hd;
        bf16x8 Qb[2][K / 16], Db[2][K / 16];
        // the images of q and dO; rows past the window are zero, and have no probabilities
        auto queries = [&]() {
            lay<LP, SRC, K>(hq, g, X, bi.qs);
            lay<LP, SG, K>(hd, g, Y, 1.f);
        };
        {
            uint32_t t[LP];
#pragma unroll
            for (int p = 0; p < LP; ++p) {
                const int n = p * (64 / LP) + l;
                t[p] = sp.pixel(g, n < g.N ? n : g.N - 1);
            }
            Held<LP> hk, hv, ho;
            float e[LP];
            if constexpr (SRC == kCkpt) {
                const int dp = ckpt_row(g.d);
                const int64_t rows = ckpt_rows(g), first = u * g.N;
                const uint8_t *ex = ckpt + 3 * rows * dp + first;
                hold<LP, SRC>(hq, g, Rows{(const char *)ckpt + first * dp, dp, ex}, t);
                hold<LP, SRC>(hk, g, Rows{(const char *)ckpt + (first + rows) * dp, dp, ex + rows}, t);
                hold<LP, SRC>(hv, g, Rows{(const char *)ckpt + (first + 2 * rows) * dp, dp, ex + 2 * rows}, t);
            } else {
                hold<LP, SRC>(hq, g, rows_at(g, sp, sh.hd, q, g.tstride), t);
                hold<LP, SRC>(hk, g, rows_at(g, sp, sh.hd, k, g.tstride), t);
                hold<LP, SRC>(hv, g, rows_at(g, sp, sh.hd, v, g.tstride), t);
            }
            hold<LP, SG>(hd, g, rows_at(g, sp, sh.hd, dout, g.C), t);
            hold<LP, SG>(ho, g, rows_at(g, sp, sh.hd, out, g.C), t);
#pragma unroll
            for (int p = 0; p < LP; ++p) {
                const int n = p * (64 / LP) + l;
                e[p] = lse[u * g.N + (n < g.N ? n : g.N - 1)];
            }
            const int c = piece_col<SG>(j, g.d);
#pragma unroll
            for (int p = 0; p < LP; ++p) {
                const int n = p * (64 / LP) + l;
                float delta = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {       // (a piece that slid back holds a neighbour's values first)
                    const uint32_t a = ho.r[p].w[i >> 1], b = hd.r[p].w[i >> 1];
                    const float x = i & 1 ? hi_bf16(a) * hi_bf16(b) : lo_bf16(a) * lo_bf16(b);
                    delta += SG == kAny || c + i >= 8 * j ? x : 0.f;
                }
#pragma unroll
                for (int m = 1; m < LP; m <<= 1) delta += __shfl_xor(delta, m);
                if (j == 0) E[n] = n >= g.N || e[p] == -INFINITY ? -kNoRow : -e[p] * kLog2e, E[64 + n] = n >= g.N ? 0.f : -delta;
            }
            queries();
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                read_rows<K / 16>(Qb[b], X + b * 32 * XS + ako);
                read_rows<K / 16>(Db[b], Y + b * 32 * XS + ako);
            }
            lay<LP, SRC, K>(hk, g, X, 1.f);
            lay<LP, SRC, K>(hv, g, Y, 1.f);
        }
        // dq and the offsets' sums: a lane owns a query
#pragma unroll
        for (int qb = 0; qb < 2; ++qb) {
            if (qb >= nb) break;
            f32x16 A[DB];
            const float mylse = E[qb * 32 + col], mydelta = E[64 + qb * 32 + col];
#pragma unroll
            for (int db = 0; db < DB; ++db) A[db] = z;
            for (int kb = 0; kb < nb; ++kb) {
                const Words16<false> at = words_of<false>(bi, ch, table, 0, kb, hf);
                bf16x8 Ak[K / 16], Av[K / 16];
                read_rows<K / 16>(Ak, X + kb * 32 * XS + ako);
                read_rows<K / 16>(Av, Y + kb * 32 * XS + ako);
                f32x16 s = bias_block<false>(B + ch.c0 - mylin[qb], at), p = z;
#pragma unroll
                for (int i = 0; i < K / 16; ++i) s = mfma(Ak[i], Qb[qb][i], s);
#pragma unroll
                for (int i = 0; i < K / 16; ++i) p = mfma(Av[i], Db[qb][i], p);
                if (kb == nb - 1) mask_rows(s, kb * 32, g.N, hf);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = prob(fmaf(s[i], bi.c, mylse)) * (p[i] + mydelta);
                if (HIST && qb * 32 + col < g.N) add_offsets<false>(H + ch.c0 - mylin[qb], at, s);      // (many lanes at one word are slow)
                uint32_t P[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) P[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    A[db] = mfma(read_tr<XS>(X + kb * 32 * XS, tro, 32 * db), as_bf16x8(P[0], P[1], P[2], P[3]), A[db]);
                    A[db] = mfma(read_tr<XS>(X + (kb * 32 + 16) * XS, tro, 32 * db), as_bf16x8(P[4], P[5], P[6], P[7]), A[db]);
                }
            }
            const int n = qb * 32 + col;
            if (n < g.N) {
                bf16_t *row = dq + (sp.img + sp.pixel(g, n)) * g.C + sh.hd * g.d;
#pragma unroll
                for (int db = 0; db < DB; ++db) store_row<SG>(row, A[db], db, g.d, hf, g.scale_c);
            }
        }
        // dk, dv: a lane owns a key; the bias of (query, key) lies where dq finds it, the other way round
        bf16x8 Kb[2][K / 16], Vb[2][K / 16];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            read_rows<K / 16>(Kb[b], X + b * 32 * XS + ako);
            read_rows<K / 16>(Vb[b], Y + b * 32 * XS + ako);
        }
        queries();
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if (kb >= nb) break;
            f32x16 Ak[DB], Av[DB];
#pragma unroll
            for (int db = 0; db < DB; ++db) Ak[db] = z, Av[db] = z;
            for (int qb = 0; qb < nb; ++qb) {
                const Words16<false> at = words_of<false>(bi, ch, table, 0, qb, hf);
                bf16x8 Aq[K / 16], Ad[K / 16];
                read_rows<K / 16>(Aq, X + qb * 32 * XS + ako);
                read_rows<K / 16>(Ad, Y + qb * 32 * XS + ako);
                f32x16 s, p;
                float4 e[4];
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float4 x = *(const float4 *)(E + 64 + qb * 32 + 8 * a + 4 * hf);
                    e[a] = *(const float4 *)(E + qb * 32 + 8 * a + 4 * hf);
                    p[4 * a] = x.x, p[4 * a + 1] = x.y, p[4 * a + 2] = x.z, p[4 * a + 3] = x.w;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = B[ch.c0 + mylin[kb] - at(i)];
#pragma unroll
                for (int i = 0; i < K / 16; ++i) s = mfma(Aq[i], Kb[kb][i], s);
#pragma unroll
                for (int i = 0; i < K / 16; ++i) p = mfma(Ad[i], Vb[kb][i], p);
                uint32_t P[8], G[8];
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = prob(fmaf(s[i], bi.c, ((const float *)&e[i >> 2])[i & 3]));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    P[i] = pack_bf16(s[2 * i], s[2 * i + 1]);
                    G[i] = pack_bf16(s[2 * i] * p[2 * i], s[2 * i + 1] * p[2 * i + 1]);
                }
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const bf16_t *x = Y + qb * 32 * XS, *y = X + qb * 32 * XS;
                    Av[db] = mfma(read_tr<XS>(x, tro, 32 * db), as_bf16x8(P[0], P[1], P[2], P[3]), Av[db]);
                    Av[db] = mfma(read_tr<XS>(x + 16 * XS, tro, 32 * db), as_bf16x8(P[4], P[5], P[6], P[7]), Av[db]);
                    Ak[db] = mfma(read_tr<XS>(y, tro, 32 * db), as_bf16x8(G[0], G[1], G[2], G[3]), Ak[db]);
                    Ak[db] = mfma(read_tr<XS>(y + 16 * XS, tro, 32 * db), as_bf16x8(G[4], G[5], G[6], G[7]), Ak[db]);
                }
            }
            const int n = kb * 32 + col;
            if (n < g.N) {
                const int64_t at = (sp.img + sp.pixel(g, n)) * g.C + sh.hd * g.d;
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    store_row<SG>(dk + at, Ak[db], db, g.d, hf, bi.ks);
                    store_row<SG>(dv + at, Av[db], db, g.d, hf, 1.f);
                }
            }
        }
    }
    if (HIST) {
        __syncthreads();
        float *dst = part + ((int64_t)sh.part * g.heads + sh.hd) * count;
        for (int e = lane; e < count; e += 64) dst[e] = (float)H[e];
    }
}

// Windows a wave: as many as leave every compute unit 12 waves.
inline hipError_t share_windows(const Geo &g, int *windows, int *per, int *parts)
{
    int cus = 0;
    const hipError_t e = compute_units(&cus);
    if (e != hipSuccess) return e;
    *windows = (int)(g.units / g.heads);
    const int64_t waves = (int64_t)cus * 12;
    *per = (int)((g.units + waves - 1) / waves);
    *parts = (*windows + *per - 1) / *per;
    return hipSuccess;
}
template <int KX, int DB, bool SUM, bool LSE, int SRC>
hipError_t launch_fwd_small_lse(const Geo &g, const FwdArgs &a)
{
    Bias bi{a.bias};
    plan_scale(g, &bi);
    plan_order(g, RIB_BF16, &bi, false);
    int windows, per, parts;
    hipError_t e = share_windows(g, &windows, &per, &parts);
    if (e != hipSuccess) return e;
    const size_t smem = (size_t)Img<KX, 32 * DB>::STAGE * 2 + 64 + (size_t)bi.w2 * bi.w2 * 4;
    auto kern = fwd_small_kernel<KX, DB, SUM, LSE, SRC>;
    e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(parts * g.heads)), dim3(64), smem, a.st, g, bi, windows, per, a.force_max, (const bf16_t *)a.q,
                       (const bf16_t *)a.k, (const bf16_t *)a.v, (bf16_t *)a.out, a.lse);
    return hipGetLastError();
}
template <int KX, int DB, bool SUM, int SRC>
hipError_t launch_fwd_small(const Geo &g, const FwdArgs &a)
{
    return a.lse != nullptr ? launch_fwd_small_lse<KX, DB, SUM, true, SRC>(g, a) : launch_fwd_small_lse<KX, DB, SUM, false, SRC>(g, a);
}
template <int K, int DB, int SRC, int SG, bool HIST>
hipError_t launch_bwd_small_one(const Geo &g, const BwdArgs &a, Ws &ws)
{
    Bias bi{a.bias};
    plan_scale(g, &bi);
    plan_order(g, RIB_BF16, &bi, false);
    int windows, per, parts;
    hipError_t e = share_windows(g, &windows, &per, &parts);
    if (e != hipSuccess) return e;
    ws.shares = parts;
    const size_t smem = ((size_t)2 * 64 * (K + 8) + 32) * 2 + 768 + (size_t)bi.w2 * bi.w2 * (HIST ? 12 : 4);
    auto kern = bwd_small_kernel<K, DB, SRC, SG, HIST>;
    e = prepare_kernel((const void *)kern, nullptr);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)(parts * g.heads)), dim3(64), smem, a.st, g, bi, windows, per, (const bf16_t *)a.q,
                       (const bf16_t *)a.k, (const bf16_t *)a.v, a.ckpt, (const bf16_t *)a.out, (const bf16_t *)a.dout, a.lse,
                       (bf16_t *)a.dq, (bf16_t *)a.dk, (bf16_t *)a.dv, (float *)((char *)a.ws + ws.part));
    return hipGetLastError();
}
template <int K, int DB, int SRC, int SG>
hipError_t launch_bwd_small(const Geo &g, const BwdArgs &a, Ws &ws)
{
    return a.dbias != nullptr ? launch_bwd_small_one<K, DB, SRC, SG, true>(g, a, ws) : launch_bwd_small_one<K, DB, SRC, SG, false>(g, a, ws);
}

// ---- which kernels ------------------------------------------------------------------------------------------------

template <int KX, int DB, bool SUM, int SRC>
hipError_t launch_fwd_src(const Geo &g, const FwdArgs &a)
{
    if (g.N <= 64) return launch_fwd_small<KX, DB, SUM, SRC>(g, a);
    const int waves = group_waves(RIB_BF16, g.N);
    const bool split = splits(g, RIB_BF16);
    if constexpr (SRC == kFast) {
        if (strip_shift(RIB_BF16, g.M) >= 0)
            return split        ? launch_fwd_one<KX, DB, SUM, SRC, true, true, 4>(g, a)
                   : waves == 3 ? launch_fwd_one<KX, DB, SUM, SRC, true, false, 3>(g, a)
                                : launch_fwd_one<KX, DB, SUM, SRC, true, false, 4>(g, a);
    }
    return split        ? launch_fwd_one<KX, DB, SUM, SRC, false, true, 4>(g, a)
           : waves == 2 ? launch_fwd_one<KX, DB, SUM, SRC, false, false, 2>(g, a)
           : waves == 3 ? launch_fwd_one<KX, DB, SUM, SRC, false, false, 3>(g, a)
                        : launch_fwd_one<KX, DB, SUM, SRC, false, false, 4>(g, a);
}

template <int K, int DB, int SRC, int SG>
hipError_t launch_bwd_src(const Geo &g, const BwdArgs &a, Ws &ws)
{
    if (g.N <= 64) return launch_bwd_small<K, DB, SRC, SG>(g, a, ws);
    const int waves = group_waves(RIB_BF16, g.N);
    const bool split = splits(g, RIB_BF16);
    if constexpr (SG == kFast) {
        if (strip_shift(RIB_BF16, g.M) >= 0)
            return split        ? launch_pair<K, DB, SRC, SG, true, true, 4>(g, a, ws)
                   : waves == 3 ? launch_pair<K, DB, SRC, SG, true, false, 3>(g, a, ws)
                                : launch_pair<K, DB, SRC, SG, true, false, 4>(g, a, ws);
    }
    return split        ? launch_pair<K, DB, SRC, SG, false, true, 4>(g, a, ws)
           : waves == 2 ? launch_pair<K, DB, SRC, SG, false, false, 2>(g, a, ws)
           : waves == 3 ? launch_pair<K, DB, SRC, SG, false, false, 3>(g, a, ws)
                        : launch_pair<K, DB, SRC, SG, false, false, 4>(g, a, ws);
}
template <int K, int DB, int SG>
hipError_t launch_bwd(const Geo &g, const BwdArgs &a, Ws &ws)
{
    return a.ckpt != nullptr ? launch_bwd_src<K, DB, kCkpt, SG>(g, a, ws) : launch_bwd_src<K, DB, SG, SG>(g, a, ws);
}

// One translation unit a width.
hipError_t bwd32(const Geo &, const BwdArgs &, Ws &);
hipError_t bwd48(const Geo &, const BwdArgs &, Ws &);
hipError_t bwd64(const Geo &, const BwdArgs &, Ws &);
hipError_t bwd_any(const Geo &, const BwdArgs &, Ws &);

}  // namespace bf
}  // namespace rpb
}  // namespace rib
