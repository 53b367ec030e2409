"""Window attention with a learned relative position bias: the calls whose time counts, and their plain forms.

The operators (public entry points of `paper_2603_06738_amd.binding`), for windows of M x M tokens of a
channel-last grid after a cyclic shift, L = (2M - 1)^2 relative offsets (query minus key, row-major):

    rib_rpb_table_fwd   bias[head][offset] = table[head][index[offset]]; an index outside the table excludes
                        the offset's pairs (a bias of minus infinity)
    rib_rpb_attn_fwd    O = softmax(scale q.k + bias[head][offset]) v, and LSE; a row without a key gives zeros
    rib_rpb_attn_bwd    dQ, dK, dV and dbias[head][offset] (sums over windows and images), the probabilities
                        made again from q, k, bias and LSE; delta is taken from O as it is stored
    rib_rpb_table_bwd   dtable[head][bucket] = sum of dbias over the bucket's offsets
    rib_checkpoint_pack q, k, v of every (window, head, token) as 8-bit codes under one power of two
    rib_rpb_attn_bwd_ckpt   the backward from such a checkpoint in place of q, k, v

Three kinds of cases:

    infer   one attention forward without LSE; the bias is laid out once, as a served model keeps it
    train   table -> bias, forward, backward, dbias -> dtable
    train8  the same, with q, k, v kept between forward and backward as an 8-bit checkpoint

A case holds kind, dtype ("bf16" / "f32": q, k, v, O, their gradients and the table), grid B x H x W, heads,
head dim d, window side M, cyclic shift s, whether q, k, v are views of one packed [B, H, W, 3C] projection,
and how offsets map to buckets:

    full    a bucket for each offset
    log     a bucket for each pair of per-axis distances, near ones exact, far ones logarithmic
    disc    a bucket for each offset no farther than 3/4 M, the others excluded
    past    a bucket for each offset to an earlier token in raster order, the others (the own token's
            too) excluded: the window's first token has no key at all
"""
import math

import torch

own = False

DEV = "cuda:0"
MAX_SCORES = 1.0e9              # scores (units * N^2) of a drawn case; the largest listed one has 1.2e9
MAX_FLOP = 3.8e11               # and its operations; the largest listed one has 4.3e11
MAX_FLOP_F32 = 9.0e10           # fp32 arithmetic is an order slower per operation
MAX_TOKENS = 150000


def _case(name, kind, dtype, B, H, W, heads, d, M, s, buckets="full", packed=False):
    return {"name": name, "kind": kind, "dtype": dtype, "B": B, "H": H, "W": W, "heads": heads, "d": d, "M": M, "s": s,
            "buckets": buckets, "packed": packed}


def listed():
    return [
        # serving one 64 x 64 tile through a layer of 8 x 8 windows: the smallest call, all latency
        _case("infer_w8_tile", "infer", "bf16", 1, 64, 64, 6, 30, 8, 4),
        # 12 x 12 windows (144 tokens: no whole tile), packed projection, an ordinary serving batch
        _case("infer_w12_packed", "infer", "bf16", 4, 96, 144, 6, 30, 12, 6, "log", packed=True),
        # the repository's headline forward shape at 32 x 32 windows
        _case("infer_w32", "infer", "bf16", 8, 96, 96, 6, 30, 32, 16),
        # part of a photograph at 64 x 64 windows
        _case("infer_w64_photo", "infer", "bf16", 1, 192, 256, 6, 30, 64, 32),
        # 7 x 7 windows (49 tokens) of 56 x 56 grids, the first stage of a window transformer: many tiny windows
        _case("train_w7", "train", "bf16", 32, 56, 56, 3, 32, 7, 3),
        # training patches at the schedule's smallest windows
        _case("train_w16", "train", "bf16", 16, 96, 96, 6, 30, 16, 8),
        # the benchmark's training step, with a table in place of the implicit bias
        _case("train_w32", "train", "bf16", 16, 96, 96, 6, 30, 32, 16),
        # attention to earlier tokens only: half of the pairs excluded, one row of a window empty
        _case("train_w24_past", "train", "bf16", 8, 96, 96, 6, 32, 24, 0, "past", packed=True),
        # the schedule's largest windows, distances in buckets
        _case("train_w96_log", "train", "bf16", 2, 96, 96, 6, 30, 96, 0, "log"),
        # the benchmark's layer in fp32 storage, a quarter of its batch, far pairs excluded
        _case("train_w32_f32", "train", "f32", 4, 96, 96, 6, 30, 32, 16, "disc"),
        # the benchmark's training step with its activations kept in 8 bits
        _case("train8_w32", "train8", "bf16", 16, 96, 96, 6, 30, 32, 16),
        # a small fp32 layer of wider heads, activations in 8 bits
        _case("train8_w16_f32", "train8", "f32", 4, 64, 64, 4, 48, 16, 8, "log"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case anywhere in the ranges above: window sides 3 to 96 (odd ones too), grids of any number of windows,
    heads 1 to 8, head dims 8 to 64 (odd ones too), every bucket map, each kind and type."""
    while True:
        kind = rng.choice(["infer", "train", "train", "train8"])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        M = _log_int(rng, 3, 96)
        d = rng.choice([8, 15, 16, 24, 28, 30, 30, 30, 32, 32, 40, 48, 64])
        heads = rng.choice([1, 2, 3, 4, 6, 6, 8])
        windows = _log_int(rng, 1, max(1.0, MAX_TOKENS / (M * M)))
        nwy = rng.randrange(1, max(1, int(math.sqrt(windows))) + 1)
        nwx = rng.randrange(1, max(1, windows // nwy) + 1)
        B = max(1, windows // (nwy * nwx))
        s = rng.choice([0, M // 2, rng.randrange(M)])
        case = _case(None, kind, dtype, B, nwy * M, nwx * M, heads, d, M, s, rng.choice(["full", "full", "log", "disc", "past"]),
                     packed=rng.random() < 0.4)
        del case["name"]
        if work(case)["flops"] <= (MAX_FLOP if dtype == "bf16" else MAX_FLOP_F32) and B * nwy * nwx * heads * M ** 4 <= MAX_SCORES:
            return case


def _dims(case):
    N = case["M"] ** 2
    tokens = case["B"] * case["H"] * case["W"]
    return N, tokens, tokens // N * case["heads"], case["heads"] * case["d"]


def work(case):
    """Bytes of every input once and every output once, and the operations of the products: forward 4 N^2 d per
    (window, head), backward 10 N^2 d; exponentials are not counted."""
    N, tokens, units, C = _dims(case)
    e = 4 if case["dtype"] == "f32" else 2
    L = (2 * case["M"] - 1) ** 2
    grid, table = tokens * C * e, case["heads"] * L * e
    if case["kind"] == "infer":                                         # q, k, v, the bias; O
        return {"bytes": float(4 * grid + case["heads"] * L * 4), "flops": 4.0 * N * N * case["d"] * units}
    # q, k, v, dO, the table and its index; O, dQ, dK, dV, dtable
    return {"bytes": float(8 * grid + 2 * table + 4 * L), "flops": 14.0 * N * N * case["d"] * units}


def _bucket_map(kind, M):
    """(index [2M-1, 2M-1] int32, number of buckets)."""
    n = 2 * M - 1
    dist = torch.arange(n, dtype=torch.int64, device=DEV) - (M - 1)     # query minus key
    dy, dx = dist[:, None].expand(n, n), dist[None, :].expand(n, n)
    if kind == "log":
        far = dist.abs().clamp(min=1).double()
        steps = torch.where(dist.abs() <= 4, dist.abs(), 4 + (2.0 * torch.log2(far / 4.0)).floor().clamp(0, 8).long())
        axis = 12 + torch.where(dist < 0, -steps, steps)                # 0 .. 24
        return (axis[:, None] * 25 + axis[None, :]).to(torch.int32).contiguous(), 625
    index = torch.arange(n * n, dtype=torch.int64, device=DEV).reshape(n, n)
    if kind == "disc":
        index = torch.where(16 * (dy * dy + dx * dx) <= 9 * M * M, index, torch.full_like(index, -1))
    if kind == "past":
        index = torch.where((dy > 0) | ((dy == 0) & (dx > 0)), index, torch.full_like(index, -1))
    return index.to(torch.int32).contiguous(), n * n


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    td = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    N, _, units, C = _dims(case)
    B, H, W, heads, d, M = (case[n] for n in ("B", "H", "W", "heads", "d", "M"))
    grid = (B, H, W, C)

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(td)

    def empty(*shape, dtype=td):
        return torch.empty(shape, device=DEV, dtype=dtype)

    st = {"case": dict(case), "scale": d ** -0.5}
    if case["packed"]:
        qkv = normal(B, H, W, 3 * C)
        st["q"], st["k"], st["v"] = qkv[..., :C], qkv[..., C:2 * C], qkv[..., 2 * C:]
    else:
        st["q"], st["k"], st["v"] = normal(*grid), normal(*grid), normal(*grid)
    st["index"], nb = _bucket_map(case["buckets"], M)
    st["table"] = normal(heads, nb, std=0.5)
    st["out"] = empty(*grid)
    L = (2 * M - 1) ** 2
    if case["kind"] == "infer":
        flat = st["index"].reshape(-1).long()
        picked = st["table"].float()[:, flat.clamp(min=0)]
        st["bias"] = torch.where(flat >= 0, picked, torch.full_like(picked, -math.inf)).contiguous()
    else:
        st["dout"] = normal(*grid)
        st["bias"], st["dbias"] = empty(heads, L, dtype=torch.float32), empty(heads, L, dtype=torch.float32)
        st["lse"] = empty(units // heads, heads, N, dtype=torch.float32)
        st["dq"], st["dk"], st["dv"], st["dtable"] = empty(*grid), empty(*grid), empty(*grid), empty(heads, nb)
    if own:
        from paper_2603_06738_amd import binding as rb
        st["p"] = rb.make_params(B, H, W, heads, d, 0, M, case["s"], st["scale"], 0.0, case["dtype"],
                                 token_stride=3 * C if case["packed"] else 0)
        if case["kind"] != "infer":
            st["tp"] = rb.make_rpb_params(M, heads, nb, case["dtype"])
            st["ws"] = empty(max(rb.rib_rpb_attn_bwd_workspace_bytes(st["p"]), 256), dtype=torch.uint8)
        if case["kind"] == "train8":
            st["ckpt"] = empty(rb.rib_checkpoint_bytes(st["p"]), dtype=torch.uint8)
    return st


# ---- plain forms -------------------------------------------------------------------------------------------------


def _windows(case, x):
    """[B, H, W, C] -> [windows, heads, N, d] after the cyclic shift."""
    B, H, W, heads, d, M, s = (case[n] for n in ("B", "H", "W", "heads", "d", "M", "s"))
    x = torch.roll(x, (-s, -s), (1, 2)).reshape(B, H // M, M, W // M, M, heads, d)
    return x.permute(0, 1, 3, 5, 2, 4, 6).reshape(-1, heads, M * M, d)


def _grid(case, x):
    """The inverse of _windows."""
    B, H, W, heads, d, M, s = (case[n] for n in ("B", "H", "W", "heads", "d", "M", "s"))
    x = x.reshape(B, H // M, W // M, heads, M, M, d).permute(0, 1, 4, 2, 5, 3, 6).reshape(B, H, W, heads * d)
    return torch.roll(x, (s, s), (1, 2))


def _offsets(M):
    """offset[i][j] of query i and key j of a window, [N, N]."""
    n = torch.arange(M * M, device=DEV)
    y, x = torch.div(n, M, rounding_mode="floor"), n % M
    return (y[:, None] - y[None, :] + M - 1) * (2 * M - 1) + (x[:, None] - x[None, :] + M - 1)


def _plain_bias(st):
    flat = st["index"].reshape(-1).long()
    table = st["table"].float()
    inside = (flat >= 0) & (flat < table.shape[1])
    return torch.where(inside, table[:, flat.clamp(0, table.shape[1] - 1)], torch.full((), -math.inf, device=DEV))


def _plain_fwd(q, k, v, bias, scale):
    """(O, LSE) of [windows, heads, N, d] in 32 bits; `bias` [heads, N, N]."""
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale).add_(bias)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = s.sub_(top).exp_()
    den = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(den == 0, torch.ones_like(den), den)
    return o, top + torch.log(den)


def _plain_8bit(x):
    """Rows of a head's d values as codes of -127 .. 127 under the smallest power of two that holds the largest; the
    values that the codes stand for."""
    big = x.abs().amax(-1, keepdim=True).double()
    m, e = torch.frexp(big)                                     # big = m 2^e, m in [1/2, 1): 127/128 still fits 2^(e-7)
    e = (torch.where(m * 128 > 127, e + 1, e) - 7).clamp(min=-126)
    step = ((e.long() + 1023) << 52).view(torch.float64)        # 2^e, exactly
    return (torch.round(x.double() / step) * step).float()


def _diagonals(x):
    """[..., M, M] (query, key) -> [..., 2M-1]: sums over query minus key."""
    M = x.shape[-1]
    x = torch.nn.functional.pad(x.flip(-1), (0, M)).flatten(-2)[..., : M * (2 * M - 1)]
    return x.reshape(*x.shape[:-1], M, 2 * M - 1).sum(-2)


def _plain_bwd(q, k, v, bias, o, do, lse, scale, M):
    """dQ, dK, dV and dbias [heads, L] (64 bits: a sum over all windows) from the stored O."""
    s = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale).add_(bias)
    p = s.sub_(torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)).exp_()
    delta = (do * o).sum(-1, keepdim=True)
    dv = torch.matmul(p.transpose(-1, -2).contiguous(), do)
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous()).sub_(delta).mul_(p)
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2).contiguous(), q) * scale
    total = ds.sum(0, dtype=torch.float64)                      # [heads, N, N]
    heads = total.shape[0]
    rows = _diagonals(total.reshape(heads, M, M, M, M).permute(0, 1, 3, 2, 4))          # [heads, yq, yk, 2M-1]
    return dq, dk, dv, _diagonals(rows.permute(0, 3, 1, 2)).transpose(1, 2).reshape(heads, -1)


def _plain_table_grad(st, dbias):
    flat = st["index"].reshape(-1).long()
    nb = st["table"].shape[1]
    inside = (flat >= 0) & (flat < nb)
    grad = torch.zeros(dbias.shape[0], nb, dtype=torch.float64, device=DEV)
    return grad.index_add_(1, flat.clamp(0, nb - 1), torch.where(inside, dbias, torch.zeros_like(dbias)))


def _plain(st):
    case = st["case"]
    td = st["q"].dtype
    q, k, v = (_windows(case, st[n].float()) for n in ("q", "k", "v"))
    offsets = _offsets(case["M"])
    if case["kind"] == "infer":
        o, _ = _plain_fwd(q, k, v, st["bias"][:, offsets], st["scale"])
        return _grid(case, o).to(td)
    bias = _plain_bias(st)[:, offsets]
    o, lse = _plain_fwd(q, k, v, bias, st["scale"])
    out = _grid(case, o).to(td)
    if case["kind"] == "train8":
        q, k, v = _plain_8bit(q), _plain_8bit(k), _plain_8bit(v)
    do = _windows(case, st["dout"].float())
    dq, dk, dv, dbias = _plain_bwd(q, k, v, bias, _windows(case, out.float()), do, lse, st["scale"], case["M"])
    return {"out": out, "dq": _grid(case, dq).to(td), "dk": _grid(case, dk).to(td), "dv": _grid(case, dv).to(td),
            "dtable": _plain_table_grad(st, dbias).to(td)}


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(st):
    if not own:
        return _plain(st)
    from paper_2603_06738_amd import binding as rb
    kind, p, q, k, v, bias, out = st["case"]["kind"], st["p"], st["q"], st["k"], st["v"], st["bias"], st["out"]
    if kind == "infer":
        rb.rib_rpb_attn_fwd(p, q, k, v, bias, out)
        return out
    rb.rib_rpb_table_fwd(st["tp"], st["table"], st["index"], bias)
    rb.rib_rpb_attn_fwd(p, q, k, v, bias, out, st["lse"])
    grads = (st["dq"], st["dk"], st["dv"], st["dbias"])
    if kind == "train8":
        rb.rib_checkpoint_pack(p, q, k, v, st["ckpt"])
        rb.rib_rpb_attn_bwd_ckpt(p, st["ckpt"], bias, out, st["dout"], st["lse"], *grads, st["ws"])
    else:
        rb.rib_rpb_attn_bwd(p, q, k, v, bias, out, st["dout"], st["lse"], *grads, st["ws"])
    rb.rib_rpb_table_bwd(st["tp"], st["dbias"], st["index"], st["dtable"])
    return {n: st[n] for n in ("out", "dq", "dk", "dv", "dtable")}


# ---- 64 bits -----------------------------------------------------------------------------------------------------


def exact(case, seed):
    """The operators' definition in 64 bits, one head at a time, windows gathered by pixel coordinates."""
    st = prepare(case, seed)
    B, H, W, heads, d, M, s = (case[n] for n in ("B", "H", "W", "heads", "d", "M", "s"))
    N = M * M
    f64 = torch.float64
    # grid pixel of token n of window (wy, wx)
    n = torch.arange(N, device=DEV)
    iy, ix = n // M, n % M
    wy, wx = torch.arange(H // M, device=DEV), torch.arange(W // M, device=DEV)
    ys = (wy[:, None, None] * M + iy + s) % H
    xs = (wx[None, :, None] * M + ix + s) % W
    pixel = (ys * W + xs).reshape(-1)                           # [windows of an image * N]
    rel = (iy[:, None] - iy[None, :] + M - 1) * (2 * M - 1) + (ix[:, None] - ix[None, :] + M - 1)

    def gather(x, h):
        return x.reshape(B, H * W, heads * d)[:, pixel, h * d:(h + 1) * d].to(f64).reshape(-1, N, d)

    td = st["q"].dtype
    full = {name: torch.zeros(B, H * W, heads * d, dtype=f64, device=DEV) for name in ("out", "dq", "dk", "dv")}
    train = case["kind"] != "infer"
    steps = torch.tensor([2.0 ** e for e in range(-126, 122)], dtype=f64, device=DEV)
    if train:
        flat, nb = st["index"].reshape(-1).long(), st["table"].shape[1]
        legal = (flat >= 0) & (flat < nb)
        dtable = torch.zeros(heads, nb, dtype=f64, device=DEV)
    for h in range(heads):
        q, k, v = (gather(st[name], h) for name in ("q", "k", "v"))
        if train:
            b = torch.full((flat.numel(),), -math.inf, dtype=f64, device=DEV)
            b[legal] = st["table"][h].to(f64)[flat[legal]]
        else:
            b = st["bias"][h].to(f64)
        b = b[rel]
        s_ = torch.baddbmm(b.expand(q.shape[0], N, N), q, k.transpose(1, 2).contiguous(), alpha=st["scale"])
        lse = torch.logsumexp(s_, -1, keepdim=True)
        p = torch.where(torch.isinf(lse), torch.zeros((), dtype=f64, device=DEV), torch.exp(s_ - lse))
        o = torch.bmm(p, v)

        def put(name, x):
            full[name][:, pixel, h * d:(h + 1) * d] = x.reshape(B, -1, d)

        put("out", o)
        if not train:
            continue
        do = gather(st["dout"], h)
        delta = (do * o.to(td).to(f64)).sum(-1, keepdim=True)   # from O as it is stored
        if case["kind"] == "train8":
            def eight(x):                                       # the smallest step in the list that holds the largest
                place = torch.searchsorted(127.0 * steps, x.abs().amax(-1, keepdim=True))
                return torch.round(x / steps[place]) * steps[place]
            q, k, v = eight(q), eight(k), eight(v)
            s_ = torch.baddbmm(b.expand(q.shape[0], N, N), q, k.transpose(1, 2).contiguous(), alpha=st["scale"])
            p = torch.where(torch.isinf(lse), torch.zeros((), dtype=f64, device=DEV), torch.exp(s_ - lse))
        del s_
        put("dv", torch.bmm(p.transpose(1, 2).contiguous(), do))
        ds = p * (torch.bmm(do, v.transpose(1, 2).contiguous()) - delta)
        del p
        put("dq", torch.bmm(ds, k) * st["scale"])
        put("dk", torch.bmm(ds.transpose(1, 2).contiguous(), q) * st["scale"])
        dbias = torch.zeros((2 * M - 1) ** 2, dtype=f64, device=DEV)
        dbias.index_add_(0, rel.reshape(-1), ds.sum(0).reshape(-1))
        dtable[h].index_add_(0, flat[legal], dbias[legal])
    if not train:
        return full["out"].reshape(B, H, W, -1)
    got = {name: x.reshape(B, H, W, -1) for name, x in full.items()}
    got["dtable"] = dtable
    return got
