"""The operators of an attention branch beyond RMSNorm, one position and full causal attention.

A case is one pass through one operator on inputs made on the GPU from a seed:

* ``layernorm``   LayerNorm over rows, forward, or backward with the gradients of its gain and bias;
* ``rope``        rotary positions with several axes on the q and k heads of a fused qkv buffer;
* ``attention``   causal grouped-query attention with a sliding window and sinks, forward or
                  backward, on full or padded batch rows.

``run`` computes them from their formulas with plain torch operations in 32 bits, or, with
``own``, calls the framework's. ``exact`` recomputes a case in float64.
"""
import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5

# what the largest case costs: the bounds of a drawn one
_MAX_ROWS = 16384 * 4096            # LayerNorm elements
_MAX_ROTATED = 16384 * 40 * 128     # rotated elements
_MAX_SCORES = 32 * 16384 * 8208     # scores that the plain form holds at once
_MAX_FLOPS = 32 * 128 * 16384 * 4096


def _layernorm(name, **kw):
    c = dict(kind="layernorm", backward=False, bias=True, resid=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _rope(name, **kw):
    c = dict(kind="rope", n_kv_heads=0, base=10000.0, interleaved=False, own_ladder=False,
             inverse=False, table=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _attention(name, **kw):
    c = dict(kind="attention", backward=False, lens="", sinks=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short sequence through a small layer's norm: latency is all of it
        _layernorm("layernorm_small", tokens=128, hidden=256),
        # the norm of an 8B-shape layer on a 16K sequence
        _layernorm("layernorm", tokens=16384, hidden=4096),
        # ragged rows of an odd width, without a bias: rows end inside a wave's share
        _layernorm("layernorm_bwd_ragged", tokens=999, hidden=2056, backward=True, bias=False),
        # the norm's backward at 16K tokens, a residual stream's gradient passing it
        _layernorm("layernorm_bwd", tokens=16384, hidden=4096, backward=True, resid=True),
        # patches of a few images, height and width with a ladder each, the tables of a new
        # image size made on the way
        _rope("rope_patches", tokens=1025, n_heads=12, n_kv_heads=4, head_dim=64, pairs="16,16",
              own_ladder=True, positions=128, table=True),
        # text and video frames of a long sequence: time, height and width on one ladder
        _rope("rope_video", tokens=16384, n_heads=32, n_kv_heads=8, head_dim=128,
              pairs="16,24,24", positions=16384, base=500000.0),
        # the gradient's way back at an odd length, the axes' pairs dealt in turn
        _rope("rope_video_bwd", tokens=4095, n_heads=16, n_kv_heads=8, head_dim=128,
              pairs="24,20,20", interleaved=True, inverse=True, positions=4096, base=1e6),
        # a padded batch of short sequences in a small layer
        _attention("window_short", batch=3, seq=333, n_heads=12, n_kv_heads=4, head_dim=64,
                   window=128, sinks=4, lens="333,200,45"),
        # an ordinary training batch, a window of a quarter of the sequence, a few sinks
        _attention("window", batch=4, seq=4096, n_heads=32, n_kv_heads=8, head_dim=128,
                   window=1024, sinks=4),
        # the smallest training step's attention backward: one short sequence, few heads
        _attention("window_bwd_short", batch=1, seq=257, n_heads=4, n_kv_heads=2, head_dim=64,
                   window=64, sinks=2, backward=True),
        # head dim 64, sequences that end inside a tile, some of them padded, no sinks
        _attention("window_bwd_ragged", batch=4, seq=2047, n_heads=32, n_kv_heads=8, head_dim=64,
                   window=500, lens="2047,2047,1500,911", backward=True),
        # the largest call: an 8B-shape layer's heads on a 16K sequence
        _attention("window_bwd_16k", batch=1, seq=16384, n_heads=32, n_kv_heads=8, head_dim=128,
                   window=4096, sinks=16, backward=True),
    ]


# ------------------------------------------------------------------ draw ----

def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step))


def _heads(rng):
    kv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 8))
    return dict(n_heads=min(kv * group, 32) // kv * kv, n_kv_heads=kv)


def draw(rng):
    kind = rng.choice(("layernorm", "rope", "attention", "attention"))
    if kind == "layernorm":
        h = _log(rng, 64, 8192, 8)
        back = rng.random() < 0.5
        return _layernorm(None, tokens=_log(rng, 1, min(16384, _MAX_ROWS // h)), hidden=h,
                          backward=back, bias=rng.random() < 0.7,
                          resid=back and rng.random() < 0.5)
    if kind == "rope":
        d, heads, n = rng.choice((64, 128)), _heads(rng), rng.choice((1, 2, 3, 3))
        rot = (heads["n_heads"] + heads["n_kv_heads"]) * d
        cuts = sorted(rng.sample(range(1, d // 2), n - 1))
        pairs = [b - a for a, b in zip([0] + cuts, cuts + [d // 2])]
        return _rope(None, tokens=_log(rng, 1, min(16384, _MAX_ROTATED // rot)), head_dim=d,
                     pairs=",".join(map(str, pairs)), positions=_log(rng, 64, 16384),
                     interleaved=rng.random() < 0.4, own_ladder=rng.random() < 0.3,
                     inverse=rng.random() < 0.4, base=rng.choice((10000.0, 500000.0, 1e6)),
                     **heads)
    while True:
        c = _attention(None, batch=rng.randint(1, 4), seq=_log(rng, 1, 16384),
                       head_dim=rng.choice((64, 128)), window=_log(rng, 1, 8192),
                       sinks=rng.choice((0, 0, 1, 4, 16, 70)), backward=rng.random() < 0.5,
                       **_heads(rng))
        if rng.random() < 0.4:
            c["lens"] = ",".join(str(rng.randint(0, c["seq"])) for _ in range(c["batch"]))
        heads, blk = c["batch"] * c["n_heads"], _block(c)
        held = heads * -(-c["seq"] // blk) * blk * (2 * blk + c["sinks"])
        if held <= _MAX_SCORES and heads * c["head_dim"] * c["seq"] * min(
                c["window"], c["seq"]) <= _MAX_FLOPS:
            return c


# --------------------------------------------------------------- prepare ----

class _Draw:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(mean, std,
                                                                           generator=self.g)

    def bf16(self, shape, std=1.0, mean=0.0):
        return self.normal(shape, std, mean).to(torch.bfloat16)

    def ints(self, n, hi):
        return torch.randint(0, hi, (n,), generator=self.g, device=DEV, dtype=torch.int32)


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV)


def _pairs(c):
    return [int(n) for n in c["pairs"].split(",")]


def _lens(c):
    return [int(n) for n in c["lens"].split(",")] if c["lens"] else [c["seq"]] * c["batch"]


def prepare(case, seed):
    return {"layernorm": _prepare_layernorm, "rope": _prepare_rope,
            "attention": _prepare_attention}[case["kind"]](case, seed)


def _prepare_layernorm(c, seed):
    d, T, h = _Draw(seed), c["tokens"], c["hidden"]
    # a residual stream's rows: their own offset each
    s = dict(c=c, x=(d.normal((T, h)) + d.normal((T, 1), 0.5)).to(torch.bfloat16),
             g=d.bf16((h,), 0.1, 1.0), b=d.bf16((h,), 0.1) if c["bias"] else None)
    if not c["backward"]:
        return dict(s, y=_empty(T, h), mean=_empty(T, dtype=torch.float32),
                    rstd=_empty(T, dtype=torch.float32))
    s["mean"], s["rstd"] = _row_statistics(s["x"].float())
    return dict(s, dy=d.bf16((T, h), 1e-2), resid=d.bf16((T, h), 1e-2) if c["resid"] else None,
                dx=_empty(T, h), dg=_empty(h, dtype=torch.float32),
                db=_empty(h, dtype=torch.float32) if c["bias"] else None)


def _axis_positions(d, c):
    """Positions [axes, T] of a sequence of texts and frames: a text token stands at one position
    on every axis, a frame's patches at its time and their row and column behind it."""
    T, n, P = c["tokens"], len(_pairs(c)), c["positions"]
    i = torch.arange(T, device=DEV)
    side = max(1, min(24, P // 4))
    patch, frame = i % (side * side), i // (side * side)
    text = (d.normal((int(frame[-1]) + 1,)) > 0.8)[frame]
    start = (frame * side) % max(1, P - 2 * side) + d.ints(1, side)
    cols = [torch.zeros_like(i), patch // side, patch % side]
    axes = cols if n == 3 else cols[1:] if n == 2 else [patch % side]
    return torch.stack([torch.where(text, start + patch % side, start + a)
                        for a in axes]).clamp(0, P - 1).to(torch.int32).contiguous()


def _prepare_rope(c, seed):
    d, T, D = _Draw(seed), c["tokens"], c["head_dim"]
    n = c["n_heads"] + c["n_kv_heads"]
    s = dict(c=c, qkv=d.bf16((T, (n + c["n_kv_heads"]) * D)), pos=_axis_positions(d, c),
             out=_empty(T, n * D), n=n)
    s["cos"], s["sin"] = (_empty(c["positions"], D // 2, dtype=torch.float32) for _ in range(2))
    if not c["table"]:
        for t, v in zip((s["cos"], s["sin"]), _angle_tables(c)):
            t.copy_(v)
    return s


def _prepare_attention(c, seed):
    d, B, S = _Draw(seed), c["batch"], c["seq"]
    hq, hkv = c["n_heads"] * c["head_dim"], c["n_kv_heads"] * c["head_dim"]
    lens = torch.tensor(_lens(c), dtype=torch.int32, device=DEV)
    s = dict(c=c, qkv=d.bf16((B * S, hq + 2 * hkv)), lens=lens if c["lens"] else None)
    if not c["backward"]:
        return dict(s, o=_empty(B * S, hq), lse=_empty(B, c["n_heads"], S, dtype=torch.float32))
    s["o"], s["lse"] = _attention_fwd(s)
    return dict(s, do=d.bf16((B * S, hq)), dqkv=torch.empty_like(s["qkv"]))


# ------------------------------------------------------------------- run ----

def run(state):
    kind = state["c"]["kind"]
    if own:
        return {"layernorm": _own_layernorm, "rope": _own_rope,
                "attention": _own_attention}[kind](state)
    back = state["c"].get("backward")
    if kind == "layernorm":
        return _layernorm_bwd(state) if back else _layernorm_fwd(state)
    if kind == "rope":
        return _rotate(state)
    return dict(dqkv=_attention_bwd(state)) if back else dict(zip(("o", "lse"),
                                                                 _attention_fwd(state)))


def _own_layernorm(s):
    from paper_2609_13645_amd import _lib
    T, h = s["x"].shape
    if not s["c"]["backward"]:
        _lib.forge_layernorm_fwd(s["x"], s["g"], s["b"], s["y"], s["mean"], s["rstd"], T, h, EPS)
        return {k: s[k] for k in ("y", "mean", "rstd")}
    if "ws" not in s:
        s["ws"] = _empty(max(1, _lib.forge_layernorm_bwd_workspace_bytes(T, h)),
                         dtype=torch.uint8)
    _lib.forge_layernorm_bwd(s["x"], s["g"], s["mean"], s["rstd"], s["dy"], s["resid"], s["dx"],
                             s["dg"], s["db"], False, T, h, s["ws"])
    return {k: s[k] for k in ("dx", "dg", "db")}


def _own_rope(s):
    from paper_2609_13645_amd import _lib
    c = s["c"]
    if "cfg" not in s:
        s["cfg"] = _lib.rope_axes_cfg(dict(c, pairs=_pairs(c)))
    if c["table"]:
        _lib.forge_rope_axes_table(s["cfg"], c["positions"], c["base"], s["cos"], s["sin"])
    _lib.forge_rope_axes_apply(s["cfg"], s["qkv"], s["qkv"].shape[1], s["out"],
                               s["out"].shape[1], s["cos"], s["sin"], s["pos"], c["tokens"],
                               c["positions"], s["n"], c["inverse"])
    return s["out"]


def _own_attention(s):
    from paper_2609_13645_amd import _lib
    c = s["c"]
    if "cfg" not in s:
        s["cfg"] = _lib.attn_window_cfg(c)
    if not c["backward"]:
        _lib.forge_attention_window_fwd(s["cfg"], s["qkv"], s["lens"], s["o"], s["lse"])
        return dict(o=s["o"], lse=s["lse"])
    if "ws" not in s:
        s["ws"] = _empty(max(1, _lib.forge_attention_window_bwd_workspace_bytes(s["cfg"])),
                         dtype=torch.uint8)
    _lib.forge_attention_window_bwd(s["cfg"], s["qkv"], s["lens"], s["o"], s["lse"], s["do"],
                                    s["dqkv"], s["ws"])
    return dict(dqkv=s["dqkv"])


# ----------------------------------------------------------- plain forms ----

def _row_statistics(x):
    mean = x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, (var + EPS).rsqrt()


def _layernorm_fwd(s):
    x = s["x"].float()
    mean, rstd = _row_statistics(x)
    y = (x - mean[:, None]) * rstd[:, None] * s["g"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    return dict(y=y.to(torch.bfloat16), mean=mean, rstd=rstd)


def _layernorm_bwd(s):
    dy, r = s["dy"].float(), s["rstd"][:, None]
    xh = (s["x"].float() - s["mean"][:, None]) * r
    gdy = dy * s["g"].float()
    dx = (gdy - gdy.mean(1, keepdim=True) - xh * (gdy * xh).mean(1, keepdim=True)) * r
    if s["resid"] is not None:
        dx = dx + s["resid"].float()
    return dict(dx=dx.to(torch.bfloat16), dg=(dy * xh).sum(0),
                db=dy.sum(0) if s["b"] is not None else None)


def _pair_axes(c):
    """The axis of every pair, and the pair's index within its axis."""
    p = _pairs(c)
    if c["interleaved"]:
        order = sorted((r, a) for a, n in enumerate(p) for r in range(n))
        return [a for _, a in order], [r for r, _ in order]
    return [a for a, n in enumerate(p) for _ in range(n)], [r for n in p for r in range(n)]


def _angle_tables(c):
    """cos and sin of every position's angle for every pair: in 64 bits, positions may be far."""
    p, (axis, index) = _pairs(c), _pair_axes(c)
    exponent = [r / p[a] for a, r in zip(axis, index)] if c["own_ladder"] else \
        [2.0 * i / c["head_dim"] for i in range(c["head_dim"] // 2)]
    freq = c["base"] ** -torch.tensor(exponent, dtype=torch.float64, device=DEV)
    angle = torch.arange(c["positions"], dtype=torch.float64, device=DEV)[:, None] * freq
    return angle.cos().float(), angle.sin().float()


def _rotate(s):
    c, half = s["c"], s["c"]["head_dim"] // 2
    cos, sin = _angle_tables(c) if c["table"] else (s["cos"], s["sin"])
    if "axis" not in s:
        s["axis"] = torch.tensor(_pair_axes(c)[0], device=DEV)
    at = s["pos"].long()[s["axis"]].t()            # [T, pairs]: the position of every pair
    cos, sin = cos.gather(0, at)[:, None], sin.gather(0, at)[:, None]
    if c["inverse"]:
        sin = -sin
    x = s["qkv"][:, :s["n"] * 2 * half].float().view(c["tokens"], s["n"], 2 * half)
    x1, x2 = x[..., :half], x[..., half:]
    y = torch.cat((x1 * cos - x2 * sin, x2 * cos + x1 * sin), 2)
    return y.view(c["tokens"], -1).to(torch.bfloat16)


def _block(c):
    """Queries of one block of the plain attention: its window lies in that block of keys and the
    one before."""
    return min(max(c["window"], 64), c["seq"])


def _bands(s):
    """q [B, blocks, kv, group * blk, d], k and v [B, blocks, kv, 2 blk + sinks, d] in 32 bits and
    the mask [B, blocks, 1, 1, blk, 2 blk + sinks] of what each query sees."""
    c, blk = s["c"], _block(s["c"])
    B, S, D, kv, sinks = c["batch"], c["seq"], c["head_dim"], c["n_kv_heads"], min(c["sinks"], c["seq"])
    grp, n = c["n_heads"] // kv, -(-c["seq"] // blk)
    x = s["qkv"].float().view(B, S, (grp + 2) * kv, D)
    x = torch.cat((x, x.new_zeros(B, n * blk - S, (grp + 2) * kv, D)), 1)
    q = _blocks_of(x[:, :, :grp * kv], c).contiguous()

    def keys(y):
        y = y.transpose(1, 2)
        own_block = y.reshape(B, kv, n, blk, D)
        before = torch.cat((torch.zeros_like(own_block[:, :, :1]), own_block[:, :, :-1]), 2)
        first = y[:, :, None, :sinks].expand(-1, -1, n, -1, -1)
        return torch.cat((before, own_block, first), 3).transpose(1, 2)

    k, v = keys(x[:, :, grp * kv:(grp + 1) * kv]), keys(x[:, :, (grp + 1) * kv:])
    b = torch.arange(n, device=DEV)[:, None, None] * blk
    i = b + torch.arange(blk, device=DEV)[:, None]
    j = b - blk + torch.arange(2 * blk, device=DEV)
    f = torch.arange(sinks, device=DEV).expand(n, 1, sinks)
    seen = torch.cat(((j >= 0) & (j <= i) & (j > i - c["window"]), f <= i - c["window"]), 2)
    lens = torch.full((B,), S, device=DEV) if s["lens"] is None else s["lens"]
    return q, k, v, (seen & (i < lens[:, None, None, None]))[:, :, None, None]


def _blocks_of(y, c):
    """[B, n blk, heads, e] -> [B, n, kv, group * blk, e]."""
    blk, kv = _block(c), c["n_kv_heads"]
    B, rows, heads, e = y.shape
    y = y.reshape(B, rows // blk, blk, kv, heads // kv, e)
    return y.permute(0, 1, 3, 4, 2, 5).reshape(B, rows // blk, kv, heads // kv * blk, e)


def _rows_of(y, c):
    """The other way, without the rows that fill the last block."""
    blk, kv, n_heads = _block(c), c["n_kv_heads"], c["n_heads"]
    B, n, _, _, e = y.shape
    y = y.view(B, n, kv, n_heads // kv, blk, e).permute(0, 1, 4, 2, 3, 5)
    return y.reshape(B, n * blk, n_heads, e)[:, :c["seq"]]


def _padded(y, c):
    B, S, heads, e = y.shape
    return torch.cat((y, y.new_zeros(B, -S % _block(c), heads, e)), 1)


def _scores(q, k, seen, c):
    grp, blk = c["n_heads"] // c["n_kv_heads"], _block(c)
    z = (q @ k.transpose(-1, -2).contiguous()) / math.sqrt(c["head_dim"])
    z = z.view(*z.shape[:3], grp, blk, z.shape[-1])
    return z.masked_fill_(~seen, -math.inf)


def _attention_fwd(s):
    c = s["c"]
    q, k, v, seen = _bands(s)
    z = _scores(q, k, seen, c)
    top = z.amax(-1, keepdim=True)
    z = z.sub_(top.clamp_min(-1e30)).exp_()
    total = z.sum(-1, keepdim=True)
    lse = top + total.log()
    o = z.flatten(3, 4) @ v / total.clamp_min(1e-30).flatten(3, 4)
    o = _rows_of(o, c).reshape(c["batch"] * c["seq"], -1).to(torch.bfloat16)
    return o, _rows_of(lse.flatten(3, 4), c)[..., 0].transpose(1, 2).contiguous()


def _attention_bwd(s):
    c = s["c"]
    B, S, D, kv, blk = c["batch"], c["seq"], c["head_dim"], c["n_kv_heads"], _block(c)
    grp = c["n_heads"] // kv
    q, k, v, seen = _bands(s)
    do = s["do"].float().view(B, S, -1, D)
    delta = (do * s["o"].float().view(B, S, -1, D)).sum(-1, keepdim=True)
    do, delta, lse = (_blocks_of(_padded(y, c), c)
                      for y in (do, delta, s["lse"].transpose(1, 2)[..., None]))
    p = _scores(q, k, seen, c).flatten(3, 4)
    p = p.sub_(lse.clamp_min(-1e30)).exp_()
    dv = p.transpose(-1, -2) @ do
    ds = do @ v.transpose(-1, -2).contiguous()
    ds = ds.sub_(delta).mul_(p).div_(math.sqrt(D))
    dq = _rows_of(ds @ k, c)
    dk = ds.transpose(-1, -2) @ q

    def keys(y):                                   # a key's shares of its blocks, and as a sink
        own_block = y[:, :, :, blk:2 * blk].clone()
        own_block[:, :-1] += y[:, 1:, :, :blk]
        y = torch.cat((own_block.transpose(1, 2).reshape(B, kv, -1, D)[:, :, :S],
                       y[:, :, :, 2 * blk:].sum(1)), 2)
        y[:, :, :y.shape[2] - S] += y[:, :, S:]
        return y[:, :, :S].transpose(1, 2)

    out = torch.cat((dq, keys(dk), keys(dv)), 2)
    return out.reshape(B * S, (grp + 2) * kv * D).to(torch.bfloat16)


# ------------------------------------------------------------------ work ----

def _seen_pairs(c):
    """(query, key) pairs that see each other, over the batch rows of one head."""
    W, sinks, n = c["window"], c["sinks"], 0
    for length in _lens(c):
        w = min(W, length)
        n += w * (w + 1) // 2 + (length - w) * w
        # sinks before the window of queries sinks + W - 1 .. and some of those between
        far = max(0, length - W)                   # queries with keys before their window
        few = min(far, sinks)
        n += few * (few + 1) // 2 + (far - few) * sinks
    return n


def work(case):
    c = case
    if c["kind"] == "layernorm":
        T, h = c["tokens"], c["hidden"]
        streams = 3 + c["resid"] if c["backward"] else 2
        vectors = (2 + 4 + 4 * c["bias"]) * h if c["backward"] else (2 + 2 * c["bias"]) * h
        return dict(bytes=2 * T * h * streams + 8 * T + vectors,
                    flops=T * h * (13 if c["backward"] else 8))
    if c["kind"] == "rope":
        T, n, D = c["tokens"], c["n_heads"] + c["n_kv_heads"], c["head_dim"]
        rows = c["positions"] if c["table"] else min(T, c["positions"])
        return dict(bytes=4 * T * n * D + 4 * len(_pairs(c)) * T + 4 * rows * D,
                    flops=3 * T * n * D)
    T, hq, hkv = sum(_lens(c)), c["n_heads"] * c["head_dim"], c["n_kv_heads"] * c["head_dim"]
    full = c["batch"] * c["seq"]
    pairs = _seen_pairs(c) * c["n_heads"] * c["head_dim"]
    if not c["backward"]:
        return dict(bytes=2 * T * (hq + 2 * hkv) + 2 * full * hq + 4 * full * c["n_heads"],
                    flops=4 * pairs)
    return dict(bytes=2 * T * (3 * hq + 2 * hkv) + 4 * T * c["n_heads"] + 2 * full * (hq + 2 * hkv),
                flops=10 * pairs)


# ----------------------------------------------------------------- exact ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"layernorm": _exact_layernorm, "rope": _exact_rope,
            "attention": _exact_attention}[case["kind"]](s)


def _exact_layernorm(s):
    x, g = s["x"].double(), s["g"].double()
    h = x.shape[1]
    if not s["c"]["backward"]:
        mean = x.sum(1) / h
        rstd = 1.0 / (((x * x).sum(1) / h - mean * mean) + EPS).sqrt()
        y = (x * rstd[:, None] - (mean * rstd)[:, None]) * g
        return dict(y=y if s["b"] is None else y + s["b"].double(), mean=mean, rstd=rstd)
    mean, rstd, dy = s["mean"].double()[:, None], s["rstd"].double()[:, None], s["dy"].double()
    centred = x - mean
    along = (dy * g * centred).sum(1, keepdim=True) * rstd ** 3 / h
    dx = dy * g * rstd - (dy * g).sum(1, keepdim=True) * rstd / h - centred * along
    return dict(dx=dx if s["resid"] is None else dx + s["resid"].double(),
                dg=((dy * rstd) * centred).sum(0), db=None if s["b"] is None else dy.sum(0))


def _exact_rope(s):
    c, D = s["c"], s["c"]["head_dim"]
    shares, turn, at, w = _pairs(c), [0] * len(_pairs(c)), [], []
    a = 0
    for i in range(D // 2):                        # whose pair is this
        if c["interleaved"]:
            while turn[a % len(shares)] >= shares[a % len(shares)]:
                a += 1
            axis = a % len(shares)
            a += 1
        else:
            axis = next(k for k in range(len(shares)) if i < sum(shares[:k + 1]))
        w.append(c["base"] ** (-turn[axis] / shares[axis] if c["own_ladder"] else -i * 2.0 / D))
        at.append(s["pos"][axis].double())
        turn[axis] += 1
    angle = torch.stack(at, 1) * torch.tensor(w, dtype=torch.float64, device=DEV)
    turn_by = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)[:, None]
    x = s["qkv"][:, :s["n"] * D].double().view(c["tokens"], s["n"], 2, D // 2)
    y = torch.complex(x[:, :, 0], x[:, :, 1]) * turn_by
    return torch.stack((y.real, y.imag), 2).reshape(c["tokens"], -1)


def _exact_attention(s):
    c = s["c"]
    B, S, D, kv, W = c["batch"], c["seq"], c["head_dim"], c["n_kv_heads"], c["window"]
    nh = c["n_heads"]
    x = s["qkv"].view(B, S, nh + 2 * kv, D)
    back = c["backward"]
    o = torch.zeros((B, S, nh, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, nh, S), -math.inf, dtype=torch.float64, device=DEV)
    dx = torch.zeros((B, S, nh + 2 * kv, D), dtype=torch.float64, device=DEV) if back else None
    for b, n in enumerate(_lens(c)):
        i, j = torch.arange(n, device=DEV)[:, None], torch.arange(n, device=DEV)
        hidden = (j > i) | ((i - j >= W) & (j >= c["sinks"]))
        for h in range(nh if n else 0):
            m = nh + h // (nh // kv)
            q, k, v = (x[b, :n, e].double() for e in (h, m, m + kv))
            z = (q @ k.t().contiguous()).mul_(D ** -0.5).masked_fill_(hidden, -math.inf)
            if not back:
                lse[b, h, :n] = z.logsumexp(1)
                o[b, :n, h] = z.softmax(1) @ v
                continue
            p = z.sub_(s["lse"][b, h, :n, None].double()).exp_()
            do = s["do"].view(B, S, nh, D)[b, :n, h].double()
            t = (do * s["o"].view(B, S, nh, D)[b, :n, h].double()).sum(1, keepdim=True)
            dx[b, :n, m + kv] += p.t() @ do
            p.mul_((do @ v.t().contiguous()).sub_(t)).mul_(D ** -0.5)
            dx[b, :n, h] = p @ k
            dx[b, :n, m] += p.t() @ q
    return dict(dqkv=dx.view(B * S, -1)) if back else dict(o=o.view(B * S, -1), lse=lse)
