"""The operators of training on packed documents of long contexts.

A case is one pass through one operator on inputs made on the GPU from a seed:

* ``attention``  causal grouped-query attention over a row packed with documents of different
                 lengths, each on its own, with or without a sliding window, forward or backward;
* ``rope``       rotary positions on a part of each head, pairs in halves or interleaved,
                 frequencies and amplitude scaled for long contexts, forward or backward;
* ``adamw``      an AdamW step over many tensors at once, its moments in 32 bits, or in 8 with
                 stochastic rounding from a given seed.

``run`` computes them from their formulas with plain torch operations in 32 bits, or, with
``own``, calls the framework's. ``exact`` recomputes a case in float64.
"""
import math

import torch

own = False

DEV = "cuda"
BETA1, BETA2, ADAM_EPS, DECAY = 0.9, 0.95, 1e-8, 0.1
BLOCK = 256                         # moments of 8 bits that share a scale

# what the largest case costs: the bounds of a drawn one
_MAX_ROTATED = 16384 * 40 * 128     # elements of the rotated heads
_MAX_SCORES = 32 * 18000 * 12000    # scores that the plain form holds at once
_MAX_FLOPS = 32 * 128 * 75_700_000  # heads x head dim x sum of squared lengths
_MAX_PARAMS = 218_112_000

# the documents of a packed batch of 16384 tokens, lengths geometric with mean 512
_DOCS = ("277,742,266,1605,405,153,558,38,15,281,124,179,43,352,955,411,87,148,423,1568,494,25,"
         "287,265,7,340,136,76,786,476,687,107,155,210,107,358,481,1463,726,45,523")
# 8000 tokens of shorter ones, some of them empty
_SHORT_DOCS = ("147,716,84,199,654,387,0,311,201,54,681,429,436,526,148,187,6,106,247,32,219,30,1,"
               "30,177,70,46,132,358,0,0,293,295,566,232")
# the parameters of an 8B-shape layer, and of the tiny model
_LAYER = "4096*2,25165824,16777216,117440512,58720256"
_TINY = "256*3,131072,65536,352256,176128,262144*2"
# adapters, norms and biases of many layers: odd sizes, from one element on
_MANY = "1,255,256,257,2056*16,777,4097*8,131*16,2056999,65537*8,98304*12,1048583*3,12345678"


def _attention(name, **kw):
    c = dict(kind="attention", backward=False, window=0, behind=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _rope(name, **kw):
    c = dict(kind="rope", n_kv_heads=0, base=10000.0, offset=0, interleaved=False, scaling="none",
             factor=1.0, low=1.0, high=32.0, original=4096, amplitude=1.0, backward=False,
             in_place=False, table=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def _adamw(name, **kw):
    c = dict(kind="adamw", bits=32, bf16_grads=False, nearest=False)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a few short documents through a small layer, one of a single token, one empty
        _attention("packed_short", lens="333,1,0,200,77", n_heads=12, n_kv_heads=4, head_dim=64),
        # an ordinary packed batch in an 8B-shape layer
        _attention("packed", lens=_DOCS, n_heads=32, n_kv_heads=8, head_dim=128),
        # short documents, head dim 64, a window, rows behind the last document
        _attention("packed_window", lens=_SHORT_DOCS, n_heads=32, n_kv_heads=8, head_dim=64,
                   window=300, behind=191),
        # the smallest training step's attention backward: three documents, few heads
        _attention("packed_bwd_short", lens="65,129,63", n_heads=4, n_kv_heads=2, head_dim=64,
                   backward=True),
        # the packed batch's backward with heads of 64
        _attention("packed_bwd", lens=_DOCS, n_heads=32, n_kv_heads=8, head_dim=64, backward=True),
        # the largest call: four long documents, an 8B-shape layer's heads
        _attention("packed_bwd_long", lens="6000,5000,3001,2383", n_heads=32, n_kv_heads=8,
                   head_dim=128, backward=True),
        # one token: latency is all of it
        _rope("rope_part_token", tokens=1, n_heads=32, n_kv_heads=8, head_dim=128, rot=64,
              positions=8192),
        # half of each head, interleaved, q and k of a fused buffer out to another
        _rope("rope_part", tokens=16384, n_heads=32, n_kv_heads=8, head_dim=128, rot=64,
              interleaved=True, positions=16384, base=500000.0),
        # whole heads in halves for a context eight times the trained one, the gradient's way
        # back in place at an odd length, the tables made on the way
        _rope("rope_long_bwd", tokens=4095, n_heads=16, n_kv_heads=8, head_dim=128, rot=128,
              positions=32768, base=500000.0, scaling="parts", factor=8.0, backward=True,
              in_place=True, table=True),
        # the tiny model's tensors, moments in 32 bits: latency
        _adamw("adamw_tiny", tensors=_TINY),
        # an 8B-shape layer's tensors, moments in 8 bits
        _adamw("adamw_layer_8bit", tensors=_LAYER, bits=8),
        # many tensors of odd sizes, gradients in bf16, moments in 8 bits
        _adamw("adamw_many_8bit", tensors=_MANY, bits=8, bf16_grads=True),
    ]


# ------------------------------------------------------------------ draw ----

def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(v) // step * step))


def _heads(rng):
    kv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 3, 4, 8))
    return dict(n_heads=min(kv * group, 32) // kv * kv, n_kv_heads=kv)


def _draw_lens(rng, tokens):
    """Documents that fill about `tokens` rows: alike, of a geometric law, or one long one."""
    mean, kind, lens = _log(rng, 8, max(8, tokens)), rng.randint(0, 2), []
    while sum(lens) < tokens and len(lens) < 300:
        n = mean if kind == 0 else 1 + int(rng.expovariate(1.0 / mean))
        if kind == 2 and not lens:
            n = max(1, tokens * 3 // 4)
        if rng.random() < 0.03:
            n = rng.choice((0, 1))
        lens.append(min(n, tokens - sum(lens)))
    return lens


def draw(rng):
    kind = rng.choice(("attention", "attention", "rope", "adamw"))
    if kind == "rope":
        d, heads = rng.choice((64, 128)), _heads(rng)
        width = (heads["n_heads"] + heads["n_kv_heads"]) * d
        rot = rng.choice((d, d, d // 2, d // 4, 2 * rng.randint(2, d // 2)))
        scaling, in_place = rng.choice(("none", "linear", "base", "parts")), rng.random() < 0.5
        return _rope(None, tokens=_log(rng, 1, min(16384, _MAX_ROTATED // width)), head_dim=d,
                     rot=rot, offset=rng.choice((0, 0, d - rot)), interleaved=rng.random() < 0.5,
                     positions=_log(rng, 64, 32768), base=rng.choice((10000.0, 500000.0, 1e6)),
                     scaling=scaling, factor=1.0 if scaling == "none" else rng.choice((2.0, 8.0)),
                     low=rng.choice((1.0, 2.0)), high=rng.choice((4.0, 32.0)),
                     original=rng.choice((2048, 4096, 8192)),
                     # (an amplitude in place would grow from pass to pass)
                     amplitude=1.0 if in_place else rng.choice((1.0, 1.2)),
                     backward=rng.random() < 0.4, in_place=in_place, table=rng.random() < 0.2,
                     **heads)
    if kind == "adamw":
        left, sizes = _log(rng, 1 << 12, _MAX_PARAMS), []
        for _ in range(_log(rng, 1, 120)):
            sizes.append(_log(rng, 1, max(1, left // 2)))
            left -= sizes[-1]
        rng.shuffle(sizes)
        return _adamw(None, tensors=",".join(map(str, sizes)), bits=rng.choice((8, 32)),
                      bf16_grads=rng.random() < 0.5, nearest=rng.random() < 0.3)
    while True:
        lens = _draw_lens(rng, _log(rng, 1, 16384))
        c = _attention(None, lens=",".join(map(str, lens)), head_dim=rng.choice((64, 128)),
                       window=rng.choice((0, 0, _log(rng, 1, 4096))),
                       behind=rng.choice((0, 0, rng.randint(1, 200))),
                       backward=rng.random() < 0.5, **_heads(rng))
        if c["n_heads"] * _held(c) <= _MAX_SCORES and \
                c["n_heads"] * c["head_dim"] * sum(n * n for n in lens) <= _MAX_FLOPS:
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

    def uniform(self, shape):
        return torch.rand(shape, generator=self.g, device=DEV)

    def ints(self, n, hi):
        return torch.randint(0, hi, (n,), generator=self.g, device=DEV, dtype=torch.int32)


def _zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype, device=DEV)


def _lens(c):
    return [int(n) for n in c["lens"].split(",")]


def _sizes(c):
    return [int(p[0]) for e in c["tensors"].split(",") for p in [e.split("*")]
            for _ in range(int(p[1]) if len(p) > 1 else 1)]


def prepare(case, seed):
    return {"attention": _prepare_attention, "rope": _prepare_rope,
            "adamw": _prepare_adamw}[case["kind"]](case, seed)


def _prepare_attention(c, seed):
    d, lens, D = _Draw(seed), _lens(c), c["head_dim"]
    T, hq, hkv = sum(lens) + c["behind"], c["n_heads"] * D, c["n_kv_heads"] * D
    ends = torch.tensor([0] + lens).cumsum(0)
    s = dict(c=c, qkv=d.bf16((T, hq + 2 * hkv)), offsets=ends.to(torch.int32).to(DEV))
    # (rows behind the last document keep what their buffers hold)
    s["o"], s["lse"] = _zeros(T, hq), _zeros(c["n_heads"], T, dtype=torch.float32)
    if not c["backward"]:
        return s
    s["o"], s["lse"] = _attention_fwd(s)
    return dict(s, do=d.bf16((T, hq)), dqkv=torch.zeros_like(s["qkv"]))


def _prepare_rope(c, seed):
    d, T, D = _Draw(seed), c["tokens"], c["head_dim"]
    n = c["n_heads"] + c["n_kv_heads"]
    # positions of documents that begin anywhere in the context
    at = torch.arange(T, device=DEV) % 700 + d.ints(1 + T // 700, c["positions"])[
        torch.arange(T, device=DEV) // 700]
    s = dict(c=c, n=n, qkv=d.bf16((T, (n + c["n_kv_heads"]) * D)),
             pos=(at % c["positions"]).to(torch.int32))
    s["out"] = s["qkv"] if c["in_place"] else _zeros(T, n * D)
    s["cos"], s["sin"] = (_zeros(c["positions"], c["rot"] // 2, dtype=torch.float32)
                          for _ in range(2))
    if not c["table"]:
        for t, v in zip((s["cos"], s["sin"]), _tables(c)):
            t.copy_(v)
    return s


def _prepare_adamw(c, seed):
    """Tensors as views of flat buffers, each at a multiple of BLOCK elements."""
    d, sizes = _Draw(seed), _sizes(c)
    blocks = [-(-n // BLOCK) for n in sizes]
    start = [0]
    for b in blocks:
        start.append(start[-1] + b)
    N = start[-1]
    kept = torch.zeros(N * BLOCK, dtype=torch.bool, device=DEV)
    for b, n in zip(start, sizes):
        kept[b * BLOCK:b * BLOCK + n] = True
    kept = kept.view(N, BLOCK)
    # (rows of an embedding that no batch has touched yet: no gradient and no moments)
    live = kept & (d.uniform((N, 1)) > 0.02)
    f = dict(master=d.normal((N, BLOCK), 0.02) * kept, param=_zeros(N, BLOCK),
             grad=d.normal((N, BLOCK), 1e-3) * live)
    if c["bf16_grads"]:
        f["grad"] = f["grad"].to(torch.bfloat16)
    f["m"] = d.normal((N, BLOCK), 3e-4) * live
    f["v"] = (0.05 + d.uniform((N, BLOCK))).square_().mul_(1e-6) * live
    if c["bits"] == 8:
        for k in "mv":
            f[k], f[k + "_scale"] = (_encode_m if k == "m" else _encode_v)(f[k], 0.5)
            f[k + "_values"] = _zeros(N, BLOCK)
    s = dict(c=c, f=f, start=start, sizes=sizes, seed=d.ints(1, 1 << 30),
             # norms and biases without decay, one tensor in five with half of the rate
             decay=[0.0 if n <= 8192 else 1.0 for n in sizes],
             rate=[0.5 if i % 5 == 4 else 1.0 for i in range(len(sizes))],
             scalars=torch.tensor([3e-4, 1 - BETA1 ** 7, 1 - BETA2 ** 7, 0.8], device=DEV))
    return s


# ------------------------------------------------------------------- run ----

def run(state):
    c = state["c"]
    if own:
        return {"attention": _own_attention, "rope": _own_rope,
                "adamw": _own_adamw}[c["kind"]](state)
    if c["kind"] == "attention":
        return dict(dqkv=_attention_bwd(state)) if c["backward"] else dict(
            zip(("o", "lse"), _attention_fwd(state)))
    return _rotate(state) if c["kind"] == "rope" else _adamw_step(state)


def _bytes(n):
    return torch.empty(max(1, n), dtype=torch.uint8, device=DEV)


def _own_attention(s):
    from paper_2609_13645_amd import _lib
    c = s["c"]
    if "cfg" not in s:
        lens = _lens(c)
        s["cfg"] = _lib.attn_packed_cfg(dict(c, tokens=s["qkv"].shape[0], n_seqs=len(lens),
                                             max_seq=max(1, max(lens))))
        s["plan"] = _bytes(_lib.forge_attention_packed_plan_bytes(s["cfg"]))
        if c["backward"]:                          # (the forward's plan)
            s["ws"] = _bytes(_lib.forge_attention_packed_bwd_workspace_bytes(s["cfg"]))
            _lib.forge_attention_packed_plan(s["cfg"], s["offsets"], s["plan"])
    if c["backward"]:
        _lib.forge_attention_packed_bwd(s["cfg"], s["plan"], s["qkv"], s["o"], s["lse"], s["do"],
                                        s["dqkv"], s["ws"])
        return dict(dqkv=s["dqkv"])
    _lib.forge_attention_packed_plan(s["cfg"], s["offsets"], s["plan"])
    _lib.forge_attention_packed_fwd(s["cfg"], s["plan"], s["qkv"], s["o"], s["lse"])
    return dict(o=s["o"], lse=s["lse"])


def _own_rope(s):
    from paper_2609_13645_amd import _lib
    c = s["c"]
    if "cfg" not in s:
        s["cfg"] = _lib.rope_part_cfg(dict(
            head_dim=c["head_dim"], rot_dim=c["rot"], rot_offset=c["offset"],
            interleaved=c["interleaved"], scaling=c["scaling"], factor=c["factor"],
            low_turns=c["low"], high_turns=c["high"], original_positions=c["original"],
            amplitude=c["amplitude"]))
    if c["table"]:
        _lib.forge_rope_part_table(s["cfg"], None, c["positions"], c["base"], s["cos"], s["sin"])
    _lib.forge_rope_part_apply(s["cfg"], s["qkv"], s["qkv"].shape[1], s["out"],
                               s["out"].shape[1], s["cos"], s["sin"], s["pos"], c["tokens"],
                               c["positions"], s["n"], c["backward"])
    return s["out"]


def _own_adamw(s):
    from paper_2609_13645_amd import _lib
    c, f = s["c"], s["f"]
    if "list" not in s:
        def view(k, i):
            if k not in f:
                return None
            return f[k][s["start"][i]:] if k.endswith("scale") else \
                f[k][s["start"][i]:s["start"][i + 1]].view(-1)
        each = [dict({k: view(k, i) for k in ("master", "param", "grad", "m", "v", "m_scale",
                                              "v_scale")},
                     n=n, lr_scale=s["rate"][i], decay_scale=s["decay"][i])
                for i, n in enumerate(s["sizes"])]
        s["list"] = _lib.adamw_multi_tensors(each)
        s["hp"] = _lib.AdamwHparams(BETA1, BETA2, ADAM_EPS, DECAY)
        if c["bits"] == 8:
            s["values"] = [_lib.pointers([view(k + "_values", i) for i in range(len(each))])
                           for k in "mv"]
    _lib.forge_adamw_multi_step(s["list"], c["bits"], c["bf16_grads"], s["hp"], s["scalars"],
                                None if c["nearest"] else s["seed"])
    if c["bits"] == 32:
        return {k: f[k] for k in ("master", "param", "m", "v")}
    # the moments as the values that their codes stand for
    _lib.forge_adamw_multi_read(s["list"], s["values"][0], s["values"][1], True)
    return dict(master=f["master"], param=f["param"], m=f["m_values"], v=f["v_values"])


# ------------------------------------------------- plain form: attention ----

def _block(c):
    """Queries of one block of the plain attention: what they see lies in that block of keys and
    the one before; a single block has none before."""
    lens = _lens(c)
    reach = min(max(lens), c["window"] or max(lens))
    return max(1, min(max(reach, 64), sum(lens) + c["behind"]))


def _held(c):
    """Scores of a head that are held at once."""
    T, blk = sum(_lens(c)) + c["behind"], _block(c)
    n = -(-T // blk)
    return n * blk * blk * min(n, 2)


def _in_blocks(y, c, heads):
    """Rows [T, heads * e] -> [blocks, kv, heads / kv * blk, e]."""
    blk, kv = _block(c), c["n_kv_heads"]
    n = -(-y.shape[0] // blk)
    y = torch.cat((y, y.new_zeros(n * blk - y.shape[0], y.shape[1])))
    y = y.view(n, blk, kv, heads // kv, -1).permute(0, 2, 3, 1, 4)
    return y.reshape(n, kv, heads // kv * blk, -1)


def _rows(y, c, heads):
    """The other way, without the rows that fill the last block."""
    blk, kv = _block(c), c["n_kv_heads"]
    T = sum(_lens(c)) + c["behind"]
    y = y.view(y.shape[0], kv, heads // kv, blk, -1).permute(0, 3, 1, 2, 4)
    return y.reshape(-1, heads * y.shape[4])[:T]


def _with_before(y):
    """Each block's keys behind those of the block before."""
    return y if len(y) == 1 else torch.cat((torch.cat((torch.zeros_like(y[:1]), y[:-1])), y), 2)


def _added_up(y, c):
    """Gradients of _with_before's keys, a block's own and its share of the next block's."""
    if len(y) == 1:
        return y
    blk = _block(c)
    out = y[:, :, blk:].clone()
    out[:-1] += y[1:, :, :blk]
    return out


def _seen(s):
    """(mask [blocks, 1, 1, blk, keys] of what each query sees, rows [T] of a document)."""
    c, blk = s["c"], _block(s["c"])
    off = s["offsets"].long()
    T = s["qkv"].shape[0]
    n = -(-T // blk)
    i = torch.arange(n * blk, device=DEV)
    doc = torch.searchsorted(off[1:], i, right=True)
    inside = i < off[-1]
    first = off[doc.clamp_max(len(off) - 2)]
    if c["window"]:
        first = torch.maximum(first, i - (c["window"] - 1))
    i, first = i.view(n, blk, 1), torch.where(inside, first, n * blk).view(n, blk, 1)
    j = torch.arange(min(n, 2) * blk, device=DEV) - (min(n, 2) - 1) * blk
    j = torch.arange(n, device=DEV).view(n, 1, 1) * blk + j
    return ((j >= first) & (j <= i))[:, None, None], inside[:T]


def _split(s):
    c, D = s["c"], s["c"]["head_dim"]
    hq, hkv = c["n_heads"] * D, c["n_kv_heads"] * D
    q, k, v = s["qkv"].float().split((hq, hkv, hkv), 1)
    kv = c["n_kv_heads"]
    return (_in_blocks(q, c, c["n_heads"]), _with_before(_in_blocks(k, c, kv)),
            _with_before(_in_blocks(v, c, kv)))


def _scores(q, k, seen, c):
    z = (q @ k.transpose(-1, -2).contiguous()).mul_(c["head_dim"] ** -0.5)
    z.view(*z.shape[:2], -1, _block(c), z.shape[-1]).masked_fill_(~seen, -math.inf)
    return z


def _attention_fwd(s):
    c = s["c"]
    q, k, v = _split(s)
    seen, inside = _seen(s)
    z = _scores(q, k, seen, c)
    top = z.amax(-1, keepdim=True).clamp_min_(-1e30)
    z = z.sub_(top).exp_()
    total = z.sum(-1, keepdim=True)
    o = _rows((z @ v) / total.clamp_min(1e-30), c, c["n_heads"]).to(torch.bfloat16)
    lse = _rows(top + total.log(), c, c["n_heads"])
    keep = inside[:, None]
    return torch.where(keep, o, s["o"]), torch.where(keep, lse, s["lse"].t()).t().contiguous()


def _attention_bwd(s):
    c, kv, nh, D = s["c"], s["c"]["n_kv_heads"], s["c"]["n_heads"], s["c"]["head_dim"]
    q, k, v = _split(s)
    seen, inside = _seen(s)
    do = s["do"].float()
    delta = (do * s["o"].float()).view(-1, nh, D).sum(-1)
    do, delta, lse = (_in_blocks(y, c, nh) for y in (do, delta, s["lse"].t()))
    p = _scores(q, k, seen, c).sub_(lse).exp_()
    dv = _added_up(p.transpose(-1, -2).contiguous() @ do, c)
    ds = (do @ v.transpose(-1, -2).contiguous()).sub_(delta).mul_(p).mul_(D ** -0.5)
    dq = _rows(ds @ k, c, nh)
    dk = _added_up(ds.transpose(-1, -2).contiguous() @ q, c)
    out = torch.cat((dq, _rows(dk, c, kv), _rows(dv, c, kv)), 1).to(torch.bfloat16)
    return torch.where(inside[:, None], out, s["dqkv"])


# ------------------------------------------------------ plain form: rope ----

def _frequencies(c):
    """Angle of every pair for one position, in 64 bits: positions may be far."""
    r, f = c["rot"], c["factor"]
    base = c["base"] * f ** (r / (r - 2)) if c["scaling"] == "base" else c["base"]
    w = base ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEV) / r)
    if c["scaling"] == "linear":
        return w / f
    if c["scaling"] == "parts":
        turns = c["original"] * w / (2 * math.pi)
        keep = ((turns - c["low"]) / (c["high"] - c["low"])).clamp(0, 1)
        return w * (keep + (1 - keep) / f)
    return w


def _tables(c):
    at = torch.arange(c["positions"], dtype=torch.float64, device=DEV)
    angle = at[:, None] * _frequencies(c)
    return (angle.cos() * c["amplitude"]).float(), (angle.sin() * c["amplitude"]).float()


def _rotate(s):
    c, T, n, r, first = s["c"], s["c"]["tokens"], s["n"], s["c"]["rot"], s["c"]["offset"]
    cos, sin = _tables(c) if c["table"] else (s["cos"], s["sin"])
    at = s["pos"].long()
    cos, sin = cos[at][:, None], sin[at][:, None]
    if c["backward"]:
        sin = -sin
    x = s["qkv"][:, :n * c["head_dim"]].view(T, n, -1)
    part = x[..., first:first + r].float()
    x1, x2 = (part[..., 0::2], part[..., 1::2]) if c["interleaved"] else part.chunk(2, -1)
    y1, y2 = x1 * cos - x2 * sin, x2 * cos + x1 * sin
    y = torch.stack((y1, y2), -1).flatten(-2) if c["interleaved"] else torch.cat((y1, y2), -1)
    out = s["out"][:, :n * c["head_dim"]].view(T, n, -1)
    if not c["in_place"]:
        out.copy_(x)
    out[..., first:first + r] = y.to(torch.bfloat16)
    return s["out"]


# ----------------------------------------------------- plain form: AdamW ----

def _mixed(x):
    """32 bits from 32: two rounds of a multiplication between shifts."""
    x = ((x ^ (x >> 16)) * 0xE699D49D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0xC570DA33) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _per_block(s, values):
    """A value of each tensor for each of its blocks, [blocks, 1]."""
    count = torch.tensor(s["start"], device=DEV).diff()
    return torch.tensor(values, device=DEV).repeat_interleave(count)[:, None]


def _random(s):
    """Two numbers in (0, 1) for each element: of the seed, its tensor and its place in that."""
    if s["c"]["nearest"]:
        return 0.5, 0.5
    first = _per_block(s, [b * BLOCK for b in s["start"][:-1]])
    key = _per_block(s, list(range(len(s["sizes"]))))
    key = _mixed(key + _mixed(s["seed"].long()))
    place = torch.arange(s["start"][-1] * BLOCK, device=DEV).view(-1, BLOCK) - first
    x = _mixed(place ^ key)
    return ((x & 0xFFFF).float() + 0.5) * 2.0 ** -16, ((x >> 16).float() + 0.5) * 2.0 ** -16


def _scale(x):
    """The largest magnitude of each block; of blocks below 2^-110 zero."""
    top = x.abs().amax(1)
    return torch.where(top < 2.0 ** -110, 0.0, top)


def _encode_m(m, u):
    """Codes -127 .. 127, q for q |q| / 127^2 of the block's largest; up with the probability
    that keeps the mean (u uniform), or to the nearest (u = 0.5)."""
    s = _scale(m)
    a = m.abs() * torch.where(s > 0, 16129.0 / s, 0.0)[:, None]
    q = a.sqrt().floor()
    q = q + (u * (2 * q + 1) < a - q * q)
    return (q.clamp_max(127) * m.sign()).to(torch.int8), s


def _encode_v(v, u):
    """Codes 0 .. 255, q for (q / 255)^4 of the block's largest; a value above zero keeps a code
    above zero."""
    s = _scale(v)
    x = v * torch.where(s > 0, 4228250625.0 / s, 0.0)[:, None]
    q = x.sqrt().sqrt().floor()
    lo, hi = (q * q).square(), ((q + 1) * (q + 1)).square()
    q = q + (u * (hi - lo) < x - lo)
    return torch.where(x > 0, q.clamp(1, 255), 0.0).to(torch.uint8), s


def _decode_m(q, s):
    q = q.float()
    return (q * q.abs()) * (s * (1 / 16129.0))[:, None]


def _decode_v(q, s):
    q = q.float()
    c = (q * q) * (1 / 65025.0)
    return (c * c) * s[:, None]


def _adamw_step(s):
    c, f = s["c"], s["f"]
    lr, bc1, bc2, clip = s["scalars"]
    b1, b2 = (float(torch.tensor(b)) for b in (BETA1, BETA2))    # (as 32 bits hold them)
    small = c["bits"] == 8
    m, v = (_decode_m(f["m"], f["m_scale"]), _decode_v(f["v"], f["v_scale"])) if small else (
        f["m"], f["v"])
    g = f["grad"].float() * clip
    m = m * b1 + (1 - b1) * g
    v = v * b2 + ((1 - b2) * g) * g
    update = (m / bc1) / ((v / bc2).sqrt() + ADAM_EPS)
    update += f["master"] * (DECAY * _per_block(s, s["decay"]))
    f["master"].sub_(update.mul_(lr * _per_block(s, s["rate"])))
    f["param"].copy_(f["master"])
    if not small:
        f["m"].copy_(m)
        f["v"].copy_(v)
        return {k: f[k] for k in ("master", "param", "m", "v")}
    for k, x, u, encode, decode in zip("mv", (m, v), _random(s), (_encode_m, _encode_v),
                                       (_decode_m, _decode_v)):
        codes, scale = encode(x, u)
        f[k].copy_(codes)
        f[k + "_scale"].copy_(scale)
        f[k + "_values"].copy_(decode(codes, scale))
    return dict(master=f["master"], param=f["param"], m=f["m_values"], v=f["v_values"])


# ------------------------------------------------------------------ work ----

def _pairs(c):
    """(query, key) pairs that see each other, of one head."""
    return sum(w * (w + 1) // 2 + (n - w) * w for n in _lens(c) for w in [min(n, c["window"] or n)])


def work(case):
    c = case
    if c["kind"] == "attention":
        T, hq, hkv = sum(_lens(c)), c["n_heads"] * c["head_dim"], c["n_kv_heads"] * c["head_dim"]
        pairs = _pairs(c) * c["n_heads"] * c["head_dim"]
        if c["backward"]:
            return dict(bytes=2 * T * (4 * hq + 4 * hkv) + 4 * T * c["n_heads"], flops=10 * pairs)
        return dict(bytes=2 * T * (2 * hq + 2 * hkv) + 4 * T * c["n_heads"], flops=4 * pairs)
    if c["kind"] == "rope":
        T, n = c["tokens"], c["n_heads"] + c["n_kv_heads"]
        width = c["rot"] if c["in_place"] else c["head_dim"]
        rows = c["positions"] if c["table"] else min(T, c["positions"])
        return dict(bytes=4 * T * n * width + 4 * T + 4 * rows * c["rot"],
                    flops=3 * T * n * c["rot"])
    n, blocks = sum(_sizes(c)), sum(-(-n // BLOCK) for n in _sizes(c))
    grad = 2 if c["bf16_grads"] else 4
    if c["bits"] == 32:
        return dict(bytes=n * (26 + grad), flops=16 * n)
    # (with the values that the moments stand for, written in bf16)
    return dict(bytes=n * (14 + grad + 4) + 16 * blocks, flops=60 * n)


# ----------------------------------------------------------------- exact ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "rope": _exact_rope,
            "adamw": _exact_adamw}[case["kind"]](s)


def _exact_attention(s):
    c, D, nh, kv = s["c"], s["c"]["head_dim"], s["c"]["n_heads"], s["c"]["n_kv_heads"]
    T = s["qkv"].shape[0]
    x = s["qkv"].view(T, nh + 2 * kv, D)
    o, lse = s["o"].double().view(T, nh, D), s["lse"].double()
    dx = torch.zeros((T, nh + 2 * kv, D), dtype=torch.float64, device=DEV)
    at = 0
    for n in _lens(c):
        rows, at = slice(at, at + n), at + n
        i, j = torch.arange(n, device=DEV)[:, None], torch.arange(n, device=DEV)
        hidden = (j > i) | (i - j >= (c["window"] or n + 1))
        for h in range(nh if n else 0):
            m = nh + h // (nh // kv)
            q, k, v = (x[rows, e].double() for e in (h, m, m + kv))
            z = (q @ k.t().contiguous()).mul_(D ** -0.5).masked_fill_(hidden, -math.inf)
            if not c["backward"]:
                lse[h, rows] = z.logsumexp(1)
                o[rows, h] = z.softmax(1) @ v
                continue
            p = z.sub_(lse[h, rows, None]).exp_()
            do = s["do"].view(T, nh, D)[rows, h].double()
            t = (do * o[rows, h]).sum(1, keepdim=True)
            dx[rows, m + kv] += p.t() @ do
            p.mul_((do @ v.t().contiguous()).sub_(t)).mul_(D ** -0.5)
            dx[rows, h] = p @ k
            dx[rows, m] += p.t() @ q
    return dict(dqkv=dx.view(T, -1)) if c["backward"] else dict(o=o.view(T, -1), lse=lse)


def _exact_rope(s):
    c, T, r = s["c"], s["c"]["tokens"], s["c"]["rot"]
    w = []
    for i in range(r // 2):
        b = c["base"] ** (-2.0 * i / r)
        if c["scaling"] == "linear":
            b /= c["factor"]
        elif c["scaling"] == "base":
            b *= c["factor"] ** (-2.0 * i / (r - 2))
        elif c["scaling"] == "parts":
            g = (c["original"] * b / (2 * math.pi) - c["low"]) / (c["high"] - c["low"])
            g = min(1.0, max(0.0, g))
            b = g * b + (1.0 - g) * b / c["factor"]
        w.append(b)
    angle = s["pos"].double()[:, None] * torch.tensor(w, dtype=torch.float64, device=DEV)
    size = torch.full_like(angle, c["amplitude"])
    turn = torch.polar(size, -angle if c["backward"] else angle)[:, None]
    y = s["out"].double()
    heads = y[:, :s["n"] * c["head_dim"]].view(T, s["n"], -1)
    heads.copy_(s["qkv"][:, :s["n"] * c["head_dim"]].view(T, s["n"], -1))
    part = heads[..., c["offset"]:c["offset"] + r]
    pairs = part.unflatten(-1, (r // 2, 2) if c["interleaved"] else (2, r // 2))
    if not c["interleaved"]:
        pairs = pairs.transpose(-1, -2)
    z = torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * turn
    z = torch.stack((z.real, z.imag), -1 if c["interleaved"] else -2)
    heads[..., c["offset"]:c["offset"] + r] = z.flatten(-2)
    return y


def _exact_adamw(s):
    c, f = s["c"], s["f"]
    lr, bc1, bc2, clip = s["scalars"].double().tolist()
    b1, b2 = (float(torch.tensor(b)) for b in (BETA1, BETA2))
    out = {k: torch.zeros_like(f["master"], dtype=torch.float64)
           for k in ("master", "param", "m", "v")}
    seed = _mixed(s["seed"].long())
    for t, n in enumerate(s["sizes"]):
        rows = slice(s["start"][t], s["start"][t + 1])
        m, v = f["m"][rows].double(), f["v"][rows].double()
        if c["bits"] == 8:
            m = m * m.abs() / 127.0 ** 2 * f["m_scale"][rows, None].double()
            v = (v / 255.0) ** 4 * f["v_scale"][rows, None].double()
        g, p = f["grad"][rows].double() * clip, f["master"][rows].double()
        m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g ** 2
        p = p - lr * s["rate"][t] * (m / bc1 / ((v / bc2) ** 0.5 + ADAM_EPS)
                                     + DECAY * s["decay"][t] * p)
        out["master"][rows], out["param"][rows] = p, p
        if c["bits"] == 8:
            x = _mixed(torch.arange(len(m) * BLOCK, device=DEV) ^ _mixed(seed + t)).view(m.shape)
            u = [0.5, 0.5] if c["nearest"] else [((x % 65536).double() + 0.5) / 65536,
                                                 ((x // 65536).double() + 0.5) / 65536]
            sm, sv = m.abs().amax(1, keepdim=True), v.amax(1, keepdim=True)
            a = m.abs() / sm.clamp_min(1e-300) * 127.0 ** 2
            q = (a ** 0.5).floor().clamp_max(126)
            q = q + (a - q ** 2 > u[0] * ((q + 1) ** 2 - q ** 2))
            m = m.sign() * q ** 2 / 127.0 ** 2 * sm
            a = v / sv.clamp_min(1e-300) * 255.0 ** 4
            q = (a ** 0.25).floor().clamp_max(254)
            q = q + (a - q ** 4 > u[1] * ((q + 1) ** 4 - q ** 4))
            v = torch.where(v > 0, q.clamp_min(1), 0.0) ** 4 / 255.0 ** 4 * sv
        out["m"][rows], out["v"][rows] = m, v
    return out
