"""What a decoder does between its projections, measured: a paged key-value cache that is written (rotary embedding,
bf16 or int8 as the layer's activations are quantised) and read back, attention of one new token per sequence over it,
and the norms before and after a block with its gate and residual scale, forward and backward.

A case is a dict of plain values; `prepare` makes a user's tensors on the GPU from a seed; `run` is one pass, in elementary
torch operations or, with `own`, through the library's entry points; `exact` is the same from the definitions in 64 bits.

Cache layout: K, V [page][head][position in the page][pitch], pitch = head_dim rounded up to 16 bytes (zeros behind head_dim); int8
codes come with one gamma = 128 / max(max|x|, 1e-5) per position and head and stand for code / gamma.
"""
import math

import torch

own = False
DEV = "cuda:0"
EPS = 1e-5


def listed():
    return [
        # ---- attention of one new token per sequence over the cache
        # a lone sequence a few pages long, 16 heads of 128 (the 1.3B decoder's): what a small call costs
        dict(name="attend_one", kind="attend", n=1, most=200, heads=16, group=1, dim=128, page=16, int8=False),
        # sixteen ragged sequences of the same decoder up to its training length, one slot idle
        dict(name="attend_16x2048", kind="attend", n=16, most=2048, heads=16, group=1, dim=128, page=64, int8=False),
        # the 3B shape, hidden 3200 in 32 heads of 100, int8 cache, sixteen ragged sequences
        dict(name="attend_16x2048_d100_int8", kind="attend", n=16, most=2048, heads=32, group=1, dim=100, page=32, int8=True),
        # one very long sequence, four query heads to a key-value head, int8 cache: few rows, a long axis
        dict(name="attend_long_int8", kind="attend", n=1, most=131072, heads=8, group=4, dim=128, page=128, int8=True),
        # a busy server: 64 ragged sequences, grouped heads
        dict(name="attend_64x4096", kind="attend", n=64, most=4096, heads=8, group=4, dim=128, page=64, int8=False),
        # a step as it is used: the new token of each of four sequences is rotated, quantised and written, then attends
        dict(name="step_4x1000_int8", kind="step", n=4, most=1000, heads=16, group=1, dim=128, page=32, int8=True),
        # ---- prompts: new tokens are written behind what a sequence holds, then its history is read back
        # four prompts of 2048 into an empty bf16 cache
        dict(name="fill_4x2048", kind="fill", n=4, past=0, new=2048, heads=16, group=1, dim=128, page=64, int8=False),
        # ragged chunks behind a ragged past, heads of 100, int8
        dict(name="fill_7x333_int8", kind="fill", n=7, past=700, new=333, heads=32, group=1, dim=100, page=32, int8=True),
        # ---- norms around a block
        # decode: one token of the 3B width, residual add and the norm in front of the next block
        dict(name="norm_1x3200", kind="norm", T=1, N=3200, post=False, gate="none"),
        # training: 8192 tokens of the 1.3B width with the norm behind the block, a gate per feature and a residual scale
        dict(name="norm_8192x2048_full", kind="norm", T=8192, N=2048, post=True, gate="vector"),
        # its backward
        dict(name="norm_grad_8192x2048_full", kind="norm_grad", T=8192, N=2048, post=True, gate="vector"),
        # backward of the plain residual add and norm, an odd number of tokens, the 3B width
        dict(name="norm_grad_999x3200", kind="norm_grad", T=999, N=3200, post=False, gate="scalar"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "step", "fill", "fill", "norm", "norm_grad"])
    if kind in ("norm", "norm_grad"):
        while True:
            T, N = _log(rng, 1, 16384), 8 * _log(rng, 8, 1080)
            if T * N <= 8192 * 2048:
                return dict(kind=kind, T=T, N=N, post=rng.random() < 0.5, gate=rng.choice(["none", "scalar", "vector"]))
    shape = dict(heads=rng.choice([1, 2, 4, 8, 16, 20, 32]), group=rng.choice([1, 1, 2, 4, 5, 8, 16]), dim=rng.choice([64, 80, 96, 100, 128, 128, 192, 256]),
                 page=rng.choice([16, 32, 48, 64, 128, 256]), int8=rng.random() < 0.5)
    cost = shape["heads"] * shape["dim"]
    if kind == "fill":
        shape["group"] = min(shape["group"], 2)
        while True:
            n, past, new = _log(rng, 1, 64), rng.choice([0, _log(rng, 1, 4096)]), _log(rng, 1, 4096)
            if n * (past + new) * cost <= 4 * 2048 * 16 * 128:
                return dict(kind=kind, n=n, past=past, new=new, **shape)
    while True:
        n, most = _log(rng, 1, 256), _log(rng, 1, 131072)
        if n * most * cost * (1 + shape["group"] / 16) <= 64 * 4096 * 8 * 128:
            return dict(kind=kind, n=n, most=most, **shape)


def _lengths(c):
    """Positions each sequence holds, the new token among them: ragged between a quarter of the longest and all of it; of eight or
    more sequences the last is an idle slot."""
    n, most = c["n"], c["most"]
    lens = [most - (i * 7919) % max(1, most - most // 4) for i in range(n)]
    if n >= 8 and c["kind"] == "attend":
        lens[-1] = 0
    return lens


def _spans(c):
    """(tokens held before, new tokens) of each sequence of a fill."""
    return [(c["past"] - (i * 331) % (c["past"] // 2 + 1), c["new"] - (i * 57) % (c["new"] // 4 + 1)) for i in range(c["n"])]


def _pitch(c):
    return -(-c["dim"] // 16) * 16 if c["int8"] else -(-c["dim"] // 8) * 8


# --------------------------------------------------------------------------- inputs
class State:
    def __init__(self, c):
        self.c = c


def _normal(g, *shape, dtype=torch.bfloat16, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(dtype)


def _cache(s, g, held):
    """Pages in no order, and a table that names a sequence's pages and -1 behind them; all pages hold tokens of some kind."""
    c, page = s.c, s.c["page"]
    need = [-(-h // page) for h in held]
    s.width, pages = max(1, max(need)), sum(need) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    row = torch.repeat_interleave(torch.arange(len(need), device=DEV), torch.tensor(need, device=DEV))
    col = torch.tensor([j for k in need for j in range(k)], device=DEV, dtype=torch.int64)
    s.table = torch.full((len(need), s.width), -1, dtype=torch.int32, device=DEV)
    s.table[row, col] = order[:len(row)]
    shape = (pages, c["heads"], page, _pitch(c))
    s.kg = s.vg = None
    if c["int8"]:
        s.k, s.v = (torch.randint(-128, 128, shape, generator=g, device=DEV, dtype=torch.int8) for _ in range(2))
        s.kg, s.vg = (128.0 / (torch.rand(shape[:3], generator=g, device=DEV) * 2 + 1.5) for _ in range(2))
    else:
        s.k, s.v = _normal(g, *shape), _normal(g, *shape)
    s.k[..., c["dim"]:] = 0
    s.v[..., c["dim"]:] = 0


def _new_tokens(s, g, seq, pos):
    """Projections of the new tokens [tokens, heads * dim], where they go, and the rotary tables."""
    c, n = s.c, len(seq)
    s.seq, s.pos = (torch.tensor(a, dtype=torch.int32, device=DEV) for a in (seq, pos))
    q_heads = c["heads"] * c["group"]
    s.q_in = _normal(g, n, q_heads * c["dim"])
    s.k_in, s.v_in = _normal(g, n, c["heads"] * c["dim"]), _normal(g, n, c["heads"] * c["dim"])
    half = c["dim"] // 2
    angle = torch.outer(torch.arange(max(pos) + 1, device=DEV, dtype=torch.float64),
                        10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half))
    s.cos, s.sin = angle.cos().float(), angle.sin().float()
    s.q = torch.empty_like(s.q_in)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s, c = State(case), case
    if c["kind"] in ("attend", "step"):
        lens = _lengths(c)
        _cache(s, g, lens)
        s.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s.q = _normal(g, c["n"], c["heads"] * c["group"] * c["dim"])
        if c["kind"] == "step":
            _new_tokens(s, g, list(range(c["n"])), [x - 1 for x in lens])
        s.out = torch.empty_like(s.q)
    elif c["kind"] == "fill":
        spans = _spans(c)
        _cache(s, g, [a + b for a, b in spans])
        _new_tokens(s, g, [i for i, (a, b) in enumerate(spans) for _ in range(b)], [j for a, b in spans for j in range(a, a + b)])
        s.all_seq = torch.tensor([i for i, (a, b) in enumerate(spans) for _ in range(a + b)], dtype=torch.int32, device=DEV)
        s.all_pos = torch.tensor([j for a, b in spans for j in range(a + b)], dtype=torch.int32, device=DEV)
        s.k_out, s.v_out = (torch.empty((len(s.all_seq), c["heads"] * c["dim"]), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    else:
        T, N = c["T"], c["N"]
        s.x, s.y = _normal(g, T, N, std=2.0), _normal(g, T, N)
        gain = lambda: (1 + 0.1 * torch.randn(N, generator=g, device=DEV)).to(torch.bfloat16)  # noqa: E731
        s.w_pre, s.w_post = gain(), gain() if c["post"] else None
        s.gate = None if c["gate"] == "none" else torch.rand(N if c["gate"] == "vector" else 1, generator=g, device=DEV) + 0.5
        s.scale = 1.0 if c["gate"] == "none" else 0.9
        if c["kind"] == "norm":
            s.x_out, s.h = torch.empty_like(s.x), torch.empty_like(s.x)
        else:   # x is the stream behind the block; dxo and dh come from what follows
            s.dxo, s.dh = (_normal(g, T, N, dtype=torch.float32) + 0.05 * s.y).to(torch.bfloat16), _normal(g, T, N)
            s.dx, s.dy = torch.empty_like(s.x), torch.empty_like(s.x)
            s.dpre = torch.empty(N, device=DEV)
            s.dpost = torch.empty(N, device=DEV) if c["post"] else None
            s.dgate = None if s.gate is None else torch.empty_like(s.gate)
    if own:
        _handles(s)
    return s


def _handles(s):
    """The descriptors and workspaces that a program keeps."""
    from paper_2602_22592_b200 import binding as pqb
    s.lib, c = pqb, s.c
    if c["kind"] in ("norm", "norm_grad"):
        s.desc = pqb.make_norm_desc(c["T"], c["N"], EPS, s.scale, c["gate"] == "vector")
        if c["kind"] == "norm_grad":
            s.ws = torch.empty(pqb.pq_block_norm_workspace_bytes(s.desc), dtype=torch.uint8, device=DEV)
        return
    s.cache = pqb.make_kv_cache(s.k, s.v, s.table, c["dim"], s.kg, s.vg)
    if c["kind"] != "fill":
        s.ws = torch.empty(pqb.pq_attn_workspace_bytes(s.cache, c["heads"] * c["group"]), dtype=torch.uint8, device=DEV)


# --------------------------------------------------------------------------- the plain forms
def _rotate(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)


def _write(s):
    """Rotates queries and keys, and writes keys and values behind what the sequences hold."""
    c, page = s.c, s.c["page"]
    pos = s.pos.long()
    cos, sin = s.cos[pos][:, None], s.sin[pos][:, None]
    q = _rotate(s.q_in.view(len(pos), -1, c["dim"]), cos, sin)
    k, v = _rotate(s.k_in.view(len(pos), -1, c["dim"]), cos, sin), s.v_in.view(len(pos), -1, c["dim"])
    slot = (s.table[s.seq.long(), pos // page].long(), slice(None), pos % page)
    for rows, to, gam in ((k, s.k, s.kg), (v, s.v, s.vg)):
        if c["int8"]:
            rows = rows.float()
            gamma = 128.0 / rows.abs().amax(-1, keepdim=True).clamp_min(1e-5)
            rows = torch.round(rows * gamma).clamp(-128, 127).to(torch.int8)
            gam[slot] = gamma[..., 0]
        to[..., :c["dim"]][slot] = rows
    return q.view(len(pos), -1)


def _values(s, pages, gam):
    """What the cached rows stand for, in 32 bits."""
    x = pages[..., :s.c["dim"]].float()
    return x if gam is None else x / gam[..., None]


def _read(s):
    pos = s.all_pos.long()
    page, at = s.table[s.all_seq.long(), pos // s.c["page"]].long(), pos % s.c["page"]
    return [_values(s, x[page, :, at], None if gam is None else gam[page, :, at]).to(torch.bfloat16).view(len(pos), -1)
            for x, gam in ((s.k, s.kg), (s.v, s.vg))]


def _attend(s, q):
    c, n = s.c, s.c["n"]
    table = s.table.long().clamp_min(0)
    held = torch.arange(s.width * c["page"], device=DEV)[None] < s.lens[:, None]              # [n, positions]
    k, v = (_values(s, x[table], None if gam is None else gam[table]).transpose(1, 2).reshape(n, c["heads"], -1, c["dim"])
            for x, gam in ((s.k, s.kg), (s.v, s.vg)))
    v = torch.where(held[:, None, :, None], v, torch.zeros((), device=DEV))
    score = q.float().view(n, c["heads"], c["group"], c["dim"]) @ k.transpose(2, 3) * c["dim"] ** -0.5
    score = score.masked_fill(~held[:, None, None], -torch.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -torch.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / torch.where(total == 0, torch.ones_like(total), total)                  # a row that sees nothing is zero
    return out.to(torch.bfloat16).view(n, -1)


def _rms(x):
    return torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)


def _norm(s):
    u = s.y.float()
    if s.w_post is not None:
        u = u * _rms(u) * s.w_post.float()
    if s.gate is not None:
        u = u * s.gate
    x = s.scale * s.x.float() + u
    return {"x": x.to(torch.bfloat16), "h": (x * _rms(x) * s.w_pre.float()).to(torch.bfloat16)}


def _norm_back(g, x, w):
    """Gradients of x rms(x) w with respect to x and, summed over the tokens, w."""
    r = _rms(x)
    n = x * r
    gw = g * w
    return r * (gw - n * (gw * n).mean(-1, keepdim=True)), (g * n).double().sum(0).float()


def _norm_grad(s):
    d, dpre = _norm_back(s.dh.float(), s.x.float(), s.w_pre.float())
    g = s.dxo.float() + d
    out = {"dx": (s.scale * g).to(torch.bfloat16), "dpre": dpre}
    u = y = s.y.float()
    if s.w_post is not None:
        u = y * _rms(y) * s.w_post.float()
    if s.gate is not None:
        gu = (g * u).double()    # long sums
        out["dgate"] = (gu.sum(0) if s.gate.numel() > 1 else gu.sum().view(1)).float()
        g = g * s.gate
    if s.w_post is not None:
        g, out["dpost"] = _norm_back(g, y, s.w_post.float())
    if s.gate is not None or s.w_post is not None:
        out["dy"] = g.to(torch.bfloat16)
    return out


# --------------------------------------------------------------------------- one pass
def run(s):
    c = s.c
    if c["kind"] in ("attend", "step"):
        if not own:
            if c["kind"] == "step":
                s.q = _write(s)
            return {"q": s.q, "out": _attend(s, s.q)} if c["kind"] == "step" else {"out": _attend(s, s.q)}
        if c["kind"] == "step":
            s.lib.pq_kv_append(s.cache, s.seq, s.pos, s.k_in, s.v_in, s.cos, s.sin, s.q_in, s.q)
        s.lib.pq_attn_decode(s.cache, s.q, s.lens, c["dim"] ** -0.5, s.out, None, s.ws)
        return {"q": s.q, "out": s.out} if c["kind"] == "step" else {"out": s.out}
    if c["kind"] == "fill":
        if not own:
            q = _write(s)
            k, v = _read(s)
            return {"q": q, "k": k, "v": v}
        s.lib.pq_kv_append(s.cache, s.seq, s.pos, s.k_in, s.v_in, s.cos, s.sin, s.q_in, s.q)
        s.lib.pq_kv_read(s.cache, s.all_seq, s.all_pos, s.k_out, s.v_out)
        return {"q": s.q, "k": s.k_out, "v": s.v_out}
    if c["kind"] == "norm":
        if not own:
            return _norm(s)
        s.lib.pq_block_norm_forward(s.desc, s.x, s.y, s.w_post, s.gate, s.w_pre, s.x_out, s.h)
        return {"x": s.x_out, "h": s.h}
    if not own:
        return _norm_grad(s)
    both = s.w_post is not None or s.gate is not None    # else the block's gradient is the stream's
    s.lib.pq_block_norm_backward(s.desc, s.dxo, s.dh, s.x, s.y if both else None, s.w_post, s.gate, s.w_pre, s.dx, s.dy if both else None,
                                 s.dpost, s.dgate, s.dpre, s.ws)
    out = {"dx": s.dx, "dpre": s.dpre}
    if s.gate is not None:
        out["dgate"] = s.dgate
    if s.w_post is not None:
        out["dpost"] = s.dpost
    if both:
        out["dy"] = s.dy
    return out


def work(case):
    c = case
    if c["kind"] in ("norm", "norm_grad"):
        T, N = c["T"], c["N"]
        if c["kind"] == "norm":
            return {"bytes": 2 * 4 * T * N + 2 * N, "flops": 8 * T * N}
        both = c["post"] or c["gate"] != "none"
        return {"bytes": 2 * (6 if both else 4) * T * N + 6 * N, "flops": 16 * T * N}
    row = 2 * c["heads"] * (c["dim"] + 4 if c["int8"] else 2 * c["dim"])        # keys and values of a position
    q = 2 * c["heads"] * c["group"] * c["dim"]
    kv = 4 * c["heads"] * c["dim"]
    if c["kind"] == "fill":
        spans = _spans(c)
        new, held = sum(b for a, b in spans), sum(a + b for a, b in spans)
        return {"bytes": new * (2 * q + kv + row) + held * (row + kv), "flops": new * 6 * (q + kv) // 2}
    held = sum(_lengths(c))
    step = c["n"] * (2 * q + kv + row) if c["kind"] == "step" else 0
    return {"bytes": held * row + c["n"] * 2 * q + step, "flops": 2 * held * q}


# --------------------------------------------------------------------------- the definitions in 64 bits
def _pair_rotation(x, angle_cos, angle_sin):
    """[tokens, heads, dim]: the pair (i, i + dim / 2) turned by its token's angle; bf16 is what the cache's definition keeps of it."""
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half], x[..., half:]) * torch.complex(angle_cos, angle_sin)[:, None, :]
    return torch.view_as_real(z).movedim(-1, -2).flatten(-2).to(torch.bfloat16).double()


def _kept(x, int8):
    """What the cache keeps of rows x (64 bits)."""
    if not int8:
        return x
    gamma = 128 / torch.clamp(torch.amax(torch.abs(x), dim=-1, keepdim=True), min=1e-5)
    return torch.clamp(torch.round(x * gamma), -128, 127) / gamma


def _held_rows(s, i, length, pages, gam):
    """Sequence i's first `length` rows as [length, heads, dim] in 64 bits."""
    c = s.c
    ids = s.table[i, :-(-length // c["page"])].long()
    rows = pages[ids].double()[..., :c["dim"]]
    if gam is not None:
        rows = rows / gam[ids].double().unsqueeze(-1)
    return rows.movedim(1, 2).reshape(-1, c["heads"], c["dim"])[:length]


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] in ("attend", "step"):
        q = s.q.double().view(c["n"], -1, c["dim"])
        if c["kind"] == "step":
            at = s.pos.long()
            turn = (s.cos[at].double(), s.sin[at].double())
            q = _pair_rotation(s.q_in.double().view(c["n"], -1, c["dim"]), *turn)
            k_new = _kept(_pair_rotation(s.k_in.double().view(c["n"], -1, c["dim"]), *turn), c["int8"])
            v_new = _kept(s.v_in.double().view(c["n"], -1, c["dim"]), c["int8"])
        out = torch.zeros_like(q)
        for i, length in enumerate(_lengths(c)):
            if length == 0:
                continue
            k, v = _held_rows(s, i, length, s.k, s.kg), _held_rows(s, i, length, s.v, s.vg)
            if c["kind"] == "step":
                k[-1], v[-1] = k_new[i], v_new[i]
            for h in range(c["heads"]):
                mine = slice(h * c["group"], (h + 1) * c["group"])
                weight = torch.softmax(torch.einsum("gd,td->gt", q[i, mine], k[:, h]) / math.sqrt(c["dim"]), dim=1)
                out[i, mine] = torch.einsum("gt,td->gd", weight, v[:, h])
        out = out.view(c["n"], -1)
        return {"q": q.view(c["n"], -1), "out": out} if c["kind"] == "step" else {"out": out}
    if c["kind"] == "fill":
        at = s.pos.long()
        turn = (s.cos[at].double(), s.sin[at].double())
        new = lambda x: x.double().view(len(at), -1, c["dim"])  # noqa: E731
        q, k_new = _pair_rotation(new(s.q_in), *turn), _kept(_pair_rotation(new(s.k_in), *turn), c["int8"])
        v_new = _kept(new(s.v_in), c["int8"])
        k, v, done = [], [], 0
        for i, (a, b) in enumerate(_spans(c)):
            for rows, pages, gam, fresh in ((k, s.k, s.kg, k_new), (v, s.v, s.vg, v_new)):
                rows += [_held_rows(s, i, a, pages, gam), fresh[done:done + b]]
            done += b
        return {"q": q.flatten(1), "k": torch.cat(k).flatten(1), "v": torch.cat(v).flatten(1)}
    x, y, w = s.x.double(), s.y.double(), s.w_pre.double()
    root = lambda z: torch.sqrt(z.pow(2).sum(1, keepdim=True) / c["N"] + EPS)  # noqa: E731
    wp = None if s.w_post is None else s.w_post.double()
    gate = 1.0 if s.gate is None else s.gate.double()
    u = y if wp is None else y / root(y) * wp
    if c["kind"] == "norm":
        x = s.scale * x + gate * u
        return {"x": x, "h": x / root(x) * w}
    dh, r = s.dh.double(), root(x)
    g = s.dxo.double() + (dh * w) / r - x * (dh * w * x).sum(1, keepdim=True) / (c["N"] * r ** 3)
    out = {"dx": s.scale * g, "dpre": torch.einsum("tn,tn->n", dh, x / r)}
    if s.gate is not None:
        out["dgate"] = torch.einsum("tn,tn->n", g, u)
        if s.gate.numel() == 1:
            out["dgate"] = out["dgate"].sum().view(1)
    g = g * gate
    if wp is not None:
        r = root(y)
        out["dpost"] = torch.einsum("tn,tn->n", g, y / r)
        g = (g * wp) / r - y * (g * wp * y).sum(1, keepdim=True) / (c["N"] * r ** 3)
    if s.gate is not None or wp is not None:
        out["dy"] = g
    return out
