"""Calls of the sizes that serving and training have: attention in equal shares of tiles with items over several CTAs, cache kernels whose
warps walk several units of several steps, every gradient of the norms against differences of the kernel.  Bounds as in test_gpu_between.py."""
import numpy as np
import pytest
import torch

from oracle import between_oracle as B
from paper_2602_22592_b200 import binding as pqb
from test_gpu_between import DEV, HALF, Cache, angles, bf, check_status, close_attention, f32t, f64, guarded, guards_whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,group,dim,page,lens,int8", [
    (8, 4, 128, 64, [9001, 8000, 8999, 0], False), (8, 4, 128, 128, [40007], True), (9, 20, 128, 32, [5000, 333, 2600, 1], False),
    (9, 20, 128, 32, [5000, 333, 2600, 1], True), (6, 9, 256, 16, [9000, 31, 4001], False), (6, 9, 256, 16, [9000, 31, 4001], True),
    (4, 20, 180, 48, [9000, -3, 4001], False), (4, 20, 180, 48, [9000, 31, 4001], True), (8, 16, 64, 16, [20000, 100], False), (8, 16, 64, 16, [20000, 100], True)])
def test_attention_in_equal_shares(heads, group, dim, page, lens, int8):
    # more chunks of 64 tiles (the longest that a form has) than SMs: the CTAs take equal shares, and long items lie in many of them
    cols = 8 if group <= 8 or dim > 128 else 16
    chunks = sum(-(-max(x, 0) // 1024) for x in lens) * heads * -(-group // cols)
    assert chunks > torch.cuda.get_device_properties(0).multi_processor_count
    rng = np.random.default_rng(dim + group + int8)
    C = Cache(rng, lens, heads, dim, page, int8)
    rows = C.fill(rng, lens)
    n, H = len(lens), heads * group
    q = B.bf16(rng.standard_normal((n, H, dim)) * 2)
    raw, O = guarded((n, H * dim))
    raw_l, lse = guarded((n, H), torch.float32)
    ws_raw, ws = guarded((pqb.pq_attn_workspace_bytes(C.c, H),), torch.uint8)
    ws.fill_(255)
    lt = torch.tensor(lens, dtype=torch.int32, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(n, -1), lt, dim ** -0.5, O, lse, ws)
    torch.cuda.synchronize()
    check_status()
    live = [s for s in range(n) if lens[s] >= 0]
    close_attention(O[live], lse[live], q[live], [rows[s] for s in live], dim ** -0.5, int8)
    assert all((O[s] == 7).all() and (lse[s] == 7).all() for s in range(n) if lens[s] < 0)
    assert guards_whole(raw) and guards_whole(raw_l) and guards_whole(ws_raw)
    O2 = torch.full_like(O, 7)
    pqb.pq_attn_decode(C.c, bf(q).view(n, -1), lt, dim ** -0.5, O2, None, ws)      # the workspace as the first call left it
    assert torch.equal(O2, O)


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dim", [16, 64, 100, 104, 180, 256])
def test_append_and_read_of_many_ragged_tokens(dim, int8):
    # 5000 tokens of 8 query heads and 4 + 4 cached ones, padding among them: four steps a unit, several units a warp
    rng = np.random.default_rng(dim + int8)
    heads, q_heads, page = 4, 8, 32
    past, new = [900, 0, 33, 511], [1700, 1, 1299, 2000]
    C = Cache(rng, [a + b for a, b in zip(past, new)], heads, dim, page, int8)
    seq = np.concatenate([np.full(b, s) for s, b in enumerate(new)])
    pos = np.concatenate([np.arange(a, a + b) for a, b in zip(past, new)])
    seq, pos = np.insert(seq, range(0, 5000, 37), 77), np.insert(pos, range(0, 5000, 37), -2)
    order = rng.permutation(len(seq))
    seq, pos = seq[order], pos[order]
    T, live = len(seq), pos >= 0
    k, v, q = (B.bf16(rng.standard_normal((T, h, dim)) * 3) for h in (heads, heads, q_heads))
    k[5] = 0
    cos, sin = angles(rng, int(pos.max()) + 1, dim)
    st, pt = (torch.from_numpy(a.astype(np.int32)).to(DEV) for a in (seq, pos))
    raw, Qo = guarded((T, q_heads * dim))
    want = C.bits()
    pqb.pq_kv_append(C.c, st, pt, bf(k).view(T, -1), bf(v).view(T, -1), torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV), bf(q).view(T, -1), Qo)
    torch.cuda.synchronize()
    check_status()
    at = np.maximum(pos, 0)
    k, q = B.rope(k, cos[at], sin[at]), B.rope(q, cos[at], sin[at])
    got = f64(Qo).reshape(q.shape)
    assert np.array_equal(got[live], q[live]) and (got[~live] == 7).all() and guards_whole(raw)
    pg, o = (torch.from_numpy(a).to(DEV).long() for a in (C.table_host[seq[live], pos[live] // page], pos[live] % page))
    stands = []
    for w, x in enumerate((k, v)):
        row = np.zeros((int(live.sum()), heads, C.k.shape[3]))
        if int8:
            codes, g = B.quantise(x[live])
            row[..., :dim] = codes
            want[w][pg, :, o] = torch.from_numpy(row).to(torch.int8).to(DEV)
            want[2 + w][pg, :, o] = torch.from_numpy(g).to(DEV).view(torch.int32)
            stands.append(B.bf16((codes.astype(np.float32) / g[..., None]).astype(np.float32)))
        else:
            row[..., :dim] = x[live]
            want[w][pg, :, o] = bf(row).view(torch.int16)
            stands.append(x[live])
    assert all(torch.equal(a, b) for a, b in zip(C.bits(), want))
    outs = [guarded((T, heads * dim)) for _ in range(2)]
    pqb.pq_kv_read(C.c, st, pt, outs[0][1], outs[1][1])
    torch.cuda.synchronize()
    check_status()
    for (r, out), x in zip(outs, stands):
        out = f64(out).reshape(T, heads, dim)
        assert np.array_equal(out[live], x) and (out[~live] == 7).all() and guards_whole(r)


def _without_mean(g, z, eps):
    return g / np.sqrt((z * z).mean(-1, keepdims=True) + eps)


def gradients_and_differences(post, gate, forward, backward, monkeypatch):
    """Every gradient against central differences of the forward along directions of random signs, which know nothing of the gradient.
    The inputs that are moved are moved to numbers of their type, and the product is with the move as it came out.  What a central
    difference is off by itself is computed in 64 bits, from the same two points.  An output's rounding to bf16 moves it by up to 2^-8 of
    itself, a deviation of 2^-8 / sqrt(3) at most: six deviations of the sum; a gradient's own rounding, and that of the stream which it
    is made from, likewise.  The same products with gradients that miss a term have to fall outside."""
    rng = np.random.default_rng(51)
    T, N, eps, scale = 48, 512, 1e-5, 0.75
    x, y = B.bf16(rng.standard_normal((T, N)) * 2), B.bf16(rng.standard_normal((T, N)))
    pre, pw = B.bf16(1 + 0.2 * rng.standard_normal(N)), B.bf16(1 + 0.2 * rng.standard_normal(N)) if post else None
    gv = None if gate == "none" else rng.uniform(0.5, 1.5, N if gate == "vector" else 1).astype(np.float32).astype(np.float64)
    # along x and y in part, so that what a norm takes off a gradient is not small
    ds, dh = B.bf16(rng.standard_normal((T, N)) + 0.5 * y), B.bf16(rng.standard_normal((T, N)) + 0.25 * x + y)
    names = ["dx", "dy", "dpost", "dgate", "dpre"]
    args = [x, y, pw, gv, pre]

    def loss(xo, h):
        return (xo * ds).sum() + (h * dh).sum()

    def exact(a):
        return loss(*B.block_norm(*a, scale, eps))

    s = B.block_norm(*args, scale, eps)[0]
    got = backward(ds, dh, *args, scale, eps)

    def formula(ds, dh, half=False):
        out = B.block_norm_backward(ds, dh, s, y, pw, gv, None if dh is None else pre, scale, eps)
        if gate == "scalar":
            out["dgate"] = out["dgate"].sum(keepdims=True)
        return {k: np.where(np.arange(v.shape[-1]) < N // 2, v, 0) if half and v.size > 1 else v for k, v in out.items()}
    right = formula(ds, dh)
    wrong = [formula(ds, None), formula(None, dh), formula(ds, dh, True)]
    with monkeypatch.context() as mp:
        mp.setattr(B, "rms_backward", _without_mean)
        wrong.append(formula(ds, dh))
    caught = {k: [False] * 4 for k in got}
    for i, name in enumerate(names):
        if name not in got:
            continue
        step = [0.25, 0.125, 0.0625, 0.25 if gate == "scalar" else 0.0625, 0.0625][i]
        for _ in range(6):
            way = rng.choice([-1.0, 1.0], args[i].shape)
            if name in ("dx", "dy"):           # in half of the rows along the row itself
                way[::2] = args[i][::2] / 2
            ends = []
            for e in (step, -step):
                a = list(args)
                a[i] = args[i] + e * way
                a[i] = a[i].astype(np.float32).astype(np.float64) if name == "dgate" else B.bf16(a[i])
                ends.append(a)
            move = ends[0][i] - ends[1][i]
            outs = [forward(*a, scale, eps) for a in ends]
            slope = loss(*outs[0]) - loss(*outs[1])
            off = abs(exact(ends[0]) - exact(ends[1]) - (right[name] * move).sum())
            noise = 6 * HALF / np.sqrt(3) * np.sqrt(sum(((xo * ds) ** 2).sum() + ((h * dh) ** 2).sum() for xo, h in outs))
            own = 6 * 2 * HALF / np.sqrt(3) * np.sqrt((right[name] ** 2 * move ** 2).sum())
            tol = off + noise + own
            assert abs(slope - (got[name] * move).sum()) <= tol, (name, slope, (got[name] * move).sum(), tol)
            for j, other in enumerate(wrong):
                caught[name][j] |= bool(abs(slope - (other.get(name, np.zeros(1)) * move).sum()) > tol)
    # the mistakes that show in a gradient: dpre has dh alone in it, one number has no half, and a norm's mean goes through dx and dy
    for name, found in caught.items():
        must = {"dpre": [1, 0, 1, 0], "dgate": [1, 1, gate == "vector", 0]}.get(name, [1, 1, 1, name != "dpost"])
        assert all(f for f, m in zip(found, must) if m), (name, found)


@pytest.mark.parametrize("post,gate", [(True, "vector"), (True, "scalar"), (False, "vector"), (False, "none")])
def test_norm_gradients_against_differences_in_other_directions(post, gate, monkeypatch):
    t = lambda a: None if a is None else bf(a)  # noqa: E731

    def forward(x, y, pw, gv, pre, scale, eps):
        xo, h = (torch.empty(x.shape, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        pqb.pq_block_norm_forward(pqb.make_norm_desc(*x.shape, eps, scale, gate == "vector"), bf(x), bf(y), t(pw), f32t(gv), bf(pre), xo, h)
        return f64(xo), f64(h)

    def backward(ds, dh, x, y, pw, gv, pre, scale, eps):
        d = pqb.make_norm_desc(*x.shape, eps, scale, gate == "vector")
        out = {k: None if a is None else torch.empty(len(a), device=DEV) for k, a in (("dpost", pw), ("dgate", gv), ("dpre", pre))}
        out.update({k: torch.empty(x.shape, dtype=torch.bfloat16, device=DEV) for k in ("dx", "dy")})
        ws = torch.empty(pqb.pq_block_norm_workspace_bytes(d), dtype=torch.uint8, device=DEV)
        pqb.pq_block_norm_backward(d, bf(ds), bf(dh), bf(forward(x, y, pw, gv, pre, scale, eps)[0]), bf(y) if post or gate != "none" else None, t(pw), f32t(gv),
                                   bf(pre), out["dx"], out["dy"], out["dpost"], out["dgate"], out["dpre"], ws)
        check_status()
        return {k: f64(v) for k, v in out.items() if v is not None}
    gradients_and_differences(post, gate, forward, backward, monkeypatch)
