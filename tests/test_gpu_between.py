"""GPU parity of what a decoder does between its projections (key-value cache, attention over it, norms around a block) against
the 64-bit forms of oracle/between_oracle.py.

Tolerances count roundings.  bf16 outputs: half a step, 2^-8 of the value.  Sums of n fp32 terms: n 2^-24 of the sum of the
terms' sizes.  Attention: a score's error d (a dot product of head_dim terms, its scale and gamma) moves a weight by the factor
e^d, and the weights p enter the second product as two bf16 numbers (bf16 cache: w = 2^-16 of p) or one fp16 number (int8 cache: half a
step, w = 2^-11 of p), while the sum that divides is of the unrounded ones.  sum (1 + a_j) p_j v_j with |a_j| <= w differs from sum
p_j v_j by at most w sum |p_j v_j|, so that an output moves by at most (2 d + w + n 2^-24) sum |p v| / sum p.
"""
import numpy as np
import pytest
import torch

from oracle import between_oracle as B
from paper_2602_22592_b200 import binding as pqb

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -8
GUARD = 64


def check_status():
    assert pqb.pq_device_status() == (0, 0)


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def bf(a):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV).to(torch.bfloat16)


class Cache:
    """A cache on the device whose every byte is known: pages in a random order, the unused ones among them, full of NaN (bf16) or
    of codes with gamma = NaN (int8); `rows` mirrors what sequences hold."""

    def __init__(self, rng, held, heads, dim, page, int8, spare=3, width=None):
        self.heads, self.dim, self.page, self.int8 = heads, dim, page, int8
        need = [-(-max(h, 0) // page) for h in held]
        pages = sum(need) + spare
        width = width or max(1, max(need))
        table = np.full((len(held), width), -1, np.int32)
        order = list(rng.permutation(pages))
        for s, k in enumerate(need):
            for j in range(k):
                table[s, j] = order.pop()
        self.table_host = table
        self.table = torch.from_numpy(table).to(DEV)
        pitch = pqb.pq_kv_pitch(pqb.PQ_KV_INT8 if int8 else pqb.PQ_KV_BF16, dim)
        shape = (pages, heads, page, pitch)
        if int8:
            self.k, self.v = (torch.full(shape, 77, dtype=torch.int8, device=DEV) for _ in range(2))
            self.kg, self.vg = (torch.full(shape[:3], float("nan"), device=DEV) for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            self.kg = self.vg = None
        self.c = pqb.make_kv_cache(self.k, self.v, self.table, dim, self.kg, self.vg)

    def fill(self, rng, held, std=1.0):
        """Rows for the first held[s] positions, written from the host; returns what they stand for, [seq] -> (k, v) [len, heads, dim]."""
        host = [(x.float().cpu().numpy() if not self.int8 else x.cpu().numpy()) for x in (self.k, self.v)]
        gam = [None if g is None else g.cpu().numpy() for g in (self.kg, self.vg)]
        out = []
        for s, n in enumerate(held):
            pair = []
            for w in range(2):
                x = B.bf16(rng.standard_normal((max(n, 0), self.heads, self.dim)) * std)
                pos = np.arange(max(n, 0))
                pg, at = self.table_host[s, pos // self.page], pos % self.page
                if self.int8:
                    codes, g = B.quantise(x)
                    host[w][pg, :, at, :self.dim], host[w][pg, :, at, self.dim:] = codes, 0
                    gam[w][pg, :, at] = g
                    x = codes.astype(np.float64) / g.astype(np.float64)[..., None]
                else:
                    host[w][pg, :, at, :self.dim], host[w][pg, :, at, self.dim:] = x, 0
                pair.append(x)
            out.append(pair)
        for w, t in enumerate((self.k, self.v)):
            t.copy_(torch.from_numpy(host[w]).to(t.dtype))
            if self.int8:
                (self.kg, self.vg)[w].copy_(torch.from_numpy(gam[w]))
        return out

    def bits(self):
        t = [x.view(torch.int16) if x.dtype == torch.bfloat16 else x for x in (self.k, self.v)] + ([self.kg.view(torch.int32), self.vg.view(torch.int32)] if self.int8 else [])
        return [x.clone() for x in t]


def guarded(shape, dtype=torch.bfloat16):
    n = int(np.prod(shape))
    raw = torch.full((n + 2 * GUARD,), 7.0, dtype=dtype, device=DEV)
    return raw, raw[GUARD:GUARD + n].view(*shape)


def guards_whole(raw):
    return bool((raw[:GUARD] == 7).all()) and bool((raw[-GUARD:] == 7).all())


def angles(rng, rows, dim):
    a = rng.uniform(-50, 50, (rows, dim // 2))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


# --------------------------------------------------------------------------- writing and reading
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dim,heads,q_heads,page,rotate,packed", [
    (128, 2, 2, 16, True, False), (64, 3, 6, 48, True, True), (100, 4, 4, 32, True, False), (8, 1, 1, 16, False, False), (256, 2, 32, 64, True, True),
    (80, 5, 5, 16, True, False), (16, 2, 0, 16, False, False), (252, 1, 2, 16, True, True), (12, 3, 3, 32, True, False), (104, 2, 2, 16, True, True)])
def test_append_then_read(dim, heads, q_heads, page, rotate, packed, int8):
    rng = np.random.default_rng(dim + 7 * heads + int8)
    held = [3 * page + 5, 1, 2 * page, 0]
    C = Cache(rng, [h + 4 for h in held], heads, dim, page, int8, width=6)
    # tokens in no order: the last four positions of each sequence, and padding
    places = [(s, h + j) for s, h in enumerate(held) for j in range(4)]
    places = [places[i] for i in rng.permutation(len(places))]
    places.insert(3, (0, -1))
    places.append((99, -5))                    # padding names no sequence
    T = len(places)
    seq, pos = (torch.tensor(a, dtype=torch.int32, device=DEV) for a in zip(*places))
    k, v = B.bf16(rng.standard_normal((T, heads, dim)) * 3), B.bf16(rng.standard_normal((T, heads, dim)))
    k[1, 0] = 0                                # an all-zero row
    q = B.bf16(rng.standard_normal((T, max(q_heads, 1), dim)))
    if packed:                                 # one projection of all three
        whole = bf(np.concatenate([q.reshape(T, -1), k.reshape(T, -1), v.reshape(T, -1)], 1))
        a, b = q.shape[1] * dim, heads * dim
        Q, K, V = whole[:, :a], whole[:, a:a + b], whole[:, a + b:]
    else:
        Q, K, V = bf(q).view(T, -1), bf(k).view(T, -1), bf(v).view(T, -1)
    cos, sin = angles(rng, max(held) + 5, dim)
    ct, st = (torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)) if rotate else (None, None)
    raw, Qo = guarded((T, q.shape[1] * dim))
    before = C.bits()
    # a packed view that begins off a 16-byte boundary is refused, not misread
    aligned = all(x.data_ptr() % 16 == 0 for x in (Q, K, V))
    if not aligned:
        with pytest.raises(pqb.PqError):
            pqb.pq_kv_append(C.c, seq, pos, K, V, ct, st, Q if q_heads else None, Qo if q_heads else None)
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
    pqb.pq_kv_append(C.c, seq, pos, K, V, ct, st, Q if q_heads else None, Qo if q_heads else None)
    torch.cuda.synchronize()
    check_status()
    at = np.maximum(pos.cpu().numpy(), 0)
    if rotate:
        k, q = B.rope(k, cos[at], sin[at]), B.rope(q, cos[at], sin[at])
    live = pos.cpu().numpy() >= 0
    if q_heads:
        assert np.array_equal(f64(Qo).reshape(q.shape)[live], q[live])
        assert (f64(Qo)[~live] == 7).all() and guards_whole(raw)
    # the cache: written rows bit for bit, zeros behind head_dim, every other byte as it was
    want = [b.clone() for b in before]
    for i, (s, p) in enumerate(places):
        if p < 0:
            continue
        pg, o = C.table_host[s, p // page], p % page
        for w, x in enumerate((k[i], v[i])):
            row = np.zeros((heads, C.k.shape[3]))
            if int8:
                codes, g = B.quantise(x)
                row[:, :dim] = codes
                want[w][pg, :, o] = torch.from_numpy(row).to(torch.int8).to(DEV)
                want[2 + w][pg, :, o] = torch.from_numpy(g).to(DEV).view(torch.int32)
            else:
                row[:, :dim] = x
                want[w][pg, :, o] = bf(row).view(torch.int16)
    for a, b in zip(C.bits(), want):
        assert torch.equal(a, b)
    # and read back
    (rk, Ko), (rv, Vo) = guarded((T, heads * dim)), guarded((T, heads * dim))
    pqb.pq_kv_read(C.c, seq, pos, Ko, Vo)
    torch.cuda.synchronize()
    check_status()
    for out, x in ((Ko, k), (Vo, v)):
        out = f64(out).reshape(T, heads, dim)
        assert (out[~live] == 7).all()
        if int8:
            codes, g = B.quantise(x)
            x = B.bf16((codes.astype(np.float32) / g[..., None]).astype(np.float32))
        assert np.array_equal(out[live], x[live])
    assert guards_whole(rk) and guards_whole(rv)


def test_append_in_place_and_many_tokens():
    # more rows than a launch has blocks for at once, queries rotated in place
    rng = np.random.default_rng(11)
    T, heads, dim, page = 5000, 4, 64, 16
    C = Cache(rng, [T], heads, dim, page, False)
    k, v, q = (B.bf16(rng.standard_normal((T, heads, dim))) for _ in range(3))
    cos, sin = angles(rng, T, dim)
    seq, pos = torch.zeros(T, dtype=torch.int32, device=DEV), torch.arange(T, dtype=torch.int32, device=DEV)
    Q = bf(q).view(T, -1)
    pqb.pq_kv_append(C.c, seq, pos, bf(k).view(T, -1), bf(v).view(T, -1), torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV), Q, Q)
    Ko, Vo = torch.empty_like(Q), torch.empty_like(Q)
    pqb.pq_kv_read(C.c, seq, pos, Ko, Vo)
    torch.cuda.synchronize()
    check_status()
    assert np.array_equal(f64(Q).reshape(q.shape), B.rope(q, cos, sin)) and np.array_equal(f64(Ko).reshape(q.shape), B.rope(k, cos, sin))
    assert np.array_equal(f64(Vo).reshape(q.shape), v)


def test_rows_that_are_not_finite_read_back_as_nan():
    rng = np.random.default_rng(12)
    C = Cache(rng, [16], 2, 64, 16, True)
    k, v = rng.standard_normal((3, 2, 64)), rng.standard_normal((3, 2, 64))
    k[0, 0, 5], k[1, 1, 63], v[2, 0, 0] = np.inf, np.nan, -np.inf
    seq, pos = torch.zeros(3, dtype=torch.int32, device=DEV), torch.arange(3, dtype=torch.int32, device=DEV)
    Ko, Vo = torch.empty((3, 128), dtype=torch.bfloat16, device=DEV), torch.empty((3, 128), dtype=torch.bfloat16, device=DEV)
    pqb.pq_kv_append(C.c, seq, pos, bf(k).view(3, -1), bf(v).view(3, -1))
    pqb.pq_kv_read(C.c, seq, pos, Ko, Vo)
    for out, bad in ((Ko, {(0, 0), (1, 1)}), (Vo, {(2, 0)})):
        nan = np.isnan(f64(out).reshape(3, 2, 64))
        for t in range(3):
            for h in range(2):
                assert nan[t, h].all() if (t, h) in bad else not nan[t, h].any()


def test_places_that_do_not_exist_are_reported_and_nothing_is_touched():
    rng = np.random.default_rng(13)
    C = Cache(rng, [32, 40], 2, 64, 16, True, width=4)
    C.table[1, 1] = C.k.shape[0]               # one past the last page
    one = lambda x: torch.tensor([x], dtype=torch.int32, device=DEV)  # noqa: E731
    k = bf(rng.standard_normal((1, 128)))
    cos, sin = (torch.ones((20, 32), device=DEV) for _ in range(2))
    before = C.bits()
    raw, Qo = guarded((1, 128))
    outs = [guarded((1, 128)) for _ in range(2)]
    for s, p in ((2, 0), (-1, 0), (1 << 30, 3), (0, 64), (0, 1 << 30), (0, 32), (1, 16)):
        pqb.pq_kv_append(C.c, one(s), one(p), k, k, None, None, k, Qo)
        assert pqb.pq_device_status()[0] == pqb.PQ_ERR_INDEX, (s, p)
        pqb.pq_kv_read(C.c, one(s), one(p), outs[0][1], outs[1][1])
        assert pqb.pq_device_status()[0] == pqb.PQ_ERR_INDEX, (s, p)
    pqb.pq_kv_append(C.c, one(0), one(20), k, k, cos, sin, k, Qo)          # no angles for position 20
    assert pqb.pq_device_status()[0] == pqb.PQ_ERR_INDEX
    assert all(torch.equal(a, b) for a, b in zip(C.bits(), before))
    assert (raw == 7).all() and all((r == 7).all() for r, _ in outs)
    pqb.pq_kv_append(C.c, one(0), one(19), k, k, cos, sin, k, Qo)
    check_status()
    # attention over a missing page and beyond the table: reported, the other sequence unharmed
    C = Cache(rng, [32, 40], 2, 64, 16, False, width=3)
    rows = C.fill(rng, [32, 40])
    q = B.bf16(rng.standard_normal((2, 2, 64)))
    O = torch.empty((2, 128), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(C.c, 2), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(2, -1), torch.tensor([33, 40], dtype=torch.int32, device=DEV), 0.125, O, None, ws)
    assert pqb.pq_device_status()[0] == pqb.PQ_ERR_INDEX
    close_attention(O[1:], None, q[1:], [rows[1]], 0.125)
    pqb.pq_attn_decode(C.c, bf(q).view(2, -1), torch.tensor([32, 49], dtype=torch.int32, device=DEV), 0.125, O, None, ws)
    assert pqb.pq_device_status()[0] == pqb.PQ_ERR_INDEX
    close_attention(O[:1], None, q[:1], [rows[0]], 0.125)


# --------------------------------------------------------------------------- attention
def close_attention(O, lse, q, rows, scale, int8=False):
    heads, dim = q.shape[1:]
    w = 2.0 ** -11 if int8 else 2.0 ** -16
    O = f64(O).reshape(len(rows), heads, dim)
    for s, (k, v) in enumerate(rows):
        want, wl, spread, big = B.attend(q[s], k, v, scale)
        d = (dim + 8) * 2.0 ** -23 * big[:, None]
        tol = HALF * np.abs(want) + (2 * d + w + len(k) * 2.0 ** -24) * spread + 1e-30
        err = np.abs(O[s] - want)
        assert (err <= tol).all(), (s, len(k), float((err / tol).max()))
        if lse is not None:
            got = f64(lse)[s]
            if len(k) == 0:
                assert (got == -np.inf).all()
            else:
                assert (np.abs(got - wl) <= d[:, 0] + (len(k) + 8) * 2.0 ** -24 + 2.0 ** -22 * np.abs(wl)).all()


ATTEND = [  # heads, group, dim, page, lengths
    (2, 1, 128, 16, [1, 15, 16, 17, 0, 129, 64]), (3, 4, 64, 48, [200, 1, 97]), (2, 1, 100, 32, [31, 333, 0, 2]), (1, 8, 128, 64, [1000]),
    (2, 5, 96, 16, [77, 50, 3]), (1, 16, 128, 16, [260, 9]), (2, 9, 64, 16, [40, 41]), (1, 20, 80, 32, [100, 0, 64]), (1, 40, 128, 16, [90]),
    (2, 3, 256, 16, [70, 1, 128]), (1, 16, 192, 32, [65, 130]), (4, 2, 8, 16, [20, 33]), (1, 1, 12, 16, [5]), (16, 1, 128, 64, [1500, 3, 700]), (3, 2, 40, 16, [33, 5]), (2, 9, 32, 16, [70, 16]), (1, 2, 112, 48, [130, 47, 200]),
    (2, 1, 180, 16, [90, 31])]


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("heads,group,dim,page,lens", ATTEND)
def test_attention(heads, group, dim, page, lens, int8):
    rng = np.random.default_rng(heads * 1000 + dim + int8)
    C = Cache(rng, lens, heads, dim, page, int8)
    rows = C.fill(rng, lens)
    n, H = len(lens), heads * group
    q = B.bf16(rng.standard_normal((n, H, dim)) * 2)
    scale = dim ** -0.5
    raw, O = guarded((n, H * dim))
    raw_l, lse = guarded((n, H), torch.float32)
    ws_raw, ws = guarded((pqb.pq_attn_workspace_bytes(C.c, H),), torch.uint8)
    ws = ws[:ws.numel()]
    lt = torch.tensor(lens, dtype=torch.int32, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(n, -1), lt, scale, O, lse, ws)
    torch.cuda.synchronize()
    check_status()
    close_attention(O, lse, q, rows, scale, int8)
    assert guards_whole(raw) and guards_whole(raw_l) and guards_whole(ws_raw)
    # rows apart, no lse, a workspace full of NaN: the same bits
    wide = torch.full((n, H * dim + 12), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, :H * dim] = bf(q).view(n, -1)
    O2 = torch.empty_like(O)
    pqb.pq_attn_decode(C.c, wide[:, :H * dim], lt, scale, O2, None, torch.full_like(ws, 255))
    assert torch.equal(O2, O)


def test_attention_leaves_padding_alone():
    rng = np.random.default_rng(21)
    lens = [20, -1, 0, 33, -7]
    for heads in (2, 400):                     # few items, and more of them than warps
        C = Cache(rng, lens, heads, 64, 16, False)
        rows = C.fill(rng, lens)
        q = B.bf16(rng.standard_normal((5, heads, 64)))
        raw, O = guarded((5, heads * 64))
        _, lse = guarded((5, heads), torch.float32)
        ws = torch.full((pqb.pq_attn_workspace_bytes(C.c, heads),), 255, dtype=torch.uint8, device=DEV)
        pqb.pq_attn_decode(C.c, bf(q).view(5, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), 0.125, O, lse, ws)
        check_status()
        for s in (1, 4):
            assert (O[s] == 7).all() and (lse[s] == 7).all()
        for s in (0, 2, 3):
            close_attention(O[s:s + 1], lse[s:s + 1], q[s:s + 1], [rows[s]], 0.125)
        assert guards_whole(raw)
        lens = [-1, -1, -1, -1, 0]             # and a batch of nothing
        O.fill_(7)
        pqb.pq_attn_decode(C.c, bf(q).view(5, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), 0.125, O, lse, ws)
        check_status()
        assert (O[:4] == 7).all() and not O[4].any() and guards_whole(raw)
        lens = [20, -1, 0, 33, -7]


@pytest.mark.parametrize("n,heads,group,dim,most,int8", [(300, 8, 1, 64, 40, False), (700, 2, 2, 64, 70, True), (37, 40, 1, 64, 130, False)])
def test_attention_of_many_sequences(n, heads, group, dim, most, int8):
    # more items than warps, more sequences than threads
    rng = np.random.default_rng(n)
    lens = [int(x) for x in rng.integers(0, most + 1, n)]
    C = Cache(rng, lens, heads, dim, 16, int8)
    rows = C.fill(rng, lens)
    q = B.bf16(rng.standard_normal((n, heads * group, dim)))
    O = torch.empty((n, heads * group * dim), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((n, heads * group), device=DEV)
    ws = torch.full((pqb.pq_attn_workspace_bytes(C.c, heads * group),), 255, dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(n, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), 0.2, O, lse, ws)
    check_status()
    close_attention(O, lse, q, rows, 0.2, int8)


@pytest.mark.parametrize("int8,group", [(False, 1), (True, 4), (False, 16)])
def test_attention_over_one_long_sequence(int8, group):
    rng = np.random.default_rng(23)
    lens = [30011]
    C = Cache(rng, lens, 1, 128, 64, int8)
    rows = C.fill(rng, lens)
    q = B.bf16(rng.standard_normal((1, group, 128)) * 3)
    O, lse = torch.empty((1, group * 128), dtype=torch.bfloat16, device=DEV), torch.empty((1, group), device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(C.c, group), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(1, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), 128 ** -0.5, O, lse, ws)
    check_status()
    close_attention(O, lse, q, rows, 128 ** -0.5, int8)


@pytest.mark.parametrize("dim", [64, 100])
def test_attention_with_extreme_scores(dim):
    # scores far apart, equal, -infinity for some positions and for all, NaN: as the definition says
    rng = np.random.default_rng(24)
    lens = [50, 50, 50, 50, 50]
    C = Cache(rng, lens, 1, dim, 16, False)
    rows = C.fill(rng, lens)
    q = B.bf16(rng.standard_normal((5, 1, dim)))
    q[0] = B.bf16(q[0] * 1000)                 # one position takes all the weight
    q[1] = 0                                   # the mean of the values
    k = C.k.float().cpu().numpy()
    for s, p, val in ((2, 10, -np.inf), (4, 7, np.nan)):
        k[C.table_host[s, p // 16], 0, p % 16, 0] = val
        rows[s][0][p, 0, 0] = val
    for p in range(50):
        k[C.table_host[3, p // 16], 0, p % 16, 0] = -np.inf
    C.k.copy_(torch.from_numpy(k))
    q[2, 0, 0] = q[3, 0, 0] = 1.0              # sign known: -infinity
    O, lse = torch.empty((5, dim), dtype=torch.bfloat16, device=DEV), torch.empty((5, 1), device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(C.c, 1), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(5, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), 1.0, O, lse, ws)
    check_status()
    assert not O[3].any() and lse[3, 0] == -float("inf")
    assert torch.isnan(O[4]).all() and torch.isnan(lse[4, 0])
    keep = np.arange(50) != 10
    rows[2] = [rows[2][0][keep], rows[2][1][keep]]
    close_attention(O[:3], lse[:3], q[:3], rows[:3], 1.0)


def test_offsets_beyond_32_bits():
    # pages whose byte and element offsets pass 2^32 in K and in V
    heads, page, dim = 8, 128, 128
    pages = (1 << 32) // (heads * page * dim) + 40
    rng = np.random.default_rng(25)
    K, V = (torch.zeros((pages, heads, page, dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.tensor([[pages - 1, 3, pages - 30]], dtype=torch.int32, device=DEV)
    c = pqb.make_kv_cache(K, V, table, dim)
    n = 300
    k, v = B.bf16(rng.standard_normal((n, heads, dim))), B.bf16(rng.standard_normal((n, heads, dim)))
    seq, pos = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV)
    pqb.pq_kv_append(c, seq, pos, bf(k).view(n, -1), bf(v).view(n, -1))
    Ko, Vo = (torch.empty((n, heads * dim), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pqb.pq_kv_read(c, seq, pos, Ko, Vo)
    assert np.array_equal(f64(Ko).reshape(k.shape), k) and np.array_equal(f64(Vo).reshape(v.shape), v)
    assert torch.equal(K[pages - 1, :, 5], bf(k[5])) and torch.equal(V[pages - 30, :, 0], bf(v[256]))
    q = B.bf16(rng.standard_normal((1, heads, dim)))
    O = torch.empty((1, heads * dim), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(c, heads), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(c, bf(q).view(1, -1), torch.tensor([n], dtype=torch.int32, device=DEV), 0.1, O, None, ws)
    check_status()
    close_attention(O, None, q, [(k, v)], 0.1)


def test_steps_replayed_from_graphs_and_on_another_stream():
    # write and attend, captured twice with workspaces of their own, replayed on two streams with new tokens and lengths
    rng = np.random.default_rng(26)
    n, heads, dim, page = 4, 4, 64, 16
    sets = []
    for _ in range(2):
        lens = [40, 1, 17, 64]
        C = Cache(rng, [80] * n, heads, dim, page, True)
        rows = C.fill(rng, [x - 1 for x in lens])
        st = dict(C=C, rows=rows, lens=torch.tensor(lens, dtype=torch.int32, device=DEV), seq=torch.arange(n, dtype=torch.int32, device=DEV),
                  q=torch.empty((n, heads * dim), dtype=torch.bfloat16, device=DEV), k=torch.empty((n, heads * dim), dtype=torch.bfloat16, device=DEV),
                  v=torch.empty((n, heads * dim), dtype=torch.bfloat16, device=DEV), O=torch.empty((n, heads * dim), dtype=torch.bfloat16, device=DEV),
                  ws=torch.empty(pqb.pq_attn_workspace_bytes(C.c, heads), dtype=torch.uint8, device=DEV))
        st["pos"] = st["lens"] - 1

        def step(st=st):
            pqb.pq_kv_append(st["C"].c, st["seq"], st["pos"], st["k"], st["v"])
            pqb.pq_attn_decode(st["C"].c, st["q"], st["lens"], 0.125, st["O"], None, st["ws"])
        st["graph"], st["stream"] = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(st["graph"]):
            step()
        sets.append(st)
    for turn in range(3):
        for st in sets:
            new = [B.bf16(rng.standard_normal((n, heads, dim))) for _ in range(3)]
            for name, x in zip("qkv", new):
                st[name].copy_(bf(x).view(n, -1))
            for s in range(n):
                for w in range(2):
                    codes, g = B.quantise(new[1 + w][s])
                    st["rows"][s][w] = np.concatenate([st["rows"][s][w], (codes / g.astype(np.float64)[:, None])[None]])
            st["want_q"] = new[0]
        torch.cuda.synchronize()
        for st in sets:
            with torch.cuda.stream(st["stream"]):
                st["graph"].replay()
        torch.cuda.synchronize()
        check_status()
        for st in sets:
            close_attention(st["O"], None, st["want_q"], st["rows"], 0.125, True)
            st["lens"] += 1
            st["pos"] += 1
    torch.cuda.synchronize()


def test_repeated_calls_give_the_same_bits():
    rng = np.random.default_rng(27)
    lens = [int(x) for x in rng.integers(1, 900, 9)]
    C = Cache(rng, lens, 3, 128, 16, False)
    C.fill(rng, lens)
    q = bf(rng.standard_normal((9, 3 * 128)))
    lt = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(C.c, 3), dtype=torch.uint8, device=DEV)
    outs = []
    for _ in range(20):
        O = torch.empty((9, 3 * 128), dtype=torch.bfloat16, device=DEV)
        pqb.pq_attn_decode(C.c, q, lt, 0.1, O, None, ws)
        outs.append(O)
    assert all(torch.equal(o, outs[0]) for o in outs)


def test_sequences_that_share_pages():
    # two sequences with the first pages of a third: they see the same rows, and rows written to their own pages stay theirs
    rng = np.random.default_rng(28)
    C = Cache(rng, [48, 16, 16], 2, 64, 16, False, width=4)
    rows = C.fill(rng, [48, 16, 16])
    table = C.table_host.copy()
    own = [table[1, 0], table[2, 0]]
    for s in (1, 2):
        table[s, :3], table[s, 3] = table[0, :3], own[s - 1]
    C.table.copy_(torch.from_numpy(table))
    lens = [48, 56, 33]
    seen = [rows[0], [np.concatenate([rows[0][w], rows[1][w][:8]]) for w in range(2)], [rows[0][w][:33] for w in range(2)]]
    q = B.bf16(rng.standard_normal((3, 4, 64)))
    O = torch.empty((3, 256), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(C.c, 4), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(3, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), 0.125, O, None, ws)
    check_status()
    close_attention(O, None, q, seen, 0.125)


@pytest.mark.parametrize("int8", [False, True])
def test_a_value_that_is_not_a_number_reaches_its_own_outputs(int8):
    rng = np.random.default_rng(29)
    C = Cache(rng, [40, 40], 2, 64, 16, int8)
    rows = C.fill(rng, [40, 40])
    pg, at = C.table_host[0, 1], 5                 # position 21 of sequence 0, head 1
    if int8:
        C.vg[pg, 1, at] = float("nan")             # the whole row
    else:
        C.v[pg, 1, at, 7] = float("nan")
    q = B.bf16(rng.standard_normal((2, 2, 64)))
    O = torch.empty((2, 128), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(C.c, 2), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(2, -1), torch.tensor([40, 40], dtype=torch.int32, device=DEV), 0.125, O, None, ws)
    check_status()
    nan = torch.isnan(O).view(2, 2, 64).cpu()
    want = torch.zeros((2, 2, 64), dtype=torch.bool)
    want[0, 1] = True if int8 else torch.arange(64) == 7
    assert torch.equal(nan, want)
    close_attention(O[1:], None, q[1:], rows[1:], 0.125, int8)


def test_two_threads_attend_on_their_own_streams():
    # one cache, two host threads with streams, queries and workspaces of their own: each call's result is the one it has alone
    import threading
    rng = np.random.default_rng(30)
    lens = [int(x) for x in rng.integers(1, 1500, 12)]
    C = Cache(rng, lens, 4, 128, 32, False)
    C.fill(rng, lens)
    lt = torch.tensor(lens, dtype=torch.int32, device=DEV)
    qs = [bf(rng.standard_normal((12, 512))) for _ in range(2)]
    new = lambda: torch.empty((12, 512), dtype=torch.bfloat16, device=DEV)  # noqa: E731
    wss = [torch.full((pqb.pq_attn_workspace_bytes(C.c, 4),), 255 * i, dtype=torch.uint8, device=DEV) for i in range(2)]
    want = [new(), new()]
    for i in range(2):
        pqb.pq_attn_decode(C.c, qs[i], lt, 0.1, want[i], None, wss[i])
    torch.cuda.synchronize()
    outs, errors = [[], []], []

    def work(i):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for _ in range(50):
                    outs[i].append(new())
                    pqb.pq_attn_decode(C.c, qs[i], lt, 0.1, outs[i][-1], None, wss[i])
            st.synchronize()
        except Exception as e:      # pragma: no cover
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    check_status()
    assert not errors and all(torch.equal(o, want[i]) for i in range(2) for o in outs[i])


# --------------------------------------------------------------------------- norms
def norm_case(rng, T, N, post, gate):
    x, y = B.bf16(rng.standard_normal((T, N)) * 2), B.bf16(rng.standard_normal((T, N)))
    pre, pw = B.bf16(1 + 0.2 * rng.standard_normal(N)), B.bf16(1 + 0.2 * rng.standard_normal(N)) if post else None
    gv = None if gate == "none" else rng.uniform(0.5, 1.5, N if gate == "vector" else 1).astype(np.float32).astype(np.float64)
    return x, y, pre, pw, gv


def f32t(a):
    return None if a is None else torch.from_numpy(a.astype(np.float32)).to(DEV)


NORMS = [(1, 8, False, "none"), (1, 3200, True, "vector"), (5, 264, True, "scalar"), (130, 512, False, "vector"), (7, 8640, True, "vector"), (700, 2048, True, "none"),
         (3, 16384, True, "vector"), (400, 1032, False, "scalar"), (600, 4104, False, "none"), (350, 264, True, "vector"), (2, 8192, False, "scalar"), (333, 8200, True, "scalar")]


@pytest.mark.parametrize("T,N,post,gate", NORMS)
def test_block_norm_forward(T, N, post, gate):
    rng = np.random.default_rng(T + N)
    x, y, pre, pw, gv = norm_case(rng, T, N, post, gate)
    if T > 2:
        x[1] = y[1] = 0                        # an all-zero row: eps keeps it finite
    scale, eps = 0.75, 1e-5
    d = pqb.make_norm_desc(T, N, eps, scale, gate == "vector")
    (ra, xo), (rb, h) = guarded((T, N)), guarded((T, N))
    X = bf(x)
    args = (bf(y), None if pw is None else bf(pw), f32t(gv), bf(pre))
    pqb.pq_block_norm_forward(d, X, *args, xo, h)
    torch.cuda.synchronize()
    check_status()
    s, hh = B.block_norm(x, y, pw, gv, pre, scale, eps)
    u = np.abs(s - scale * x)
    ds = (N + 16) * 2.0 ** -24 * u + 4 * 2.0 ** -24 * (np.abs(scale * x) + u)       # u holds a norm of its own; then products and a sum
    r = hh / np.where(s == 0, 1, s)
    assert (np.abs(f64(xo) - s) <= HALF * np.abs(s) + ds + 1e-38).all()
    tol = HALF * np.abs(hh) + (N + 16) * 2.0 ** -24 * np.abs(hh) + ds * np.abs(np.where(s == 0, pre / np.sqrt(eps), r)) + np.abs(hh) * (ds * ds).sum(-1, keepdims=True) ** 0.5 / np.sqrt((s * s).sum(-1, keepdims=True) + eps) + 1e-38
    assert (np.abs(f64(h) - hh) <= tol).all()
    assert guards_whole(ra) and guards_whole(rb)
    # in place, and each output alone: the same bits
    X2, Y2 = X.clone(), args[0].clone()
    pqb.pq_block_norm_forward(d, X2, Y2, *args[1:], X2, Y2)
    assert torch.equal(X2, xo) and torch.equal(Y2, h)
    only = torch.empty_like(X)
    pqb.pq_block_norm_forward(d, X, args[0], args[1], args[2], None, only, None)
    assert torch.equal(only, xo)
    pqb.pq_block_norm_forward(d, X, *args, None, only)
    assert torch.equal(only, h)


def test_block_norm_of_the_stream_alone():
    rng = np.random.default_rng(31)
    x, pre = B.bf16(rng.standard_normal((6, 320))), B.bf16(1 + rng.standard_normal(320))
    d = pqb.make_norm_desc(6, 320, 1e-6)
    h = torch.empty((6, 320), dtype=torch.bfloat16, device=DEV)
    pqb.pq_block_norm_forward(d, bf(x), None, None, None, bf(pre), None, h)
    want = B.block_norm(x, None, None, None, pre, 1.0, 1e-6)[1]
    assert (np.abs(f64(h) - want) <= (HALF + 340 * 2.0 ** -24) * np.abs(want)).all()
    check_status()


@pytest.mark.parametrize("parts", ["both", "stream", "next"])
@pytest.mark.parametrize("T,N,post,gate", NORMS)
def test_block_norm_backward(T, N, post, gate, parts):
    rng = np.random.default_rng(T + 3 * N)
    s, y, pre, pw, gv = norm_case(rng, T, N, post, gate)
    if T > 2:
        s[1] = y[1] = 0
    scale, eps = 0.75, 1e-5
    ds, dh = B.bf16(rng.standard_normal((T, N))), B.bf16(rng.standard_normal((T, N)))
    ds = None if parts == "next" else ds
    if parts == "stream":
        dh = pre = None
    d = pqb.make_norm_desc(T, N, eps, scale, gate == "vector")
    t = lambda a: None if a is None else bf(a)  # noqa: E731
    (ra, dx), (rb, dy) = guarded((T, N)), guarded((T, N))
    sums = {"dpost": guarded((N,), torch.float32) if post else (None, None), "dgate": guarded((len(gv),), torch.float32) if gv is not None else (None, None),
            "dpre": guarded((N,), torch.float32) if dh is not None else (None, None)}
    ws_raw, ws = guarded((pqb.pq_block_norm_workspace_bytes(d),), torch.uint8)
    both = post or gate != "none"
    args = (t(ds), t(dh), t(s) if dh is not None else None, t(y) if both else None, t(pw), f32t(gv), t(pre))
    pqb.pq_block_norm_backward(d, *args, dx, dy, sums["dpost"][1], sums["dgate"][1], sums["dpre"][1], ws)
    torch.cuda.synchronize()
    check_status()
    want = B.block_norm_backward(ds, dh, s, y, pw, gv, pre, scale, eps)
    # sizes of the terms, for the fp32 steps: (N + 16) of them along a row, T along a column
    one, e = (N + 24) * 2.0 ** -24, eps
    r = 1 / np.sqrt((s * s).mean(-1, keepdims=True) + e)
    size = np.zeros((T, N)) if ds is None else np.abs(ds)
    if dh is not None:
        size = size + r * (np.abs(dh * pre) + np.abs(s * r) * np.abs(dh * pre * s * r).mean(-1, keepdims=True))
    tol = {"dx": HALF * np.abs(want["dx"]) + one * scale * size}
    # a block adds its rows one after another, then 148 blocks, then fp32 -- T terms at most
    col = (T + N + 32) * 2.0 ** -24
    if dh is not None:
        tol["dpre"] = col * np.abs(dh * s * r).sum(0)
    g = np.ones(1) if gv is None else gv
    ry = 1 / np.sqrt((y * y).mean(-1, keepdims=True) + e)
    m = y * ry if post else y
    u = m * pw if post else m
    if gv is not None:
        tol["dgate"] = col * (size * np.abs(u)).sum(0)
        if gate == "scalar":
            want["dgate"], tol["dgate"] = want["dgate"].sum(keepdims=True), tol["dgate"].sum(keepdims=True)
    es = size * g
    if post:
        tol["dpost"] = col * (es * np.abs(m)).sum(0)
        es = ry * (es * np.abs(pw) + np.abs(m) * (es * np.abs(pw * m)).mean(-1, keepdims=True))
    tol["dy"] = HALF * np.abs(want["dy"]) + 2 * one * es
    got = {"dx": dx, "dy": dy, **{k: v[1] for k, v in sums.items() if v[1] is not None}}
    assert set(got) == set(want)
    for k, v in got.items():
        err = np.abs(f64(v) - want[k])
        assert (err <= tol[k] + 1e-38).all(), (k, float((err / (tol[k] + 1e-38)).max()))
    assert all(guards_whole(x) for x in (ra, rb, ws_raw) + tuple(v[0] for v in sums.values() if v[0] is not None))
    # in place over what comes in, and again: the same bits
    again = [None if a is None else a.clone() for a in args[:2]]
    into = again[0] if again[0] is not None else again[1]
    dy2 = torch.empty_like(dx)
    sums2 = {k: None if v[1] is None else torch.full_like(v[1], float("nan")) for k, v in sums.items()}
    pqb.pq_block_norm_backward(d, *again, *args[2:], into, dy2, sums2["dpost"], sums2["dgate"], sums2["dpre"], torch.full_like(ws, 255))
    assert torch.equal(into, dx) and torch.equal(dy2, dy) and all(v[1] is None or torch.equal(v[1], sums2[k]) for k, v in sums.items())


def test_norm_gradients_against_differences_of_the_kernel():
    # the forward kernel's own differences: h and s are bf16, so that a step large enough to rise above their rounding is taken and many
    # values are averaged; the direction is the gradient itself
    rng = np.random.default_rng(33)
    T, N, eps = 64, 256, 1e-5
    x, y, pre, pw, gv = norm_case(rng, T, N, True, "vector")
    ds, dh = B.bf16(rng.standard_normal((T, N))), B.bf16(rng.standard_normal((T, N)))
    d = pqb.make_norm_desc(T, N, eps, 0.75, True)
    xo, h = (torch.empty((T, N), dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def loss(gate):
        pqb.pq_block_norm_forward(d, bf(x), bf(y), bf(pw), f32t(gate), bf(pre), xo, h)
        return float((f64(xo) * ds).sum() + (f64(h) * dh).sum())

    pqb.pq_block_norm_forward(d, bf(x), bf(y), bf(pw), f32t(gv), bf(pre), xo, h)
    dx, dy = torch.empty_like(xo), torch.empty_like(xo)
    dpost, dgate, dpre = (torch.empty(N, device=DEV) for _ in range(3))
    ws = torch.empty(pqb.pq_block_norm_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    pqb.pq_block_norm_backward(d, bf(ds), bf(dh), xo, bf(y), bf(pw), f32t(gv), bf(pre), dx, dy, dpost, dgate, dpre, ws)
    g = f64(dgate)
    step = 0.05 / np.abs(g).max()
    slope = (loss(gv + step * g) - loss(gv - step * g)) / (2 * step)
    # 2 T N outputs, each rounded by up to 2^-8 of about 2 in both calls, weighted by N(0, 1): six standard deviations of that noise
    noise = 6 * np.sqrt(2 * 2 * T * N) * 2 * HALF / np.sqrt(3) / (2 * step)
    # x_out's rounding reaches g through the backward as well (2^-8 of g), and the cubic term of the difference: 0.05^2
    assert abs(slope - (g * g).sum()) <= noise + (HALF + 0.01) * (g * g).sum()


# --------------------------------------------------------------------------- together, as a decoder uses them
from paper_2602_22592_b200.decoder_harness import NORM_EPS, PQDecoder, PQServer  # noqa: E402


def bf16_sum_tol(x, y):
    return HALF * np.abs(x + y) + 2.0 ** -23 * (np.abs(x) + np.abs(y)) + 1e-38


def close_norm(h, s, w, tol_s):
    """h against the norm of s (64 bits), s known to tol_s."""
    want = B.rms(s, NORM_EPS) * w
    r = 1 / np.sqrt((s * s).mean(-1, keepdims=True) + NORM_EPS)
    whole = np.sqrt((tol_s * tol_s).sum(-1, keepdims=True) / ((s * s).sum(-1, keepdims=True) + 1e-30))
    tol = HALF * np.abs(want) + (s.shape[-1] + 16) * 2.0 ** -24 * np.abs(want) + np.abs(tol_s * r * w) + np.abs(want) * whole + 1e-38
    assert (np.abs(h - want) <= tol).all()


@pytest.mark.parametrize("int8,heads,page", [(False, 4, 16), (True, 4, 32), (True, 2, 16)])
def test_server_prompts_and_steps(int8, heads, page):
    # prompts of different lengths, steps, a further ragged prompt, steps across page ends; every attention and norm of the steps against the
    # 64-bit forms on what the cache holds
    m = PQDecoder(layers=2, hidden=256, heads=heads, ffn=512, vocab=500, batch=1, seq=64, r=32, E=4, seed=7)
    n, D = 3, 256 // heads
    S = PQServer(m, n, 70, page, int8)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    ids = lambda *shape: torch.randint(0, 500, shape, generator=gen, device=DEV)  # noqa: E731
    logits = S.prompt(ids(n, 29), [29, 1, 13])
    assert logits.shape == (n, 500) and torch.isfinite(logits.float()).all()

    def steps(k):
        for _ in range(k):
            S.capture = []
            out = S.step(ids(n))
            torch.cuda.synchronize()
            check_status()
            assert torch.isfinite(out.float()).all() and len(S.capture) == 2
            for i, cap in enumerate(S.capture):
                lens = [int(v) for v in cap["lens"]]
                assert lens == S.held
                cos, sin = S.cos[[v - 1 for v in lens]].cpu().numpy(), S.sin[[v - 1 for v in lens]].cpu().numpy()
                q = B.rope(f64(cap["q"]).reshape(n, heads, D), cos, sin)
                assert np.array_equal(f64(cap["q_rot"]).reshape(q.shape), q)
                k_new = B.rope(f64(cap["k"]).reshape(n, heads, D), cos, sin)
                rows = []
                for s in range(n):
                    seq = torch.full((lens[s],), s, dtype=torch.int32, device=DEV)
                    pos = torch.arange(lens[s], dtype=torch.int32, device=DEV)
                    ko, vo = (torch.empty((lens[s], heads * D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
                    pqb.pq_kv_read(S.caches[i], seq, pos, ko, vo)
                    pair = []
                    table = S.table.cpu().numpy()
                    p = np.arange(lens[s])
                    for pages, gam in ((S.caches[i].tensors[0], S.caches[i].tensors[3]), (S.caches[i].tensors[1], S.caches[i].tensors[4])):
                        x = pages.float().cpu().numpy().astype(np.float64)[table[s, p // page], :, p % page, :D]
                        if int8:
                            x = x / gam.cpu().numpy().astype(np.float64)[table[s, p // page], :, p % page][..., None]
                        pair.append(x)
                    assert np.array_equal(f64(ko).reshape(pair[0].shape), B.bf16(pair[0].astype(np.float32)) if int8 else pair[0])
                    last = k_new[s] if not int8 else (lambda c, g: c / g.astype(np.float64)[:, None])(*B.quantise(k_new[s]))
                    assert np.array_equal(pair[0][-1], last)
                    rows.append(pair)
                close_attention(cap["a"], None, q, rows, D ** -0.5, int8)
                x, o = f64(cap["x"]), f64(cap["o"])
                tol = bf16_sum_tol(x, o)
                assert (np.abs(f64(cap["x_out"]) - (x + o)) <= tol).all()
                close_norm(f64(cap["h"]), x + o, f64(m.blocks[i]["norm2"]), 2.0 ** -23 * (np.abs(x) + np.abs(o)))
            S.capture = None

    steps(4)
    S.prompt(ids(n, 9), [1, 9, 4])
    assert S.held == [34, 14, 21]
    steps(2)
    with pytest.raises(ValueError):
        S.prompt(ids(n, 60), [60, 60, 60])


def test_server_refuses_nothing_it_has_room_for():
    m = PQDecoder(layers=1, hidden=128, heads=2, ffn=256, vocab=100, batch=1, seq=32, r=0, E=0, seed=8)
    S = PQServer(m, 2, 33, 16)
    S.prompt(torch.zeros((2, 33), dtype=torch.int64, device=DEV), [33, 20])
    assert S.held == [33, 20] and len({int(v) for v in S.table.flatten() if v >= 0}) == 5
    torch.cuda.synchronize()
    check_status()


def test_training_step_with_library_norms():
    # every norm of a step, forward and backward, against the 64-bit forms on its own inputs
    m = PQDecoder(layers=2, hidden=256, heads=4, ffn=512, vocab=400, batch=2, seq=32, r=32, E=4, seed=9, library_norms=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(2)
    with torch.no_grad():
        for p in [m.norm_f] + [b[k] for b in m.blocks for k in ("norm1", "norm2")]:
            p.copy_(1 + 0.2 * torch.randn(256, generator=g, device=DEV))
    ids, tgt = m.random_batch()
    m.norm_capture = []
    loss = m.step(ids, tgt)
    torch.cuda.synchronize()
    check_status()
    assert torch.isfinite(loss) and len(m.norm_capture) == 5
    weights = [m.blocks[0]["norm1"], m.blocks[0]["norm2"], m.blocks[1]["norm1"], m.blocks[1]["norm2"], m.norm_f]
    for cap, weight in zip(m.norm_capture, weights):
        x, w = f64(cap["x"]), f64(cap["weight"])
        y = None if cap["y"] is None else f64(cap["y"])
        s = x if y is None else x + y
        if y is not None:
            assert (np.abs(f64(cap["x_out"]) - s) <= bf16_sum_tol(x, y)).all()
        close_norm(f64(cap["h"]), s, w, np.zeros_like(s) if y is None else 2.0 ** -23 * (np.abs(x) + np.abs(y)))
        ds = None if cap.get("dx_out") is None else f64(cap["dx_out"])
        dh, st = f64(cap["dh"]), f64(cap["x_out"])
        want = B.block_norm_backward(ds, dh, st, None, None, None, w, 1.0, NORM_EPS)
        r = 1 / np.sqrt((st * st).mean(-1, keepdims=True) + NORM_EPS)
        size = (0 if ds is None else np.abs(ds)) + r * (np.abs(dh * w) + np.abs(st * r) * np.abs(dh * w * st * r).mean(-1, keepdims=True))
        assert (np.abs(f64(cap["dx"]) - want["dx"]) <= HALF * np.abs(want["dx"]) + (256 + 24) * 2.0 ** -24 * size + 1e-38).all()
        tol = (len(st) + 256 + 32) * 2.0 ** -24 * np.abs(dh * st * r).sum(0)
        assert (np.abs(f64(cap["dweight"]) - want["dpre"]) <= tol + 1e-38).all()
        assert torch.equal(weight.grad, cap["dweight"].to(torch.bfloat16))
    assert (m.norm_capture[-1]["dx_out"] if "dx_out" in m.norm_capture[-1] else None) is None      # nothing reads the stream behind the last norm
