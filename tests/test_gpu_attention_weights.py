"""How far the weights of pq_attn_decode are off, seen where nothing else is: values that cancel, values far apart, infinities.

Tolerances count roundings.  Relative errors of one weight: exp2 2^-22, the reciprocal of an int8 row's gamma 2^-23, products and
differences in fp32 2^-24 each; of an int8 cache two fp16 numbers, 2^-11 2^-11 = 2^-22.  A sum inside a tensor core may cut each of its
17 terms at 2^-23 of the largest one.  Together W = 2^-18 of sum |p v| / sum p for a handful of positions (2^-22 + 2^-23 + 4 2^-24 + 2^-22 +
17 2^-23 = 2^-18.6); a score's error is counted apart."""
import numpy as np
import pytest
import torch

from oracle import between_oracle as B
from paper_2602_22592_b200 import binding as pqb
from test_gpu_between import DEV, HALF, Cache, bf, check_status, f64

pytestmark = pytest.mark.gpu
W = 2.0 ** -18


def attend(C, q, lens, scale, lse=None):
    n, H = q.shape[:2]
    O = torch.empty((n, q.shape[1] * q.shape[2]), dtype=torch.bfloat16, device=DEV)
    ws = torch.full((pqb.pq_attn_workspace_bytes(C.c, H),), 255, dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(C.c, bf(q).view(n, -1), torch.tensor(lens, dtype=torch.int32, device=DEV), scale, O, lse, ws)
    check_status()
    return f64(O).reshape(q.shape)


@pytest.mark.parametrize("dim,group", [(8, 1), (64, 12), (128, 1), (128, 12), (256, 3)])
def test_int8_weights_where_values_cancel(dim, group):
    # two positions a sequence whose first values cancel: gamma_v of the second is chosen for it (to fp32's rounding), so that the
    # output there is the weights' own error
    rng = np.random.default_rng(41)
    n, scale = 48, 0.25
    C = Cache(rng, [2] * n, 1, dim, 16, True)
    rows = C.fill(rng, [2] * n)
    k, v = C.k.cpu().numpy(), C.v.cpu().numpy()
    kg, vg = C.kg.cpu().numpy(), C.vg.cpu().numpy()
    q = np.zeros((n, group, dim))
    q[:, :, 0] = 1
    for s in range(n):
        pg = C.table_host[s, 0]
        k[pg, 0, :2] = 0
        k[pg, 0, :2, 0] = rng.integers(-128, 128, 2)
        kg[pg, 0, :2] = rng.uniform(60, 250, 2).astype(np.float32)
        keys = k[pg, 0, :2].astype(np.float64) / kg[pg, 0, :2].astype(np.float64)[:, None]
        p = np.exp(scale * keys[:, 0])
        a, b = rng.integers(60, 128), -rng.integers(60, 128)
        v[pg, 0, 0, 0], v[pg, 0, 1, 0] = a, b
        vg[pg, 0, 0] = np.float32(rng.uniform(10, 100))
        vg[pg, 0, 1] = np.float32(-(p[1] * b) / (p[0] * a) * np.float64(vg[pg, 0, 0]))
        rows[s] = [keys[:, None], (v[pg, 0, :2, :dim].astype(np.float64) / vg[pg, 0, :2].astype(np.float64)[:, None])[:, None]]
        rows[s][0] = rows[s][0][..., :dim]
    for t, h in ((C.k, k), (C.v, v), (C.kg, kg), (C.vg, vg)):
        t.copy_(torch.from_numpy(h))
    O = attend(C, q, [2] * n, scale)
    for s in range(n):
        want, _, spread, big = B.attend(q[s], *rows[s], scale)
        assert (np.abs(want[:, 0]) < 2.0 ** -20 * spread[:, 0]).all()                    # they cancel
        tol = HALF * np.abs(want) + (2 * (dim + 8) * 2.0 ** -23 * big[:, None] + W) * spread
        assert (np.abs(O[s] - want) <= tol).all(), (s, float((np.abs(O[s] - want) / tol).max()))


@pytest.mark.parametrize("length,at", [(3, 1), (40, 39), (40, 0), (700, 333), (9000, 8999), (9000, 0)])
def test_int8_rows_of_zeros_beside_very_large_ones(length, at):
    # equal scores; one row of 2^126 (gamma 2^-119), the others zeros (gamma 2^23): every position counts in the weights' sum
    rng = np.random.default_rng(42)
    dim = 64
    C = Cache(rng, [length], 1, dim, 16, True)
    rows = C.fill(rng, [length])
    x = np.zeros((length, 1, dim))
    x[at] = 2.0 ** 126
    codes, gamma = B.quantise(x)
    pos = np.arange(length)
    pg, o = (torch.from_numpy(a).to(DEV).long() for a in (C.table_host[0, pos // 16], pos % 16))
    C.v[pg, 0, o, :dim], C.vg[pg, 0, o] = torch.from_numpy(codes[:, 0]).to(DEV), torch.from_numpy(gamma[:, 0]).to(DEV)
    q, lse = np.zeros((1, 1, dim)), torch.empty((1, 1), device=DEV)
    O = attend(C, q, [length], 0.125, lse)
    v = codes.astype(np.float64) / gamma.astype(np.float64)[..., None]
    want, wl, spread, _ = B.attend(q[0], rows[0][0], v, 0.125)
    assert (np.abs(O[0] - want) <= HALF * np.abs(want) + (W + length * 2.0 ** -24) * spread).all(), (O[0, 0, 0], want[0, 0])
    assert abs(float(lse[0, 0]) - wl[0]) <= (length + 8) * 2.0 ** -24 + 2.0 ** -22 * abs(wl[0])


def test_the_sum_of_weights_knows_nothing_of_the_values():
    # int8 rows of values that are not numbers: NaN in the outputs, the log of the weights' sum as ever
    rng = np.random.default_rng(45)
    lens = [40, 17, 900]
    C = Cache(rng, lens, 1, 64, 16, True)
    rows = C.fill(rng, lens)
    C.vg[int(C.table_host[0, 1]), 0, 3] = float("nan")
    C.vg[int(C.table_host[1, 0])] = C.vg[int(C.table_host[1, 1]), :, 0] = float("nan")
    C.vg[int(C.table_host[2, 30]), 0] = float("nan")
    q, lse = B.bf16(rng.standard_normal((3, 2, 64))), torch.empty((3, 2), device=DEV)
    O = attend(C, q, lens, 0.125, lse)
    assert np.isnan(O).all()
    for s in range(3):
        _, wl, _, big = B.attend(q[s], *rows[s], 0.125)
        assert (np.abs(f64(lse)[s] - wl) <= 72 * 2.0 ** -23 * big + (lens[s] + 8) * 2.0 ** -24 + 2.0 ** -22 * np.abs(wl)).all()


def two_bf16_error(p):
    """What p loses as the sum of two bf16 numbers, each rounded to nearest, relative to p."""
    hi = B.bf16(p)
    return (p - hi - B.bf16(p - hi)) / p


@pytest.mark.parametrize("dim,group", [(8, 1), (64, 12), (128, 1), (256, 3)])
def test_bf16_weights_where_values_cancel(dim, group):
    # three positions: one takes the maximum and has no value; the weights of the others are such that two bf16 numbers miss one by
    # +2^-17.x and the other by -2^-17.x, and their values cancel to 2^-12.  The score is one product, 2^k0 after scale = ln 2: its fp32
    # roundings (of scale log2 e, of the product, of the difference) are 2^-24 of at most 1 each
    rng = np.random.default_rng(43)
    scale = float(np.float32(np.log(2)))
    k0 = -(128 + np.arange(128)) / 256.0                                                   # bf16 numbers in (-1, -1/2]
    k0 = np.concatenate([k0, k0 / 2])
    e = two_bf16_error(np.exp(scale * k0).astype(np.float32).astype(np.float64)) * 2.0 ** 17
    up, down = k0[(e > 0.55) & (e < 0.97)], k0[(e < -0.55) & (e > -0.97)]
    assert len(up) and len(down)
    sets = []
    for ku in up:
        for kd in down:
            pu, pd = np.exp(scale * ku), np.exp(scale * kd)
            a = np.arange(128, 256)
            b = np.rint(a * pu / pd)
            off = np.where((b >= 128) & (b < 256), np.abs(a * pu - b * pd) / (a * pu), 1)
            if off.min() < 2.0 ** -13:
                sets.append((ku, kd, a[off.argmin()], b[off.argmin()]))
    assert len(sets) >= 3
    n = len(sets)
    C = Cache(rng, [3] * n, 1, dim, 16, False)
    C.fill(rng, [3] * n)
    q = np.zeros((n, group, dim))
    q[:, :, 0] = 1
    rows = []
    for s, (ku, kd, a, b) in enumerate(sets):
        k, v = np.zeros((3, 1, dim)), np.zeros((3, 1, dim))
        k[:, 0, 0] = [0, ku, kd]
        v[1, 0], v[2, 0] = a, -b
        pg = int(C.table_host[s, 0])
        C.k[pg, 0, :3, :dim], C.v[pg, 0, :3, :dim] = bf(k[:, 0]), bf(v[:, 0])
        rows.append((k, v))
    O = attend(C, q, [3] * n, scale)
    for s in range(n):
        want, _, spread, _ = B.attend(q[s], *rows[s], scale)
        # weights: exp2 2^-22, three roundings of the score 3 2^-24 ln 2; the sum: 4 terms cut at 2^-23 of the largest, half of spread.  The
        # sum that divides moves an output of 2^-12 of spread by nothing that counts
        tol = HALF * np.abs(want) + (2.0 ** -22 + 3 * 2.0 ** -24 + 4 * 2.0 ** -24) * spread
        assert (np.abs(O[s] - want) <= tol).all(), (s, float((np.abs(O[s] - want) / tol).max()))


@pytest.mark.parametrize("dim,group,length", [(64, 1, 1), (64, 12, 40), (128, 1, 700), (128, 12, 5000), (100, 2, 37), (256, 3, 90)])
def test_an_infinity_among_the_values(dim, group, length):
    # in one value of some positions: that infinity in the outputs it reaches, NaN where both signs meet, the others as ever
    rng = np.random.default_rng(44)
    C = Cache(rng, [length], 1, dim, 16, False)
    (k, v), = C.fill(rng, [length])
    q = B.bf16(rng.standard_normal((1, group, dim)))
    scale = dim ** -0.5
    where = {0: [0], 3: [length - 1], 9: list(range(length)), 20: [length // 2, 0], 31: [length // 3]}
    for d, at in where.items():
        v[at, 0, d] = -np.inf if d in (3, 31) else np.inf
    if length > 1:
        v[0, 0, 40], v[length - 1, 0, 40] = np.inf, -np.inf
    pos = np.arange(length)
    pg, o = (torch.from_numpy(a).to(DEV).long() for a in (C.table_host[0, pos // 16], pos % 16))
    C.v[pg, 0, o, :dim] = bf(v[:, 0])
    O = attend(C, q, [length], scale)[0]
    with np.errstate(invalid="ignore"):
        want = B.attend(q[0], k, v, scale)[0]
    assert np.array_equal(np.isnan(want[0]), (np.arange(dim) == 40) & (length > 1)) and np.isposinf(want[:, 9]).all()
    special = ~np.isfinite(want)
    assert np.array_equal(O[special], want[special], equal_nan=True), O[special]
    want, _, spread, big = B.attend(q[0], k, np.where(np.isfinite(v), v, 0), scale)
    tol = HALF * np.abs(want) + (2 * (dim + 8) * 2.0 ** -23 * big[:, None] + 2.0 ** -16 + length * 2.0 ** -24) * spread + 1e-30
    assert (np.abs(O - want) <= tol)[~special].all()


@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("dim,group", [(64, 1), (64, 16), (128, 1), (128, 16), (256, 3)])
def test_long_sums_lean_to_neither_side(dim, group, int8):
    # 131072 positions, the same eight pages over and over, values of one sign; enough sequences that a warp has thousands of tiles of one.  An
    # output's rounding to bf16 is at most 2^-8 either way, a deviation of 2^-8 / sqrt(3): the mean over all outputs stays within six
    # of its own deviations, and 2^-20 for what a tile's sum (cut off at 2^-23) and a reciprocal (2^-23) may lean by
    g = torch.Generator(device=DEV)
    g.manual_seed(46)
    page, pages, length, n, heads = 128, 8, 131072, 148, 8 if group == 1 else 2
    k, v = (torch.randn((pages, heads, page, dim), generator=g, device=DEV) for _ in range(2))
    v = v * 0.3 + 1.5
    kg = vg = None
    if int8:
        kg, vg = 128 / k.abs().amax(-1), 128 / v.abs().amax(-1)
        k, v = ((x * y[..., None]).round().clamp(-128, 127).to(torch.int8) for x, y in ((k, kg), (v, vg)))
        rows = [x.double() / y.double()[..., None] for x, y in ((k, kg), (v, vg))]
    else:
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        rows = [k.double(), v.double()]
    table = (torch.arange(length // page, device=DEV, dtype=torch.int32) % pages).repeat(n, 1)
    c = pqb.make_kv_cache(k, v, table, dim, kg, vg)
    H = heads * group
    q = torch.randn((n, H * dim), generator=g, device=DEV).to(torch.bfloat16)
    O = torch.empty_like(q)
    ws = torch.empty(pqb.pq_attn_workspace_bytes(c, H), dtype=torch.uint8, device=DEV)
    pqb.pq_attn_decode(c, q, torch.full((n,), length, dtype=torch.int32, device=DEV), dim ** -0.5, O, None, ws)
    check_status()
    keys, values = (x.transpose(0, 1).reshape(heads, -1, dim) for x in rows)
    weight = torch.softmax(torch.einsum("nhgd,hpd->nhgp", q.double().view(n, heads, group, dim), keys) * dim ** -0.5, -1)
    want = torch.einsum("nhgp,hpd->nhgd", weight, values).reshape(n, -1)
    lean = float(((O.double() - want) / want).mean())
    assert abs(lean) <= 6 * HALF / np.sqrt(3 * want.numel()) + 2.0 ** -20, lean
