"""Pins of the 64-bit forms in oracle/between_oracle.py, and the refusals of the entry points (host logic, no kernel runs)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import between_oracle as B


def test_bf16_rounding_against_torch_and_at_ties():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(20000) * 10.0 ** rng.integers(-20, 20, 20000)
    want = torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).double().numpy()
    assert np.array_equal(B.bf16(x.astype(np.float32)), want)
    assert B.bf16(1 + 2.0 ** -8) == 1 and B.bf16(1 + 3 * 2.0 ** -8) == 1 + 2.0 ** -6       # ties to even
    assert B.bf16(1 + 2.0 ** -8 + 2.0 ** -40) == 1 + 2.0 ** -7                              # not twice: fp32 alone would drop the last term
    assert B.bf16(1 + 3 * 2.0 ** -8 - 2.0 ** -40) == 1 + 2.0 ** -7
    assert np.isnan(B.bf16(np.nan)) and B.bf16(np.inf) == np.inf


def test_rope_is_a_rotation():
    rng = np.random.default_rng(1)
    x = B.bf16(rng.standard_normal((5, 3, 16)))
    ang = rng.uniform(0, 100, (5, 8))
    c, s = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    y = B.rope(x, c, s)
    z = (x[..., :8] + 1j * x[..., 8:]) * np.exp(1j * ang)[:, None]
    assert np.abs(y - np.concatenate([z.real, z.imag], -1)).max() <= 2.0 ** -8 * np.abs(z).max() + 1e-5
    assert np.array_equal(B.rope(x, np.ones((5, 8)), np.zeros((5, 8))), x)


def test_quantiser_bounds_and_special_rows():
    rng = np.random.default_rng(2)
    x = B.bf16(rng.standard_normal((50, 64)))
    codes, gamma = B.quantise(x)
    back = codes.astype(np.float64) / gamma.astype(np.float64)[:, None]
    assert np.abs(back - x).max() <= np.abs(x).max() / 128 * 1.0001          # half a step, the whole of one at +max (128 is clipped to 127)
    assert codes.min() >= -128 and codes.max() == 127
    codes, gamma = B.quantise(np.zeros((1, 8)))
    assert not codes.any() and gamma[0] == np.float32(128) / np.float32(1e-5)
    codes, gamma = B.quantise(np.array([[1.0, np.inf], [np.nan, 1.0], [1.0, 2.0]]))
    assert np.isnan(gamma[:2]).all() and np.isfinite(gamma[2])


def test_attention_special_cases():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    q = rng.standard_normal((6, 8))
    out, lse, spread, _ = B.attend(q, k, v, 0.3)
    for h in range(6):
        w = [np.exp(0.3 * sum(q[h, d] * k[j, h // 3, d] for d in range(8))) for j in range(7)]
        assert np.allclose(out[h], sum(w[j] * v[j, h // 3] for j in range(7)) / sum(w), atol=1e-12)
        assert abs(lse[h] - np.log(sum(w))) < 1e-12
    assert (spread >= np.abs(out)).all()
    one = B.attend(q, k[:1], v[:1], 0.3)[0]
    assert np.array_equal(one, np.repeat(v[0], 3, 0))
    none = B.attend(q, k[:0], v[:0], 0.3)
    assert not none[0].any() and (none[1] == -np.inf).all()


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", ["none", "scalar", "vector"])
def test_norm_gradients_against_differences(post, gate):
    rng = np.random.default_rng(4)
    T, N, eps, scale = 3, 8, 1e-5, 0.7
    x, y = rng.standard_normal((2, T, N))
    pre, pw = rng.standard_normal((2, N))
    pw = pw if post else None
    gv = None if gate == "none" else rng.standard_normal(N if gate == "vector" else 1)
    ds, dh = rng.standard_normal((2, T, N))

    def loss(x, y, pw, gv, pre):
        s, h = B.block_norm(x, y, pw, gv, pre, scale, eps)
        return (s * ds).sum() + (h * dh).sum()

    s, _ = B.block_norm(x, y, pw, gv, pre, scale, eps)
    got = B.block_norm_backward(ds, dh, s, y, pw, gv, pre, scale, eps)
    if gate == "scalar":
        got["dgate"] = got["dgate"].sum(keepdims=True)
    args = [x, y, pw, gv, pre]
    for i, name in enumerate(["dx", "dy", "dpost", "dgate", "dpre"]):
        if args[i] is None:
            continue
        num = np.zeros_like(args[i])
        for j in np.ndindex(args[i].shape):
            d = []
            for e in (1e-6, -1e-6):
                a = [None if v is None else v.copy() for v in args]
                a[i][j] += e
                d.append(loss(*a))
            num[j] = (d[0] - d[1]) / 2e-6
        assert np.abs(num - got[name]).max() < 1e-7 * max(1, np.abs(num).max()) * 10, name


# --------------------------------------------------------------------------- refusals
@pytest.fixture(scope="module")
def lib():
    from paper_2602_22592_b200 import build
    build.build()
    from paper_2602_22592_b200 import binding
    return binding


P = 1 << 20      # an aligned address that is never touched: every call below is refused before a launch


def cache(lib, **kw):
    f = dict(size=ctypes.sizeof(lib.pq_kv_cache), flags=0, format=lib.PQ_KV_INT8, heads=4, head_dim=100, page_size=32, num_pages=8, num_seqs=3,
             max_pages=5, reserved=0, K=P, V=P, k_gamma=P, v_gamma=P, page_table=P)
    f.update(kw)
    return lib.pq_kv_cache(*[f[n] for n, _ in lib.pq_kv_cache._fields_])


def test_struct_layouts_match_the_header(lib, tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    structs = {"pq_kv_cache": lib.pq_kv_cache, "pq_norm_desc": lib.pq_norm_desc}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "pquant.h"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    lines += ["return 0; }"]
    src, exe = tmp_path / "l.c", tmp_path / "l"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for cls in structs.values():
        want += [ctypes.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_status_string_and_pitch(lib):
    assert "range" in lib.pq_status_string(lib.PQ_ERR_INDEX)
    assert [lib.pq_kv_pitch(lib.PQ_KV_BF16, d) for d in (8, 100, 128, 252)] == [8, 104, 128, 256]
    assert [lib.pq_kv_pitch(lib.PQ_KV_INT8, d) for d in (8, 100, 128, 256)] == [16, 112, 128, 256]
    assert [lib.pq_kv_pitch(f, d) for f, d in ((0, 4), (0, 98), (1, 260), (2, 64), (-1, 64))] == [0] * 5


def test_cache_refusals(lib):
    L = lib.lib()

    def append(c, tokens=2, seq=P, pos=P, K=P, ks=0, V=P, vs=0, cos=None, sin=None, rows=0, Q=None, qs=0, qh=0, Qo=None):
        return L.pq_kv_append(ctypes.byref(c) if c else None, tokens, seq, pos, K, ks, V, vs, cos, sin, rows, Q, qs, qh, Qo, None)

    def read(c, tokens=2, seq=P, pos=P, K=P, V=P):
        return L.pq_kv_read(ctypes.byref(c) if c else None, tokens, seq, pos, K, V, None)

    def attend(c, heads=8, Q=P, qs=0, lens=P, scale=1.0, O=P, lse=None, ws=P, wb=1 << 40):
        return L.pq_attn_decode(ctypes.byref(c) if c else None, heads, Q, qs, lens, scale, O, lse, ws, wb, None)

    good = cache(lib)
    for call in (append, read, attend):
        assert call(None) == lib.PQ_ERR_NULL
        for field in ("K", "V", "k_gamma", "v_gamma", "page_table"):
            assert call(cache(lib, **{field: None})) == lib.PQ_ERR_NULL, field
            assert call(cache(lib, **{field: P + 8})) == lib.PQ_ERR_ALIGN, field
        for bad in (dict(size=4), dict(flags=1), dict(format=2), dict(heads=0), dict(head_dim=98), dict(head_dim=4), dict(head_dim=260),
                    dict(page_size=0), dict(page_size=24), dict(num_pages=0), dict(num_seqs=0), dict(max_pages=0), dict(max_pages=1 << 30)):
            assert call(cache(lib, **bad)) == lib.PQ_ERR_SHAPE, bad
    # tokens: none is a call that does nothing, fewer is an error
    assert append(good, tokens=0) == lib.PQ_OK and read(good, tokens=0) == lib.PQ_OK
    assert append(good, tokens=0, seq=None, pos=None, K=None, V=None) == lib.PQ_OK and read(good, tokens=0, seq=None, pos=None, K=None, V=None) == lib.PQ_OK
    assert append(good, tokens=-1) == lib.PQ_ERR_SHAPE and read(good, tokens=-1) == lib.PQ_ERR_SHAPE
    for name in ("seq", "pos", "K", "V"):
        assert append(good, **{name: None}) == lib.PQ_ERR_NULL and append(good, **{name: P + 4}) == lib.PQ_ERR_ALIGN
        assert read(good, **{name: None}) == lib.PQ_ERR_NULL and read(good, **{name: P + 4}) == lib.PQ_ERR_ALIGN
    assert append(good, cos=P) == lib.PQ_ERR_NULL and append(good, sin=P, rows=4) == lib.PQ_ERR_NULL
    assert append(good, cos=P, sin=P, rows=0) == lib.PQ_ERR_SHAPE and append(good, cos=P, sin=P + 4, rows=1) == lib.PQ_ERR_ALIGN
    assert append(good, Q=P, qh=4) == lib.PQ_ERR_NULL and append(good, Q=P, Qo=P, qh=0) == lib.PQ_ERR_SHAPE and append(good, qh=4) == lib.PQ_ERR_SHAPE
    assert append(good, ks=396) == lib.PQ_ERR_SHAPE and append(good, vs=402) == lib.PQ_ERR_SHAPE and append(good, ks=-400) == lib.PQ_ERR_SHAPE
    assert append(good, Q=P, Qo=P, qh=4, qs=1000) == lib.PQ_ERR_SHAPE      # in place needs dense rows
    # attention
    for name in ("Q", "lens", "O", "ws"):
        assert attend(good, **{name: None}) == lib.PQ_ERR_NULL and attend(good, **{name: P + 8}) == lib.PQ_ERR_ALIGN
    assert attend(good, lse=P + 4) == lib.PQ_ERR_ALIGN
    for heads in (0, 3, 6, -4):
        assert attend(good, heads=heads) == lib.PQ_ERR_SHAPE and lib.pq_attn_workspace_bytes(good, heads) == 0
    assert attend(good, qs=798) == lib.PQ_ERR_SHAPE and attend(good, qs=802) == lib.PQ_ERR_SHAPE
    for scale in (float("nan"), float("inf")):
        assert attend(good, scale=scale) == lib.PQ_ERR_SHAPE
    need = lib.pq_attn_workspace_bytes(good, 8)
    assert need > 0 and attend(good, wb=need - 1) == lib.PQ_ERR_WORKSPACE
    assert lib.pq_attn_workspace_bytes(cache(lib, K=None, V=None, page_table=None), 8) == need      # sizes alone


def test_norm_refusals(lib):
    L = lib.lib()

    def fwd(d, x=P, y=P, post=None, gate=None, pre=P, xo=P, h=P):
        return L.pq_block_norm_forward(ctypes.byref(d) if d else None, x, y, post, gate, pre, xo, h, None)

    def bwd(d, dxo=P, dh=P, xo=P, y=P, post=None, gate=None, pre=P, dx=P, dy=P, dpost=None, dgate=None, dpre=P, ws=P, wb=1 << 40):
        return L.pq_block_norm_backward(ctypes.byref(d) if d else None, dxo, dh, xo, y, post, gate, pre, dx, dy, dpost, dgate, dpre, ws, wb, None)

    good = lib.make_norm_desc(4, 64)
    bad = [lib.make_norm_desc(0, 64), lib.make_norm_desc(4, 4), lib.make_norm_desc(4, 68), lib.make_norm_desc(4, 16392), lib.make_norm_desc(4, 64, 0.0),
           lib.make_norm_desc(4, 64, float("nan")), lib.make_norm_desc(4, 64, 1e-5, float("inf"))]
    flagged = lib.make_norm_desc(4, 64)
    flagged.flags = 2
    sized = lib.make_norm_desc(4, 64)
    sized.size = 8
    for call in (fwd, bwd):
        assert call(None) == lib.PQ_ERR_NULL
        for d in bad + [flagged, sized]:
            assert call(d) == lib.PQ_ERR_SHAPE
            assert lib.pq_block_norm_workspace_bytes(d) == 0
    for kw in (dict(x=None), dict(xo=None, h=None, pre=None), dict(h=None), dict(pre=None), dict(y=None, post=P), dict(y=None, gate=P)):
        assert fwd(good, **kw) == lib.PQ_ERR_NULL, kw
    for name in ("x", "y", "post", "gate", "pre", "xo", "h"):
        assert fwd(good, **{name: P + 8}) == lib.PQ_ERR_ALIGN, name
    for kw in (dict(dxo=None, dh=None, pre=None), dict(dx=None), dict(ws=None), dict(dh=None), dict(pre=None), dict(xo=None), dict(dpre=None),
               dict(post=P, dpost=P, y=None), dict(gate=P, dgate=P, dy=None), dict(post=P), dict(gate=P)):
        assert bwd(good, **kw) == lib.PQ_ERR_NULL, kw
    for name in ("dxo", "dh", "xo", "y", "pre", "dx", "dy", "dpre", "ws"):
        assert bwd(good, **{name: P + 8}) == lib.PQ_ERR_ALIGN, name
    assert bwd(good, wb=lib.pq_block_norm_workspace_bytes(good) - 1) == lib.PQ_ERR_WORKSPACE


def test_binding_checks_types_shapes_and_layouts(lib):
    t = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype)  # noqa: E731
    table = t(3, 5, dtype=torch.int32)
    gam = t(8, 4, 32, dtype=torch.float32)
    for kw in (dict(K=t(8, 4, 32, 96)), dict(K=t(8, 4, 32, 104, dtype=torch.float16)), dict(V=t(8, 4, 32, 96)), dict(table=table.long()), dict(table=table[:, 0]),
               dict(K=t(8, 32, 4, 104).transpose(1, 2)), dict(kg=gam), dict(K=t(8, 4, 32, 112, dtype=torch.int8)), dict(table=table.t())):
        a = dict(K=t(8, 4, 32, 104), V=t(8, 4, 32, 104), table=table, kg=None)
        a.update(kw)
        with pytest.raises(lib.PqArgumentError):
            lib.make_kv_cache(a["K"], a["V"], a["table"], 100, a["kg"])
    c = lib.make_kv_cache(t(8, 4, 32, 104), t(8, 4, 32, 104), table, 100)
    assert (c.heads, c.head_dim, c.page_size, c.num_pages, c.num_seqs, c.max_pages) == (4, 100, 32, 8, 3, 5)
    # rows: dense or with a stride; on another device than the current one they are refused (here: the CPU, device -1)
    assert lib._rows_at("f", "x", t(5, 64), 5, 64, -1)[1] == 0 and lib._rows_at("f", "x", t(5, 2, 32), 5, 64, -1)[1] == 0
    assert lib._rows_at("f", "x", t(5, 96)[:, 32:], 5, 64, -1)[1] == 96 and lib._rows_at("f", "x", t(1, 96)[:, 32:], 1, 64, -1)[1] == 0
    for bad in (t(5, 64, dtype=torch.float16), t(64, 5).t(), t(4, 64), t(5, 2, 64)[:, :, :32], t(5, 128)[:, ::2]):
        with pytest.raises(lib.PqArgumentError):
            lib._rows_at("f", "x", bad, 5, 64, -1)
    for x in (t(5, 64), t(5, 96)[:, 32:]):
        with pytest.raises(lib.PqArgumentError, match="current device"):
            lib._rows_at("f", "x", x, 5, 64, 0)
    with pytest.raises(lib.PqArgumentError, match="contiguous"):
        lib._at("f", "x", t(64, 5).t(), torch.bfloat16, 320, -1)
    with pytest.raises(lib.PqArgumentError):
        lib._whole("f", "x", t(5, 64), 100)
    assert lib._at("f", "x", None, torch.int32, 7, 0) is None


def test_rows_that_lie_on_one_another_are_refused(lib):
    # one row for all (stride 0, which the library takes for dense rows: they would be read far behind the tensor's end) and overlapping ones
    one = torch.zeros(64, dtype=torch.bfloat16)
    for bad in (one.expand(5, 64), one[None].expand(5, 64), torch.zeros(320, dtype=torch.bfloat16).as_strided((5, 64), (32, 1))):
        with pytest.raises(lib.PqArgumentError):
            lib._rows_at("f", "x", bad, 5, 64, -1)
    assert lib._rows_at("f", "x", one.expand(1, 64), 1, 64, -1)[1] == 0


def test_empty_rotary_tables_are_refused(lib, monkeypatch):
    # an empty tensor has no address, which the library takes for a call without a rotation
    monkeypatch.setattr(lib, "_device", lambda: -1)
    cache = lib.make_kv_cache(torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16),
                              torch.zeros(1, 2, dtype=torch.int32), 64)
    row, at = torch.zeros(1, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    empty = torch.zeros(0, 32)
    monkeypatch.setattr(lib, "_stream", lambda s: None)
    monkeypatch.setattr(lib, "_check", lambda fn, status: pytest.fail("the call went through"))
    monkeypatch.setattr(lib, "lib", lambda: type("L", (), {"pq_kv_append": staticmethod(lambda *a: 0)}))
    with pytest.raises(lib.PqArgumentError):
        lib.pq_kv_append(cache, at, at, row, row, empty, empty)


@pytest.mark.parametrize("scale", [2.5e38, -3.4e38, float("inf"), float("-inf"), float("nan")])
def test_attention_scales_that_overflow_in_powers_of_two_are_refused(lib, scale):
    # the kernel takes scale log2(e): infinite for these, and a score of 0 would come out as NaN
    c = cache(lib)
    assert lib.lib().pq_attn_decode(ctypes.byref(c), 8, P, 0, P, scale, P, None, P, 1 << 40, None) == lib.PQ_ERR_SHAPE
