"""PQServer: weights that change behind a server, padding, the numbers of a prompt stage by stage, prompts in one piece and in several."""
import numpy as np
import pytest
import torch

from oracle import between_oracle as B
from paper_2602_22592_b200 import decoder_harness as harness
from paper_2602_22592_b200.decoder_harness import NORM_EPS, PQDecoder, PQServer
from test_gpu_between import DEV, HALF, bf16_sum_tol, check_status, close_norm, f64

pytestmark = pytest.mark.gpu


def model(seed, **kw):
    a = dict(layers=2, hidden=256, heads=4, ffn=512, vocab=300, batch=1, seq=64, r=32, E=4)
    return PQDecoder(**{**a, **kw}, seed=seed)


def tokens(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(0, 300, shape, generator=g, device=DEV)


def kept(S, layer, s, length):
    """What the cache keeps of the first positions of a sequence, from its bytes: keys and values [length, heads, dim] in 64 bits."""
    K, V, table, kg, vg = S.caches[layer].tensors
    p = np.arange(length)
    pg, at, D = table.cpu().numpy()[s, p // S.page_size], p % S.page_size, S.caches[layer].head_dim
    out = []
    for pages, gam in ((K, kg), (V, vg)):
        x = f64(pages)[pg, :, at, :D]
        out.append(x if gam is None else x / f64(gam)[pg, :, at][..., None])
    return out


class Recorder:
    """The calls that a prompt makes, with what they were given and what they left."""

    def __init__(self, mp):
        self.appends, self.norms, self.attentions = [], [], []
        append, norm, sdpa = harness.pqb.pq_kv_append, harness.pqb.pq_block_norm_forward, harness.F.scaled_dot_product_attention

        def pq_kv_append(cache, seq, pos, K, V, cos, sin, Q, Q_out, stream=None):
            append(cache, seq, pos, K, V, cos, sin, Q, Q_out, stream)
            self.appends.append(dict(pos=pos.cpu().numpy(), seq=seq.cpu().numpy(), k=f64(K), v=f64(V), q=f64(Q), q_rot=f64(Q_out)))

        def pq_block_norm_forward(d, x, y, post, gate, pre, x_out, h, stream=None):
            before = f64(x), None if y is None else f64(y)
            norm(d, x, y, post, gate, pre, x_out, h, stream)
            self.norms.append((*before, f64(pre), None if x_out is None else f64(x_out), f64(h)))

        def attention(q, k, v, attn_mask=None, **kw):
            out = sdpa(q, k, v, attn_mask=attn_mask, **kw)
            self.attentions.append((f64(q), f64(k), f64(v), attn_mask.cpu().numpy(), f64(out)))
            return out
        mp.setattr(harness.pqb, "pq_kv_append", pq_kv_append)
        mp.setattr(harness.pqb, "pq_block_norm_forward", pq_block_norm_forward)
        mp.setattr(harness.F, "scaled_dot_product_attention", attention)


def test_a_server_serves_the_weights_it_was_made_with():
    # the model's weights change and are packed again by a training step: a server made before answers as before, bit for bit
    m = model(63)
    first, second = (PQServer(m, 2, 40, 16, True) for _ in range(2))

    def answers(S):
        return [S.prompt(tokens(6, 2, 7), [7, 3])] + [S.step(tokens(7 + t, 2)) for t in range(2)] + [S.prompt(tokens(9, 2, 4), [2, 4])]
    want = answers(first)
    with torch.no_grad():
        for lin in m.linears():
            for t in (lin.W, lin.A, lin.B, lin.Wr):
                t.copy_((0.03 * torch.randn(t.shape, device=DEV)).to(t.dtype))
            lin.alpha.fill_(1.5)
            lin.beta.fill_(0.7)
        for t in m._torch_params():
            t.copy_((t + 0.1 * torch.randn(t.shape, device=DEV)).to(t.dtype))
    m.step(*m.random_batch())
    got = answers(second)
    torch.cuda.synchronize()
    check_status()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert not torch.equal(answers(PQServer(m, 2, 40, 16, True))[0], want[0])


@pytest.mark.parametrize("pad", [0, -100, 300, -301, 1 << 40])
def test_what_lies_behind_a_sequences_tokens_names_no_token(pad):
    m = model(64)
    lengths = [9, 2, 5]
    ids = tokens(8, 3, 9)
    behind = torch.arange(9, device=DEV)[None] >= torch.tensor(lengths, device=DEV)[:, None]
    want = PQServer(m, 3, 20, 16).prompt(torch.where(behind, 7, ids), lengths)
    assert torch.equal(PQServer(m, 3, 20, 16).prompt(torch.where(behind, pad, ids), lengths), want)


@pytest.mark.parametrize("int8", [False, True])
def test_prompt_stage_by_stage(int8, monkeypatch):
    # a first ragged prompt and a second one behind it: rotation and cache bit for bit, the mask, the attention, every norm, the logits
    m = model(61)
    n, H, D = 3, 4, 64
    S = PQServer(m, n, 60, 16, int8)
    for lengths in ([21, 1, 16], [5, 17, 2]):
        past, ids = list(S.held), tokens(len(S.held) + lengths[0], n, max(lengths))
        with monkeypatch.context() as mp:
            R = Recorder(mp)
            logits = S.prompt(ids, lengths)
        torch.cuda.synchronize()
        check_status()
        T = max(lengths)
        assert S.held == [a + b for a, b in zip(past, lengths)] and len(R.appends) == len(R.attentions) == 2 and len(R.norms) == 5
        assert np.array_equal(R.norms[0][0].reshape(n, T, -1)[[0, 1, 2], [x - 1 for x in lengths]], f64(m.embed)[ids.cpu().numpy()[[0, 1, 2], [x - 1 for x in lengths]]])
        for layer, (a, (q, k, v, mask, out)) in enumerate(zip(R.appends, R.attentions)):
            pos = a["pos"].reshape(n, T)
            for s in range(n):
                L, P = lengths[s], past[s]
                assert np.array_equal(pos[s], np.where(np.arange(T) < L, P + np.arange(T), -1))
                assert (a["seq"].reshape(n, T)[s] == s).all()
                cos, sin = (t[P:P + L].cpu().numpy() for t in (S.cos, S.sin))
                mine = lambda x: x.reshape(n, T, H, D)[s, :L]  # noqa: E731
                q_rot = B.rope(mine(a["q"]), cos, sin)
                assert np.array_equal(mine(a["q_rot"]), q_rot) and np.array_equal(q[s, :, :L], q_rot.transpose(1, 0, 2))
                keys, values = kept(S, layer, s, P + L)
                for rows, new in ((keys, B.rope(mine(a["k"]), cos, sin)), (values, mine(a["v"]))):
                    codes, g = B.quantise(new)
                    assert np.array_equal(rows[P:], codes / g.astype(np.float64)[..., None] if int8 else new)
                for dense, rows in ((k, keys), (v, values)):
                    want = B.bf16(rows.astype(np.float32)) if int8 else rows
                    assert np.array_equal(dense[s, :, :P + L], want.transpose(1, 0, 2)) and not dense[s, :, P + L:].any()
                for t in range(L):
                    assert np.array_equal(mask[s, 0, t], np.arange(mask.shape[-1]) <= P + t)
                    want, _, spread, big = B.attend(q_rot[t], k[s, :, :P + t + 1].transpose(1, 0, 2), v[s, :, :P + t + 1].transpose(1, 0, 2), D ** -0.5)
                    # torch's: scores and weights may be rounded to bf16
                    assert (np.abs(out[s, :, t] - want) <= HALF * np.abs(want) + (2 * 2 * HALF * big[:, None] + HALF) * spread).all(), (layer, s, t)
        for i, (x, y, w, x_out, h) in enumerate(R.norms):
            total = x if y is None else x + y
            if y is not None:
                assert (np.abs(x_out - total) <= bf16_sum_tol(x, y)).all()
                if i + 1 < len(R.norms):
                    assert np.array_equal(R.norms[i + 1][0], x_out)
            close_norm(h, total, w, np.zeros_like(total) if y is None else 2.0 ** -23 * (np.abs(x) + np.abs(y)))
        last = R.norms[-1][4].reshape(n, T, -1)[[0, 1, 2], [x - 1 for x in lengths]]
        head = f64(m.head)
        want = last @ head.T
        assert (np.abs(f64(logits) - want) <= HALF * np.abs(want) + (256 + 8) * 2.0 ** -23 * (np.abs(last) @ np.abs(head).T)).all()


@pytest.mark.parametrize("int8", [False, True])
def test_a_prompt_in_pieces_and_by_steps_keeps_what_one_prompt_keeps(int8):
    # the first layer's keys and values are functions of a token and its place.  Without experts a projection is an exact integer sum, scaled
    # and rounded to bf16, on every path: outputs a rounding apart at most (2^-7), which a rotation spreads over a pair, and int8 adds
    # half a step of either (128 codes)
    m = model(62, r=0, E=0)
    ids = tokens(5, 2, 24)
    whole, pieces = PQServer(m, 2, 30, 16, int8), PQServer(m, 2, 30, 16, int8)
    whole.prompt(ids, [24, 24])
    pieces.prompt(ids[:, :9], [9, 9])
    pieces.prompt(ids[:, 9:20], [11, 11])
    for t in range(20, 24):
        pieces.step(ids[:, t])
    torch.cuda.synchronize()
    check_status()
    assert whole.held == pieces.held == [24, 24]
    for s in range(2):
        for a, b in zip(kept(whole, 0, s, 24), kept(pieces, 0, s, 24)):
            pair = np.abs(a) + np.abs(np.roll(a, 32, -1)) + np.abs(b)
            tol = 4 * HALF * pair + (np.abs(a).max(-1, keepdims=True) / 128 * 1.01 if int8 else 0)
            assert (np.abs(a - b) <= tol).all() and np.abs(a).max() > 0


def test_a_refused_call_changes_nothing():
    # ids of another shape: refused before the sequences grow, so that the next call's tokens stand where they belong
    m = model(65)
    S, other = PQServer(m, 2, 20, 16), PQServer(m, 2, 20, 16)
    S.prompt(tokens(1, 2, 3), [3, 2])
    for bad in (lambda: S.step(tokens(2, 3)), lambda: S.step(tokens(2, 2, 1)), lambda: S.prompt(tokens(2, 3, 4), [4, 4]), lambda: S.prompt(tokens(2, 4), [4, 4]),
                lambda: S.prompt(tokens(2, 2, 4), [4, 3, 1]), lambda: S.prompt(tokens(2, 2, 4), [3, 3]), lambda: S.prompt(tokens(2, 2, 4), [4, 0])):
        with pytest.raises(ValueError):
            bad()
    for n in (0, 17):
        with pytest.raises(ValueError):
            PQServer(m, n, 20, 16)
    assert S.held == [3, 2]
    other.prompt(tokens(1, 2, 3), [3, 2])
    assert torch.equal(S.step(tokens(4, 2)), other.step(tokens(4, 2)))
