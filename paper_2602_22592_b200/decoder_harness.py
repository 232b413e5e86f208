"""A LLaMA-style decoder whose every projection is a pQuant linear: the harness around the C entry points for the
"whole training step" workload (24 layers, hidden 2048, 16 heads, FFN 5632, RMSNorm, RoPE, vocabulary 32000 at
full size).

Training (`PQDecoder.step`): each projection is `pq_pack_weights` + `pq_linear_forward` in the forward pass and
`pq_linear_backward` in the backward pass, reached through a torch.autograd.Function that marshals pointers and
nothing else.  Embedding, rotary embedding, attention, SiLU gating, LM head and cross-entropy are ordinary torch; so are the norms and
the residual additions unless the model is made with `library_norms=True`: then `pq_block_norm_forward` /
`pq_block_norm_backward` add a block's output to the stream and norm it for the next one in one pass each way.

Serving (`PQServer`): prompts and then one token per sequence at a time.  Projections run from the packed sign bits
(`pq_decode_batch`) or, for prompts, on the tensor cores; keys and values live in a paged cache (`pq_kv_append`, bf16 or int8), a new
token attends over it with `pq_attn_decode`, a prompt over its history as `pq_kv_read` gives it back, and
`pq_block_norm_forward` stands between the blocks.  SiLU gating, the prompt's attention and the LM head are torch.

CUDA events around every pq_* call let the caller report the pQuant-linear time of a step apart from the rest.
"""
from __future__ import annotations

import math

import torch
import torch.nn.functional as F

from . import binding as pqb

NORM_EPS = 1e-5


class _Workspaces:
    """Forward / backward / pack workspaces shared by all linears of one model (calls are serial on one stream)."""

    def __init__(self, device):
        self.dev = device
        self.fwd = self.bwd = self.pack = None

    def reserve(self, desc):
        def grow(buf, n):
            return buf if buf is not None and buf.numel() >= n else torch.empty(max(n, 16), dtype=torch.uint8, device=self.dev)
        self.fwd = grow(self.fwd, pqb.pq_workspace_bytes(desc, pqb.PQ_PHASE_FWD))
        self.bwd = grow(self.bwd, pqb.pq_workspace_bytes(desc, pqb.PQ_PHASE_BWD))
        self.pack = grow(self.pack, pqb.pq_workspace_bytes(desc, pqb.PQ_PHASE_PACK))


class Timer:
    """Sums the device time of the pq_* calls of a step: one event pair per call, read after the step."""

    def __init__(self):
        self.pairs = []
        self.enabled = False

    def begin(self):
        if not self.enabled:
            return None
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        self.pairs.append((a, b))
        return b

    @staticmethod
    def end(b):
        if b is not None:
            b.record()

    def total_ms(self):
        """Call after a synchronise.  Clears the recorded pairs."""
        t = sum(a.elapsed_time(b) for a, b in self.pairs)
        self.pairs = []
        return t


class _PQLinearFn(torch.autograd.Function):
    """x [T,K] bf16 -> y [T,N] bf16 through the C ABI.  Parameter gradients are not returned to autograd: the
    library overwrites the module's gradient buffers (dW, dA, dB, dWr, dalpha, dbeta), which is what the ABI
    promises; accumulation over micro-batches would be the optimiser's business."""

    @staticmethod
    def forward(ctx, x, mod):
        ctx.mod = mod
        x = x.contiguous()
        ctx.save_for_backward(x)
        return mod._forward(x)

    @staticmethod
    def backward(ctx, dy):
        (x,) = ctx.saved_tensors
        return ctx.mod._backward(x, dy.contiguous()), None


class PQLinearModule:
    """One pQuant linear (Eq. 10-11, Sec. 3.3) of a model: latent fp32 W, bf16 experts A, B, router Wr, scalar feature
    scales; `saved` is its own (it lives from forward to backward), workspaces are the model's."""

    def __init__(self, T, K, N, r, E, ws: _Workspaces, timer: Timer, gen, device, name=""):
        self.T, self.K, self.N, self.r, self.E, self.name = T, K, N, r, (E if r > 0 else 0), name
        self.ws, self.timer = ws, timer
        self.desc = pqb.make_desc(T, K, N, r, self.E, 1, False)
        ws.reserve(self.desc)
        dev = device
        std = 0.02
        self.W = torch.randn((N, K), generator=gen, device=dev, dtype=torch.float32) * std
        Ee = max(self.E, 1)
        if r > 0:
            self.A = (torch.randn((Ee, r, K), generator=gen, device=dev) * std).to(torch.bfloat16)
            self.B = (torch.randn((Ee, N, r), generator=gen, device=dev) * std).to(torch.bfloat16)
            self.Wr = (torch.randn((Ee, K), generator=gen, device=dev) * std).to(torch.bfloat16) if Ee > 1 else None
            self.dA = torch.empty((Ee, r, K), dtype=torch.float32, device=dev)
            self.dB = torch.empty((Ee, N, r), dtype=torch.float32, device=dev)
            self.dWr = torch.empty((Ee, K), dtype=torch.float32, device=dev) if Ee > 1 else None
        else:
            self.A = self.B = self.Wr = self.dA = self.dB = self.dWr = None
        self.alpha = torch.full((1,), 2.0, device=dev)     # the paper's initial feature scales (Sec. 3.2)
        self.beta = torch.full((1,), 0.2, device=dev)
        self.dalpha = torch.empty(1, dtype=torch.float32, device=dev)
        self.dbeta = torch.empty(1, dtype=torch.float32, device=dev)
        self.dW = torch.empty((N, K), dtype=torch.float32, device=dev)
        self.w_bits = torch.empty((N, K // 32), dtype=torch.int32, device=dev)
        self.w_s8 = torch.empty((N, K), dtype=torch.int8, device=dev)
        self.w_scales = torch.empty(2, dtype=torch.float32, device=dev)
        self.saved = torch.empty(pqb.pq_saved_bytes(self.desc), dtype=torch.uint8, device=dev)
        self.capture = None        # set to a dict by tests: receives x, y, dy, dx of the next call

    def __call__(self, x):
        return _PQLinearFn.apply(x, self)

    def _forward(self, x):
        assert x.shape == (self.T, self.K) and x.dtype == torch.bfloat16
        y = torch.empty((self.T, self.N), dtype=torch.bfloat16, device=x.device)
        ev = self.timer.begin()
        # QAT re-quantises the latent weights in every forward pass
        pqb.pq_pack_weights(self.desc, self.W, self.w_bits, self.w_s8, self.w_scales, self.ws.pack)
        pqb.pq_linear_forward(self.desc, x, self.w_bits, self.w_s8, self.w_scales, self.A, self.B, self.Wr, self.alpha, self.beta, y,
                              self.saved, self.ws.fwd)
        self.timer.end(ev)
        if self.capture is not None:
            self.capture.update(x=x.detach().clone(), y=y.detach().clone())
        return y

    def _backward(self, x, dy):
        dx = torch.empty((self.T, self.K), dtype=torch.bfloat16, device=x.device)
        ev = self.timer.begin()
        pqb.pq_linear_backward(self.desc, dy, x, self.w_s8, self.w_scales, self.A, self.B, self.Wr, self.alpha, self.beta, self.saved,
                               dx, self.dW, self.dA, self.dB, self.dWr, self.dalpha, self.dbeta, self.ws.bwd)
        self.timer.end(ev)
        if self.capture is not None:
            self.capture.update(dy=dy.detach().clone(), dx=dx.detach().clone())
        return dx


class _NormFn(torch.autograd.Function):
    """(x, y, weight) -> x + y and its RMSNorm times weight; without y the norm of x alone (the first one of a model)."""

    @staticmethod
    def forward(ctx, x, y, weight, mod):
        ctx.set_materialize_grads(False)
        x = x.contiguous()
        h = torch.empty_like(x)
        out = x if y is None else torch.empty_like(x)
        y = None if y is None else y.contiguous()
        pqb.pq_block_norm_forward(mod.norm_desc, x, y, None, None, weight.detach(), None if y is None else out, h)
        ctx.mod, ctx.joined = mod, y is not None
        ctx.save_for_backward(out, weight)
        if mod.norm_capture is not None:
            mod.norm_capture.append(dict(x=x.detach().clone(), y=None if y is None else y.detach().clone(), weight=weight.detach().clone(), h=h.clone(),
                                         x_out=out.detach().clone()))
            ctx.capture = mod.norm_capture[-1]
        return (out, h) if ctx.joined else h

    @staticmethod
    def backward(ctx, *grads):
        out, weight = ctx.saved_tensors
        dx_out, dh = grads if ctx.joined else (None, grads[0])
        dx_out, dh = (None if g is None else g.contiguous() for g in (dx_out, dh))
        if dh is None:                        # nothing came back through the norm
            return dx_out, dx_out if ctx.joined else None, None, None
        dx = torch.empty_like(out)
        dweight = torch.empty(weight.numel(), dtype=torch.float32, device=out.device)
        pqb.pq_block_norm_backward(ctx.mod.norm_desc, dx_out, dh, out, None, None, None, weight.detach(), dx, None, None, None, dweight, ctx.mod.norm_ws)
        if ctx.mod.norm_capture is not None:
            ctx.capture.update(dx_out=None if dx_out is None else dx_out.clone(), dh=dh.clone(), dx=dx.clone(), dweight=dweight.clone())
        return dx, dx if ctx.joined else None, dweight.to(weight.dtype), None


def _rope_tables(seq, head_dim, device, base=10000.0):
    inv = 1.0 / (base ** (torch.arange(0, head_dim, 2, device=device, dtype=torch.float32) / head_dim))
    ang = torch.outer(torch.arange(seq, device=device, dtype=torch.float32), inv)     # [S, D/2]
    return ang.cos(), ang.sin()


def _apply_rope(x, cos, sin):
    # x [B, H, S, D]; rotate pairs (even, odd halves)
    d = x.shape[-1] // 2
    x1, x2 = x[..., :d].float(), x[..., d:].float()
    return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], dim=-1).to(x.dtype)


class PQDecoder:
    """The decoder.  `attn_hp=False` makes the four attention projections pure 1-bit linears (r = 0), the form the
    paper gives its attention blocks (Sec. 3); True gives them the same routed HP branch as the MLP projections."""

    def __init__(self, layers=24, hidden=2048, heads=16, ffn=5632, vocab=32000, batch=4, seq=2048, r=128, E=8, attn_hp=True,
                 device="cuda:0", seed=3, library_norms=False):
        self.dev = torch.device(device)
        self.layers, self.hidden, self.heads, self.ffn, self.vocab, self.batch, self.seq = layers, hidden, heads, ffn, vocab, batch, seq
        self.head_dim = hidden // heads
        gen = torch.Generator(device=self.dev)
        gen.manual_seed(seed)
        T = batch * seq
        self.T = T
        self.ws = _Workspaces(self.dev)
        self.timer = Timer()
        mk = lambda K, N, rr, name: PQLinearModule(T, K, N, rr, E, self.ws, self.timer, gen, self.dev, name)
        ra = r if attn_hp else 0
        self.blocks = []
        for i in range(layers):
            blk = dict(q=mk(hidden, hidden, ra, f"L{i}.q"), k=mk(hidden, hidden, ra, f"L{i}.k"), v=mk(hidden, hidden, ra, f"L{i}.v"),
                       o=mk(hidden, hidden, ra, f"L{i}.o"), gate=mk(hidden, ffn, r, f"L{i}.gate"), up=mk(hidden, ffn, r, f"L{i}.up"),
                       down=mk(ffn, hidden, r, f"L{i}.down"),
                       norm1=torch.ones(hidden, device=self.dev, dtype=torch.bfloat16, requires_grad=True),
                       norm2=torch.ones(hidden, device=self.dev, dtype=torch.bfloat16, requires_grad=True))
            self.blocks.append(blk)
        self.embed = (torch.randn((vocab, hidden), generator=gen, device=self.dev) * 0.02).to(torch.bfloat16).requires_grad_(True)
        self.head = (torch.randn((vocab, hidden), generator=gen, device=self.dev) * 0.02).to(torch.bfloat16).requires_grad_(True)
        self.norm_f = torch.ones(hidden, device=self.dev, dtype=torch.bfloat16, requires_grad=True)
        self.cos, self.sin = _rope_tables(seq, self.head_dim, self.dev)
        self.gen = gen
        self.library_norms = library_norms
        self.norm_capture = None      # set to a list by tests: receives a dict for every norm of the next step
        if library_norms:
            self.norm_desc = pqb.make_norm_desc(T, hidden, NORM_EPS)
            self.norm_ws = torch.empty(pqb.pq_block_norm_workspace_bytes(self.norm_desc), dtype=torch.uint8, device=self.dev)

    def linears(self):
        for blk in self.blocks:
            for k in ("q", "k", "v", "o", "gate", "up", "down"):
                yield blk[k]

    def random_batch(self):
        ids = torch.randint(0, self.vocab, (self.batch, self.seq), generator=self.gen, device=self.dev)
        tgt = torch.randint(0, self.vocab, (self.batch, self.seq), generator=self.gen, device=self.dev)
        return ids, tgt

    def _torch_params(self):
        ps = [self.embed, self.head, self.norm_f]
        for blk in self.blocks:
            ps += [blk["norm1"], blk["norm2"]]
        return ps

    def step(self, ids, tgt):
        """One forward + backward (no optimiser).  Returns the loss tensor."""
        for p in self._torch_params():
            p.grad = None
        B, S, H, D = self.batch, self.seq, self.heads, self.head_dim
        lib = self.library_norms
        norm = lambda x, w: _NormFn.apply(x, None, w, self) if lib else F.rms_norm(x, (self.hidden,), w, NORM_EPS)

        def join(x, y, w):
            """The stream behind a block, and the next block's input."""
            if lib:
                return _NormFn.apply(x, y, w, self)
            x = x + y
            return x, F.rms_norm(x, (self.hidden,), w, NORM_EPS)

        x = F.embedding(ids, self.embed).view(B * S, self.hidden)
        h = norm(x, self.blocks[0]["norm1"])
        for i, blk in enumerate(self.blocks):
            q = blk["q"](h).view(B, S, H, D).transpose(1, 2)
            k = blk["k"](h).view(B, S, H, D).transpose(1, 2)
            v = blk["v"](h).view(B, S, H, D).transpose(1, 2)
            q, k = _apply_rope(q, self.cos, self.sin), _apply_rope(k, self.cos, self.sin)
            a = F.scaled_dot_product_attention(q, k, v, is_causal=True)
            a = a.transpose(1, 2).reshape(B * S, self.hidden)
            x, h = join(x, blk["o"](a), blk["norm2"])
            m = F.silu(blk["gate"](h)) * blk["up"](h)
            x, h = join(x, blk["down"](m), self.blocks[i + 1]["norm1"] if i + 1 < self.layers else self.norm_f)
        logits = h @ self.head.t()
        loss = F.cross_entropy(logits.float(), tgt.view(-1))
        loss.backward()
        return loss.detach()

    def roofline_time_s(self, p_bf16, p_i8):
        """Sum over the linears of 2TNK / P_i8 + (4TNK + 6Tr(K+N)) / P_bf16."""
        t = 0.0
        for L in self.linears():
            tnk = L.T * L.N * L.K
            t += 2 * tnk / p_i8 + (4 * tnk + 6 * L.T * L.r * (L.K + L.N)) / p_bf16
        return t


class _ServedLinear:
    """A linear's weights as a server keeps them: packed once, every tensor its own."""

    def __init__(self, lin: PQLinearModule):
        self.K, self.N, self.r, self.E = lin.K, lin.N, lin.r, lin.E
        self.w_bits, self.w_s8, self.w_scales = (torch.empty_like(t) for t in (lin.w_bits, lin.w_s8, lin.w_scales))
        pqb.pq_pack_weights(lin.desc, lin.W, self.w_bits, self.w_s8, self.w_scales, lin.ws.pack)
        self.A, self.B, self.Wr, self.alpha, self.beta = (None if t is None else t.clone() for t in (lin.A, lin.B, lin.Wr, lin.alpha, lin.beta))


class PQServer:
    """Serves a PQDecoder's weights to `n` sequences (16 at most: the decode path's tokens): `prompt` takes their first tokens, or more of
    them later, `step` one new token each; both return the logits of every sequence's last token [n, vocab].

    The cache has room for `positions` tokens a sequence in pages of `page_size`, handed out as sequences grow; lengths live on the
    host (a program that admits and frees sequences does so there) and on the device.  Weights are packed and every other parameter is
    copied when the server is made: what becomes of the model afterwards does not reach it."""

    def __init__(self, model: PQDecoder, n, positions, page_size=64, int8_cache=False):
        if not 1 <= n <= 16:
            raise ValueError(f"{n} sequences: the decode path takes 1 to 16")
        self.m, self.n, self.positions = model, n, positions
        dev, H, D, L = model.dev, model.heads, model.head_dim, model.layers
        self.dev = dev
        self.entries = -(-positions // page_size)
        pages = n * self.entries
        pitch = pqb.pq_kv_pitch(pqb.PQ_KV_INT8 if int8_cache else pqb.PQ_KV_BF16, D)
        self.table = torch.full((n, self.entries), -1, dtype=torch.int32, device=dev)
        self.free = list(range(pages - 1, -1, -1))
        self.page_size, self.held = page_size, [0] * n
        shape = (pages, H, page_size, pitch)
        pages_of = lambda: torch.zeros(shape, dtype=torch.int8 if int8_cache else torch.bfloat16, device=dev)
        gammas = lambda: torch.ones(shape[:3], device=dev) if int8_cache else None
        self.caches = [pqb.make_kv_cache(pages_of(), pages_of(), self.table, D, gammas(), gammas()) for _ in range(L)]     # one table, a cache a layer
        self.cos, self.sin = _rope_tables(positions, D, dev)
        self.attn_ws = torch.empty(pqb.pq_attn_workspace_bytes(self.caches[0], H), dtype=torch.uint8, device=dev)
        self.seq = torch.arange(n, dtype=torch.int32, device=dev)
        self.desc = pqb.make_norm_desc(n, model.hidden, NORM_EPS)
        self.capture = None       # set to a list by tests: receives a dict for every layer of the next call
        own = lambda t: t.detach().clone()
        self.blocks = [{name: own(p) if name.startswith("norm") else _ServedLinear(p) for name, p in blk.items()} for blk in model.blocks]
        self.embed, self.head, self.norm_f = own(model.embed), own(model.head), own(model.norm_f)
        self.items = [{names: self._items(blk, names) for names in (("q", "k", "v"), ("o",), ("gate", "up"), ("down",))} for blk in self.blocks]

    def _items(self, blk, names):
        """Decode descriptors of linears that read the same tokens, with their inputs, outputs and workspaces."""
        lins = [blk[k] for k in names]
        x = torch.empty((self.n, lins[0].K), dtype=torch.bfloat16, device=self.dev)
        ys, entries, keep = [], [], []
        for lin in lins:
            d = pqb.make_desc(self.n, lin.K, lin.N, lin.r, lin.E)
            ys.append(torch.empty((self.n, lin.N), dtype=torch.bfloat16, device=self.dev))
            nb, nB = pqb.pq_decode_pack_bytes(d)
            bits = torch.empty(nb, dtype=torch.uint8, device=self.dev)
            b_il = torch.empty(nB, dtype=torch.uint8, device=self.dev) if nB else None
            pqb.pq_pack_decode(d, lin.w_bits, lin.B, bits, b_il)
            ws = torch.zeros(max(16, pqb.pq_workspace_bytes(d, pqb.PQ_PHASE_DECODE)), dtype=torch.uint8, device=self.dev)
            entries.append((d, x, lin.w_bits, lin.w_scales, lin.A, lin.B, lin.Wr, lin.alpha, lin.beta, ys[-1], ws, None, 0.0, bits, b_il))
            keep += [bits, b_il, ws]
        return x, ys, pqb.make_decode_items(entries), keep

    def _grow(self, more):
        """Pages for more[s] further tokens of sequence s; nothing changes where one of them has no room."""
        for s, k in enumerate(more):
            if self.held[s] + k > self.positions:
                raise ValueError(f"sequence {s}: {self.held[s] + k} tokens, there is room for {self.positions}")
        for s, k in enumerate(more):
            have, need = -(-self.held[s] // self.page_size), -(-(self.held[s] + k) // self.page_size)
            if need > have:
                ids = [self.free.pop() for _ in range(need - have)]
                self.table[s, have:need] = torch.tensor(ids, dtype=torch.int32, device=self.dev)
        self.held = [h + k for h, k in zip(self.held, more)]

    def _decode(self, i, names, x):
        xin, ys, items, _ = self.items[i][names]
        xin.copy_(x)
        pqb.pq_decode_batch(items)
        return ys

    def step(self, ids):
        """One new token of every sequence: ids [n]."""
        m, n = self.m, self.n
        if ids.shape != (n,):
            raise ValueError(f"ids has to be [{n}], one token of every sequence")
        self._grow([1] * n)
        lens = torch.tensor(self.held, dtype=torch.int32, device=self.dev)
        pos = lens - 1
        x = self.embed[ids]
        h, q_rot, a = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
        pqb.pq_block_norm_forward(self.desc, x, None, None, None, self.blocks[0]["norm1"], None, h)
        for i, blk in enumerate(self.blocks):
            q, k, v = self._decode(i, ("q", "k", "v"), h)
            pqb.pq_kv_append(self.caches[i], self.seq, pos, k, v, self.cos, self.sin, q, q_rot)
            pqb.pq_attn_decode(self.caches[i], q_rot, lens, m.head_dim ** -0.5, a, None, self.attn_ws)
            if self.capture is not None:
                self.capture.append(dict(q=q.clone(), k=k.clone(), v=v.clone(), q_rot=q_rot.clone(), a=a.clone(), lens=lens.clone(), x=x.clone()))
            y, = self._decode(i, ("o",), a)
            pqb.pq_block_norm_forward(self.desc, x, y, None, None, blk["norm2"], x, h)
            if self.capture is not None:
                self.capture[-1].update(o=y.clone(), x_out=x.clone(), h=h.clone())
            gate, up = self._decode(i, ("gate", "up"), h)
            y, = self._decode(i, ("down",), F.silu(gate) * up)
            pqb.pq_block_norm_forward(self.desc, x, y, None, None, self.blocks[i + 1]["norm1"] if i + 1 < m.layers else self.norm_f, x, h)
        return h @ self.head.t()

    def prompt(self, ids, lengths):
        """lengths[s] further tokens of every sequence (host integers, at least 1), ids [n, max(lengths)]; what lies behind a sequence's own
        tokens is padding and may be any number.  They attend over what the sequence holds already, and over one another in order."""
        m, n, S = self.m, self.n, ids.shape[-1]
        if ids.shape != (n, S) or len(lengths) != n or max(lengths) != S or min(lengths) < 1:
            raise ValueError(f"ids has to be [{n}, longest of lengths], and every sequence has to get a token")
        past = list(self.held)
        self._grow(lengths)
        T, H, D, dev = n * S, m.heads, m.head_dim, self.dev
        at = torch.arange(S, device=dev)[None]
        begin, count = torch.tensor(past, device=dev)[:, None], torch.tensor(lengths, device=dev)[:, None]
        pos = torch.where(at < count, begin + at, -1).to(torch.int32).reshape(-1)
        seq = torch.arange(n, dtype=torch.int32, device=dev).repeat_interleave(S)
        most = max(self.held)
        all_at = torch.arange(most, device=dev)[None]
        held = torch.tensor(self.held, device=dev)[:, None]
        all_pos = torch.where(all_at < held, all_at, -1).to(torch.int32).reshape(-1)
        all_seq = torch.arange(n, dtype=torch.int32, device=dev).repeat_interleave(most)
        mask = all_at[:, None, :] <= (begin + at)[:, :, None]                                  # [n, S, most]
        desc = pqb.make_norm_desc(T, m.hidden, NORM_EPS)
        x = self.embed[torch.where(at < count, ids.to(dev), 0)].reshape(T, m.hidden)           # a padding id need not be in the vocabulary
        h, q_rot = torch.empty_like(x), torch.empty_like(x)
        pqb.pq_block_norm_forward(desc, x, None, None, None, self.blocks[0]["norm1"], None, h)

        def linear(lin, x):
            d = pqb.make_desc(T, lin.K, lin.N, lin.r, lin.E)
            y = torch.empty((T, lin.N), dtype=torch.bfloat16, device=dev)
            ws = torch.empty(pqb.pq_workspace_bytes(d, pqb.PQ_PHASE_FWD), dtype=torch.uint8, device=dev)
            pqb.pq_linear_forward(d, x, lin.w_bits, lin.w_s8, lin.w_scales, lin.A, lin.B, lin.Wr, lin.alpha, lin.beta, y, None, ws)
            return y

        for i, blk in enumerate(self.blocks):
            q, k, v = (linear(blk[name], h) for name in "qkv")
            q_rot.zero_()                                       # rows of padding are left as they are
            pqb.pq_kv_append(self.caches[i], seq, pos, k, v, self.cos, self.sin, q, q_rot)
            ks, vs = (torch.zeros((n * most, H * D), dtype=torch.bfloat16, device=dev) for _ in range(2))
            pqb.pq_kv_read(self.caches[i], all_seq, all_pos, ks, vs)
            heads = lambda t, rows: t.view(n, rows, H, D).transpose(1, 2)
            a = F.scaled_dot_product_attention(heads(q_rot, S), heads(ks, most), heads(vs, most), attn_mask=mask[:, None])
            y = linear(blk["o"], a.transpose(1, 2).reshape(T, m.hidden))
            pqb.pq_block_norm_forward(desc, x, y, None, None, blk["norm2"], x, h)
            y = linear(blk["down"], F.silu(linear(blk["gate"], h)) * linear(blk["up"], h))
            pqb.pq_block_norm_forward(desc, x, y, None, None, self.blocks[i + 1]["norm1"] if i + 1 < m.layers else self.norm_f, x, h)
        last = torch.arange(n, device=dev) * S + count[:, 0] - 1
        return h[last] @ self.head.t()


def softmax_entropy_bound(vocab):
    """Loss of a uniform prediction, ln(vocab): what a randomly initialised model should be near."""
    return math.log(vocab)
