"""PQServer: weights that change behind a server, padding, the numbers of a prompt stage by stage, prompts in one piece and in several."""
import pytest
import torch

from paper_2602_22592_b200.decoder_harness import PQDecoder, PQServer
from test_gpu_between import DEV, check_status

pytestmark = pytest.mark.gpu


def model(seed, **kw):
    a = dict(layers=2, hidden=256, heads=4, ffn=512, vocab=300, batch=1, seq=64, r=32, E=4)
    return PQDecoder(**{**a, **kw}, seed=seed)


def tokens(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(0, 300, shape, generator=g, device=DEV)


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
