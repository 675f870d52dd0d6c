"""The example decoder: the operators of one block run together, in training
and in serving, against the same model written out in elementary torch."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

LENS = (5, 130, 1, 64)


def _patterns(seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, (6, 9), generator=gen), gen


@pytest.fixture(scope="module")
def dec():
    import decoder
    return decoder


def _model(dec, seed=1):
    torch.manual_seed(seed)
    return dec.Decoder(width=256, layers=2).cuda()


def _norm(x, w, eps=1e-6):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w


def _plain(model, tokens):
    """Logits of one sequence (L,) in the model's weights and 64 bits, step by step."""
    d = lambda t: t.double()
    x = d(model.embed.weight)[tokens]
    res = torch.zeros_like(x)
    for b in model.blocks:
        res = res + d(b.res_scale) * x
        q, k, v, z, a = (_norm(res, d(b.norm)) @ d(b.inp.weight).T).split(b.cols, dim=-1)
        q, k = (torch.nn.functional.normalize(t.unflatten(-1, (b.Hk, b.head)), dim=-1)
                .repeat_interleave(b.H // b.Hk, dim=1) for t in (q, k))
        v = v.unflatten(-1, (b.H, b.head))
        decay = torch.exp(-torch.nn.functional.softplus(a) * d(b.rate).exp())
        S, o = torch.zeros(b.H, b.head, b.head, dtype=torch.float64, device=x.device), []
        for t in range(len(tokens)):
            S = decay[t, :, None, None] * S + k[t, :, :, None] * v[t, :, None, :]
            o.append((q[t, :, :, None] * S).sum(1))
        u = torch.stack(o) * (z * torch.sigmoid(z)).unflatten(-1, (b.H, b.head))
        x = _norm(u, d(b.out_norm).view(b.H, b.head)).flatten(-2) @ d(b.out.weight).T
    return _norm(res + x, d(model.norm)) @ d(model.head.weight).T


# Twelve or so roundings to bf16 (2^-9 each, as a share of a vector's length) stand
# between the tokens and the logits; two layers of norms pass each on with a gain of
# about one: 12 x 2^-9 = 2.3 %, and twice that is allowed.
TOL = 2 * 12 * 2.0 ** -9


def test_prompt_is_the_recurrence(dec):
    model = _model(dec)
    tokens, cu = dec.packed(LENS, *_patterns(2), "cuda")
    logits, _ = model.prompt(tokens, cu)
    with torch.no_grad():
        want = torch.cat([_plain(model, tokens[0, a:b]) for a, b in zip(cu[:-1].tolist(), cu[1:].tolist())])
    err = (logits[0].double() - want).norm() / want.norm()
    assert err < TOL, err


def test_decode_continues_the_prompt(dec):
    """Prompts cut at any step and continued token by token give the whole's logits."""
    model = _model(dec)
    tokens, cu = dec.packed((40, 40, 40), *_patterns(3), "cuda")
    whole, _ = model.prompt(tokens, cu)
    rows = tokens.view(3, 40)
    first = (33, 7, 1)
    head = torch.cat([rows[n, :m] for n, m in enumerate(first)])[None]
    at = torch.tensor([0] + list(first)).cumsum(0).to(torch.int32).cuda()
    _, states = model.prompt(head, at)
    # the pool holds the sequences in another order, beside a slot of no sequence
    pools = [torch.stack([s[2], torch.full_like(s[0], 7.0), s[0], s[1]]) for s in states]
    slots = torch.tensor([2, 3, 0], dtype=torch.int32, device="cuda")
    for i in range(7):
        t = torch.tensor([rows[n, m + i].item() for n, m in enumerate(first)], device="cuda")
        got = model.decode(t, pools, slots)
        want = torch.stack([whole[0, 40 * n + m + i] for n, m in enumerate(first)])
        err = (got.double() - want.double()).norm() / want.double().norm()
        assert err < TOL, (i, err)
    assert all((p[1] == 7.0).all() for p in pools)


def test_gradients_reach_every_weight(dec):
    """Every weight's gradient is that of the 64-bit model."""
    model = _model(dec)
    tokens, cu = dec.packed((65,), *_patterns(4), "cuda")
    target = tokens[0, 1:]
    loss = torch.nn.functional.cross_entropy(model(tokens, cu)[0, :-1].float(), target)
    loss.backward()
    names = [n for n, p in model.named_parameters() if p.grad is None or not p.grad.isfinite().all()
             or (p.grad == 0).all()]
    assert not names, names
    wrt = list(model.parameters())
    plain = torch.nn.functional.cross_entropy(_plain(model, tokens[0])[:-1], target)
    want = torch.autograd.grad(plain, wrt)
    for (n, p), w in zip(model.named_parameters(), want):
        err = (p.grad.double() - w.double()).norm() / w.double().norm()
        # backwards as many roundings again
        assert err < 2 * TOL, (n, err)


def test_training_learns_and_repeats(dec):
    """The loss falls, and the same run gives the same losses to the bit."""
    runs = []
    for _ in range(2):
        model = _model(dec, seed=5)
        runs.append(dec.train(model, _patterns(6)[0], 12, _patterns(7)[1], lens=(128, 33, 64), log=None))
    assert runs[0][-1] < 0.9 * runs[0][0]
    assert runs[0] == runs[1]


def test_generate_runs(dec):
    model = _model(dec)
    tokens, cu = dec.packed(LENS, *_patterns(8), "cuda")
    out = dec.generate(model, tokens, cu, 4)
    assert out.shape == (len(LENS), 4) and int(out.min()) >= 0 and int(out.max()) < 256
