"""The example decoder with gated blocks between attention blocks and turned queries and
keys: embedding, head norm, gated recurrence and the operators around them run together,
in training and in serving, against the same model written out in elementary torch."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

LENS = (5, 130, 1, 0, 64)
F = torch.nn.functional


@pytest.fixture(scope="module")
def dec():
    import decoder
    return decoder


def _model(dec, seed=1, blocks="ga", rotary=32):
    torch.manual_seed(seed)
    return dec.Decoder(width=256, layers=2, blocks=blocks, rotary=rotary).cuda()


def _patterns(seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, (6, 9), generator=gen), gen


def _norm(x, w, eps=1e-6):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w


def _turn(x, freq):
    """x (L, heads, K): the first columns of step t turned by t * freq."""
    n = len(freq)
    angle = torch.arange(x.shape[0], device=x.device).double()[:, None] * freq.double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    p, q = x[..., :n], x[..., n:2 * n]
    return torch.cat([p * c - q * s, q * c + p * s, x[..., 2 * n:]], -1)


def _plain(model, tokens):
    """Logits of one sequence (L,) in the model's weights and 64 bits, step by step."""
    d = lambda t: t.double()  # noqa: E731
    x = d(model.embed.weight)[tokens]
    res = torch.zeros_like(x)
    for b in model.blocks:
        res = res + d(b.res_scale) * x
        y = _norm(res, d(b.norm)) @ d(b.inp.weight).T
        o = []
        if hasattr(b, "lam"):
            u, r, i, z = y.split(b.width, dim=-1)
            a = torch.exp(-8.0 * F.softplus(d(b.lam)) * torch.sigmoid(r))
            u = torch.sqrt(1 - a * a) * torch.sigmoid(i) * u
            h = torch.zeros_like(u[0])
            for t in range(len(tokens)):
                h = a[t] * h + u[t]
                o.append(h)
            o = torch.stack(o).unflatten(-1, (-1, b.head))
        else:
            q, k, v, z, g = y.split(b.cols, dim=-1)
            q, k = (t.unflatten(-1, (b.Hk, b.head)) for t in (q, k))
            q, k = (_turn(_norm(t, 1.0), b.freq).repeat_interleave(b.H // b.Hk, dim=1) / b.head ** 0.5
                    for t in (q, k))
            v = v.unflatten(-1, (b.H, b.head))
            decay = torch.exp(-F.softplus(g) * d(b.rate).exp())
            S = torch.zeros(b.H, b.head, b.head, dtype=torch.float64, device=x.device)
            for t in range(len(tokens)):
                S = decay[t, :, None, None] * S + k[t, :, :, None] * v[t, :, None, :]
                o.append((q[t, :, :, None] * S).sum(1))
            o = torch.stack(o)
        u = o * (z * torch.sigmoid(z)).unflatten(-1, (-1, b.head))
        x = _norm(u, d(b.out_norm).view(-1, b.head)).flatten(-2) @ d(b.out.weight).T
    return _norm(res + x, d(model.norm)) @ d(model.head.weight).T


# Some fourteen roundings to bf16 (2^-9 each, as a share of a vector's length) stand between
# the tokens and the logits; two layers of norms pass each on with a gain of about one: 14 x
# 2^-9 = 2.7 %, and twice that is allowed.
TOL = 2 * 14 * 2.0 ** -9


def test_prompt_is_the_recurrence(dec):
    model = _model(dec)
    tokens, cu = dec.packed(LENS, *_patterns(2), "cuda")
    logits, states = model.prompt(tokens, cu)
    with torch.no_grad():
        want = torch.cat([_plain(model, tokens[0, a:b]) for a, b in zip(cu[:-1].tolist(), cu[1:].tolist())
                          if b > a])
    err = (logits[0].double() - want).norm() / want.norm()
    assert err < TOL, err
    assert all((s[3] == 0).all() for s in states)  # the sequence of no tokens


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
    positions = torch.tensor(first, dtype=torch.int32, device="cuda")
    for i in range(7):
        t = torch.tensor([rows[n, m + i].item() for n, m in enumerate(first)], device="cuda")
        got = model.decode(t, pools, slots, positions + i)
        want = torch.stack([whole[0, 40 * n + m + i] for n, m in enumerate(first)])
        err = (got.double() - want.double()).norm() / want.double().norm()
        assert err < TOL, (i, err)
    assert all((p[1] == 7.0).all() for p in pools)


def test_gradients_reach_every_weight(dec):
    """Every weight's gradient is that of the 64-bit model."""
    model = _model(dec)
    tokens, cu = dec.packed((65,), *_patterns(4), "cuda")
    target = tokens[0, 1:]
    loss = F.cross_entropy(model(tokens, cu)[0, :-1].float(), target)
    loss.backward()
    names = [n for n, p in model.named_parameters() if p.grad is None or not p.grad.isfinite().all()
             or (p.grad == 0).all()]
    assert not names, names
    wrt = list(model.parameters())
    want = torch.autograd.grad(F.cross_entropy(_plain(model, tokens[0])[:-1], target), wrt)
    for (n, p), w in zip(model.named_parameters(), want):
        err = (p.grad.double() - w.double()).norm() / w.double().norm()
        # backwards as many roundings again
        assert err < 2 * TOL, (n, err)


def test_training_repeats_and_generates(dec):
    """The same run gives the same losses to the bit; prompts go on."""
    runs = []
    for _ in range(2):
        model = _model(dec, seed=5, blocks="gag")
        runs.append(dec.train(model, _patterns(6)[0], 6, _patterns(7)[1], lens=(128, 33, 64), log=None))
    assert runs[0] == runs[1]
    lens = tuple(n for n in LENS if n)
    tokens, cu = dec.packed(lens, *_patterns(8), "cuda")
    out = dec.generate(model, tokens, cu, 4)
    assert out.shape == (len(lens), 4) and int(out.min()) >= 0 and int(out.max()) < 256


def test_a_captured_decode_step(dec):
    """One token of each sequence through every operator, captured once and replayed."""
    model = _model(dec)
    tokens, cu = dec.packed((12, 20), *_patterns(9), "cuda")
    _, states = model.prompt(tokens, cu)
    slots = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    token = torch.tensor([3, 250], device="cuda")
    positions = torch.tensor([20, 12], dtype=torch.int32, device="cuda")
    pools = [s.clone() for s in states]
    model.decode(token, pools, slots, positions)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        logits = model.decode(token, pools, slots, positions)
    for p, s in zip(pools, states):
        p.copy_(s)
    eager = [s.clone() for s in states]
    for i in range(3):
        token.copy_(torch.tensor([7 * i, 11 * i + 1]))
        graph.replay()
        torch.cuda.synchronize()
        want = model.decode(token, eager, slots, positions)
        assert torch.equal(logits, want) and all(torch.equal(a, b) for a, b in zip(pools, eager)), i
        positions.add_(1)
