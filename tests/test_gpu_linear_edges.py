"""Linear attention at the edges of its contract: packed rows padded to a fixed length,
no heads, many sequences, graphs of the backward, offsets past 32 bits."""
import numpy as np
import pytest

import linear_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _rand(seed, dtype, **shapes):
    r = np.random.Generator(np.random.PCG64(seed))
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    return {n: torch.from_numpy(r.standard_normal(s)).to(dt if n in ("q", "k", "v", "do") else torch.float32)
            .cuda() for n, s in shapes.items()}


def _poison():
    """Freed blocks full of NaN, where the next allocations lie."""
    for n in (1 << 10, 1 << 14, 1 << 18, 1 << 22):
        blocks = [torch.full((n,), float("nan"), device="cuda") for _ in range(8)]
        del blocks


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hk, H, K, V, const", [(2, 2, 32, 64, False), (1, 3, 13, 7, False),
                                                (2, 8, 64, 64, True), (1, 2, 136, 65, False)])
@pytest.mark.parametrize("L, cu", [(700, [0, 5, 5, 300]), (260, [3, 64, 259]), (9, [9, 9]), (40, [0, 0]),
                                   (64, [0, 10, 64])])
def test_steps_that_no_sequence_covers(sw, L, cu, Hk, H, K, V, const, dtype):
    """Zero in o and in every gradient, whatever the inputs hold there; the covered
    steps are those of the row cut to them."""
    print("case uncovered", L, cu, Hk, H, K, V, dtype, flush=True)
    n = len(cu) - 1
    t = _rand(L + K, dtype, q=(1, L, Hk, K), k=(1, L, Hk, K), v=(1, L, H, V), do=(1, L, H, V),
              g=(H,) if const else (1, L, H), h0=(n, H, K, V), dh=(n, H, K, V))
    t["g"] = -0.1 * t["g"].abs()
    for name in ("q", "k", "v", "do") + (() if const else ("g",)):
        t[name][:, :cu[0]] = float("nan")
        t[name][:, cu[-1]:] = float("nan")
    c = torch.tensor(cu, dtype=torch.int32, device="cuda")
    _poison()
    o = torch.full((1, L, H, V), float("nan"), dtype=t["v"].dtype, device="cuda")
    o, h = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], h0=t["h0"], cu_seqlens=c, o=o)
    _poison()
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"], cu_seqlens=c)
    a, e = cu[0], cu[-1]
    for name, x in dict(o=o, **r).items():
        if name == "dh0" or (const and name == "dg"):
            continue
        assert (x[:, :a] == 0).all() and (x[:, e:] == 0).all(), name
    if a == e:
        assert torch.equal(h, t["h0"]) and torch.equal(r["dh0"], t["dh"])
        return
    x = {m: t[m].double().cpu().numpy() for m in t}
    cut = {m: x[m][:, a:e] for m in ("q", "k", "v", "do")}
    g = np.broadcast_to(x["g"], (1, e - a, H)) if const else x["g"][:, a:e]
    spans = [(0, i - a, j - a) for i, j in zip(cu[:-1], cu[1:])]
    args = (cut["q"], cut["k"], cut["v"], g, K ** -0.5, x["h0"], spans, cut["do"], x["dh"])
    w = ref.attn(*args)
    if const:
        w["dg"] = w["dg"].sum((0, 1))
    for name, got in dict(o=o, h_last=h, **r).items():
        got = got.double().cpu().numpy()
        if name in ("o", "dq", "dk", "dv") or (name == "dg" and not const):
            got = got[:, a:e]
        # the root mean square error of a result: bf16's rounding of it and of its operands
        # are 2^-9 each (uniform: over sqrt 3), fp32 sums 2^-19 of its size at most here
        rel = 2.0 ** -8 if dtype == "bf16" and name in ("o", "dq", "dk", "dv") else 2.0 ** -17
        size = np.sqrt((w[name] ** 2).mean())
        assert np.sqrt(((got - w[name]) ** 2).mean()) <= rel * size, name


def test_padded_row_through_autograd(sw):
    """A padded row's gradients reach the parameters finite and as of the row cut short."""
    L, e, H, K = 300, 211, 2, 32
    t = _rand(7, "f32", x=(L, 48), w=(48, 3 * H * K), g=(1, L, H))
    c = torch.tensor([0, 100, e], dtype=torch.int32, device="cuda")
    g = -t["g"].abs()

    def grad(n):
        w = t["w"].clone().requires_grad_(True)
        _poison()
        q, k, v = (t["x"][:n] @ w).view(1, n, 3 * H, K).split(H, 2)
        o = sw.linear_attn_fn(q, k, v, g[:, :n].contiguous(), cu_seqlens=c)
        return torch.autograd.grad(o[:, :e].square().sum(), w)[0]

    long, short = grad(L), grad(e)
    assert torch.isfinite(long).all()
    assert torch.allclose(long, short, rtol=0, atol=1e-4 * short.abs().max().item())


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_no_heads(sw, dtype, packed):
    """q's and k's are sums over no heads; many sequences."""
    B, L, Hk, K = (1, 50, 2, 24) if packed else (3, 50, 2, 24)
    t = _rand(3, dtype, q=(B, L, Hk, K), k=(B, L, Hk, K))
    v = t["q"].new_empty(B, L, 0, 16)
    c = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda") if packed else None
    for g in (torch.empty(B, L, 0, device="cuda"), torch.empty(0, device="cuda")):
        _poison()
        o, h = sw.linear_attn_fwd(t["q"], t["k"], v, g, cu_seqlens=c)
        assert o.shape == v.shape and h.numel() == 0
        r = sw.linear_attn_bwd(t["q"], t["k"], v, g, v, cu_seqlens=c)
        assert (r["dq"] == 0).all() and (r["dk"] == 0).all() and r["dq"].shape == t["q"].shape
        assert r["dv"].shape == v.shape and r["dg"].shape == g.shape


def test_many_short_sequences_of_wide_heads(sw):
    """Each launch is held to the limit by its own workgroups: 2^17 sequences of one step
    with K = V = 256 take 2^19."""
    B, K = 2 ** 17, 256
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(B, 1, 1, K, generator=gen, device="cuda").bfloat16() for _ in range(3))
    o, _ = sw.linear_attn_fwd(q, k, v, torch.zeros(B, 1, 1, device="cuda"), want_h_last=False)
    want = (q.float() * k.float()).sum(-1, keepdim=True) * K ** -0.5 * v.float()
    # q.k and the result are rounded to bf16; the sums of q.k to fp32
    assert ((o.float() - want).abs() <= 2.0 ** -7 * want.abs() + 1e-6 * v.abs()).all()


@pytest.mark.parametrize("const", [False, True])
def test_backward_captured(sw, const):
    """As a graph replayed on new inputs, a packed and padded row with shared heads."""
    L, Hk, H, K, V = 900, 2, 4, 64, 64
    t = _rand(31, "bf16", q=(1, L, Hk, K), k=(1, L, Hk, K), v=(1, L, H, V), do=(1, L, H, V),
              g=(H,) if const else (1, L, H), h0=(3, H, K, V), dh=(3, H, K, V))
    t["g"] = -0.1 * t["g"].abs()
    c = torch.tensor([0, 500, 512, 850], dtype=torch.int32, device="cuda")
    q = t["q"].clone()

    def run():
        return sw.linear_attn_bwd(q, t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"], cu_seqlens=c)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for i in range(3):
        q.copy_(t["q"] * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = run()
        for n in want:
            assert torch.equal(out[n], want[n]), (i, n)


def test_offsets_past_32_bits(sw):
    """2^31 elements and more in v, o, dout and dv, the heads' rows far apart: the last
    head as of a call of its own."""
    L, H, K, V = 2 ** 18, 66, 16, 128
    gen = torch.Generator(device="cuda").manual_seed(17)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    q, k = rand(1, L, 1, K), rand(1, L, 1, K)
    v, do = rand(1, H, L, V).transpose(1, 2), rand(1, L, H, V)
    assert v.numel() > 2 ** 31
    g = -0.1 * torch.rand(1, L, H, generator=gen, device="cuda")
    last = lambda x: x[:, :, H - 1:]  # noqa: E731
    near = lambda a, b, rel: ((a.double() - b.double()).square().mean()  # noqa: E731
                              <= rel ** 2 * b.double().square().mean()).item()
    print("case far offsets, forward", flush=True)
    o, h = sw.linear_attn_fwd(q, k, v, g)
    o1, h1 = sw.linear_attn_fwd(q, k, last(v), last(g))
    # single bf16 roundings that fall the other way, and fp32 sums
    assert near(last(o), o1, 2.0 ** -11) and near(h[:, H - 1:], h1, 2.0 ** -18)
    del o, o1
    print("case far offsets, backward", flush=True)
    r = sw.linear_attn_bwd(q, k, v, g, do)
    r1 = sw.linear_attn_bwd(q, k, last(v), last(g), last(do))
    assert near(last(r["dv"]), r1["dv"], 2.0 ** -11) and near(last(r["dg"]), r1["dg"], 2.0 ** -18)
    assert torch.isfinite(r["dq"]).all() and torch.isfinite(r["dk"]).all()
