"""How often linear attention's outputs are rounded: in bf16 once, in calls of any
size, and fp32 sums beside it.

One rounding to bf16's 8 bits errs by at most half of the last, evenly spread; over
values whose leading digits are spread as usual that is 2^-8 / sqrt(3) sqrt(3 / (8 ln
2)) = 1.66e-3 of a result by root mean square.  Two in a row make 2.35e-3; the bound,
1.9e-3, lies between.  fp32 results: sums of up to 256 terms of 2^-24 each and as many
chunks, at random 2^-20; 2^-19."""
import numpy as np
import pytest

import linear_ref as ref

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu

ONCE = 1.9e-3


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _rms(err, want):
    return float(np.sqrt((err ** 2).mean() / (want ** 2).mean()))


def _bf16(a):
    return torch.from_numpy(a).bfloat16().double().numpy()


def test_the_bound_tells_one_rounding_from_two():
    r = np.random.Generator(np.random.PCG64(1))
    x, y = r.standard_normal((2, 40000))
    assert _rms(_bf16(x) - x, x) <= ONCE
    # an operand's rounding and the result's
    assert _rms(_bf16(_bf16(x) * y) - x * y, x * y) > ONCE


def _make(B, L, Hk, H, K, V, dtype, seed):
    r = np.random.Generator(np.random.PCG64(seed))
    x = {"q": r.standard_normal((B, L, Hk, K)), "k": r.standard_normal((B, L, Hk, K)),
         "v": r.standard_normal((B, L, H, V)), "do": r.standard_normal((B, L, H, V)),
         "g": -0.1 * r.random((B, L, H)), "h0": r.standard_normal((B, H, K, V)),
         "dh": r.standard_normal((B, H, K, V))}
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    return {n: torch.from_numpy(a).to(dt if n in ("q", "k", "v", "do") else torch.float32)
            for n, a in x.items()}


def _results(sw, t):
    d = {n: a.cuda() for n, a in t.items()}
    o, h = sw.linear_attn_fwd(d["q"], d["k"], d["v"], d["g"], h0=d["h0"])
    r = sw.linear_attn_bwd(d["q"], d["k"], d["v"], d["g"], d["do"], d["dh"], h0=d["h0"])
    return dict(o=o, h_last=h, **r)


# one chunk, several, cut sequences; widths of every instance, and of more than one tile
_SHAPES = [(1, 64, 1, 1, 64, 64), (1, 64, 2, 4, 128, 128), (2, 300, 1, 2, 32, 64), (1, 700, 1, 3, 64, 128),
           (1, 500, 2, 2, 128, 64), (2, 257, 2, 2, 128, 128), (1, 200, 1, 2, 136, 96), (1, 130, 1, 1, 256, 256),
           (1, 1900, 1, 1, 64, 64), (1, 3, 1, 2, 24, 40), (1, 1, 1, 1, 96, 112)]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", _SHAPES)
def test_every_result(sw, shape, dtype):
    print("case rounding", shape, dtype, flush=True)
    t = _make(*shape, dtype, 50 + sum(shape))
    x = {n: a.double().numpy() for n, a in t.items()}
    w = ref.attn(x["q"], x["k"], x["v"], x["g"], shape[4] ** -0.5, x["h0"], None, x["do"], x["dh"])
    got = _results(sw, t)
    e = {n: _rms(got[n].double().cpu().numpy() - w[n], w[n]) for n in w}
    print("  " + ", ".join(f"{n} {v:.3g}" for n, v in e.items()), flush=True)
    for n, v in e.items():
        assert v <= (ONCE if got[n].dtype is torch.bfloat16 else 2.0 ** -19), n


@gpu
@pytest.mark.parametrize("L", [1, 64, 100, 128, 129, 300])
def test_a_sequence_alone_and_in_a_batch(sw, L):
    """The same sequence has the same accuracy wherever it runs, and results that differ
    by fp32 sums: single roundings that fall the other way."""
    t = _make(1, L, 2, 4, 64, 64, "bf16", 7)
    alone = _results(sw, t)
    many = _results(sw, {n: a.expand(130, *a.shape[1:]).contiguous() for n, a in t.items()})
    for n, a in alone.items():
        a, b = a.double().cpu().numpy(), many[n][129:].double().cpu().numpy()
        # fp32 sums move a result by 2^-19 of its size: over one of bf16's steps of 2^-8
        # that is a chance of 2^-11 to fall the other way, by 2^-8: 2^-13.5 by root mean square
        assert _rms(a - b, a) <= (2.0 ** -12 if alone[n].dtype is torch.bfloat16 else 2.0 ** -18), n
