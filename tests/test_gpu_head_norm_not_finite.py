"""Infinities and NaN in heads of which only some columns are turned: they reach the
columns that the definition mixes them with, and no others.

    u = w x / rms(x),  y = u with the pairs of its first R columns turned
    g = dy turned back,  dw = sum g x / rms(x)

An infinite x makes rms(x) infinite: its own u is NaN, the head's others are zero.  Zero
and NaN are compared as such; finite weight gradients with those of the same call in which
the head's dy is zero: its terms are then zero as well, and the sums the same bits."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BAD = [float("inf"), -float("inf"), float("nan")]


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _mixed(c, R, adjacent):
    """The columns that the turn mixes column c with, itself among them."""
    if c >= R:
        return [c]
    if adjacent:
        return [c, c ^ 1]
    return [c, (c + R // 2) % R]


def _inputs(K, R, dtype):
    g = torch.Generator(device="cuda").manual_seed(K + R)
    make = lambda n: torch.randn(2, 5, n, K, generator=g, device="cuda").to(TYPES[dtype])  # noqa: E731
    t = {"q": make(3), "k": make(2), "dq": make(3), "dk": make(2)}
    w = [torch.rand(K, generator=g, device="cuda") + 0.5 for _ in "qk"]
    freq = torch.tensor(100.0 ** (-np.arange(0, R, 2) / R), dtype=torch.float32, device="cuda") if R else None
    # away from where a cosine or sine is zero: there a product with an infinity is NaN, too
    pos = torch.tensor([[1, 2, 4, 5, 7], [8, 10, 11, 13, 14]], device="cuda")
    return t, w, dict(positions=pos, inv_freq=freq)


_CASES = [(64, 32), (64, 16), (100, 50), (33, 14), (256, 250), (17, 16), (24, 2), (40, 0), (64, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("K,R", _CASES)
def test_inputs(sw, K, R, adjacent, dtype):
    print("case not finite x", K, R, adjacent, dtype, flush=True)
    t, (wq, wk), how = _inputs(K, R, dtype)
    how["adjacent"] = adjacent
    for side, heads in (("q", 3), ("k", 2)):
        for n, c in enumerate(sorted({0, 1, max(R - 1, 0), min(R, K - 1), min(R + 9, K - 1), K - 1})):
            bad, at = BAD[n % 3], (n % 2, n % 5, n % heads)
            x = {**t, side: t[side].clone()}
            x[side][at][c] = bad
            y = dict(zip("qk", sw.head_norm_fwd(x["q"], x["k"], wq, wk, **how)))[side][at]
            if bad != bad:
                assert torch.isnan(y).all()
            else:
                want = torch.zeros(K, dtype=torch.bool, device="cuda")
                want[_mixed(c, R, adjacent)] = True
                assert torch.equal(torch.isnan(y), want), (side, c, bad, torch.nonzero(torch.isnan(y) != want))
                assert (y[~want] == 0).all()
            # the weights' gradients: of an infinite x only its own column's is not finite
            g = sw.head_norm_bwd(x["dq"], x["dk"], x["q"], x["k"], wq, wk, **how)["dweight_" + side]
            if bad != bad:
                assert torch.isnan(g).all()
                continue
            none = {**t, "d" + side: t["d" + side].clone()}
            none["d" + side][at] = 0
            clean = sw.head_norm_bwd(none["dq"], none["dk"], t["q"], t["k"], wq, wk, **how)["dweight_" + side]
            other = torch.arange(K, device="cuda") != c
            assert torch.isnan(g[c]) and torch.equal(g[other], clean[other]), (side, c, bad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("K,R", _CASES)
def test_gradients(sw, K, R, adjacent, dtype):
    print("case not finite dy", K, R, adjacent, dtype, flush=True)
    t, (wq, wk), how = _inputs(K, R, dtype)
    how["adjacent"] = adjacent
    clean = sw.head_norm_bwd(t["dq"], t["dk"], t["q"], t["k"], wq, wk, **how)
    for side, heads in (("q", 3), ("k", 2)):
        for n, c in enumerate(sorted({0, 1, max(R - 1, 0), min(R, K - 1), min(R + 9, K - 1), K - 1})):
            bad, at = BAD[n % 3], (n % 2, n % 5, n % heads)
            x = {**t, "d" + side: t["d" + side].clone()}
            x["d" + side][at][c] = bad
            g = sw.head_norm_bwd(x["dq"], x["dk"], x["q"], x["k"], wq, wk, **how)
            hit = torch.zeros(K, dtype=torch.bool, device="cuda")
            hit[_mixed(c, R, adjacent)] = True
            dw = g["dweight_" + side]
            assert not torch.isfinite(dw[hit]).any(), (side, c, bad)
            assert torch.equal(dw[~hit], clean["dweight_" + side][~hit]), (side, c, bad, dw[~hit])
            # the head's own dx holds its mean; every other head is as it was
            dx, want = g["d" + side], clean["d" + side]
            assert not torch.isfinite(dx[at]).any()
            keep = torch.ones(dx.shape[:-1], dtype=torch.bool, device="cuda")
            keep[at] = False
            assert torch.equal(dx[keep], want[keep])
            assert torch.equal(g["dk" if side == "q" else "dq"], clean["dk" if side == "q" else "dq"])
