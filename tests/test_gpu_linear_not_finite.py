"""Where an infinity or a NaN reaches in linear attention's gradients and in sequences
cut into segments: as in the definition, every value finite there is finite, and
right."""
import numpy as np
import pytest

import linear_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _case(B, L, Hk, H, K, V, seed, dtype):
    r = np.random.Generator(np.random.PCG64(seed))
    x = {"q": r.standard_normal((B, L, Hk, K)), "k": r.standard_normal((B, L, Hk, K)),
         "v": r.standard_normal((B, L, H, V)), "do": r.standard_normal((B, L, H, V)),
         "g": -0.2 * r.random((B, L, H)), "h0": r.standard_normal((B, H, K, V)),
         "dh": r.standard_normal((B, H, K, V))}
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    t = {n: torch.from_numpy(a).to(dt if n in ("q", "k", "v", "do") else torch.float32)
         for n, a in x.items()}
    return t


def _all(sw, t):
    d = {n: a.cuda() for n, a in t.items()}
    o, h = sw.linear_attn_fwd(d["q"], d["k"], d["v"], d["g"], scale=0.5, h0=d["h0"])
    r = sw.linear_attn_bwd(d["q"], d["k"], d["v"], d["g"], d["do"], d["dh"], scale=0.5, h0=d["h0"])
    return {n: a.double().cpu().numpy() for n, a in dict(o=o, h_last=h, **r).items()}


def _want(t):
    x = {n: a.double().numpy() for n, a in t.items()}
    with np.errstate(invalid="ignore", over="ignore"):
        return ref.attn(x["q"], x["k"], x["v"], x["g"], 0.5, x["h0"], None, x["do"], x["dh"])


def _same(got, want, dtype):
    """Finite where the definition is, and there within a root mean square of one
    rounding (bf16: 2^-8 with the operands'; 2^-18 for fp32)."""
    for n, w in want.items():
        fine = np.isfinite(w)
        assert np.array_equal(np.isfinite(got[n]), fine), n
        if fine.any():
            rel = 2.0 ** -8 if dtype == "bf16" and n in ("o", "dq", "dk", "dv") else 2.0 ** -18
            rms = lambda a: np.sqrt((a[fine] ** 2).mean())  # noqa: E731
            with np.errstate(invalid="ignore"):
                assert rms(got[n] - w) <= rel * rms(w), n


_PLACES = {"q": (0, 100, 0, 7), "k": (0, 70, 0, 3), "v": (0, 100, 1, 5), "do": (0, 127, 0, 0),
           "g": (0, 65, 0), "h0": (0, 1, 3, 4), "dh": (0, 0, 2, 2)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", list(_PLACES))
@pytest.mark.parametrize("value", [np.inf, np.nan])
def test_gradients(sw, what, value, dtype):
    """Each input in turn; with q and k the chunk goes step by step in the walks whose
    values they are (dk's, dq's), with do in dv's."""
    print("case not finite", what, value, dtype, flush=True)
    t = _case(1, 200, 1, 2, 40, 72, 37, dtype)
    t[what][_PLACES[what]] = value
    _same(_all(sw, t), _want(t), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "v", "do", "g"])
def test_inner_segment(sw, what, dtype):
    """One head and some thousand steps: cut into segments, with the value inside one,
    so that its carries go step by step too."""
    L = 3000
    print("case not finite, cut", what, dtype, flush=True)
    t = _case(1, L, 1, 1, 32, 32, 41, dtype)
    t[what][(0, 1490, 0) + ((5,) if what != "g" else ())] = np.nan
    f = sw.fast()
    args = (1, L, 1, 1, 32, 32, 1, 1 if dtype == "bf16" else 0, 0, 0)
    assert f.sw_linear_attn_fwd_workspace(*args) > 0  # carries: the sequence is cut
    _same(_all(sw, t), _want(t), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k"])
def test_decays_gradient_beside_them(sw, what, dtype):
    """In the chunk of the value dg is finite and right on the steps that it does not
    reach: k's those up to it, q's those after it."""
    t = _case(1, 150, 1, 1, 64, 64, 43, dtype)
    at = 90
    t[what][0, at, 0, 9] = np.inf
    got, want = _all(sw, t)["dg"][0, :, 0], _want(t)["dg"][0, :, 0]
    fine = np.s_[:at + 1] if what == "k" else np.s_[at + 1:]
    assert np.isfinite(want[fine]).all()
    assert (np.abs(got[fine] - want[fine]) <= 2.0 ** -17 * np.sqrt((want[fine] ** 2).mean())).all()
