"""The decays' gradient, dg_t = e^{g_t} <dS_t, S_{t-1}>, over the range of the decays.

Each dg_t is a sum of pairs of steps with t between them, fp32 operands and sums of
up to some hundred terms in each product, and the decay between the steps: 2^x of an
x of up to 126 that is known to 2^-24 of itself, 126 2^-24 ln 2 = 5e-6 at the far
end.  So: by step 1e-5 of it in the middle of the steps, and everywhere 2^-18 of its
own terms' sizes, e^{g_t} <|dS_t|, |S_{t-1}|> with both states of absolute values; by
root mean square 2^-19 where the decays are weak; a head's sum 2^-19 of its steps'
sizes."""
import numpy as np
import pytest

import linear_ref as ref

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _values(B, L, Hk, H, K, V, seed, dtype, g, h0=True, dh=True):
    """The inputs in 64 bits, as their type holds them."""
    r = np.random.Generator(np.random.PCG64(seed))
    x = {"q": r.standard_normal((B, L, Hk, K)), "k": r.standard_normal((B, L, Hk, K)),
         "v": r.standard_normal((B, L, H, V)), "do": r.standard_normal((B, L, H, V)),
         "h0": r.standard_normal((B, H, K, V)) if h0 else None,
         "dh": r.standard_normal((B, H, K, V)) if dh else None, "g": g(r)}
    for n, a in x.items():
        if a is not None:
            t = torch.from_numpy(np.ascontiguousarray(a)).float()
            x[n] = (t.bfloat16() if dtype == "bf16" and n in ("q", "k", "v", "do") else t).double().numpy()
    return x


def _want(x, spans=None, scale=0.125):
    """(dg by step, its terms' sizes)."""
    B, L = x["q"].shape[:2]
    g = np.broadcast_to(x["g"], (B, L, x["v"].shape[2]))
    ab = lambda a: None if a is None else np.abs(a)  # noqa: E731
    w = ref.attn(x["q"], x["k"], x["v"], g, scale, x["h0"], spans, x["do"], x["dh"])["dg"]
    m = ref.attn(*(ab(x[n]) for n in "qkv"), g, abs(scale), ab(x["h0"]), spans, ab(x["do"]), ab(x["dh"]))["dg"]
    return w, m


def _got(sw, x, dtype, cu=None, scale=0.125):
    t = {n: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).float().cuda()
         for n, a in x.items()}
    if dtype == "bf16":
        for n in ("q", "k", "v", "do"):
            t[n] = t[n].bfloat16()
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], scale=scale, h0=t["h0"],
                           cu_seqlens=cu)
    return r["dg"].double().cpu().numpy()


def _steps_ok(got, want, terms):
    """Whether a gradient by step is within the bounds of the header above."""
    there = terms > 1e-36  # fp32 holds it
    err = np.abs(got - want)
    if not (err <= 2.0 ** -18 * terms + 1e-37).all():
        return False
    return bool(np.median(err[there] / np.maximum(np.abs(want[there]), 1e-300)) <= 1e-5)


def _heads_ok(got, want):
    return bool((np.abs(got - want.sum((0, 1))) <= 2.0 ** -19 * np.abs(want).sum((0, 1))).all())


def _uniform(B, L, H, rate):
    return lambda r: -rate * (0.5 + 0.5 * r.random((B, L, H)))


def _resets(B, L, H, rate):
    """Weak decays, and now and then one step that forgets almost everything."""
    def g(r):
        a = -0.05 * r.random((B, L, H))
        a[r.random((B, L, H)) < 0.02] = -rate
        a[0, L // 2, 0] = -rate
        return a
    return g


_SHAPES = [(1, 256, 1, 1, 64, 64), (2, 301, 1, 2, 128, 128), (1, 200, 2, 2, 136, 40), (1, 130, 1, 3, 24, 100)]


def difference_form(x, w, scale=0.125):
    """dg as the running difference of q . dq and k . dk, both rounded to fp32 once, from
    the exact value at the end: the shorter way, which strong decays take the digits of."""
    r = ref.attn(x["q"], x["k"], x["v"], x["g"], scale, x["h0"], None, x["do"], x["dh"])
    H, Hk = x["v"].shape[2], x["q"].shape[2]
    assert H == Hk
    f = lambda a: a.astype(np.float32).astype(np.float64)  # noqa: E731
    d = f((f(r["dq"]) * x["q"]).sum(-1)) - f((f(r["dk"]) * x["k"]).sum(-1))
    last = (x["dh"] * r["h_last"]).sum((2, 3))
    return last[:, None] + np.cumsum(d[:, ::-1], 1)[:, ::-1]


def test_the_checks_can_fail():
    """Zero, a gradient without h0 or without dh_last, and the difference of sums at
    strong decays are all outside the bounds; the exact one in fp32 is inside."""
    B, L, H = 1, 200, 1
    for rate in (1.0, 12.0):
        x = _values(B, L, 1, H, 64, 64, 3, "f32", _uniform(B, L, H, rate))
        w, m = _want(x)
        assert _steps_ok(w.astype(np.float32).astype(np.float64), w, m)
        assert not _steps_ok(np.zeros_like(w), w, m)
        assert _heads_ok(w.sum((0, 1)), w) and not _heads_ok(np.zeros(H), w)
        if rate == 1.0:
            for gone in ("h0", "dh"):
                other = _want({**x, gone: None})[0]
                assert not _steps_ok(other, w, m) and not _heads_ok(other.sum((0, 1)), w), gone
        else:
            assert not _steps_ok(difference_form(x, w), w, m)
            assert not _heads_ok(difference_form(x, w).sum((0, 1)), w)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("how", [_uniform, _resets])
@pytest.mark.parametrize("rate", [0.1, 1.0, 4.0, 8.0, 12.0, 16.0, 20.0, 60.0])
@pytest.mark.parametrize("shape", _SHAPES)
def test_by_step(sw, shape, rate, how, dtype):
    print("case dg by step", shape, rate, how.__name__, dtype, flush=True)
    B, L, Hk, H, K, V = shape
    x = _values(*shape, 100 + L, dtype, how(B, L, H, rate))
    w, m = _want(x)
    got = _got(sw, x, dtype)
    there = m > 1e-36
    err = np.abs(got - w)
    print("  worst of terms 2^-18: %.3g, median relative %.3g" % (
        (err / (2.0 ** -18 * m + 1e-37)).max(), np.median(err[there] / np.abs(w[there]))), flush=True)
    assert _steps_ok(got, w, m)
    if how is _uniform and rate <= 1.0:
        assert np.sqrt((err ** 2).mean()) <= 2.0 ** -19 * np.sqrt((w ** 2).mean())


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rate", [0.1, 1.0, 8.0, 12.0, 16.0])
@pytest.mark.parametrize("shape", [(1, 1024, 1, 2, 64, 64), (2, 300, 2, 4, 136, 24), (2, 321, 2, 6, 40, 24)])
def test_by_head(sw, shape, rate, dtype):
    print("case dg by head", shape, rate, dtype, flush=True)
    B, L, Hk, H, K, V = shape
    x = _values(*shape, 7 + L, dtype, lambda r: -rate * (0.5 + 0.5 * r.random(H)))
    w, _ = _want(x)
    assert _heads_ok(_got(sw, x, dtype), w)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("h0, dh", [(False, False), (True, False), (False, True)])
def test_packed_and_cut(sw, h0, dh, dtype):
    """Packed sequences of all lengths, long enough for few heads to be cut; each
    boundary state comes from another place."""
    lens = [1, 0, 64, 65, 2300, 33, 128, 700, 31]
    e = np.concatenate([[0], np.cumsum(lens)])
    L = int(e[-1])
    spans = [(0, int(i), int(j)) for i, j in zip(e[:-1], e[1:])]
    r = np.random.Generator(np.random.PCG64(5))
    x = _values(1, L, 1, 1, 32, 48, 11, dtype, _resets(1, L, 1, 9.0), False, False)
    n = len(lens)
    if h0:
        x["h0"] = r.standard_normal((n, 1, 32, 48)).astype(np.float32).astype(np.float64)
    if dh:
        x["dh"] = r.standard_normal((n, 1, 32, 48)).astype(np.float32).astype(np.float64)
    w, m = _want(x, spans)
    got = _got(sw, x, dtype, torch.tensor(e, dtype=torch.int32, device="cuda"))
    err = np.abs(got - w)
    print("  worst of terms 2^-18: %.3g" % (err / (2.0 ** -18 * m + 1e-37)).max(), flush=True)
    assert _steps_ok(got, w, m)


@gpu
@pytest.mark.parametrize("scale", [-0.7, 1e-3])
def test_scales_with_both_signs(sw, scale):
    B, L, Hk, H, K, V = 1, 150, 1, 2, 64, 32
    for dtype in ("bf16", "f32"):
        x = _values(B, L, Hk, H, K, V, 23, dtype, _uniform(B, L, H, 3.0))
        w, m = _want(x, scale=scale)
        assert _steps_ok(_got(sw, x, dtype, scale=scale), w, m)
