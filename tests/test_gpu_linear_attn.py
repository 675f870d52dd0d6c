"""Linear attention with a log decay for each head against its 64-bit definition:
forward, every gradient, packed sequences, shared heads, strides, resets, values
that are not finite, the one-step form, and refusals.

Tolerances, in units of the terms' magnitude (the same sums of absolute values):
fp32 results: products of up to 256 terms, sums of 64 steps and the decays'
exponentials round some 400 times, 2^-24 each; three times the square root of
that is 60, so 2^-18.  bf16 results: rounding to 8 bits errs by 2^-8 at most; the
output rounds once, and the chunk's weights and the state, each a part of the
terms, once as operands: 2^-7."""
import numpy as np
import pytest

import linear_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = 2.0 ** -18
BF16 = 2.0 ** -7


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def _inputs(B, L, Hk, H, K, V, seed, dtype, n=None, h0=False, dh=False, const_g=False, rate=0.2):
    """Device tensors and the same values in 64 bits."""
    r = np.random.Generator(np.random.PCG64(seed))
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    n = B if n is None else n
    x = {"q": r.standard_normal((B, L, Hk, K)), "k": r.standard_normal((B, L, Hk, K)),
         "v": r.standard_normal((B, L, H, V)), "do": r.standard_normal((B, L, H, V)),
         "g": -rate * r.random((H,) if const_g else (B, L, H)),
         "h0": r.standard_normal((n, H, K, V)) if h0 else None,
         "dh": r.standard_normal((n, H, K, V)) if dh else None}
    t = {}
    for name, a in x.items():
        if a is not None:
            t[name] = torch.from_numpy(a).to(dt if name in ("q", "k", "v", "do") else torch.float32)
            x[name] = t[name].double().numpy()
            t[name] = t[name].cuda()
        else:
            t[name] = None
    if const_g:
        x["g"] = np.broadcast_to(x["g"], (B, L, H))
    return t, x


def _near(got, want, mag, tol, what):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isfinite(got), np.isfinite(want)), what
    fine = np.isfinite(want)
    err, most = np.abs(got - want)[fine], (tol * mag)[fine]
    assert (err <= most).all(), f"{what}: {np.max(err / np.maximum(most, 1e-300)):.3g} of the bound"


def _check(sw, t, x, scale, dtype, cu=None, spans=None, bwd=True):
    tol = BF16 if dtype == "bf16" else F32
    args = (x["q"], x["k"], x["v"], x["g"], scale, x["h0"], spans)
    w = ref.attn(*args, do=x["do"] if bwd else None, dh=x["dh"])
    m = ref.magnitudes(*args, do=x["do"] if bwd else None, dh=x["dh"])
    o, h = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], scale=scale, h0=t["h0"],
                              cu_seqlens=cu)
    _near(o, w["o"], m["o"], tol, "o")
    _near(h, w["h_last"], m["h_last"], F32, "h_last")
    if not bwd:
        return
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], scale=scale,
                           h0=t["h0"], cu_seqlens=cu)
    for name in ("dq", "dk", "dv"):
        _near(r[name], w[name], m[name], tol, name)
    _near(r["dh0"], w["dh0"], m["dh0"], F32, "dh0")
    if t["g"].dim() == 1:
        w["dg"], m["dg"] = w["dg"].sum((0, 1)), m["dg"].sum((0, 1))
    _near(r["dg"], w["dg"], m["dg"], F32, "dg")


# lengths at and around the chunk (32 and 64 steps), the kept states (256) and a
# segment; widths at and around the instances' 32, 64, 128, 256 and the tiles' 64, 128
_SHAPES = [(1, 1, 1, 1, 1, 1), (2, 2, 1, 2, 3, 5), (1, 31, 2, 2, 32, 64), (1, 33, 1, 3, 33, 65),
           (2, 63, 1, 1, 64, 64), (1, 64, 2, 4, 64, 128), (1, 65, 1, 1, 68, 68),
           (1, 130, 1, 2, 128, 128), (1, 256, 1, 1, 16, 16), (1, 257, 2, 2, 129, 130),
           (1, 300, 1, 1, 256, 256), (1, 700, 1, 5, 24, 40), (2, 1029, 1, 1, 48, 17)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", _SHAPES)
def test_forward_and_gradients(sw, shape, dtype):
    print("case linear", dtype, shape, flush=True)
    odd = sum(shape) % 2 == 1
    t, x = _inputs(*shape, 11 + sum(shape), dtype, h0=odd, dh=not odd)
    _check(sw, t, x, 0.3, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decay_for_each_head_and_both_states(sw, dtype):
    t, x = _inputs(2, 321, 2, 6, 40, 24, 5, dtype, h0=True, dh=True, const_g=True)
    _check(sw, t, x, 1.0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[1], [5, 0, 64, 1, 0, 300, 63], [700, 3], [0, 0], [256, 512, 1]])
def test_packed_sequences(sw, lens, dtype):
    """Of no step and of many; an empty one hands its initial state on."""
    e = np.concatenate([[0], np.cumsum(lens)])
    spans = [(0, int(e[i]), int(e[i + 1])) for i in range(len(lens))]
    t, x = _inputs(1, int(e[-1]), 2, 4, 36, 72, 17, dtype, n=len(lens), h0=True, dh=True)
    cu = torch.tensor(e, dtype=torch.int32, device="cuda")
    _check(sw, t, x, 0.5, dtype, cu, spans)


def test_many_segments_agree_with_few(sw):
    """A long sequence of one head, cut into segments, against the same steps beside
    many others, walked whole: the composition's rounding apart."""
    t, x = _inputs(1, 5000, 1, 1, 64, 64, 23, "f32", h0=True, dh=True)
    one = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"])
    rep = lambda a: a.expand(600, *a.shape[1:])  # noqa: E731
    many = sw.linear_attn_bwd(*(rep(t[n]) for n in ("q", "k", "v", "g", "do")),
                              rep(t["dh"]).contiguous(), h0=rep(t["h0"]).contiguous())
    m = ref.magnitudes(x["q"], x["k"], x["v"], x["g"], 0.125, x["h0"], None, x["do"], x["dh"])
    for name in one:
        a, b = one[name], many[name][599:600]
        _near(a, b.double().cpu().numpy(), m[name], 2 * F32, name)


def test_strides(sw):
    """Parts of a fused projection, a broadcast key, heads before steps, offsets off
    16 bytes: the same bits as of dense copies."""
    B, L, H, K, V = 2, 200, 4, 32, 64
    r = torch.Generator(device="cuda").manual_seed(3)
    for dt in (torch.bfloat16, torch.float32):
        rand = lambda *s: torch.randn(*s, generator=r, device="cuda").to(dt)  # noqa: E731
        fused = rand(B, L, H * (2 * K + V) + 3)[..., 3:]
        q, k, v = (p.unflatten(-1, (H, -1)) for p in fused.split([H * K, H * K, H * V], -1))
        shared = rand(B, L, 1, K).expand(B, L, H, K)
        swapped = rand(B, H, L, V).transpose(1, 2)
        g = -torch.rand(B, H, L, generator=r, device="cuda").transpose(1, 2)
        do = rand(L, B, H, V).transpose(0, 1)
        for args in ((q, k, v, g), (q, shared, swapped, g)):
            dense = [a.contiguous() for a in args]
            assert all(torch.equal(a, b) for a, b in zip(sw.linear_attn_fwd(*args),
                                                         sw.linear_attn_fwd(*dense)))
            a, b = sw.linear_attn_bwd(*args, do), sw.linear_attn_bwd(*dense, do.contiguous())
            assert all(torch.equal(a[n], b[n]) for n in a)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_resets_and_lowest_decays(sw, dtype):
    """-inf and the type's lowest value forget everything before, exactly."""
    t, x = _inputs(1, 150, 1, 2, 32, 64, 29, dtype, h0=True, dh=True)
    for at, low in ((0, -np.inf), (40, -np.inf), (64, -3.4e38), (65, -np.inf), (149, -3.4e38)):
        t["g"][0, at, 0] = low
        x["g"][0, at, 0] = -np.inf
    _check(sw, t, x, 0.25, dtype)
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"])
    assert (r["dg"][0, [0, 40, 64, 65, 149], 0] == 0).all()
    assert (r["dh0"][0, 0] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.7, 1e-3])
def test_scales(sw, scale, dtype):
    t, x = _inputs(1, 140, 1, 2, 32, 64, 33, dtype, h0=True, dh=True)
    _check(sw, t, x, scale, dtype)
    t["v"][0, 70, 0, 5] = float("inf")
    x["v"][0, 70, 0, 5] = 1.0  # magnitudes alone
    o = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], scale=scale, h0=t["h0"])[0]
    w = ref.attn(x["q"], x["k"], x["v"], x["g"], scale, x["h0"])["o"]
    m = ref.magnitudes(x["q"], x["k"], x["v"], x["g"], scale, x["h0"])["o"]
    for part in (np.s_[:, :70], np.s_[:, 70:, 0, :5], np.s_[:, 70:, 1]):
        _near(o[part], w[part], m[part], BF16 if dtype == "bf16" else F32, "o")


def test_strong_and_growing_decays(sw):
    """Decays that underflow within a chunk, and states that grow."""
    t, x = _inputs(1, 200, 1, 2, 32, 32, 31, "f32", rate=40.0)
    _check(sw, t, x, 0.25, "f32")
    t, x = _inputs(1, 200, 1, 2, 32, 32, 31, "f32", rate=-0.2)
    _check(sw, t, x, 0.25, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "v"])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_what_is_not_finite_reaches_no_earlier_step(sw, what, value, dtype):
    """As in the recurrence: from its step on, and in its own columns."""
    t, x = _inputs(1, 200, 1, 2, 40, 72, 37, dtype)
    t[what][0, 100, 0, 7] = value
    x[what][0, 100, 0, 7] = value
    w = ref.attn(x["q"], x["k"], x["v"], x["g"], 0.5)
    clean = {n: np.nan_to_num(a, nan=1.0, posinf=1.0, neginf=1.0) if n in "qkv" else a
             for n, a in x.items()}
    m = ref.magnitudes(clean["q"], clean["k"], clean["v"], clean["g"], 0.5)
    o, h = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], scale=0.5)
    _near(o, w["o"], m["o"], BF16 if dtype == "bf16" else F32, "o")
    _near(h, w["h_last"], m["h_last"], F32, "h_last")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_what_is_not_finite(sw, dtype):
    """A NaN in do reaches dq of its step and dk, dv, dg of it and earlier ones."""
    t, x = _inputs(1, 200, 1, 1, 32, 64, 41, dtype)
    t["do"][0, 100, 0, 3] = np.nan
    x["do"][0, 100, 0, 3] = np.nan
    w = ref.attn(x["q"], x["k"], x["v"], x["g"], 0.5, do=x["do"])
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], scale=0.5)
    for name in ("dq", "dk", "dv"):
        assert np.array_equal(np.isfinite(r[name].float().cpu().numpy()), np.isfinite(w[name])), name
    assert torch.isfinite(r["dg"][0, 101:]).all() and torch.isnan(r["dg"][0, 1:101]).all()


def test_gradients_against_differences(sw):
    """sum(do o) + sum(dh h_last) is linear in each of q, k, v and h0, so a difference
    over any distance is the gradient along it; in g a central one over 2^-7."""
    t, x = _inputs(1, 130, 1, 2, 32, 32, 43, "f32", h0=True, dh=True)

    def loss(**new):
        a = {**t, **new}
        o, h = sw.linear_attn_fwd(a["q"], a["k"], a["v"], a["g"], h0=a["h0"])
        return ((o.double() * t["do"].double()).sum() + (h.double() * t["dh"].double()).sum()).item()

    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"])
    gen = torch.Generator(device="cuda").manual_seed(5)
    for name in ("q", "k", "v", "h0", "g"):
        e = 2.0 ** -7 if name == "g" else 1.0
        d = torch.randn(t[name].shape, generator=gen, device="cuda")
        got = (loss(**{name: t[name] + e * d}) - loss(**{name: t[name] - e * d})) / (2 * e)
        want = (r["d" + name].double() * d.double()).sum().item()
        size = (r["d" + name].double() * d.double()).abs().sum().item()
        # the loss's terms add up to some thousand times its gradient's; e^2 / 6 in g
        assert abs(got - want) <= 2e-4 * size, (name, got, want, size)


def test_autograd_matches_backward_and_both_outputs_train(sw):
    t, x = _inputs(2, 100, 2, 4, 32, 32, 47, "bf16", h0=True, dh=True, const_g=True)
    leaf = {n: t[n].clone().requires_grad_(True) for n in ("q", "k", "v", "g", "h0")}
    o, h = sw.linear_attn_fn(leaf["q"], leaf["k"], leaf["v"], leaf["g"], h0=leaf["h0"],
                             return_last_state=True)
    got = torch.autograd.grad([o, h], list(leaf.values()), [t["do"], t["dh"]])
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"])
    for a, n in zip(got, leaf):
        assert torch.equal(a, r["d" + n]), n
    last = sw.linear_attn_fn(leaf["q"], leaf["k"], leaf["v"], leaf["g"], return_last_state=True)[1]
    (gq,) = torch.autograd.grad(last.sum(), [leaf["q"]])
    assert (gq == 0).all()  # h_last does not read q


def test_deterministic(sw):
    t, _ = _inputs(2, 3000, 2, 8, 64, 64, 53, "bf16", h0=True, dh=True, const_g=True)
    run = lambda: sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"],  # noqa: E731
                                     h0=t["h0"])
    a, b = run(), run()
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_another_stream_and_capture(sw):
    """On a stream of the caller's, and as a graph replayed on new inputs."""
    t, x = _inputs(1, 2000, 1, 2, 64, 64, 59, "bf16", h0=True)
    eager = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], h0=t["h0"])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], h0=t["h0"])
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    q = t["q"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sw.linear_attn_fwd(q, t["k"], t["v"], t["g"], h0=t["h0"])
    for i in range(3):
        q.copy_(t["q"] * (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        want = sw.linear_attn_fwd(q, t["k"], t["v"], t["g"], h0=t["h0"])
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i


# ---- one step

_STEPS = [(1, 1, 1, 1, 1), (3, 1, 2, 5, 7), (2, 2, 2, 64, 64), (5, 1, 3, 128, 128), (2, 1, 1, 256, 256),
          (70, 2, 4, 33, 130), (1, 1, 4, 200, 3)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", _STEPS)
def test_step(sw, shape, dtype):
    """Against the definition; a token at a time is the prompt form."""
    B, Hk, H, K, V = shape
    t, x = _inputs(B, 3, Hk, H, K, V, 61 + sum(shape), dtype, h0=True, const_g=B == 3)
    w = ref.attn(x["q"], x["k"], x["v"], x["g"], 0.5, x["h0"])
    m = ref.magnitudes(x["q"], x["k"], x["v"], x["g"], 0.5, x["h0"])
    state = t["h0"].clone()
    for i in range(3):
        g = t["g"] if t["g"].dim() == 1 else t["g"][:, i]
        o = sw.linear_attn_step(t["q"][:, i], t["k"][:, i], t["v"][:, i], g, state, scale=0.5)
        # no bf16 operands here: the output's rounding alone
        _near(o, w["o"][:, i], m["o"][:, i], 2.0 ** -8 * 1.01 if dtype == "bf16" else F32, "o")
    _near(state, w["h_last"], m["h_last"], F32, "state")


def test_step_slots(sw):
    """Slots in any order; those outside the pool are no sequences."""
    t, x = _inputs(6, 1, 2, 4, 32, 64, 67, "f32")
    pool = torch.randn(9, 4, 32, 64, device="cuda")
    before = pool.clone()
    slots = torch.tensor([4, -1, 0, 9, 8, -2 ** 31], dtype=torch.int32, device="cuda")
    one = lambda a: a[:, 0]  # noqa: E731
    o = sw.linear_attn_step(one(t["q"]), one(t["k"]), one(t["v"]), one(t["g"]), pool, slots=slots)
    for i, s in enumerate(slots.tolist()):
        if not 0 <= s < 9:
            assert (o[i] == 0).all()
            continue
        st = before[s:s + 1].clone()
        want = sw.linear_attn_step(*(one(t[n])[i:i + 1] for n in ("q", "k", "v", "g")), st)
        assert torch.equal(o[i:i + 1], want) and torch.equal(pool[s:s + 1], st)
    for s in (1, 2, 3, 5, 6, 7):
        assert torch.equal(pool[s], before[s])


def test_step_far_slots(sw):
    """A pool whose offsets pass 2^31 elements."""
    H, K, V = 8, 128, 128
    n = 2 ** 31 // (H * K * V) + 3
    pool = torch.zeros(n, H, K, V, device="cuda")
    t, _ = _inputs(2, 1, 8, H, K, V, 71, "bf16")
    slots = torch.tensor([n - 1, 0], dtype=torch.int32, device="cuda")
    args = [t[a][:, 0] for a in ("q", "k", "v", "g")]
    o = sw.linear_attn_step(*args, pool, slots=slots)
    small = torch.zeros(2, H, K, V, device="cuda")
    assert torch.equal(o, sw.linear_attn_step(*args, small))
    assert torch.equal(pool[n - 1], small[0]) and torch.equal(pool[0], small[1])
    assert (pool[1:n - 1].abs().amax() == 0).item()


def test_step_captured(sw):
    t, _ = _inputs(4, 1, 2, 4, 64, 64, 73, "bf16", h0=True)
    args = [t[a][:, 0].contiguous() for a in ("q", "k", "v", "g")]
    want, state = t["h0"].clone(), t["h0"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = sw.linear_attn_step(*args, state)
    for i in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, sw.linear_attn_step(*args, want)) and torch.equal(state, want), i


# ---- refusals


def test_refusals(sw):
    t, _ = _inputs(2, 8, 2, 4, 16, 16, 79, "f32", h0=True)
    q, k, v, g, h0 = (t[n] for n in ("q", "k", "v", "g", "h0"))
    f = sw.linear_attn_fwd
    with pytest.raises(TypeError):
        f(q, k.bfloat16(), v, g)
    with pytest.raises(TypeError):
        f(q.half(), k.half(), v.half(), g)
    with pytest.raises(TypeError):
        f(q, k, v, g.double())
    with pytest.raises(ValueError):
        f(q, k[:, :-1], v, g)
    with pytest.raises(ValueError):
        f(q, k, v, g[:, :, :2])
    with pytest.raises(ValueError):
        f(q.cpu(), k.cpu(), v.cpu(), g.cpu())
    with pytest.raises(ValueError):
        f(q.transpose(2, 3).contiguous().transpose(2, 3), k, v, g)
    with pytest.raises(ValueError):
        f(q, k, v, g, h0=h0[:1])
    with pytest.raises(ValueError):
        f(q, k, v, g, cu_seqlens=torch.tensor([0, 8], dtype=torch.int32, device="cuda"))  # B = 2
    with pytest.raises(TypeError):
        f(q[:1], k[:1], v[:1], g[:1], cu_seqlens=torch.tensor([0, 8], device="cuda"))
    with pytest.raises(sw.ScanWeaverError) as e:
        f(q[:, :, :, :], k, v[:, :, :3], g[:, :, :3])  # 3 heads of 2 key heads
    assert e.value.status == 1
    wide = torch.zeros(1, 4, 1, 257, device="cuda")
    with pytest.raises(sw.ScanWeaverError) as e:
        f(wide, wide, wide[..., :16], torch.zeros(1, 4, 1, device="cuda"))
    assert e.value.status == 2
    with pytest.raises(sw.ScanWeaverError) as e:  # the output over an input
        f(q, k, v, g, o=v)
    assert e.value.status == 1 and "overlaps" in str(e.value)
    with pytest.raises(ValueError):
        sw.linear_attn_bwd(q, k, v, g, v[:, :4])
    with pytest.raises(ValueError):
        sw.linear_attn_step(q[:, 0], k[:, 0], v[:, 0], g[:, 0], h0[:1])
    with pytest.raises(TypeError):
        sw.linear_attn_step(q[:, 0], k[:, 0], v[:, 0], g[:, 0], h0,
                            slots=torch.zeros(2, dtype=torch.int64, device="cuda"))


def test_pool_workspace_and_too_small_a_workspace(sw):
    """Without a workspace the call takes the pool's; a smaller one is refused."""
    t, _ = _inputs(1, 4000, 1, 1, 32, 64, 83, "f32")
    from paper_2606_00601_amd._bind import _on
    o = torch.empty_like(t["v"])
    sizes, st = (1, 4000, 1, 1, 32, 64, 1), (0, 32, 0) * 2 + (0, 64, 0) + (0, 1, 0)
    f = sw.fast()
    need = f.sw_linear_attn_fwd_workspace(*sizes, 0, 0, 0)
    assert need > 0
    ptr = [t[n].data_ptr() for n in ("q", "k", "v", "g")]
    small = torch.empty(need - 1, dtype=torch.uint8, device="cuda")
    with _on(o.device):
        assert f.sw_linear_attn_fwd(*ptr, None, None, o.data_ptr(), None, *sizes, st, 0, 0, 0.5, None,
                                    0) == 0
        assert f.sw_linear_attn_fwd(*ptr, None, None, o.data_ptr(), None, *sizes, st, 0, 0, 0.5,
                                    small.data_ptr(), need - 1) == 1
    assert torch.equal(o, sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], scale=0.5)[0])


def test_no_steps_and_no_heads(sw):
    t, _ = _inputs(2, 0, 1, 2, 16, 16, 89, "bf16", h0=True, dh=True, const_g=True)
    o, h = sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"], h0=t["h0"])
    assert o.shape == (2, 0, 2, 16) and torch.equal(h, t["h0"])
    r = sw.linear_attn_bwd(t["q"], t["k"], t["v"], t["g"], t["do"], t["dh"], h0=t["h0"])
    assert torch.equal(r["dh0"], t["dh"]) and (r["dg"] == 0).all()
    t, _ = _inputs(0, 5, 1, 2, 16, 16, 89, "bf16")
    assert sw.linear_attn_fwd(t["q"], t["k"], t["v"], t["g"])[0].shape == (0, 5, 2, 16)
