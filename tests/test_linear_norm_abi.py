"""Host-side checks of linear attention and the block norms: what the C ABI
refuses before any HIP call, through ctypes and the call extension alike."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2606_00601_amd as pkg
    return pkg.lib()


def _fwd(B=1, L=4, Hk=1, H=2, K=8, V=8, n=1, strides=(0,) * 12, dtype=0, flags=0, ws=0, cu=None):
    return (*[None] * 5, cu, None, None, B, L, Hk, H, K, V, n, strides, dtype, flags, 1.0, None, ws)


def _both(lib, name, args, at):
    import paper_2606_00601_amd as pkg
    got = getattr(pkg.fast(), name)(*args)
    msg = pkg.last_error()
    c = list(args)
    c[at] = (ctypes.c_int64 * len(c[at]))(*c[at])
    assert getattr(lib, name)(*c) == got
    assert pkg.last_error() == msg
    return got, msg


@pytest.mark.parametrize("kw, status, says", [
    (dict(L=-1), 1, "negative size"), (dict(K=0), 2, "outside"), (dict(V=257), 2, "outside"),
    (dict(H=3, Hk=2), 1, "multiple"), (dict(Hk=0), 1, "multiple"), (dict(n=2), 1, "nseq"),
    (dict(dtype=7), 1, "dtype"), (dict(flags=2), 1, "flags"), (dict(ws=-1), 1, "workspace"),
    (dict(strides=(0, -1) + (0,) * 10), 1, "negative stride"), (dict(L=2 ** 31), 2, "steps"),
    (dict(B=2 ** 59, n=2 ** 59), 2, "overflow"), (dict(B=0, n=0), 0, ""), (dict(H=0), 0, ""),
    (dict(cu=0x1000, B=2, n=2), 1, "packed"),
])
def test_linear_forward_sizes(lib, kw, status, says):
    got, msg = _both(lib, "sw_linear_attn_fwd", _fwd(**kw), 15)
    assert got == status
    if status:
        assert says in msg


def test_linear_backward_and_step_sizes(lib):
    bwd = (*[None] * 13, 1, 4, 1, 2, 300, 8, 1, (0,) * 15, 0, 0, 1.0, None, 0)
    assert _both(lib, "sw_linear_attn_bwd", bwd, 20)[0] == 2
    step = lambda **k: (*[None] * 7, *(k.get(n, d) for n, d in  # noqa: E731
                                        (("B", 2), ("Hk", 1), ("H", 2), ("K", 8), ("V", 8), ("pool", 2))),
                        k.get("strides", (0,) * 8), 0, k.get("flags", 0), 1.0)
    for kw, status in ((dict(pool=1), 1), (dict(K=257), 2), (dict(Hk=3), 1), (dict(flags=4), 1),
                       (dict(strides=(-1,) + (0,) * 7), 1), (dict(B=-1), 1), (dict(B=0), 0)):
        assert _both(lib, "sw_linear_attn_step", step(**kw), 13)[0] == status, kw
    assert lib.sw_linear_attn_fwd(*[None] * 8, 1, 4, 1, 2, 8, 8, 1, None, 0, 0, 1.0, None, 0) == 1


def test_strides_are_counted(lib):
    import paper_2606_00601_amd as pkg
    with pytest.raises(TypeError):
        pkg.fast().sw_linear_attn_fwd(*_fwd(strides=(0,) * 11))
    with pytest.raises(TypeError):
        pkg.fast().sw_linear_attn_fwd(*_fwd(strides=[0] * 12))


def test_norm_sizes(lib):
    res = lambda M=1, D=8, xs=8, rs=8, dt=0, rt=0, x=None, r=None, s=None, out=None: (  # noqa: E731
        x, r, None, s, None, out, M, D, xs, rs, dt, rt, 1e-6)
    f = lib.sw_residual_norm_fwd
    assert f(*res(M=-1)) == 1
    assert f(*res(D=16385)) == 2
    assert f(*res(D=0)) == 2
    assert f(*res(xs=-8)) == 1
    assert f(*res(dt=3)) == 1
    assert f(*res(dt=0, rt=1)) == 1  # a stream narrower than x
    assert f(*res(s=0x1000)) == 1 and b"require residual" in lib.sw_last_error()
    assert f(*res(M=0)) == 0
    g = lib.sw_gated_norm_fwd
    assert g(None, None, None, None, 1, 8, 3, 8, 8, 0, 0, 1e-6) == 1
    assert g(None, None, None, None, 1, 8, 8, 8, 8, 0, 2, 1e-6) == 1
    assert g(None, None, None, None, 0, 8, 8, 8, 8, 0, 0, 1e-6) == 0
    b = lib.sw_gated_norm_bwd
    assert b(*[None] * 5, 0x1000, None, 1, 8, 8, 8, 8, 8, 0, 0, 1e-6, None, 0) == 1
    assert b"dz requires z" in lib.sw_last_error()
    assert b(*[None] * 7, 1, 8, 8, 8, 8, 8, 0, 0, 1e-6, None, -1) == 1
    assert lib.sw_norm_bwd_workspace(4, 8, 8, 3) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    import paper_2606_00601_amd as pkg
    q = torch.zeros(1, 4, 1, 8)
    with pytest.raises(ValueError):
        pkg.linear_attn_fwd(q, q, q, torch.zeros(1, 4, 1))
    with pytest.raises(ValueError):
        pkg.gated_norm_fwd(q, q, torch.zeros(8))
