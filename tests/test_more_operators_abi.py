"""Host-side checks of the gated recurrence, the head norm and the embedding: what the C
ABI refuses before any HIP call, through ctypes and the call extension alike."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2606_00601_amd as pkg
    return pkg.lib()


def _both(lib, name, args):
    import paper_2606_00601_amd as pkg
    got = getattr(pkg.fast(), name)(*args)
    msg = pkg.last_error()
    c = [(ctypes.c_int64 * len(a))(*a) if isinstance(a, tuple) else a for a in args]
    assert getattr(lib, name)(*c) == got
    assert pkg.last_error() == msg
    return got, msg


def _scan(B=1, L=4, D=8, n=1, strides=(0,) * 6, dtype=0, c=8.0, ws=0, cu=None):
    return (*[None] * 5, cu, None, None, None, B, L, D, n, strides, dtype, c, None, ws)


@pytest.mark.parametrize("kw, status, says", [
    (dict(L=-1), 1, "negative size"), (dict(D=-1), 1, "negative size"), (dict(n=2), 1, "nseq"),
    (dict(dtype=7), 1, "dtype"), (dict(c=0.0), 1, "c="), (dict(c=float("nan")), 1, "c="),
    (dict(c=float("inf")), 1, "c="), (dict(ws=-1), 1, "workspace"),
    (dict(strides=(0, -1) + (0,) * 4), 1, "negative stride"), (dict(L=2 ** 31), 2, "steps"),
    (dict(D=2 ** 28), 2, "channels"), (dict(B=2 ** 50, n=2 ** 50, L=2 ** 20), 2, "overflow"),
    (dict(B=2 ** 61, n=2 ** 61), 2, "overflow"), (dict(B=0, n=0), 0, ""), (dict(D=0), 0, ""),
    (dict(L=0), 0, ""), (dict(cu=0x1000, B=2, n=2), 1, "packed")])
def test_scan_sizes(lib, kw, status, says):
    got, msg = _both(lib, "sw_gated_scan_fwd", _scan(**kw))
    assert got == status
    if status:
        assert says in msg


def test_scan_backward_and_step_sizes(lib):
    bwd = lambda D=8, c=1.0, ws=0: (*[None] * 14, 1, 4, D, 1, (0,) * 8, 0, c, None, ws)  # noqa: E731
    for kw, status in ((dict(D=-1), 1), (dict(c=-1.0), 1), (dict(ws=-1), 1), (dict(D=0), 0)):
        assert _both(lib, "sw_gated_scan_bwd", bwd(**kw))[0] == status, kw
    step = lambda B=2, D=8, pool=2, st=(8, 8, 8), c=8.0: (*[None] * 7, B, D, pool, st, 0, c)  # noqa: E731
    for kw, status in ((dict(pool=1), 1), (dict(B=-1), 1), (dict(c=0.0), 1), (dict(st=(-8, 8, 8)), 1),
                       (dict(D=2 ** 28), 2), (dict(B=0), 0), (dict(D=0), 0)):
        assert _both(lib, "sw_gated_scan_step", step(**kw))[0] == status, kw
    assert lib.sw_gated_scan_fwd(*[None] * 9, 1, 4, 8, 1, None, 0, 1.0, None, 0) == 1
    assert lib.sw_gated_scan_fwd_workspace(-1, 4, 8) == 0
    assert lib.sw_gated_scan_bwd_workspace(1, 0, 8, 0) == 0


def _head(B=1, L=4, H=2, Hk=1, K=8, R=8, strides=(0,) * 8, dtype=0, flags=0):
    return (*[None] * 8, B, L, H, Hk, K, R, strides, dtype, flags, 1e-6)


@pytest.mark.parametrize("kw, status, says", [
    (dict(L=-1), 1, "negative size"), (dict(K=0, R=0), 2, "outside"), (dict(K=257, R=0), 2, "outside"),
    (dict(R=10), 1, "even number"), (dict(R=3), 1, "even number"), (dict(dtype=3), 1, "dtype"),
    (dict(flags=4), 1, "flags"), (dict(strides=(0, 0, -1) + (0,) * 5), 1, "negative stride"),
    (dict(strides=(0,) * 7 + (-1,)), 1, "negative stride"), (dict(B=2 ** 60), 2, "overflow"),
    (dict(B=2 ** 20, L=2 ** 10), 2, "launch limit"), (dict(H=2 ** 31), 2, "launch limit"),
    (dict(B=0), 0, ""), (dict(H=0, Hk=0), 0, "")])
def test_head_norm_sizes(lib, kw, status, says):
    got, msg = _both(lib, "sw_head_norm_fwd", _head(**kw))
    assert got == status
    if status:
        assert says in msg


def test_head_norm_backward_sizes(lib):
    bwd = lambda dw=None, K=8, ws=0: (*[None] * 10, dw, None, 1, 4, 2, 1, K, 8, (0,) * 14, 0, 0, 1e-6,  # noqa: E731
                                      None, ws)
    assert "both given" in _both(lib, "sw_head_norm_bwd", bwd(dw=0x1000))[1]
    assert _both(lib, "sw_head_norm_bwd", bwd(K=300))[0] == 2
    assert _both(lib, "sw_head_norm_bwd", bwd(ws=-1))[0] == 1
    assert lib.sw_head_norm_bwd_workspace(1, 4, 2, 1, 300) == 0


def test_embedding_sizes(lib):
    f = lambda T=2, V=4, D=8, td=0, yd=0, flags=0: (None, None, None, T, V, D, td, yd, flags, 1.0)  # noqa: E731
    for kw, status in ((dict(T=-1), 1), (dict(V=-1), 1), (dict(td=2), 1), (dict(yd=-1), 1), (dict(flags=2), 1),
                       (dict(T=2 ** 31), 2), (dict(V=2 ** 31), 2), (dict(D=2 ** 24), 2),
                       (dict(T=2 ** 60, D=2 ** 20), 2), (dict(T=0), 0), (dict(D=0), 0)):
        assert _both(lib, "sw_embedding_fwd", f(**kw))[0] == status, kw
    b = lambda T=2, V=4, D=8, st=8, flags=0, ws=0: (None, None, None, T, V, D, st, 0, 0, flags, 1.0, None, ws)  # noqa: E731
    for kw, status in ((dict(T=-1), 1), (dict(st=-8), 1), (dict(flags=2), 1), (dict(ws=-1), 1),
                       (dict(T=2 ** 31), 2), (dict(st=2 ** 62), 2), (dict(V=0), 0), (dict(D=0), 0)):
        assert _both(lib, "sw_embedding_bwd", b(**kw))[0] == status, kw
    assert lib.sw_embedding_bwd_workspace(-1, 4, 8) == 0
    assert lib.sw_embedding_bwd_workspace(0, 4, 8) == 0


def test_binding_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    import paper_2606_00601_amd as pkg
    x = torch.zeros(1, 4, 8)
    with pytest.raises(ValueError):
        pkg.gated_scan_fwd(x, x, x, torch.zeros(8))
    with pytest.raises(ValueError):
        pkg.gated_scan_step(x[0], x[0], x[0], torch.zeros(8), x[0])
    with pytest.raises(ValueError):
        pkg.head_norm_fwd(x.view(1, 4, 1, 8), x.view(1, 4, 1, 8))
    with pytest.raises(ValueError):
        pkg.embedding_fwd(torch.zeros(3, dtype=torch.int64), x[0])
    with pytest.raises(ValueError):
        pkg.embedding_bwd(torch.zeros(4, dtype=torch.int64), x[0], 9)
