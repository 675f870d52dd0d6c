"""The gated recurrence where its walks differ by the size of a call: how many chunks a
workgroup looks back over (16 up to 15 groups of 64 channels in all rows, 8 up to 31, 4
from 32 on), words between workgroups in the stream's scratch or in a cleared workspace
(past 16 MiB), rows addressed in 64 bits.  Against the 64-bit definition with gated_ref's
bounds, or, where the same steps are walked in the same chunks, to the bit."""
import numpy as np
import pytest

import gated_ref as ref
from test_gpu_gated_scan import TYPES, _check, _make, _near

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,L,D", [(1, 1500, 1010), (2, 1500, 1100), (1, 1300, 2113), (9, 700, 200)])
def test_many_groups(sw, B, L, D, dtype):
    """16, 36, 34 and 36 groups, 24 chunks backward."""
    print("case gated groups", B, L, D, dtype, flush=True)
    t, v = _make(B + L + D, B, L, D, dtype)
    _check(sw, t, v, D % 2 == 0, None, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,D,edges", [
    (1500, 1100, [0, 0, 300, 301, 1290, 1480]), (2100, 2050, [10, 250, 250, 1800, 2100]),
    (1200, 2111, [0, 1200])])
def test_many_groups_packed(sw, L, D, edges, dtype):
    """18, 33 and 33 groups; sequences over dozens of chunks and within one."""
    print("case gated groups packed", L, D, edges, dtype, flush=True)
    n = len(edges) - 1
    t, v = _make(L + D, 1, L, D, dtype, n)
    for t0, t1 in ((0, edges[0]), (edges[-1], L)):
        for name in ("x", "r", "i", "dh"):
            t[name][:, t0:t1] = float("nan")
    _check(sw, t, v, True, torch.tensor(edges, dtype=torch.int32, device="cuda"),
           [(0, edges[j], edges[j + 1]) for j in range(n)])


@pytest.mark.parametrize("packed", [False, True])
def test_words_past_the_scratch(sw, packed):
    """An eager call whose words take more than 16 MiB clears a workspace for them: 256 chunks
    of 65 groups forward, 1024 of 17 backward.  A channel knows nothing of the others, so
    slices of 1, 8, 20 and 36 groups, whose words lie in the scratch, give the same bits; so
    does a call that brings no workspace."""
    from paper_2606_00601_amd._bind import _on
    L = 65536
    gen = torch.Generator(device="cuda").manual_seed(3)
    make = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    how, n = {}, 1
    if packed:
        cu = torch.tensor([100, 7000, 7000, 7001, 60000, 65500], dtype=torch.int32, device="cuda")
        how, n = dict(cu_seqlens=cu), 5
    for D, cuts in ((4160, (0, 64, 576, 1856, 4160)), (1088, (0, 64, 576, 1088))):
        print("case gated words", D, packed, flush=True)
        x, r, i, dh = (make(1, L, D).bfloat16() for _ in range(4))
        lam, h0, tail = make(D) * 2 - 4, make(n, D), make(n, D)
        h, last = sw.gated_scan_fwd(x, r, i, lam, h0=h0, **how)
        if D == 4160:
            ws = sw.fast().sw_gated_scan_fwd_workspace(1, L, D)
            assert ws > 2 ** 24
        else:
            g = sw.gated_scan_bwd(x, r, i, lam, dh, tail, h0=h0, **how)
        for c0, c1 in zip(cuts, cuts[1:]):
            part = [t[..., c0:c1] for t in (x, r, i)]
            some = dict(h0=h0[:, c0:c1].contiguous(), **how)
            a, b = sw.gated_scan_fwd(*part, lam[c0:c1], **some)
            assert torch.equal(a, h[..., c0:c1]) and torch.equal(b, last[:, c0:c1]), (c0, c1)
            if D == 1088:
                k = sw.gated_scan_bwd(*part, lam[c0:c1], dh[..., c0:c1], tail[:, c0:c1].contiguous(), **some)
                assert all(torch.equal(k[m], g[m][..., c0:c1]) for m in k), (c0, c1)
        if D == 4160:
            out = torch.full_like(h, 7.0)
            ptr = [t.data_ptr() for t in (x, r, i, lam, h0)]
            with _on(h.device):
                assert sw.fast().sw_gated_scan_fwd(*ptr, how["cu_seqlens"].data_ptr() if packed else None,
                                                   out.data_ptr(), None, None, 1, L, D, n, (L * D, D) * 3, 1,
                                                   8.0, None, 0) == 0
            assert torch.equal(out, h)


@pytest.mark.parametrize("edges", [None, [3, 90, 90, 250, 329]])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L,D", [(330, 9), (330, 64), (100, 9)])
def test_rows_far_apart(sw, L, D, dtype, edges):
    """Rows so far apart that a chunk's reach over 2^31 bytes, forward and backward: several
    chunks of 16 steps a lane (L = 330) and one of 8, odd widths and whole ones; the inputs
    are columns of the same rows of one buffer, of which nothing else is touched."""
    print("case gated far", L, D, dtype, edges, flush=True)
    if edges and L < 330:
        edges = [min(e, L) for e in edges]
    n = len(edges) - 1 if edges else 1
    t, v = _make(L + D, 1, L, D, dtype, n)
    es = 4 if dtype == "f32" else 2
    step = 2 ** 31 // (64 * es) + 1  # of 64 steps of the backward; the forward's have 128 or 256
    names = ("x", "r", "i", "dh")
    big = torch.empty((L - 1) * step + 4 * 70, dtype=TYPES[dtype], device="cuda")
    for j, name in enumerate(names):
        far = big.as_strided((1, L, D), (0, step, 1), j * 70)
        far.copy_(t[name])
        t["far " + name] = far
    spans, cu = None, None
    if edges:
        cu = torch.tensor(edges, dtype=torch.int32, device="cuda")
        spans = [(0, edges[j], edges[j + 1]) for j in range(n)]
    how = dict(c=8.0, h0=t["h0"], cu_seqlens=cu)
    ins = [t["far " + name] for name in ("x", "r", "i")]
    want, off = ref.scan(v["x"], v["r"], v["i"], v["lam"], 8.0, v["h0"], spans, v["dh"], v["dh_last"])
    h, last = sw.gated_scan_fwd(*ins, t["lam"], **how)
    _near(h, want["h"], off["h"], "h")
    _near(last, want["h_last"], off["h_last"], "h_last")
    g = sw.gated_scan_bwd(*ins, t["lam"], t["far dh"], t["dh_last"], **how)
    for name in ("dx", "dr", "di", "dlam", "dh0"):
        _near(g[name], want[name], off[name], name)
    # the same steps in the same chunks, near
    near = [t[name] for name in ("x", "r", "i")]
    a, b = sw.gated_scan_fwd(*near, t["lam"], **how)
    assert torch.equal(a, h) and torch.equal(b, last)
    k = sw.gated_scan_bwd(*near, t["lam"], t["dh"], t["dh_last"], **how)
    assert all(torch.equal(k[m], g[m]) for m in k)
    covered = np.zeros(L, dtype=bool)
    for _, t0, t1 in spans or [(0, 0, L)]:
        covered[t0:t1] = True
    assert (h[0, torch.from_numpy(~covered).cuda()] == 0).all()
