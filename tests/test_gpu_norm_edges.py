"""The norms' gradients at the edges of their contract."""
import numpy as np
import pytest

import linear_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sw():
    import paper_2606_00601_amd as pkg
    return pkg


def test_no_rows_read_no_input(sw):
    """Of no rows the parameters' gradients are zero and every input may be NULL."""
    from paper_2606_00601_amd._bind import _on
    f = sw.fast()
    for D, group in ((256, 64), (77, 11)):
        dw, ds = (torch.full((D,), float("nan"), device="cuda") for _ in range(2))
        with _on(dw.device):
            for flags in (0, 1):
                print("case no rows, gated", D, group, flags, flush=True)
                dw.fill_(float("nan"))
                assert f.sw_gated_norm_bwd(None, None, None, None, None, None, dw.data_ptr(), 0, D, group,
                                           D, D, D, 1, flags, 1e-6, None, 0) == 0
                assert (dw == 0).all()
            print("case no rows, residual", D, flush=True)
            dw.fill_(float("nan"))
            scale = torch.ones(D, device="cuda")
            assert f.sw_residual_norm_bwd(None, None, None, None, None, scale.data_ptr(), None, None,
                                          dw.data_ptr(), ds.data_ptr(), 0, D, D, D, D, D, 1, 0, 1e-6,
                                          None, 0) == 0
            assert (dw == 0).all() and (ds == 0).all()


@pytest.mark.parametrize("after", [False, True])
def test_large_gates(sw, after):
    """The sigmoid keeps fp32 accuracy for gates of any size: some ten roundings of 2^-24
    in each value, 2^-20."""
    M, D, group = 40, 256, 64
    r = np.random.Generator(np.random.PCG64(3))
    x, dy = r.standard_normal((2, M, D)).astype(np.float32)
    z = np.linspace(-80, 80, M * D, dtype=np.float32).reshape(M, D)
    z = r.permutation(z.reshape(M, -1, group), axis=0).reshape(M, D)  # each group's alike in size
    w = (1 + 0.1 * r.standard_normal(D)).astype(np.float32)
    t = {n: torch.from_numpy(a).cuda() for n, a in dict(x=x, z=z, w=w, dy=dy).items()}
    # eps far below the smallest group's mean square, e^-160
    eps = 1e-38 if after else 0.0
    want = ref.gated(*(a.astype(np.float64) for a in (x, z, w)), group, after, eps, dy.astype(np.float64))
    y = sw.gated_norm_fwd(t["x"], t["z"], t["w"], group=group, gate_after=after, eps=eps)
    g = sw.gated_norm_bwd(t["dy"], t["x"], t["z"], t["w"], group=group, gate_after=after, eps=eps)
    rows = np.s_[:] if after else np.abs(z).max(1) < 40  # u^2 within fp32's range
    for name, got in (("y", y), ("dz", g["dz"])):
        err = np.abs(got.double().cpu().numpy() - want[name])[rows]
        size = (want["t_y"] if name == "y" else want["t_dz"])[rows]
        assert size.size and (err <= 2.0 ** -20 * size + 1e-36).all(), (name, (err / size).max() * 2 ** 20)
