"""The norms' gradients at the edges of their contract."""
import pytest

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
