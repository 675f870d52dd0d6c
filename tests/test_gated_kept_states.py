"""When the gated recurrence's autograd function keeps states for its backward: where a
gradient can be asked for, and only there (no GPU: the forward itself is replaced)."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

import paper_2606_00601_amd._gated as gated  # noqa: E402


@pytest.mark.parametrize("leaf", ["x", "r", "i", "lam", "h0", None])
@pytest.mark.parametrize("grad", [True, False])
def test_states_are_kept_for_a_backward_only(monkeypatch, leaf, grad):
    kept = []

    def forward(x, r, i, lam, c, h0, cu_seqlens, h, h_last, keep):
        kept.append(keep)
        return torch.zeros_like(x), None, torch.zeros(1) if keep else None

    monkeypatch.setattr(gated, "_forward", forward)
    t = {n: torch.zeros(1, 4, 8) for n in ("x", "r", "i")}
    t["lam"], t["h0"] = torch.zeros(8), torch.zeros(1, 8)
    if leaf:
        t[leaf].requires_grad_(True)
    with contextlib.nullcontext() if grad else torch.no_grad():
        h = gated.gated_scan_fn(t["x"], t["r"], t["i"], t["lam"], h0=t["h0"])
    assert kept == [grad and leaf is not None]
    assert h.requires_grad == kept[0]
