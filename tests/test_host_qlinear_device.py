"""Buffers in host memory never reach a kernel: the binding refuses them by itself (the library sees addresses alone)."""
import pytest
import torch


def test_rows_on_the_host_are_refused(monkeypatch):
    from paper_2511_13587_amd import binding as vb
    calls = []
    for name in ("vvs_qrows_round", "vvs_qrows_norm", "vvs_qrows_read"):
        monkeypatch.setattr(vb.lib, name, lambda *a: calls.append(a) or 0)
    r, x = vb.QRows(3, 20, device="cpu"), torch.zeros(3, 20)
    for call in (lambda: vb.vvs_qrows_round(x, r), lambda: vb.vvs_qrows_read(r, x), lambda: vb.vvs_qrows_norm(x, torch.ones(20), 1e-5, r), lambda: vb.vvs_qrows_round(x[:2], r.first(2))):
        with pytest.raises(ValueError, match="host"):
            call()
    assert not calls


@pytest.mark.parametrize("device", ["cpu", "meta", torch.device("cpu")])
def test_maps_and_caches_on_the_host_are_refused(device):
    from paper_2511_13587_amd import binding as vb
    with pytest.raises(ValueError, match="GPU"):
        vb.QLinear(300, 200, 4, vb.VVS_BF16, device=device)
    with pytest.raises(ValueError, match="GPU"):
        vb.QCache(1, 2, 4, 4, 64, 64, 4, vb.VVS_BF16, device=device)
