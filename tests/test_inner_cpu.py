"""Sequencing of the inner and outer steps of adapters on the host: nothing is launched."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from paper_2506_21263_amd import inner
from paper_2506_21263_amd.stage import MatrixState


@pytest.mark.parametrize("size,K,outer,r,mma", [(512, 2, 8, 64, dlcx.MMA_BF16), (512, 2, 8, 64, dlcx.MMA_F32),
                                                (512, 2, 4, 256, dlcx.MMA_F32), (1024, 4, 16, 256, dlcx.MMA_F16),
                                                (512, 2, 64, 8, dlcx.MMA_F32), (512, 2, 8, 64, dlcx.MMA_FMA)])
def test_every_call_of_an_outer_step_has_the_workspace_of_its_own_rank(monkeypatch, size, K, outer, r, mma):
    theta = torch.zeros(size, size)
    M = MatrixState(theta, K, torch.zeros(outer, size), 8, 64, mma)
    proj = inner.AdapterProjection(theta, torch.zeros(K, r, size), 1.0, 16, torch.float32)
    step = inner.AdapterOuterStep(M, 0.7, 0.9)
    ranks = []

    def decompress(d, p, q, out, ef=(), workspace=None, stream=None):
        ranks.append(d.r)
        if mma != dlcx.MMA_FMA:
            assert workspace.numel() >= dlcx.dlcx_workspace_bytes(d, 1), d.r

    def compress(d, phase, ef, basis, codes, scales, mean, workspace, stream=None):
        assert workspace.numel() >= dlcx.dlcx_workspace_bytes(d, len(ef))

    monkeypatch.setattr(inner, "dlcx_decompress", decompress)
    monkeypatch.setattr(inner, "dlcx_compress_average", compress)
    monkeypatch.setattr(inner, "dlcx_orthonormalize", lambda *a, **k: None)
    monkeypatch.setattr(inner, "dlcx_outer_nesterov", lambda *a, **k: None)
    step.step(proj)
    step.step(proj)
    assert ranks.count(r) >= 2 * K and outer in ranks


def test_fold_refuses_a_workspace_that_is_too_small(monkeypatch):
    theta = torch.zeros(512, 512)
    proj = inner.AdapterProjection(theta, torch.zeros(2, 64, 512), 1.0, 16, torch.float32)
    monkeypatch.setattr(inner, "dlcx_decompress", lambda *a, **k: pytest.fail("was called"))
    need = proj.fold_workspace_bytes(64, dlcx.MMA_F32)
    assert need > 0 and proj.fold_workspace_bytes(64, dlcx.MMA_FMA) == 0
    for ws in (None, torch.empty(need - 1, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            proj.fold([theta, theta], ws, 64, dlcx.MMA_F32)
