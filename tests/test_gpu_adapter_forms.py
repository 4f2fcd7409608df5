"""Which of its two forms a call takes: a row to a workgroup, or rows sorted into tiles."""
import pytest
import torch

import paper_2506_21263_amd as dlcx
from gpu_util import DEV

pytestmark = pytest.mark.gpu


def kernels(rows, m, n, r, count, dtype, backward):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    d = dlcx.adapter_desc(m, n, r, count, dlcx.BF16 if dtype == "bf16" else dlcx.F32)
    z = lambda *s, t=dt: torch.zeros(*s, device=DEV, dtype=t)  # noqa: E731
    x, y, h, ids = z(rows, n), z(rows, m), z(rows, r, t=torch.float32), z(rows, t=torch.int32)
    q, p, ws = z(count, r, n), z(count, r, m), z(dlcx.dlcx_adapter_workspace_bytes(d, rows), t=torch.uint8)
    dlcx.dlcx_profile_enable(True)
    if backward:
        dlcx.dlcx_adapter_backward(d, x, y, ids, q, p, h, x, x, z(count, r, n, t=torch.float32),
                                   z(count, r, m, t=torch.float32), ws)
    else:
        dlcx.dlcx_adapter_forward(d, x, ids, q, p, y, y, h, ws)
    torch.cuda.synchronize()
    names = set(dlcx.dlcx_profile_read())
    dlcx.dlcx_profile_enable(False)
    return names


# both forms were timed at these sizes, and the one named took clearly less
@pytest.mark.parametrize("rows,m,n,r,count,backward,form", [
    (1024, 8192, 8192, 1, 1, False, "up"), (4096, 8192, 8192, 1, 1, False, "up"), (4096, 8192, 8192, 1, 64, False, "up"),
    (1024, 8192, 8192, 4, 1, False, "up"), (512, 8192, 8192, 8, 1, False, "up"), (256, 28672, 8192, 16, 1, False, "up"),
    (4096, 2048, 2048, 1, 1, False, "up"), (128, 28672, 8192, 64, 1, False, "up"), (512, 28672, 8192, 64, 64, False, "up"),
    (1024, 8192, 8192, 1, 1, True, "up"), (256, 8192, 8192, 16, 1, True, "up"), (64, 8192, 8192, 256, 1, True, "up"),
    (96, 28672, 8192, 16, 64, False, "rows"), (256, 28672, 8192, 16, 64, False, "rows"), (1, 8192, 8192, 256, 1, False, "rows"),
    (512, 2048, 2048, 16, 1, False, "rows"), (32, 8192, 8192, 256, 64, False, "rows"), (64, 8192, 8192, 16, 64, True, "rows"),
    (128, 28672, 8192, 64, 64, False, "rows"), (512, 1024, 8192, 1, 1, False, "rows"), (1024, 512, 512, 8, 1, False, "rows"),
    (16, 512, 512, 8, 4, True, "rows"), (8000, 64, 64, 1, 1, False, "up")])
def test_the_form_that_takes_less(rows, m, n, r, count, backward, form):
    names = kernels(rows, m, n, r, count, "bf16", backward)
    assert ("adapter_rows" in names) == (form == "rows") and ("adapter_up" in names) == (form == "up"), names
