"""Norm and gradient where a workgroup takes several rows, one of each width of group and with rows that end anywhere: the
next row's loads, the places of the sums and the parts of dw change from turn to turn."""
import pytest

from test_gpu_norm import check_backward, check_forward

pytestmark = pytest.mark.gpu

# rows, n: more rows than workgroups (8192 up to 512 columns, 2048, 1280, 768, 256 above), turns of the last one left out
TURNS = [(8200, 130), (8213, 512), (16500, 8), (2100, 1021), (4101, 2048), (1300, 2050), (2600, 4096), (800, 8190), (1600, 8192)]
LONG = [(300, 16384, "f32"), (600, 16384, "bf16"), (300, 32768, "bf16"), (300, 9001, "bf16")]


@pytest.mark.parametrize("rows,n,dtype", [(r, n, d) for r, n in TURNS for d in ("f32", "bf16")] + LONG)
def test_norm(rows, n, dtype):
    """With and without a residual, whose sum goes over x; to the type, to 8 bits and to both."""
    check_forward(rows, n, dtype, True, True, True, pad=3, shift=1, in_place=True)
    check_forward(rows, n, dtype, False, False, True)
    check_forward(rows, n, dtype, True, True, False, pad=2)


@pytest.mark.parametrize("rows,n,dtype", [(r, n, d) for r, n in [(8200, 130), (3100, 2050), (2000, 4096), (1100, 8190), (1536, 8192)]
                                          for d in ("f32", "bf16")] + [(600, 16384, "bf16"), (600, 9001, "f32")])
def test_gradient(rows, n, dtype):
    check_backward(rows, n, dtype, True, pad=1, shift=1)
    check_backward(rows, n, dtype, False)
    check_backward(rows, n, dtype, True, alias="dx_in")
