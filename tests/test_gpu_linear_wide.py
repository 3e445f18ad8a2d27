"""Layers with bfloat16 results and an outlier list through the 256 x 128 tile: the sums of such layers are not carried, with a
list either, and the columns are whole or shared by up to 16 workgroups."""
import pytest
import torch

from test_gpu_linear import Matrix, check, randn
from test_host_gemm_plan import WIDE
from test_host_layer_plan import layers  # noqa: F401 (a fixture: the host's choice of the kernel for layers)

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32

# rows, cols, tokens, workgroups that share the columns; rows and tokens that end inside tiles
LISTED = [(14875, 576, 201, 1), (22016, 4096, 230, 1), (4161, 992, 174, 2), (4096, 4096, 400, 4), (2749, 2752, 131, 5), (610, 8992, 162, 16)]


def workgroups(plan, rows, cols, n_tokens):
    """Workgroups along the columns, from the workspace that the plan needs: x in order, then a binary32 part of each."""
    x = -(-n_tokens // 32) * 32 * -(-cols // 64) * 128
    return max(1, round((plan.need - x) / (n_tokens * rows * 4)))


@pytest.mark.parametrize("rows,cols,n_tokens,split", LISTED)
def test_listed_layers_with_uncarried_sums(layers, rows, cols, n_tokens, split):  # noqa: F811
    plan = layers(rows, cols, n_tokens, True, True)
    assert plan.way == WIDE and not plan.carry and workgroups(plan, rows, cols, n_tokens) == split
    m = Matrix(rows, cols, 0.006)
    check(m, "gemm", n_tokens)
    check(m, "gemm", n_tokens, "silu", mul=BF16, pre=BF16)
    check(m, "gemm", n_tokens, "gelu", bias=F32, mul=F32, residual=F32)


def test_every_listed_entry_is_in_its_place():
    """x of unit vectors: each column of the decoded matrix comes out alone, exactly, entries of the list among them."""
    rows, cols, n_tokens = 4161, 992, 174
    m = Matrix(rows, cols, 0.02)
    for first in (0, 400, cols - n_tokens):
        x = torch.zeros((n_tokens, cols), dtype=BF16, device="cuda")
        x[torch.arange(n_tokens), first + torch.arange(n_tokens)] = 1.0
        y = m.linear("gemm", x, residual=torch.zeros((n_tokens, rows), dtype=BF16, device="cuda"))
        assert torch.equal(y.double(), m.gemm_w[:, first:first + n_tokens].t())


def test_result_over_the_residual():
    for rows, cols, n_tokens, _ in LISTED[:3]:
        m, x = Matrix(rows, cols, 0.006), randn((n_tokens, cols), 1)
        r = randn((n_tokens, rows), 2)
        want = m.linear("gemm", x, residual=r)
        m.linear("gemm", x, residual=r, out=r)
        assert torch.equal(r, want)
