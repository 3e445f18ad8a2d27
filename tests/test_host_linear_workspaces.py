"""The workspace of a linear layer's gradients on the CPU: a host formula that covers every type of dy and dx."""
import pytest

from paper_2505_06653_amd import binding


@pytest.mark.parametrize("rows,cols", [(1 << 18, 96), (1 << 18, 32768), (100000, 4096), (4096, 11008)])
def test_gradient_workspace_holds_every_number_of_terms_and_never_falls(rows, cols):
    sizes = [binding.bof4_gemm_linear_backward_workspace_bytes(rows, cols, n) for n in
             (1, 100, 2000, 2687, 2688, 2689, 2720, 2816, 5376, 7000, 7168, 7169, 9000, 20000, 65536)]
    assert sizes == sorted(sizes)
    # dz in one term, or as much of it as several terms take at a time (4 GiB), partial sums of up to 16 workgroups and slabs
    least = 65536 * rows * 2
    assert least <= sizes[-1] <= max(least, 4 << 30) + 16 * 65536 * cols * 4 + (300 << 20) + 64 * 50 * rows * 4
