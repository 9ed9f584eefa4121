"""More rows than one launch of the norm has threads for."""
import pytest
import torch

from paper_1712_01084_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols", [(70_000_001, 1), (2_200_003, 513), (4_300_001, 65)])
def test_more_rows_than_a_launch_has(rows, cols):
    """The limit is 2^32 threads: 67 million short rows, 16.7 million of up to 2048 columns; slices of a launch begin below it."""
    x = torch.empty(rows, cols, dtype=torch.float16, device="cuda").normal_()
    out = torch.full_like(x, 99.0)
    B.pivot_norm_run(x.data_ptr(), B.PIVOT_F16, cols, out.data_ptr(), B.PIVOT_F16, cols, rows, cols, eps=1e-3, stream=torch.cuda.current_stream().cuda_stream)
    for a in range(0, rows, 1 << 22 if cols > 1 else 1 << 26):
        h = x[a:a + (1 << 22 if cols > 1 else 1 << 26)].float()
        want = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-3)
        # half a step of fp16, 2^-11, or of its subnormal numbers, and what two evaluations in fp32 differ by
        assert ((out[a:a + len(h)].float() - want).abs() <= want.abs() * (2.0 ** -11 + (cols + 8) * 2.0 ** -23) + 2.0 ** -25).all()
