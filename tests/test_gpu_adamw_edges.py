"""AdamW and gradient norms beyond what one launch or 32 bits hold."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_norm_of_more_elements_than_a_launch_takes():
    """One gradient of 2^31 elements listed eighty times: 2^24 workgroups of 256 threads and more."""
    import paper_1511_08486_amd as sfb
    g = torch.empty(1 << 31, dtype=torch.bfloat16, device=DEV)
    g.normal_(0.0, 1.0, generator=torch.Generator(device=DEV).manual_seed(1))
    one, many = torch.zeros(2, device=DEV), torch.zeros(2, device=DEV)
    sfb.GradNorm([g])(1.0, one)
    norm = sfb.GradNorm([g] * 80)
    norm(1.0, many)
    norm.sync()
    assert abs(float(one[0]) / 2.0 ** 15.5 - 1.0) < 1e-3                 # 2^31 squares of a unit normal: 3e-5 deviation
    # sums in 64 bits: what is left is the two results' rounding to fp32
    assert abs(float(many[0]) / (float(one[0]) * 80.0 ** 0.5) - 1.0) <= 2.0 ** -23
    assert abs(float(many[1]) * float(many[0]) - 1.0) <= 2.0 ** -22
