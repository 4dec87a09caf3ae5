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


def test_8_bit_moments_of_elements_beyond_32_bits():
    """An element's number, of which its rounding is drawn, does not end at 2^32: the same tensor behind 2^32 elements is drawn anew, and
    every code is one of the two about the value."""
    import paper_1511_08486_amd as sfb
    from test_gpu_adamw import HYPER, _formula, _values
    n, big = 5000, 1 << 32
    g = torch.randn(n, generator=torch.Generator().manual_seed(3)).to(DEV) * 1e-2
    step = torch.zeros(1, dtype=torch.int32, device=DEV)
    u8 = lambda k: torch.zeros(k, dtype=torch.uint8, device=DEV)  # noqa: E731

    def state():
        return torch.zeros(n, device=DEV), u8(n), u8(n), u8((n + 127) // 128), u8((n + 127) // 128)
    front, behind = state(), state()
    p = torch.zeros(big, device=DEV)
    opt = sfb.AdamW([front[0], p, behind[0]], [g.bfloat16(), torch.zeros(big, dtype=torch.bfloat16, device=DEV), g.bfloat16()], [front[1], u8(big), behind[1]],
                    [front[2], u8(big), behind[2]], step, m_scales=[front[3], u8(big // 128), behind[3]], v_scales=[front[4], u8(big // 128), behind[4]])
    opt.step(**HYPER, seed=5)
    opt.sync()
    assert (p[:: 1 << 20] == 0).all() and int(step) == 1
    zero, gd = torch.zeros(n).double().numpy(), g.bfloat16().double().cpu().numpy()
    want, m, v, _ = _formula(zero, gd, zero, zero, 1, **HYPER)
    for s in (front, behind):
        err = abs(s[0].double().cpu().numpy() - want)
        assert (err <= HYPER["lr"] * 2e-4).all()                         # a dozen roundings, 1 - b2 as an fp32 number
        # codes are an eighth of their binade apart, or 2^-9 and 2^-17 of the scale at their lowest
        for codes, scales, x, second in ((s[1], s[3], m, False), (s[2], s[4], v, True)):
            at = _values(codes, scales, second)
            lowest = (2.0 ** -17 if second else 2.0 ** -9) * 2.0 ** (scales.cpu().numpy().astype(float).repeat(128)[:n] - 127.0)
            assert (abs(at - x) <= abs(x) / 8.0 + lowest + 1e-5 * abs(x)).all()
    assert torch.equal(front[3], behind[3]) and torch.equal(front[4], behind[4]) and torch.equal(front[0], behind[0])
    # of elements that round up with a probability p, two draws differ with 2 p (1 - p): a third on average where p is anything
    moved = float((front[1] != behind[1]).double().mean())
    assert 0.2 < moved < 0.45, moved


def test_norm_beyond_fp32_is_clipped_all_the_same():
    import paper_1511_08486_amd as sfb
    out = torch.zeros(2, device=DEV)
    norm = sfb.GradNorm([torch.full((4,), 3e38, device=DEV)])
    norm(1e3, out)
    norm.sync()
    assert float(out[0]) == float("inf")
    assert abs(float(out[1]) / (1e3 / 6e38) - 1.0) <= 2.0 ** -22         # 3e38 and the factor as fp32 numbers
