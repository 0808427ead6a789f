"""Values of the RMS norm that a bound on the error does not pin."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def _codes(gs, x, w, group):
    """The codes and scales of rows whose y is x w exactly: x = +-1, eps = 0, so that the mean square is 1."""
    y8, sc, _ = gs.add_rms_norm_fp8(x, w, None, 0.0, group)
    y = x.float() * w.float()                     # 8 bits times a sign
    width = group or x.shape[1]
    amax = torch.stack([y[:, i: i + width].abs().amax(1) for i in range(0, x.shape[1], width)], 1)
    assert torch.equal(sc, (amax.double() / 448).float())     # 32-bit tensors on a GPU are multiplied by 1 / 448
    q = (y / sc.repeat_interleave(width, 1)).to(torch.float8_e4m3fn)
    assert torch.equal(y8.view(torch.uint8), q.view(torch.uint8))


def _groups_of_every_mantissa():
    """128 groups of 128 columns: every 8-bit mantissa as the largest, the others below it."""
    w = torch.arange(128, 256, device="cuda")[None].repeat(128, 1) / 256
    w[:, 0] = torch.arange(128, 256, device="cuda") / 128
    return w.to(torch.bfloat16)


# a row in registers; read again for each pass (2^16 columns)
@pytest.mark.parametrize("repeat", [1, 4])
def test_codes_are_those_of_the_quotient(gs, repeat):
    w = _groups_of_every_mantissa().flatten().repeat(repeat)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(0, 2, (3, w.numel()), generator=g, device="cuda").mul_(2).sub_(1).to(torch.bfloat16)
    _codes(gs, x, w, 128)


@pytest.mark.parametrize("exponent", [0, -100, 60, 119])
def test_codes_of_whole_rows(gs, exponent):
    x = torch.ones((2, 128), dtype=torch.bfloat16, device="cuda")
    for w in _groups_of_every_mantissa() * 2.0 ** exponent:
        _codes(gs, x, w, 0)


@pytest.mark.parametrize("n", [128, 515])
def test_codes_beside_an_infinity(gs, n):
    """An infinite y is NaN in 8 bits, the finite ones of its group zero."""
    x, w = (torch.ones(s, dtype=torch.bfloat16, device="cuda") for s in ((2, n), (n,)))
    w[3] = float("inf")
    y8, sc, _ = gs.add_rms_norm_fp8(x, w)
    assert (sc == float("inf")).all() and y8[:, 3].float().isnan().all()
    assert (y8[:, :3].float() == 0).all() and (y8[:, 4:].float() == 0).all()
