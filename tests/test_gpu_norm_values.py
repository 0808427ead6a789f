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


@pytest.mark.parametrize("n", [8, 512, 515, 4096, 16384, 40000])
@pytest.mark.parametrize("size,eps", [(1e20, 1e-5), (2.0 ** 126, 1e-5), (1e-21, 0.0), (1e-25, 1e-50), (1e-30, 1e-36), (1e-38, 0.0),
                                      (3e18, 1e-5), (1e-20, 1e-5)])
def test_rows_whose_squares_leave_the_range(gs, n, size, eps):
    """Finite rows have finite norms, however large or small they are; ordinary rows beside them keep their bits."""
    from tests import _block_ref as ref
    g = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").clamp(-3.9, 3.9)  # noqa: E731
    x, r, w = (rand(4, n) / 4).bfloat16(), (rand(4, n) / 4).bfloat16(), rand(n).bfloat16()
    plain = gs.add_rms_norm(x, w, r, eps)[0]
    x[1], r[1] = (x[1].double() * size).bfloat16(), (r[1].double() * size).bfloat16()
    x[2, 0] = size                                # one element alone is out of range
    y, h = gs.add_rms_norm(x, w, r, eps)
    eps32 = float(torch.tensor(eps, dtype=torch.float32))
    hr, yr = ref.norm(x, r, w, eps32)
    assert yr.isfinite().all()
    ref.assert_close(y, yr, yr.abs() * (ref.BF + n * 2.0 ** -24) + 1e-30, "y")
    ref.assert_close(h, hr, hr.abs() * ref.BF + 2.0 ** -134, "h")
    assert torch.equal(y[[0, 3]], plain[[0, 3]])
    y8, sc, _ = gs.add_rms_norm_fp8(x, w, r, eps, 128)
    want = torch.stack([yr[:, i: i + 128].abs().amax(1) for i in range(0, n, 128)], 1) / 448
    ref.assert_close(sc, want.clamp(min=2.0 ** -126), want * (n * 2.0 ** -24 + 2.0 ** -20) + 1e-37, "scales")


def test_empty_and_infinite_rows(gs):
    for n in (512, 515):
        x, w = torch.zeros((3, n), dtype=torch.bfloat16, device="cuda"), torch.ones((n,), dtype=torch.bfloat16, device="cuda")
        x[1, 5], x[2, 7] = float("inf"), float("nan")
        for eps in (1e-5, 1e-38):
            y, _ = gs.add_rms_norm(x, w, None, eps)
            assert (y[0] == 0).all() and y[1, 5].isnan() and (y[1, 6:] == 0).all() and y[2].isnan().all()
