"""Adapters whose B holds an infinity."""
import pytest
import torch

from tests import _block_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


@pytest.mark.parametrize("rank,inp,out", [(8, 64, 40), (16, 512, 96), (24, 264, 37), (32, 512, 200), (64, 256, 96),
                                          (128, 256, 72), (48, 520, 33)])
@pytest.mark.parametrize("lens,ids", [([1, 2, 1], [0, 1, 0]), ([80, 90], [1, 0])])
def test_infinite_elements_of_b(gs, rank, inp, out, lens, ids):
    """They give base + s inf (A x) = an infinity of A x's sign; every other output keeps its bits."""
    g = torch.Generator(device="cuda").manual_seed(rank)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    T, off, i = sum(lens), ref.offsets(lens), ref.i32(ids)
    x, base, A, B = rand(T, inp), rand(T, out), rand(2, rank, inp), rand(2, out, rank)
    scale = torch.tensor([0.5, 2.0], device="cuda")
    clean = gs.adapters_into(x, base, gs.Adapters(A, B, scale), off, i, torch.empty_like(base))
    at = [(a, o, k) for a in (0, 1) for o, k in ((0, 0), (3, rank - 1), (out - 1, rank // 2), (17, 5))]
    for n, (a, o, k) in enumerate(at):
        B[a, o, k] = float("inf") * (-1) ** n
    B[0, 20, 1], B[0, 20, 2] = float("inf"), float("inf")     # two: an infinity or NaN
    for inplace in (False, True):
        y = base.clone()
        gs.adapters_into(x, y if inplace else base, gs.Adapters(A, B, scale), off, i, y)
        seq = torch.repeat_interleave(torch.tensor(ids), torch.tensor(lens)).cuda()
        hit = torch.zeros((T, out), dtype=torch.bool, device="cuda")
        for n, (a, o, k) in enumerate(at):
            rows = (seq == a).nonzero()[:, 0]
            low = x[rows].double() @ A[a, k].double()
            # far enough from 0 for float32 sums to have its sign
            sure = low.abs() > inp * 2.0 ** -24 * (x[rows].double().abs() @ A[a, k].double().abs())
            assert (y[rows, o][sure].double() == low[sure].sign() * (-1) ** n * float("inf")).all()
            hit[rows, o] = True
        rows = (seq == 0).nonzero()[:, 0]
        low = x[rows].double() @ A[0, 1:3].double().T
        want = (low.sign() * float("inf")).sum(1)
        assert torch.equal(y[rows, 20].double().nan_to_num(7.0), want.nan_to_num(7.0))
        hit[rows, 20] = True
        assert torch.equal(y[~hit], clean[~hit])
