"""Tokens of no sequence, and lengths that the page table does not hold, in each launch of the attention and beside it."""
import pytest
import torch

from tests import _block_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def _rand(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


# (tokens, offsets, lengths, max_new): the kernel for few rows, the one for many (all sequences as long as the longest, by
# the sizes alone), both; tokens of no sequence before the first one, behind the last one, at both ends, all of them
@pytest.mark.parametrize("tokens,offsets,kv,max_new", [
    (6, [2, 5], [40], 6), (6, [0, 0], [0], 6), (100, [0, 60], [90], 100), (100, [40, 100], [90], 100),
    (200, [7, 150], [500], 200), (64, [0, 0], [0], 64), (120, [3, 63, 64, 70], [90, 33, 8], 60), (80, [0, 70, 71], [70, 300], 70)])
@pytest.mark.parametrize("d", [64, 128])
def test_tokens_of_no_sequence_are_zero(gs, tokens, offsets, kv, max_new, d):
    cache, table = ref.make_cache(gs, kv, 2, d, 16, 1)
    q = _rand((tokens, 8, d), 2)
    out = torch.full_like(q, 7.0)
    gs.paged_attention(q, cache, gs.Batch(ref.i32(offsets), ref.i32(kv), table, max_new), out=out)
    new = [b - a for a, b in zip(offsets, offsets[1:])]
    inside = slice(offsets[0], offsets[-1])
    want, bound = ref.attention(q[inside], cache.k_pages, cache.v_pages, table, new, kv, d ** -0.5)
    ref.assert_close(out[inside], want, bound)
    assert (out[: offsets[0]] == 0).all() and (out[offsets[-1]:] == 0).all()
    assert gs.device_status() == gs.GS_OK


@pytest.mark.parametrize("new,told", [([1], 1), ([3, 1], 3), ([100], 100), ([100, 1], 100)])
def test_lengths_outside_the_table(gs, new, told):
    """Longer than the table: every token sees what the table holds.  Negative: no token sees anything."""
    d, page, hq, hkv = 64, 16, 4, 2
    cache, table = ref.make_cache(gs, [64] * len(new), hkv, d, page, 3)
    T = sum(new)
    q = _rand((T, hq, d), 4)
    seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
    K, V = (p[table.long()].permute(0, 2, 1, 3, 4).reshape(len(new), hkv, 64, d).double()[seq] for p in (cache.k_pages, cache.v_pages))
    K, V = (t.repeat_interleave(hq // hkv, 1) for t in (K, V))
    p = (torch.einsum("thd,thjd->thj", q.double(), K) * d ** -0.5).softmax(-1)
    want, size = torch.einsum("thj,thjd->thd", p, V), torch.einsum("thj,thjd->thd", p, V.abs())
    for length in (64 + told - 1, 4000, 2 ** 31 - 1):
        out = gs.paged_attention(q, cache, gs.Batch(ref.offsets(new), ref.i32([length] * len(new)), table, told))
        ref.assert_close(out, want, ref.BF * want.abs() + size * (2.0 ** -8 + 2.0 ** -14), f"length {length}")
    for length in (-1, -5000, -2 ** 31):
        out = torch.full_like(q, 7.0)
        gs.paged_attention(q, cache, gs.Batch(ref.offsets(new), ref.i32([length] * len(new)), table, told), out=out)
        assert (out == 0).all()
    assert gs.device_status() == gs.GS_OK


def test_append_and_adapters_leave_tokens_of_no_sequence(gs):
    d, T, off, kv = 64, 9, ref.i32([2, 5, 7]), [40, 2]
    cache, table = ref.make_cache(gs, kv, 2, d, 16, 5)
    k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
    q, k, v = _rand((T, 4, d), 6), _rand((T, 2, d), 7), _rand((T, 2, d), 8)
    a = torch.rand((64, d // 2), device="cuda") * 6
    out = gs.cache_append(cache, gs.Batch(off, ref.i32(kv), table, 3), q, k, v, a.cos(), a.sin())
    assert torch.equal(out[:2], q[:2]) and torch.equal(out[7:], q[7:])
    for i, (t0, n, m) in enumerate(((2, 3, 40), (5, 2, 2))):
        for j in range(n):
            pos = m - n + j
            at = int(table[i, pos // 16]), slice(None), pos % 16
            assert torch.equal(cache.v_pages[at], v[t0 + j])
            k0[at], v0[at] = cache.k_pages[at], v[t0 + j]
    same = lambda x, y: torch.equal(x.view(torch.int16), y.view(torch.int16))  # noqa: E731
    assert same(cache.k_pages, k0) and same(cache.v_pages, v0)
    x, base = _rand((T, 128), 9), _rand((T, 40), 10)
    ad = gs.Adapters(_rand((2, 8, 128), 11), _rand((2, 40, 8), 12), torch.ones(2, device="cuda"))
    y = torch.full_like(base, 7.0)
    gs.adapters_into(x, base, ad, off, ref.i32([1, -1]), y)
    assert (y[:2] == 7).all() and (y[7:] == 7).all() and torch.equal(y[5:7], base[5:7])
    want, bound = ref.adapters(x[2:7], base[2:7], ad.A, ad.B, ad.scale, [3, 2], [1, -1])
    ref.assert_close(y[2:7], want, bound)


def test_a_batch_refuses_more_new_tokens_than_32_bits(gs):
    for bad in (2 ** 32 + 1, 2 ** 31, -1):
        with pytest.raises(ValueError, match="max_new"):
            gs.Batch(ref.offsets([1]), ref.i32([5]), ref.i32([[0]]), bad)
