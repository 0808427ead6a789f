"""Attention over a cache in 8 bits against 64 bits, each form held to its own arithmetic and to nothing looser.

With p the softmax's weights, s the values' powers of two and q their codes, a = sum_j p_j |v_j| of a row's channel:

  output  bf16: 2^-8 of itself.
  scores  float32: a weight is off by 2 (sum |q||k| scale) (d 2^-24 + 2^-22) of itself, and by 2^-15 for exponents that a power has
          been added to (below 2^8, so three roundings of 2^-17) and for ex2.
  sums    float32: a unit in the last place for each 16 keys and for each of the joins, 2^-23 (keys / 16 + 64) of a.
  weights many rows (chunk): bf16, 2^-8 of themselves; below 2^-126 of the row's largest, zero.
          few rows: f16, 2^-11 of themselves, or, where p s is below 2^-20 of the row's largest, half of f16's least step: the largest
          is 2^6 at least there, so 2^-25 is 2^-31 of it, times the key's codes.

There is no absolute term but float32's least numbers, so values of any size count.
"""
import math

import pytest
import torch

from tests import _block_ref as ref
from tests import _fp8_ref as f8

pytestmark = pytest.mark.gpu

# (query heads, key heads, width, new tokens, lengths).  At most 32 rows a key head, or 64 where sequences x key heads are few.  40000
# keys of one key head lie in so many parts that they are joined in two levels.
FEW = [(4, 4, 128, [1], [90]), (4, 4, 64, [1, 1], [700, 33]), (7, 1, 128, [1], [9000]), (28, 4, 128, [4], [300]), (28, 4, 128, [2, 1], [70, 2000]),
       (16, 2, 64, [4, 2, 3], [500, 130, 1500]), (7, 1, 128, [1], [40000]), (28, 4, 128, [9], [2000]), (8, 1, 64, [8, 5], [400, 90])]
CHUNK = [(4, 4, 128, [150], [444]), (28, 4, 128, [100], [3000]), (16, 2, 64, [77, 200], [900, 200])]
FORMS = [pytest.param(True, *f, id="few-" + "-".join(map(str, f))) for f in FEW] + [pytest.param(False, *f, id="chunk-" + "-".join(map(str, f))) for f in CHUNK]


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def _rand(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def reference(q, cache, table, new, kv, scale, few, weight=None):
    """(out, bound) in 64 bits.  weight: what to round the weights (largest: 1) to, to see what a bound tells apart."""
    T, hq, d = q.shape
    hkv, g = cache.kv_heads, hq // cache.kv_heads
    codes_of, s_of = cache.v_pages.float().double(), f8.scale_values(cache.v_scales)
    K_of = f8.values(cache.k_pages, cache.k_scales)
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    t = 0
    for i, (n, m) in enumerate(zip(new, kv)):
        ids = table[i, : -(-m // cache.page_size)].long()
        K, C = (x[ids].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :m] for x in (K_of, codes_of))
        S = s_of[ids].permute(1, 0, 2).reshape(hkv, 1, -1)[..., :m]
        rows = q[t: t + n].double().permute(1, 0, 2).reshape(hkv, g * n, d)
        sc = rows @ K.transpose(1, 2) * scale
        mags = (rows.abs() @ K.abs().transpose(1, 2) * abs(scale)).amax(-1, keepdim=True)
        seen = (torch.arange(m, device=q.device)[None] <= (m - n + torch.arange(n, device=q.device)).repeat(g)[:, None])
        w = (sc - sc.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)).exp() * seen
        total = w.sum(-1, keepdim=True)
        if weight is not None:
            w = w.to(weight).double()
        p = w / total
        V = C * S.transpose(1, 2)
        o, a = p @ V, p @ V.abs()
        err = ref.BF * o.abs() + a * (2 * mags * (d * 2.0 ** -24 + 2.0 ** -22) + 2.0 ** -15 + 2.0 ** -23 * (m / 16 + 64)) + 2.0 ** -126
        if few:
            err += a * 1.02 * 2.0 ** -11 + 1.02 * 2.0 ** -31 * (p * S).amax(-1, keepdim=True) * (seen.double() @ C.abs())
        else:
            err += a * 1.02 * 2.0 ** -8 + 2.0 ** -126 * (seen.double() @ V.abs())
        out[t: t + n] = o.reshape(hq, n, d).permute(1, 0, 2)
        bound[t: t + n] = err.reshape(hq, n, d).permute(1, 0, 2)
        t += n
    return out, bound


def _check(gs, cache, table, q, few, new, kv, scale, what):
    b = gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new))
    got = gs.paged_attention(q, cache, b, scale)
    want, bound = reference(q, cache, table, new, kv, scale, few)
    ref.assert_close(got, want, bound, what)
    assert torch.equal(got, gs.paged_attention(q, cache, b, scale)) and gs.device_status() == gs.GS_OK
    return got


@pytest.mark.parametrize("few,hq,hkv,d,new,kv", FORMS)
@pytest.mark.parametrize("vscale", [1.0, 2.0 ** -60, 2.0 ** -90, 2.0 ** 40])
def test_each_form_within_its_own_bound(gs, few, hq, hkv, d, new, kv, vscale):
    cache, table = f8.make_cache(gs, kv, hkv, d, 32, 200, vscale=vscale)
    _check(gs, cache, table, _rand((sum(new), hq, d), 201, 1.0), few, new, kv, d ** -0.5, f"values of {vscale}")


@pytest.mark.parametrize("few,hq,hkv,d,new,kv", FORMS)
@pytest.mark.parametrize("more", [10, 24, 32, 40, 57, 64, 90])
@pytest.mark.parametrize("at", [0.0, 0.4, 0.9])
def test_a_large_value_of_little_weight_takes_nothing_from_the_others(gs, few, hq, hkv, d, new, kv, more, at):
    """A key that all rows see, with a weight of about 2^-58, and a value 2^more times as large as the others: before, among and
    behind them."""
    cache, table = f8.make_cache(gs, kv, hkv, d, 32, 210)
    q = (1.0 + 0.1 * _rand((sum(new), hq, d), 211).float()).to(torch.bfloat16)
    ks, vs = cache.k_scales.view(torch.uint8), cache.v_scales.view(torch.uint8)
    ks -= 4 * (ks != 255)
    for i, (n, m) in enumerate(zip(new, kv)):
        pos = int(at * (m - n))
        page, slot = int(table[i, pos // 32]), pos % 32
        cache.k_pages.view(torch.uint8)[page, :, slot] = 0xB2 if d == 64 else 0xAA       # -0.625, -0.3125: a score of -40
        ks[page, :, slot] = 127
        vs[page, :, slot] += more
    _check(gs, cache, table, q, few, new, kv, 1.0, f"2^{more} at {at}")


@pytest.mark.parametrize("few,hq,hkv,d,new,kv", FORMS)
@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_values_of_all_sizes_under_weights_of_all_sizes(gs, few, hq, hkv, d, new, kv, scale):
    """Powers from 2^-60 to 2^60 at random, under scores that make the large ones count in some rows and not in others."""
    cache, table = f8.make_cache(gs, kv, hkv, d, 32, 220)
    vs = cache.v_scales.view(torch.uint8)
    g = torch.Generator(device="cuda").manual_seed(221)
    vs += torch.where(vs == 255, 0, torch.randint(-60, 61, vs.shape, generator=g, device="cuda")).to(torch.uint8)
    _check(gs, cache, table, _rand((sum(new), hq, d), 222), few, new, kv, scale * d ** -0.5, "powers at random")


@pytest.mark.parametrize("few,hq,hkv,d,new,kv", FORMS)
@pytest.mark.parametrize("which", ["first", "all", "some", "keys"])
def test_scales_of_zero_read_as_zero(gs, few, hq, hkv, d, new, kv, which):
    """Heads whose scale byte is 0, whatever their codes: values of the first keys, of all keys, of some; or keys (a score of 0)."""
    cache, table = f8.make_cache(gs, kv, hkv, d, 32, 250)
    sc = (cache.k_scales if which == "keys" else cache.v_scales).view(torch.uint8)
    some = torch.rand(sc.shape, generator=torch.Generator(device="cuda").manual_seed(251), device="cuda") < 0.7
    if which == "all":
        some.fill_(True)
    if which == "first":
        some.fill_(False)
        for i, m in enumerate(kv):
            pages = table[i, : -(-m // 32)].long()
            for at, page in enumerate(pages.tolist()):
                some[page, :, : max(0, min(32, m * 2 // 3 - 32 * at))] = True
    sc.masked_fill_(some & (sc != 255), 0)
    got = _check(gs, cache, table, _rand((sum(new), hq, d), 252), few, new, kv, d ** -0.5, which)
    assert (got == 0).all() == (which == "all")


@pytest.mark.parametrize("few,hq,hkv,d,new,kv", FORMS)
@pytest.mark.parametrize("operand", [0, 1])
def test_nan_at_the_first_key_stays_with_its_head(gs, few, hq, hkv, d, new, kv, operand):
    cache, table = f8.make_cache(gs, kv, hkv, d, 32, 260)
    q = _rand((sum(new), hq, d), 261)
    b = gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new))
    clean = gs.paged_attention(q, cache, b)
    (cache.k_scales, cache.v_scales)[operand].view(torch.uint8)[int(table[0, 0]), hkv - 1, 0] = 255
    got = gs.paged_attention(q, cache, b)
    own = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    own[: new[0], hq - hq // hkv:] = True
    assert got[own].isnan().all() and torch.equal(got[~own], clean[~own])


@pytest.mark.parametrize("few,hq,hkv,d,new,kv", FORMS)
def test_sums_of_the_largest_values_are_finite(gs, few, hq, hkv, d, new, kv):
    """Many keys of the same weight, all with the largest value that append writes: their mean is that value."""
    cache, table = f8.make_cache(gs, kv, hkv, d, 32, 230)
    cache.k_pages.view(torch.uint8).zero_()
    cache.k_scales.view(torch.uint8).fill_(127)
    sign = torch.where(torch.arange(d, device="cuda") % 3 == 0, 0xFE, 0x7E).to(torch.uint8)
    cache.v_pages.view(torch.uint8).copy_(sign.expand(cache.v_pages.shape))
    cache.v_scales.view(torch.uint8).fill_(246)
    b = gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new))
    got = gs.paged_attention(_rand((sum(new), hq, d), 231), cache, b)
    want = (sign.view(torch.float8_e4m3fn).double() * 2.0 ** 119).to(torch.bfloat16)
    assert torch.equal(got, want.expand(got.shape))


@pytest.mark.parametrize("d", [64, 128])
def test_weights_of_few_rows_keep_eleven_bits(gs, d):
    """A few keys whose values are one vector and its opposite: what is left of them is the weights' differences.  Weights
    rounded to bf16 are outside the bound, rounded to f16 inside."""
    n, hkv = 96, 4
    kv = [2 + i % 5 for i in range(n)]
    cache, table = f8.make_cache(gs, kv, hkv, d, 16, 240)
    ks = cache.k_scales.view(torch.uint8)
    ks -= 4 * (ks != 255)
    u = f8.bytes_of(f8.quantise(_rand((hkv, 1, d), 241).double())[0]) & 127
    cache.v_pages.view(torch.uint8).copy_((u + 128 * (torch.arange(16, device="cuda") % 2)[:, None].to(torch.uint8)).expand(cache.v_pages.shape))
    cache.v_scales.view(torch.uint8).fill_(127)
    q = _rand((n, hkv, d), 242)
    _check(gs, cache, table, q, True, [1] * n, kv, d ** -0.5, "opposite values")
    want, bound = reference(q, cache, table, [1] * n, kv, d ** -0.5, True)
    for weight, inside in ((torch.bfloat16, False), (torch.float16, True)):
        other, _ = reference(q, cache, table, [1] * n, kv, d ** -0.5, True, weight)
        assert bool(((other - want).abs() <= bound).all()) == inside
