"""Norm, adapters, cache writes and attention over a paged cache against 64-bit references."""
import pytest
import torch

from tests import _block_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def _rand(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


# -------------------------------------------------------------------- norm

@pytest.mark.parametrize("T,n", [(1, 4096), (3, 5120), (2, 1), (5, 7), (4, 8), (7, 264), (2, 8200), (3, 16384), (2, 16392),
                                 (1, 20001), (33, 3584), (2, 129)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_norm(gs, T, n, with_residual):
    x, w = _rand((T, n), 1), _rand((n,), 2)
    r = _rand((T, n), 3, 4.0) if with_residual else None
    y, h = gs.add_rms_norm(x, w, r, 1e-5)
    hr, yr = ref.norm(x, r, w, 1e-5)
    ref.assert_close(y, yr, yr.abs() * (ref.BF + n * 2.0 ** -24) + 1e-30, "y")
    if with_residual:
        ref.assert_close(h, hr, hr.abs() * ref.BF, "h")
    else:
        assert h is None


@pytest.mark.parametrize("T,n,group", [(1, 4096, 0), (3, 4096, 128), (2, 264, 128), (5, 7, 0), (4, 300, 128), (2, 16384, 128),
                                       (2, 16392, 0), (1, 128, 128), (2, 8200, 128)])
def test_norm_8_bits(gs, T, n, group):
    x, r, w = _rand((T, n), 4), _rand((T, n), 5, 3.0), _rand((n,), 6)
    x[-1, : n // 2] = 0
    r[-1, : n // 2] = 0        # groups of zeros
    y8, sc, h = gs.add_rms_norm_fp8(x, w, r, 1e-6, group)
    hr, yr = ref.norm(x, r, w, 1e-6)
    ref.assert_close(h, hr, hr.abs() * ref.BF, "h")
    width = group or n
    assert sc.shape == (T, -(-n // width))
    want = torch.stack([yr[:, i: i + width].abs().amax(1) for i in range(0, n, width)], 1) / 448
    want = want.clamp(min=2.0 ** -126)
    rel = n * 2.0 ** -24 + 2.0 ** -20
    ref.assert_close(sc, want, want * rel, "scales")
    each = want.repeat_interleave(width, 1)[:, :n]
    # e4m3: 4 significant bits (2^-4 of the value at most), steps of 2^-9 at the bottom
    ref.assert_close(y8.float(), yr / each, (yr / each).abs() * (1.02 * 2.0 ** -4 + rel) + 1.02 * 2.0 ** -10, "y8")


@pytest.mark.parametrize("T,n", [(160, 4096), (160, 4104), (153, 8200), (3, 32768), (2, 32776), (200, 1000)])
def test_norm_many_rows_and_long_ones(gs, T, n):
    x, r, w = _rand((T, n), 41), _rand((T, n), 42, 2.0), _rand((n,), 43)
    y, h = gs.add_rms_norm(x, w, r, 1e-5)
    hr, yr = ref.norm(x, r, w, 1e-5)
    ref.assert_close(y, yr, yr.abs() * (ref.BF + n * 2.0 ** -24) + 1e-30, "y")
    ref.assert_close(h, hr, hr.abs() * ref.BF, "h")
    y8, sc, h = gs.add_rms_norm_fp8(x, w, r, 1e-5, 128)
    want = torch.stack([yr[:, i: i + 128].abs().amax(1) for i in range(0, n, 128)], 1) / 448
    rel = n * 2.0 ** -24 + 2.0 ** -20
    ref.assert_close(sc, want, want * rel, "scales")
    at = yr / want.repeat_interleave(128, 1)[:, :n]
    ref.assert_close(y8.float(), at, at.abs() * (1.02 * 2.0 ** -4 + rel) + 1.02 * 2.0 ** -10, "y8")
    ref.assert_close(h, hr, hr.abs() * ref.BF, "h")


def test_norm_in_place_and_nonfinite(gs):
    for n in (512, 515):
        x, r, w = _rand((3, n), 7), _rand((3, n), 8), _rand((n,), 9)
        want_y, want_h = gs.add_rms_norm(x, w, r)
        x2, r2 = x.clone(), r.clone()
        y, h = gs.add_rms_norm(x2, w, r2, h=r2, y=x2)
        assert y is x2 and h is r2 and torch.equal(y, want_y) and torch.equal(h, want_h)
        x[1, 3] = float("inf")
        y, _ = gs.add_rms_norm(x, w, r)
        assert torch.equal(y[0], want_y[0]) and torch.equal(y[2], want_y[2])
        assert y[1, 3].isnan() and (y[1, 4:] == 0).all()
        y8, sc, _ = gs.add_rms_norm_fp8(x, w, r)
        assert y8[1, 3].float().isnan() and y8[0].float().isfinite().all()


def test_norm_both_outputs(gs):
    """One call may write bf16 and 8 bits."""
    x, w = _rand((4, 640), 10), _rand((640,), 11)
    y, y8 = torch.empty_like(x), torch.empty((4, 640), dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.empty((4, 5), device="cuda")
    st = gs.lib.gs_add_rms_norm(x.data_ptr(), None, w.data_ptr(), 4, 640, 1e-5, None, y.data_ptr(), y8.data_ptr(), sc.data_ptr(),
                                128, torch.cuda.current_stream().cuda_stream)
    assert st == gs.GS_OK
    assert torch.equal(y, gs.add_rms_norm(x, w)[0])
    a, b, _ = gs.add_rms_norm_fp8(x, w, group=128)
    assert torch.equal(a.view(torch.uint8), y8.view(torch.uint8)) and torch.equal(b, sc)


# -------------------------------------------------------------------- adapters

def _adapters(gs, n, rank, inp, out, seed):
    A, B = _rand((n, rank, inp), seed, inp ** -0.5), _rand((n, out, rank), seed + 1, 0.1)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    return gs.Adapters(A, B, torch.rand((n,), generator=g, device="cuda") + 0.5), A, B


CASES = [([1], [0]), ([1] * 16, list(range(-2, 14))), ([0, 3, 0, 1, 17], [1, 2, 0, -1, 0]), ([64], [1]), ([65, 1, 130], [0, 5, 2]),
         ([200], [-1]), ([15, 16, 17, 33], [3, 3, 1, 9999]), ([1] * 300, [i % 5 for i in range(300)]), ([700], [2])]


@pytest.mark.parametrize("lens,ids", CASES)
@pytest.mark.parametrize("rank,inp,out", [(8, 256, 128), (16, 1024, 512), (24, 264, 40), (32, 3584, 512), (64, 128, 1000),
                                          (48, 520, 37), (128, 768, 333), (5, 8, 1)])
def test_adapters(gs, lens, ids, rank, inp, out):
    T = sum(lens)
    ad, A, B = _adapters(gs, 6, rank, inp, out, 20)
    x, base = _rand((T, inp), 24), _rand((T, out), 25)
    want, bound = ref.adapters(x, base, A, B, ad.scale, lens, ids)
    y = torch.full((T, out), float("nan"), dtype=torch.bfloat16, device="cuda")
    gs.adapters_into(x, base, ad, ref.offsets(lens), ref.i32(ids), y)
    ref.assert_close(y, want, bound)
    inplace = base.clone()
    gs.adapters_into(x, inplace, ad, ref.offsets(lens), ref.i32(ids), inplace)
    assert torch.equal(inplace, y)


def test_adapters_batched_equals_single(gs):
    lens, ids = [1, 40, 0, 7], [2, 0, 1, -1]
    T, off, i = sum(lens), ref.offsets(lens), ref.i32(ids)
    ads = [_adapters(gs, 3, r, inp, out, 30 + 3 * r)[0] for r, inp, out in ((16, 256, 512), (32, 256, 128), (32, 512, 72))]
    xs, bases = [_rand((T, a.inp), 40) for a in ads], [_rand((T, a.out), 41) for a in ads]
    outs = [torch.empty_like(b) for b in bases]
    gs.adapters_batched_into(xs, bases, ads, off, i, outs)
    for x, b, a, o in zip(xs, bases, ads, outs):
        assert torch.equal(o, gs.adapters_into(x, b, a, off, i, torch.empty_like(b)))


@pytest.mark.parametrize("lens", [[1, 2, 1], [80, 90]])
def test_adapters_nonfinite_stay_with_their_token(gs, lens):
    """NaN in one token's input, in another adapter, or in the padding of ranks reaches no other token."""
    T, ids = sum(lens), list(range(len(lens)))
    ad, A, B = _adapters(gs, 4, 16, 512, 96, 50)
    x, base = _rand((T, 512), 54), _rand((T, 96), 55)
    off, i = ref.offsets(lens), ref.i32(ids)
    want = gs.adapters_into(x, base, ad, off, i, torch.empty_like(base))
    ad.A[3], ad.B[3] = float("nan"), float("inf")      # used by nobody
    x[T - 1, 5] = float("nan")
    got = gs.adapters_into(x, base, ad, off, i, torch.empty_like(base))
    assert torch.equal(got[: T - 1], want[: T - 1]) and got[T - 1].isnan().all()


def test_adapters_huge_product(gs):
    """A x that is infinite stays an infinity of the right sign (it is split in two parts on the way)."""
    A = torch.full((1, 8, 64), 1e19, dtype=torch.bfloat16, device="cuda")
    B = torch.tensor([1.0, -1.0, 2.0, -0.5], device="cuda").to(torch.bfloat16)[None, :, None].repeat(1, 1, 8).contiguous()
    ad = gs.Adapters(A, B, torch.ones((1,), device="cuda"))
    x = torch.full((1, 64), 1e19, dtype=torch.bfloat16, device="cuda")
    y = gs.adapters_into(x, torch.zeros((1, 4), dtype=torch.bfloat16, device="cuda"), ad, ref.offsets([1]), ref.i32([0]),
                         torch.empty((1, 4), dtype=torch.bfloat16, device="cuda"))
    assert y[0].tolist() == [float("inf"), -float("inf"), float("inf"), -float("inf")]


def test_linear_adapted(gs):
    out, inp, lens, ids = 512, 768, [1, 20, 3], [0, -1, 1]
    W, x = _rand((out, inp), 60, 0.02), _rand((sum(lens), inp), 61)
    mask = (torch.rand((out, inp // 256), device="cuda") < 0.5).to(torch.uint8)
    p = gs.pack(W, mask)
    ad, A, B = _adapters(gs, 2, 16, inp, out, 62)
    y = gs.linear_adapted(x, p, ad, ref.offsets(lens), ref.i32(ids))
    base = gs.linear(x, p)
    want, bound = ref.adapters(x, base, A, B, ad.scale, lens, ids)
    ref.assert_close(y, want, bound)


# -------------------------------------------------------------------- cache

def _angles(n, d):
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    return a.cos().float(), a.sin().float()


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 4, 128, 16), (28, 4, 128, 64), (5, 1, 64, 32), (16, 2, 64, 256), (40, 40, 128, 128)])
@pytest.mark.parametrize("new,kv", [([1], [1]), ([1, 1, 1], [17, 1, 300]), ([40, 0, 3, 1], [40, 0, 99, 16]), ([5, 7], [2, 7])])
def test_append(gs, hq, hkv, d, page, new, kv):
    cache, table = ref.make_cache(gs, kv, hkv, d, page, 70)
    k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
    T = sum(new)
    joint = _rand((T, (hq + 2 * hkv) * d + 8), 71)     # slices of a joint projection, rows not contiguous
    q = joint[:, : hq * d].unflatten(1, (hq, d))
    k = joint[:, hq * d: (hq + hkv) * d].unflatten(1, (hkv, d))
    v = joint[:, (hq + hkv) * d: (hq + 2 * hkv) * d].unflatten(1, (hkv, d))
    cos, sin = _angles(max(kv), d)
    out = gs.cache_append(cache, gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new)), q, k, v, cos, sin)
    t = 0
    for i, (n, m) in enumerate(zip(new, kv)):
        for j in range(n):
            pos = m - n + j
            if pos < 0:                                # no such position
                assert torch.equal(out[t], q[t])
            else:
                for x, got in ((q, out), (k, None)):
                    want, bound = ref.turned(x[t: t + 1], cos[pos: pos + 1], sin[pos: pos + 1])
                    p = int(table[i, pos // page])
                    row = got[t] if got is not None else cache.k_pages[p, :, pos % page]
                    ref.assert_close(row, want[0], bound[0])
                assert torch.equal(cache.v_pages[p, :, pos % page], v[t])
                k0[p, :, pos % page], v0[p, :, pos % page] = cache.k_pages[p, :, pos % page], v[t]
            t += 1
    same = lambda a, b: torch.equal(a.view(torch.int16), b.view(torch.int16))  # noqa: E731
    assert same(cache.k_pages, k0) and same(cache.v_pages, v0)   # nothing else was written


def test_append_without_a_place(gs):
    """Pages that do not exist and positions past the angle table or the page table are not followed."""
    cache, table = ref.make_cache(gs, [40, 40, 40], 2, 64, 16, 72)
    k0 = cache.k_pages.clone()
    table[0, 2], table[1, 2] = -1, cache.pages
    q, k, v = _rand((3, 4, 64), 73), _rand((3, 2, 64), 74), _rand((3, 2, 64), 75)
    cos, sin = _angles(40, 64)
    b = gs.Batch(ref.offsets([1, 1, 1]), ref.i32([40, 40, 4000]), table, 1)
    out = gs.cache_append(cache, b, q, k, v, cos, sin)
    assert torch.equal(cache.k_pages.view(torch.int16), k0.view(torch.int16))
    assert torch.equal(out[2], q[2]) and not torch.equal(out[0], q[0])
    inplace = q.clone()
    assert gs.cache_append(cache, b, inplace, k, v, cos, sin, inplace) is inplace and torch.equal(inplace, out)


# -------------------------------------------------------------------- attention

def _attend(gs, new, kv, hq, hkv, d, page, seed=80, fill=float("nan"), qscale=1.5, scale=None, cache=None):
    cache, table = cache or ref.make_cache(gs, kv, hkv, d, page, seed, fill)
    q = _rand((sum(new), hq, d), seed + 1, qscale)
    b = gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new))
    out = gs.paged_attention(q, cache, b, scale)
    want, bound = ref.attention(q, cache.k_pages, cache.v_pages, table, new, kv, d ** -0.5 if scale is None else scale)
    ref.assert_close(out, want, bound, f"new {new} kv {kv} heads {hq}/{hkv} d {d} page {page}")
    assert torch.equal(out, gs.paged_attention(q, cache, b, scale))     # the same bits again (and a clean workspace)
    assert gs.device_status() == gs.GS_OK
    return out, q, cache, table, b


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 128), (7, 1, 128), (28, 4, 128), (16, 2, 64), (64, 1, 128), (3, 3, 64), (20, 1, 64),
                                      (66, 2, 128)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("kv", [[1], [2, 15, 16, 17], [63, 64, 65, 127, 128, 129], [0, 300, 1000, 4], [5000]])
def test_single_tokens(gs, hq, hkv, d, page, kv):
    _attend(gs, [0 if v == 0 else 1 for v in kv], kv, hq, hkv, d, page)


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 4, 128, 16), (28, 4, 128, 32), (7, 1, 128, 128), (16, 2, 64, 256), (6, 6, 64, 16),
                                           (64, 1, 64, 64), (3, 1, 128, 64)])
@pytest.mark.parametrize("new,kv", [([2], [2]), ([3, 1], [400, 17]), ([64], [64]), ([129], [129]), ([300], [777]),
                                    ([1, 200, 0, 33, 5], [900, 200, 0, 1033, 5]), ([37, 1, 260], [1500, 1, 261]),
                                    ([16, 9, 17], [16, 2000, 145])])
def test_chunks(gs, hq, hkv, d, page, new, kv):
    _attend(gs, new, kv, hq, hkv, d, page)


@pytest.mark.parametrize("new,kv", [([5], [3]), ([1], [0]), ([200], [150]), ([300, 4], [10, 0])])
def test_rows_without_keys_are_zero(gs, new, kv):
    out, *_ = _attend(gs, new, kv, 4, 2, 128, 16)
    assert (out[: max(0, new[0] - kv[0])] == 0).all()


@pytest.mark.parametrize("q,kvlen", [(1, 100), (6, 100), (90, 300), (300, 300), (257, 2000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_masked_values_do_not_reach_earlier_rows(gs, q, kvlen, bad):
    """A later token's key and value, whatever they are, leave the rows before it as they were."""
    kv, page = [kvlen], 16
    cache, table = ref.make_cache(gs, kv, 2, 128, page, 90)
    x = _rand((q, 4, 128), 91)
    b = gs.Batch(ref.offsets([q]), ref.i32(kv), table, q)
    clean = gs.paged_attention(x, cache, b)
    for back in {0, q // 2, min(q - 1, 70)}:
        pos = kvlen - 1 - back
        k2, v2 = cache.k_pages.clone(), cache.v_pages.clone()
        p = int(table[0, pos // page])
        v2[p, :, pos % page, 3] = bad
        out = gs.paged_attention(x, gs.PagedCache(k2, v2), b)
        row = q - 1 - back
        assert torch.equal(out[:row], clean[:row])
        assert (~out[row:, :, 3].isfinite()).all()
        assert torch.equal(out[row:, :, 4:], clean[row:, :, 4:])
        k2[p, :, pos % page] = bad
        v2 = cache.v_pages.clone()
        out = gs.paged_attention(x, gs.PagedCache(k2, v2), b)
        assert torch.equal(out[:row], clean[:row])
        if bad != bad:
            assert out[row:].isnan().all()


def test_missing_pages_read_as_zeros(gs):
    for new, kv in (([1], [100]), ([70], [100]), ([200], [200])):
        cache, table = ref.make_cache(gs, kv, 2, 64, 16, 92, fill=0.0)
        full = gs.PagedCache(torch.cat([cache.k_pages, torch.zeros_like(cache.k_pages[:1])]),
                             torch.cat([cache.v_pages, torch.zeros_like(cache.v_pages[:1])]))
        x = _rand((new[0], 4, 64), 93)
        t2 = table.clone()
        t2[0, 1] = cache.pages                       # the page of zeros
        want = gs.paged_attention(x, full, gs.Batch(ref.offsets(new), ref.i32(kv), t2, new[0]))
        for bad in (-1, cache.pages, 2 ** 31 - 1, -2 ** 31):
            t2[0, 1] = bad
            got = gs.paged_attention(x, cache, gs.Batch(ref.offsets(new), ref.i32(kv), t2, new[0]))
            assert torch.equal(got, want)


def test_lengths_past_the_table_are_cut(gs):
    cache, table = ref.make_cache(gs, [64], 2, 64, 16, 94)
    x = _rand((1, 2, 64), 95)
    want = gs.paged_attention(x, cache, gs.Batch(ref.offsets([1]), ref.i32([64]), table, 1))
    got = gs.paged_attention(x, cache, gs.Batch(ref.offsets([1]), ref.i32([2 ** 30]), table, 1))
    assert torch.equal(got, want)


def test_strided_queries_scales_and_large_scores(gs):
    new, kv = [3, 90], [50, 400]
    cache, table = ref.make_cache(gs, kv, 2, 128, 32, 96)
    joint = _rand((93, 10 * 128 + 24), 97, 1.0)
    q = joint[:, 8: 8 + 6 * 128].unflatten(1, (6, 128))
    b = gs.Batch(ref.offsets(new), ref.i32(kv), table, 90)
    assert torch.equal(gs.paged_attention(q, cache, b), gs.paged_attention(q.contiguous(), cache, b))
    for scale, qscale in ((0.0, 1.0), (-0.1, 1.0), (1.0, 10.0), (0.088, 1e-3)):
        _attend(gs, new, kv, 6, 2, 128, 32, 98, qscale=qscale, scale=scale)


@pytest.mark.parametrize("hq,hkv,d,page", [(7, 1, 128, 64), (2, 2, 64, 16)])
@pytest.mark.parametrize("new,kv", [([1], [20011]), ([4], [9000]), ([9, 2], [16000, 3]), ([40], [8191]), ([300], [5000])])
def test_one_sequence_in_many_parts(gs, hq, hkv, d, page, new, kv):
    _attend(gs, new, kv, hq, hkv, d, page, seed=120)


@pytest.mark.parametrize("new,kv", [([3], [70]), ([90], [400]), ([200, 2], [4000, 9])])
def test_output_off_a_sector(gs, new, kv):
    cache, table = ref.make_cache(gs, kv, 2, 128, 32, 130)
    q = _rand((sum(new), 4, 128), 131)
    b = gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new))
    room = torch.full((q.numel() + 16,), 7.0, device="cuda", dtype=torch.bfloat16)
    out = room[8: 8 + q.numel()].view(q.shape)        # 16 bytes past a 32-byte boundary
    assert torch.equal(gs.paged_attention(q, cache, b, out=out), gs.paged_attention(q, cache, b))
    assert (room[:8] == 7).all() and (room[-8:] == 7).all()


def test_tokens_of_no_sequence_and_more_tokens_than_told(gs):
    cache, table = ref.make_cache(gs, [40], 1, 64, 16, 99)
    q = _rand((5, 2, 64), 100)
    b = gs.Batch(ref.i32([0, 3]), ref.i32([40]), table, 3)
    out = gs.paged_attention(q, cache, b)
    want, bound = ref.attention(q[:3], cache.k_pages, cache.v_pages, table, [3], [40], 64 ** -0.5)
    ref.assert_close(out[:3], want, bound)
    assert (out[3:] == 0).all()


def test_many_sequences(gs):
    kv = [(37 * i) % 211 + 1 for i in range(700)]
    _attend(gs, [1] * 700, kv, 4, 2, 64, 16)
    new = [(i * i) % 5 for i in range(300)]
    _attend(gs, new, [n + (13 * i) % 90 for i, n in enumerate(new)], 4, 1, 64, 32)


def test_many_chunks(gs):
    """More sequences than threads of a block, each of more rows than the few-row kernel's."""
    new = [17 + i % 9 for i in range(600)]
    _attend(gs, new, [n + (29 * i) % 170 for i, n in enumerate(new)], 4, 1, 64, 32)


@pytest.mark.parametrize("told", [1, 4, 5, 8, 16])
def test_more_new_tokens_than_told(gs, told):
    """A sequence of more new tokens than max_new is right or zero, and its neighbours are right."""
    new, kv = [1, 20, 3, 9, 1], [30, 50, 70, 9, 200]
    cache, table = ref.make_cache(gs, kv, 1, 128, 16, 130)
    q = _rand((sum(new), 4, 128), 131)
    out = gs.paged_attention(q, cache, gs.Batch(ref.offsets(new), ref.i32(kv), table, told))
    want, bound = ref.attention(q, cache.k_pages, cache.v_pages, table, new, kv, 128 ** -0.5)
    t = 0
    for n in new:
        rows = slice(t, t + n)
        if n <= told or (out[rows] != 0).any():
            ref.assert_close(out[rows], want[rows], bound[rows], f"{n} tokens, told {told}")
        t += n


def test_streams_and_graphs(gs):
    """A captured step follows new lengths, pages and tokens in the tensors it was captured with."""
    kv, hq, hkv, d, page = [100, 33, 260], 8, 2, 128, 16
    cache, table = ref.make_cache(gs, kv, hkv, d, page, 101)
    wide = torch.zeros((3, 40), dtype=torch.int32, device="cuda")
    wide[:, : table.shape[1]] = table
    lens = ref.i32([v - 7 for v in kv])
    b = gs.Batch(ref.offsets([1, 1, 1]), lens, wide, 1)
    q, k, v = _rand((3, hq, d), 102), _rand((3, hkv, d), 103), _rand((3, hkv, d), 104)
    cos, sin = _angles(512, d)
    qr, out = torch.empty_like(q), torch.empty_like(q)

    def step():
        gs.cache_append(cache, b, q, k, v, cos, sin, qr)
        gs.paged_attention(qr, cache, b, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        step()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step()
    for n in range(7):
        lens += 1
        q.copy_(_rand(q.shape, 110 + n))
        g.replay()
        want, bound = ref.attention(qr, cache.k_pages, cache.v_pages, wide, [1, 1, 1], lens.tolist(), d ** -0.5)
        ref.assert_close(out, want, bound, f"replay {n}")
    # an explicit stream: its own workspace, the same bits
    torch.cuda.synchronize()
    got = gs.paged_attention(qr, cache, b, stream=side)
    side.synchronize()
    assert torch.equal(got, out)


def test_offsets_past_32_bits(gs):
    """Pages whose elements lie more than 2^32 bytes, and 2^31 elements, into the cache."""
    hkv, d, page = 8, 128, 256
    pages = (2 ** 31) // (hkv * d * page) + 8
    k = torch.zeros((pages, hkv, page, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    ids = [pages - 1, 0, pages - 3]
    for i in ids:
        k[i], v[i] = _rand((hkv, page, d), 120 + i), _rand((hkv, page, d), 220 + i)
    cache, table = gs.PagedCache(k, v), ref.i32([ids])
    for n in (1, 100):
        _attend(gs, [n], [700], 8, hkv, d, page, 121, cache=(cache, table))
    kk, vv = _rand((2, hkv, d), 122), _rand((2, hkv, d), 123)
    cos, sin = _angles(800, d)
    gs.cache_append(cache, gs.Batch(ref.offsets([2]), ref.i32([700]), table, 2), kk, kk, vv, cos, sin)
    assert torch.equal(v[pages - 3, :, 699 - 512], vv[1])
