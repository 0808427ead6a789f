"""A wait of the attention kernels that runs out: the status says so, and what follows is right.

The test hook makes the copying warp of the first CTA give up on a word that nothing sets; the CTA's other warps then
leave their waits for it, the CTA brings no part of the items that it shares, and arrivals stay half counted.
"""
import pytest
import torch

from tests import _block_ref as ref

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE = 7, 1, 128, 64


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


def _step(gs, new, kv):
    cache, table = ref.make_cache(gs, kv, HKV, D, PAGE, 1)
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn((sum(new), HQ, D), generator=g, device="cuda").to(torch.bfloat16)
    batch, out = gs.Batch(ref.offsets(new), ref.i32(kv), table, max(new)), torch.empty_like(q)
    want, bound = ref.attention(q, cache.k_pages, cache.v_pages, table, new, kv, D ** -0.5)
    return (lambda: gs.paged_attention(q, cache, batch, out=out)), out, lambda what: ref.assert_close(out, want, bound, what)


# the kernel for few rows alone, the one for many alone, each of both; long enough that the first CTA has a part of an
# item (a share of a few units is moved to the item's beginning)
@pytest.mark.parametrize("chunk,new,kv", [(0, [1], [60000]), (1, [40], [60000]), (0, [40, 1], [60000, 50000]),
                                          (1, [40, 1], [60000, 50000])])
def test_timeout_then_recovery(gs, chunk, new, kv):
    step, out, check = _step(gs, new, kv)
    assert gs.device_status() == gs.GS_OK
    step()
    check("before")
    ws = gs._attention_ws[(0, torch.cuda.current_stream().cuda_stream)]
    counters = ws[: gs.ATTENTION_COUNTER_BYTES].view(torch.int32)
    assert not counters.any()
    gs.debug_inject_attention_wait(chunk, 1_000_000)
    step()
    torch.cuda.synchronize()
    assert counters.any()                             # some CTA waits for the one that gave up, in vain
    assert gs.device_status() == gs.GS_ERR_DEVICE_TIMEOUT
    assert gs.device_status() == gs.GS_OK             # reading it cleared it
    for i in range(2):
        out.zero_()
        step()
        check(f"call {i} after the timeout")
    assert gs.device_status() == gs.GS_OK


@pytest.mark.parametrize("chunk,new,kv", [(0, [1], [60000]), (1, [40], [60000])])
def test_timeout_inside_a_graph(gs, chunk, new, kv):
    """A graph whose every replay gives up, and one without the hook whose workspace takes no harm from it."""
    step, out, check = _step(gs, new, kv)
    step()
    side, graphs = torch.cuda.Stream(), []
    for limit in (0, 1_000_000):
        gs.debug_inject_attention_wait(chunk, limit)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
        graphs.append(g)
    whole, broken = graphs
    for i in range(2):
        broken.replay()
        assert gs.device_status() == gs.GS_ERR_DEVICE_TIMEOUT
        out.zero_()
        whole.replay()
        check(f"replay {i} after a timeout")
        out.zero_()
        step()
        check(f"call {i} after a timeout")
    assert gs.device_status() == gs.GS_OK
