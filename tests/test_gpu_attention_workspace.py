"""Who uses which workspace of the attention: streams, graphs, replays beside one another."""
import gc

import pytest
import torch

from tests import _block_ref as ref

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE = 7, 1, 128, 64


@pytest.fixture(scope="module")
def gs(built_lib):
    from paper_2609_33977_gb300 import groupsparse
    return groupsparse


@pytest.fixture
def used(gs, monkeypatch):
    """The workspace of every attention call."""
    call, seen = gs.lib.gs_paged_attention, []

    def record(*args):
        seen.append(args[7])
        return call(*args)
    monkeypatch.setattr(gs.lib, "gs_paged_attention", record)
    return seen


class Step:
    """Attention of one step, split over CTAs; its inputs and its output stay where they are."""

    def __init__(self, gs, new, kv, seed):
        self.gs, self.new, self.kv = gs, new, kv
        self.cache, self.table = ref.make_cache(gs, kv, HKV, D, PAGE, seed)
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.q = torch.randn((sum(new), HQ, D), generator=g, device="cuda").to(torch.bfloat16)
        self.lens = ref.i32(kv)
        self.batch = gs.Batch(ref.offsets(new), self.lens, self.table, max(new))
        self.out = torch.empty_like(self.q)

    def __call__(self):
        self.gs.paged_attention(self.q, self.cache, self.batch, out=self.out)

    def check(self, what=""):
        want, bound = ref.attention(self.q, self.cache.k_pages, self.cache.v_pages, self.table, self.new, self.lens.tolist(),
                                    D ** -0.5)
        ref.assert_close(self.out, want, bound, what)


def _capture(step, stream, calls=1):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        for _ in range(calls):
            step()
    return g


def _on(stream, step):
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)


def test_graphs_and_eager_calls_of_one_stream_use_different_workspaces(gs, used):
    side = torch.cuda.Stream()
    a, b = Step(gs, [1], [20011], 1), Step(gs, [3], [9000], 2)
    _on(side, a)
    _on(side, b)                                  # the stream has a workspace
    ga, gb = _capture(a, side, calls=2), _capture(b, side)
    _on(side, a)
    e0, e1, a0, a1, b0, e2 = used
    assert e0 == e1 == e2 and a0 == a1            # calls in order share one
    assert len({e0, a0, b0}) == 3
    for step, g in ((a, ga), (b, gb)):
        step.out.zero_()
        g.replay()
        step.check()
    assert gs.device_status() == gs.GS_OK


@pytest.mark.parametrize("new,kv", [([1], [20011]), ([40], [8191]), ([40, 1], [6000, 3000])])
def test_a_capture_on_a_stream_that_ran_nothing(gs, new, kv):
    """Split sequences, new lengths, replays on another stream than the capture's."""
    gs.device_status()
    step = Step(gs, new, kv, 3)
    g = _capture(step, torch.cuda.Stream())
    for back in (0, 5, 1000):
        step.lens.copy_(ref.i32([v - back for v in kv]))
        step.out.zero_()
        g.replay()
        step.check(f"{back} keys fewer")
    assert gs.device_status() == gs.GS_OK


@pytest.mark.parametrize("new,kv", [([1], [20011]), ([300], [5000])])
def test_a_replay_does_not_depend_on_the_counters_it_finds(gs, used, new, kv):
    """A replay that gave up leaves half-counted arrivals in its graph's workspace."""
    step, side = Step(gs, new, kv, 4), torch.cuda.Stream()
    _on(side, step)
    g = _capture(step, side)
    ws, = (w for _, w in gs._captured_ws.values() if w.data_ptr() == used[-1])
    for left in (1, 0, 3):
        ws[: gs.ATTENTION_COUNTER_BYTES].view(torch.int32).fill_(left)
        step.out.zero_()
        g.replay()
        step.check(f"counters at {left}")
    assert gs.device_status() == gs.GS_OK


def test_replays_beside_one_another(gs):
    """Two graphs of one capture stream and eager calls on it, all at the same time."""
    side, others = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    steps = [Step(gs, [1], [20011], 5), Step(gs, [3], [9000], 6), Step(gs, [60], [4001], 7)]
    for s in steps:
        _on(side, s)
    graphs = [_capture(s, side) for s in steps[:2]]
    torch.cuda.synchronize()
    for _ in range(50):
        for s, g in zip(others, graphs):
            with torch.cuda.stream(s):
                g.replay()
        with torch.cuda.stream(side):
            steps[2]()
    torch.cuda.synchronize()
    for s in steps:
        s.check()
    assert gs.device_status() == gs.GS_OK


def test_a_graphs_workspace_goes_with_the_graph(gs, used):
    step = Step(gs, [1], [3000], 8)
    g = _capture(step, torch.cuda.Stream())
    at = used[-1]
    assert gs._graph_owned(gs._captured_ws[max(gs._captured_ws, key=lambda k: gs._captured_ws[k][0])][1])
    assert not gs._graph_owned(step.q)
    held = lambda: any(s["address"] <= at < s["address"] + s["total_size"] for s in torch.cuda.memory_snapshot())  # noqa: E731
    assert held()
    gs.trim()
    g.replay()                                    # the graph's pool keeps it
    step.check()
    torch.cuda.synchronize()
    del g
    gc.collect()
    torch.cuda.empty_cache()
    assert not held()
