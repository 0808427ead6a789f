"""The serving example against the same blocks in 64 bits: prompts, then decoding steps replayed from a graph."""
import importlib.util
import math
from pathlib import Path

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = Path(__file__).resolve().parent.parent


@pytest.fixture(scope="module")
def ex(built_lib):
    spec = importlib.util.spec_from_file_location("serve_block", ROOT / "examples" / "serve_block.py")
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _reference(weights, heads, kv_heads, rows, lens, ids, steps, cos, sin):
    """rows[i]: all inputs of request i, prompt then steps; the residual stream of every input, in 64 bits."""
    outs = []
    for x, n, a in zip(rows, lens, ids):
        x, h = x.double(), None
        T = x.shape[0]
        for w in weights:
            W = {k: w["W"][k].double() * w["M"][k].bool().repeat_interleave(256, 1) for k in w["W"]}

            def proj(v, k):
                y = v @ W[k].T
                if 0 <= a < w["A"][k].shape[0]:
                    y = y + float(w["scale"][a]) * (v @ w["A"][k][a].double().T @ w["B"][k][a].double().T)
                return y

            def norm(v, g):
                return v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-5) * g.double()
            h = x if h is None else x + h
            y = norm(h, w["norms"][0])
            q, k, v = (proj(y, t).view(T, -1, h.shape[1] // heads) for t in "qkv")
            c, s = cos[:T].double()[:, None], sin[:T].double()[:, None]

            def turn(t):
                p, r = t.chunk(2, -1)
                return torch.cat([p * c - r * s, r * c + p * s], -1)
            q, k = turn(q), turn(k)
            k, v = (t.repeat_interleave(heads // kv_heads, 1) for t in (k, v))
            sc = torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(q.shape[-1])
            sc = sc.masked_fill(~torch.tril(torch.ones(T, T, dtype=torch.bool, device="cuda")), -math.inf)
            x = proj(torch.einsum("hqk,khd->qhd", sc.softmax(-1), v).reshape(T, -1), "o")
            h = x + h
            y = norm(h, w["norms"][1])
            x = proj(torch.nn.functional.silu(proj(y, "gate")) * proj(y, "up"), "down")
        outs.append(x + h)
    return outs


@pytest.mark.parametrize("heads,kv_heads,hidden,inter", [(4, 4, 512, 1024), (8, 2, 1024, 1536)])
def test_prompts_and_decoding(ex, heads, kv_heads, hidden, inter):
    lens, ids, steps, page = [70, 1, 333, 16], [1, -1, 0, 2], 3, 16
    weights = [ex.random_block(hidden, inter, heads, kv_heads, 0.5, 3, 16, seed) for seed in (1, 2)]
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = [torch.randn((n + steps, hidden), generator=g, device="cuda").to(torch.bfloat16) for n in lens]
    per = -(-(max(lens) + steps + 1) // page)
    table = torch.randperm(per * len(lens), generator=g, device="cuda").to(torch.int32).view(len(lens), per)
    blocks = [ex.Block(w, heads, kv_heads, per * len(lens), page) for w in weights]
    outs = ex.run(blocks, [r[:n] for r, n in zip(rows, lens)],
                  torch.stack([torch.stack([r[n + i] for r, n in zip(rows, lens)]) for i in range(steps)]), ids, table, per * page)
    want = _reference(weights, heads, kv_heads, rows, lens, ids, steps, *ex.angles(per * page, hidden // heads))
    got = [torch.cat([o] + [outs[1 + i][j: j + 1] for i in range(steps)]) for j, o in enumerate(outs[0].split(lens))]
    for a, b in zip(got, want):
        # about a dozen roundings to bf16 a block, each 2^-9 of its values in the mean, that add up like noise:
        # sqrt(24) 2^-9 = 1 % of the stream over both blocks; three times that here
        err = torch.linalg.vector_norm(a.double() - b, dim=1) / torch.linalg.vector_norm(b, dim=1)
        assert float(err.max()) < 0.03
