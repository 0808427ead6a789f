"""The operators that serve a pruned Transformer block around its projections, as cases that can be timed and compared.

A case is one pass through one operator of `paper_2609_33977_gb300.groupsparse`:

  norm      h = x + residual, y = h / sqrt(mean(h^2) + eps) * w; in bf16, or in 8 bits (e4m3) with scales;
  adapters  out = base + s_a B_a (A_a x) with the low-rank adapter a of each request, for the layers of one call;
  append    rotary embedding of a chunk's queries and keys, keys and values written into the pages of a cache;
  attend    causal attention of every sequence's new tokens over its pages, grouped heads, any mix of lengths.

Widths, heads and projections are those of the LLaMA-2-7B / 13B and Qwen2.5-7B blocks that the workload module lists
(heads of 128: 32/32, 40/40 and 28/4), and 64-wide heads. Weights are drawn as there (N(0, 0.02^2), activations N(0, 1)).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
E4M3_MAX = 448.0
TINY = 2.0 ** -126

HEADS = {"llama2-7b": (32, 32, 128), "llama2-13b": (40, 40, 128), "qwen2.5-7b": (28, 4, 128), "narrow": (16, 2, 64)}
PROJ = {"llama2-7b": ["4096x4096", "4096x4096 4096x4096 4096x4096", "11008x4096 11008x4096", "4096x11008"],
        "llama2-13b": ["5120x5120", "13824x5120 13824x5120", "5120x13824"],
        "qwen2.5-7b": ["3584x3584 512x3584 512x3584", "18944x3584", "3584x18944"]}


def listed():
    return [
        # one token of one sequence enters a 7B block
        {"name": "norm_t1", "kind": "norm", "T": 1, "n": 4096, "residual": True, "eight_bit": False, "group": 0},
        # a prompt of no round length in a 13B model
        {"name": "norm_t2047", "kind": "norm", "T": 2047, "n": 5120, "residual": True, "eight_bit": False, "group": 0},
        # the last norm of a prompt batch, in 8 bits with a scale per 128 columns, for an 8-bit product behind it
        {"name": "norm_8bit_t777", "kind": "norm", "T": 777, "n": 3584, "residual": True, "eight_bit": True, "group": 128},
        # 16 sequences decode through q, k and v of a 7B block, 12 adapters among them, two sequences without
        {"name": "adapters_qkv_t16", "kind": "adapters", "layers": "4096x4096 4096x4096 4096x4096", "rank": 16, "n_adapters": 32,
         "lens": "1 1 1 1 1 1 1 1 1 1 1 1 1 1 1 1", "ids": "0 5 5 -1 17 3 8 30 8 8 21 2 -1 11 14 9"},
        # prompts of several tenants through a 7B block's down projection
        {"name": "adapters_down_t2048", "kind": "adapters", "layers": "4096x11008", "rank": 32, "n_adapters": 8,
         "lens": "901 1 333 70 513 230", "ids": "3 0 7 -1 1 3"},
        # keys and values of 16 decoding sequences of a 7B model
        {"name": "append_t16", "kind": "append", "heads": "llama2-7b", "page": 16, "q_lens": " ".join(["1"] * 16),
         "kv_lens": "130 1 517 2048 999 1024 16 17 700 64 1500 333 801 90 1999 255"},
        # a long prompt's chunk and short ones beside it
        {"name": "append_t3000", "kind": "append", "heads": "qwen2.5-7b", "page": 64, "q_lens": "2048 1 900 51",
         "kv_lens": "4096 777 900 1000"},
        # one sequence at the start of its answer: latency is all
        {"name": "attend_t1", "kind": "attend", "heads": "qwen2.5-7b", "page": 16, "q_lens": "1", "kv_lens": "129"},
        # 16 sequences decode with a 7B model, one key head a query head
        {"name": "attend_7b_t16", "kind": "attend", "heads": "llama2-7b", "page": 16, "q_lens": " ".join(["1"] * 16),
         "kv_lens": "1301 4000 517 2048 999 1024 2900 317 1700 640 1500 333 3801 90 1999 2555"},
        # three long documents answered token by token, seven query heads a key head
        {"name": "attend_long_t3", "kind": "attend", "heads": "qwen2.5-7b", "page": 64, "q_lens": "1 1 1",
         "kv_lens": "65536 30001 49999"},
        # continuous batching: the next chunk of one prompt, the end of another, decoding sequences, an idle slot
        {"name": "attend_mixed_t681", "kind": "attend", "heads": "qwen2.5-7b", "page": 32, "q_lens": "1 512 1 0 1 163 1 1 1",
         "kv_lens": "3000 8192 1111 0 4097 163 7777 64 2500"},
        # whole prompts of different lengths through a 13B model
        {"name": "attend_13b_prompts", "kind": "attend", "heads": "llama2-13b", "page": 64, "q_lens": "4096 1023 1777 300",
         "kv_lens": "4096 1023 1777 300"},
    ]


def _ints(text):
    return [int(v) for v in str(text).split()]


def _text(values):
    return " ".join(str(v) for v in values)


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _parts(rng, total, n):
    cuts = sorted(rng.randint(0, total) for _ in range(n - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [total])]


def _seconds(case):
    """A rough lower bound of a pass, for keeping drawn cases below the largest listed one."""
    w = work(case)
    return max(w["bytes"] / 6.0e12, w["flops"] / 1.0e15)


def draw(rng):
    """One more case: any operator, lengths over the whole range, odd ones among them."""
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), _seconds(c))
    while True:
        kind = rng.choice(["norm", "adapters", "adapters", "append", "attend", "attend", "attend"])
        case = {"kind": kind}
        if kind == "norm":
            n = rng.choice([3584, 4096, 5120, 11008, _log_int(rng, 64, 13824)])
            case.update(T=_log_int(rng, 1, 4096), n=n, residual=rng.random() < 0.8, eight_bit=rng.random() < 0.4, group=0)
            if case["eight_bit"] and rng.random() < 0.5:
                case["group"] = 128
        elif kind == "adapters":
            case["layers"] = rng.choice(PROJ[rng.choice(sorted(PROJ))])
            if rng.random() < 0.25:   # widths of no model: the input in whole groups, any number of outputs
                case["layers"] = "%dx%d" % (_log_int(rng, 100, 16000), 128 * _log_int(rng, 4, 100))
            case.update(rank=rng.choice([8, 16, 32, 64]), n_adapters=_log_int(rng, 1, 48))
            lens = [1] * _log_int(rng, 1, 64)
            if rng.random() < 0.6:
                lens = _parts(rng, _log_int(rng, 17, 2048), rng.randint(1, 12))
            case.update(lens=_text(lens), ids=_text(rng.randint(-1, case["n_adapters"] - 1) for _ in lens))
        else:
            case.update(heads=rng.choice(sorted(HEADS)), page=rng.choice([16, 32, 64, 128]))
            mode = rng.choice(["decode", "chunk", "mixed", "prompts"])
            n = _log_int(rng, 1, 32) if mode == "decode" else rng.randint(1, 8)
            top = _log_int(rng, 40, 65536 if mode == "decode" else 8192 if mode != "prompts" else 4096)
            past = [max(0, int(top * rng.random() ** 1.5) - 1) for _ in range(n)]
            if mode == "decode":
                new = [1] * n
            elif mode == "chunk":
                new = [_log_int(rng, 2, 1024) for _ in range(n)]
            elif mode == "mixed":
                new = [rng.choice([1, 1, 0, _log_int(rng, 2, 512)]) for _ in range(n)]
            else:
                new, past = [max(1, p) for p in past], [0] * n
            if sum(new) == 0:
                new[0] = 1
            case.update(q_lens=_text(new), kv_lens=_text(p + q if q else 0 for p, q in zip(past, new)))
            if kind == "attend":   # what the plain form holds: a padded score for every pair
                hq = HEADS[case["heads"]][0]
                if n * hq * max(new) * max(p + q for p, q in zip(past, new)) > 2.8e9:
                    continue
                # its copy of the gathered keys
                if n * max(p + q for p, q in zip(past, new)) * hq * HEADS[case["heads"]][2] > 8e9:
                    continue
        if _seconds(case) <= most[kind]:
            return case


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _randn(g, shape, scale=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(torch.bfloat16)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lens):
    at = [0]
    for v in lens:
        at.append(at[-1] + v)
    return at


def _shapes(case):
    return [tuple(map(int, s.split("x"))) for s in case["layers"].split()]


def _inputs(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    if kind == "norm":
        T, n = case["T"], case["n"]
        # the residual stream grows with depth, and a few channels are much larger than the others
        r = _randn(g, (T, n), 3.0) if case["residual"] else None
        if r is not None:
            r[:, torch.randperm(n, generator=g, device="cuda")[: max(1, n // 200)]] *= 20.0
        return {"x": _randn(g, (T, n)), "residual": r,
                "w": (1.0 + 0.1 * torch.randn((n,), generator=g, device="cuda")).to(torch.bfloat16)}
    if kind == "adapters":
        lens, ids, r, n = _ints(case["lens"]), _ints(case["ids"]), case["rank"], case["n_adapters"]
        T = sum(lens)
        xs, layers = {}, []
        for out, inp in _shapes(case):
            if inp not in xs:   # q, k and v (gate and up) read the same activations
                xs[inp] = _randn(g, (T, inp))
            layers.append({"x": xs[inp], "base": _randn(g, (T, out)), "A": _randn(g, (n, r, inp), inp ** -0.5),
                           "B": _randn(g, (n, out, r), 0.02), "out": torch.empty((T, out), dtype=torch.bfloat16, device="cuda")})
        return {"layers": layers, "offsets": _i32(_offsets(lens)), "ids": _i32(ids),
                "scale": 0.5 + torch.rand((n,), generator=g, device="cuda", dtype=torch.float32)}
    hq, hkv, d = HEADS[case["heads"]]
    new, kv, page = _ints(case["q_lens"]), _ints(case["kv_lens"]), case["page"]
    T = sum(new)
    need = [-(-v // page) for v in kv]
    n_pages = sum(need) + 8
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)   # pages come and go: no order
    table = torch.full((len(kv), max(1, max(need))), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, v in enumerate(need):
        table[i, :v] = order[at: at + v]
        at += v
    s = {"k_pages": _randn(g, (n_pages, hkv, page, d)), "v_pages": _randn(g, (n_pages, hkv, page, d)), "table": table,
         "offsets": _i32(_offsets(new)), "kv_lens": _i32(kv), "max_q": max(new), "q": _randn(g, (T, hq, d), 1.5)}
    if kind == "append":
        top = max(kv) + 1
        angle = torch.arange(top, device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
        s.update(k=_randn(g, (T, hkv, d)), v=_randn(g, (T, hkv, d)), cos=angle.cos().float(), sin=angle.sin().float(),
                 q_out=torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda"))
    else:
        s["out"] = torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        # a serving program keeps these: the stacked adapters, the cache, and a step's batch (made once for all layers)
        from paper_2609_33977_gb300 import groupsparse as gs
        s["gs"] = gs
        if case["kind"] == "adapters":
            s["ads"] = [gs.Adapters(l["A"], l["B"], s["scale"]) for l in s["layers"]]
        elif case["kind"] in ("append", "attend"):
            s["cache"] = gs.PagedCache(s["k_pages"], s["v_pages"])
            s["batch"] = gs.Batch(s["offsets"], s["kv_lens"], s["table"], s["max_q"])
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------

def run(s):
    case = s["case"]
    return _KINDS[case["kind"]][1 if own else 0](s, case)


def _norm_own(s, case):
    if case["eight_bit"]:
        y, scales, h = s["gs"].add_rms_norm_fp8(s["x"], s["w"], s["residual"], EPS, case["group"])
        return {"y": y, "scales": scales, "h": h}
    y, h = s["gs"].add_rms_norm(s["x"], s["w"], s["residual"], EPS)
    return {"y": y, "h": h}


def _norm_plain(s, case):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + EPS) * s["w"].float()
    kept = h.to(torch.bfloat16) if s["residual"] is not None else None
    if not case["eight_bit"]:
        return {"y": y.to(torch.bfloat16), "h": kept}
    n = case["n"]
    group = case["group"] or n
    wide = torch.nn.functional.pad(y, (0, -n % group)).reshape(case["T"], -1, group)
    scales = (wide.abs().amax(-1) / E4M3_MAX).clamp(min=TINY)
    q = (wide / scales[..., None]).clamp(-E4M3_MAX, E4M3_MAX).reshape(case["T"], -1)[:, :n]
    return {"y": q.to(torch.float8_e4m3fn), "scales": scales, "h": kept}


def _adapters_own(s, case):
    ls = s["layers"]
    if len(ls) == 1:
        s["gs"].adapters_into(ls[0]["x"], ls[0]["base"], s["ads"][0], s["offsets"], s["ids"], ls[0]["out"])
    else:
        s["gs"].adapters_batched_into([l["x"] for l in ls], [l["base"] for l in ls], s["ads"], s["offsets"], s["ids"],
                                      [l["out"] for l in ls])
    return [l["out"] for l in ls]


def _adapters_plain(s, case):
    T = s["layers"][0]["x"].shape[0]
    token = torch.arange(T, device="cuda")
    seg = (token[:, None] >= s["offsets"][None, 1:]).sum(1)
    mine = s["ids"].long()[seg]                                                    # the adapter of every token
    use = (mine[:, None] == torch.arange(case["n_adapters"], device="cuda")[None]).float() * s["scale"][None]

    def one(l):
        v = torch.einsum("tk,ark->tar", l["x"].float(), l["A"].float()) * use[:, :, None]
        return (l["base"].float() + torch.einsum("tar,aor->to", v, l["B"].float())).to(torch.bfloat16)
    return list(map(one, s["layers"]))


def _append_own(s, case):
    q = s["gs"].cache_append(s["cache"], s["batch"], s["q"], s["k"], s["v"], s["cos"], s["sin"], s["q_out"])
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _places(s):
    """Every token's sequence and position."""
    T = s["q"].shape[0]
    token = torch.arange(T, device="cuda")
    at = s["offsets"].long()
    seq = (token[:, None] >= at[None, 1:]).sum(1)
    return seq, s["kv_lens"].long()[seq] - (at[seq + 1] - at[seq]) + token - at[seq]


def _append_plain(s, case):
    seq, pos = _places(s)
    c, n = s["cos"][pos][:, None], s["sin"][pos][:, None]

    def turn(x):
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * c - b * n, b * c + a * n], -1).to(torch.bfloat16)
    page = s["table"][seq, pos // case["page"]].long()
    s["k_pages"][page, :, pos % case["page"]] = turn(s["k"])
    s["v_pages"][page, :, pos % case["page"]] = s["v"]
    return {"q": turn(s["q"]), "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _attend_own(s, case):
    return s["gs"].paged_attention(s["q"], s["cache"], s["batch"], out=s["out"])


def _attend_plain(s, case):
    hq, hkv, d = HEADS[case["heads"]]
    n, g, top = s["table"].shape[0], hq // hkv, s["max_q"]
    seq, pos = _places(s)
    row = torch.arange(seq.shape[0], device="cuda") - s["offsets"].long()[seq]
    q = torch.zeros((n, top, hq, d), device="cuda")
    q[seq, row] = s["q"].float()
    limit = torch.full((n, top), -1, dtype=torch.int64, device="cuda")   # the last key a row sees
    limit[seq, row] = pos
    pages = s["table"].long().clamp(min=0)
    k = s["k_pages"][pages].permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d).float()
    v = s["v_pages"][pages].permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d).float()
    qg = q.reshape(n, top, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, g * top, d)
    a = torch.matmul(qg, k.transpose(-1, -2)).mul_(d ** -0.5).reshape(n, hkv, g, top, -1)
    seen = torch.arange(k.shape[2], device="cuda")[None, None] <= limit[:, :, None]
    a.masked_fill_(~seen[:, None, None], float("-inf"))
    a.sub_(a.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    total = a.sum(-1, keepdim=True)
    o = torch.matmul(a.reshape(n, hkv, g * top, -1), v).reshape(n, hkv, g, top, d)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return o.permute(0, 3, 1, 2, 4).reshape(n, top, hq, d)[seq, row].to(torch.bfloat16)


_KINDS = {"norm": (_norm_plain, _norm_own), "adapters": (_adapters_plain, _adapters_own),
          "append": (_append_plain, _append_own), "attend": (_attend_plain, _attend_own)}


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "norm":
        T, n = case["T"], case["n"]
        groups = -(-n // case["group"]) if case["group"] else 1
        per = 2.0 + (4.0 if case["residual"] else 0.0) + (1.0 if case["eight_bit"] else 2.0)
        return {"bytes": per * T * n + 2.0 * n + (4.0 * T * groups if case["eight_bit"] else 0.0), "flops": 4.0 * T * n}
    if kind == "adapters":
        lens, ids, r = _ints(case["lens"]), _ints(case["ids"]), case["rank"]
        T, used = sum(lens), len({i for i, n in zip(ids, lens) if i >= 0 and n > 0})
        mine = sum(n for i, n in zip(ids, lens) if i >= 0)
        shapes = _shapes(case)
        return {"bytes": 2.0 * mine * sum({i for _, i in shapes}) +
                sum(4.0 * T * o + 2.0 * used * r * (o + i) for o, i in shapes),
                "flops": sum(2.0 * mine * r * (o + i) for o, i in shapes)}
    hq, hkv, d = HEADS[case["heads"]]
    new, kv = _ints(case["q_lens"]), _ints(case["kv_lens"])
    T = sum(new)
    if kind == "append":   # q, k, v in; q out, k and v into the pages; a row of the table of angles each
        return {"bytes": T * (4.0 * d * (hq + 2 * hkv) + 4.0 * d), "flops": 3.0 * T * d * (hq + hkv)}
    pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(new, kv))
    seen = sum(k for n, k in zip(new, kv) if n)
    return {"bytes": 4.0 * T * hq * d + 4.0 * seen * hkv * d, "flops": 4.0 * pairs * hq * d}


# --------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence
# --------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        T, n = case["T"], case["n"]
        h = s["x"].double() + (s["residual"].double() if case["residual"] else 0.0)
        rms = (torch.linalg.vector_norm(h, dim=1) ** 2 / n + EPS) ** 0.5
        y = h / rms[:, None] * s["w"].double()[None]
        h = h if case["residual"] else None
        if not case["eight_bit"]:
            return {"y": y, "h": h}
        group = case["group"] or n
        scales = torch.stack([y[:, i: i + group].abs().max(1).values for i in range(0, n, group)], 1) / E4M3_MAX
        scales = torch.maximum(scales, torch.full_like(scales, TINY))
        return {"y": y / scales.repeat_interleave(group, 1)[:, :n], "scales": scales, "h": h}
    if kind == "adapters":
        lens, ids = _ints(case["lens"]), _ints(case["ids"])
        outs = []
        for l in s["layers"]:
            y = l["base"].double()
            t = 0
            for n, i in zip(lens, ids):
                if i >= 0 and n:
                    low = l["x"][t: t + n].double() @ l["A"][i].double().T
                    y[t: t + n] += float(s["scale"][i]) * (low @ l["B"][i].double().T)
                t += n
            outs.append(y)
        return outs
    new, kv, page = _ints(case["q_lens"]), _ints(case["kv_lens"]), case["page"]
    hq, hkv, d = HEADS[case["heads"]]
    t = 0
    if kind == "append":
        q, kp, vp = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda"), s["k_pages"].double(), s["v_pages"].double()
        half = d // 2
        for i, (n, m) in enumerate(zip(new, kv)):
            if n == 0:
                continue
            pos = torch.arange(m - n, m, device="cuda")
            z = torch.complex(s["cos"][pos].double(), s["sin"][pos].double())[:, None]   # one turn of each pair of channels
            for x, to in ((s["q"], q), (s["k"], None)):
                w = x[t: t + n].double()
                w = torch.complex(w[..., :half], w[..., half:]) * z
                w = torch.cat([w.real, w.imag], -1)
                if to is not None:
                    to[t: t + n] = w
                else:
                    kp[s["table"][i].long()[pos // page], :, pos % page] = w
            vp[s["table"][i].long()[pos // page], :, pos % page] = s["v"][t: t + n].double()
            t += n
        return {"q": q, "k_pages": kp, "v_pages": vp}
    out = torch.zeros((sum(new), hq, d), dtype=torch.float64, device="cuda")
    for i, (n, m) in enumerate(zip(new, kv)):
        if n == 0:
            continue
        pages = s["table"][i, : -(-m // page)].long()
        last = torch.arange(m - n, m, device="cuda")
        for h in range(hkv):
            k = s["k_pages"][pages, h].reshape(-1, d)[:m].double()
            v = s["v_pages"][pages, h].reshape(-1, d)[:m].double()
            for j in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                a = s["q"][t: t + n, j].double() @ k.T / math.sqrt(d)
                a = torch.where(torch.arange(m, device="cuda")[None] <= last[:, None], a, -math.inf)
                out[t: t + n, j] = torch.softmax(a, 1) @ v
        t += n
    return out
