"""The operators around a block's projections in 64 bits, sequence by sequence, with error bounds.

Bounds: bf16 keeps 8 significant bits (values in [1, 2) are 2^-7 apart), so rounding to it is off by at
most 2^-8 of the value; float32 sums of n terms by at most n 2^-24 of the sum of magnitudes.  BF is 2^-8 with a margin of 2 % for the
rounding's dependence on a value that is itself off.
"""
import math

import torch

BF = 1.02 * 2.0 ** -8


def norm(x, residual, w, eps):
    h = x.double() + (residual.double() if residual is not None else 0.0)
    return h, h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * w.double()


def adapters(x, base, A, B, scale, lens, ids):
    """(out, bound): A x and its product with B in float32 (or nearly: hi + lo bf16 keeps 16 bits)."""
    out, mag = base.double().clone(), torch.zeros(base.shape, dtype=torch.float64, device=base.device)
    t = 0
    for n, i in zip(lens, ids):
        if n and 0 <= i < A.shape[0]:
            s, xd, a, b = float(scale[i]), x[t: t + n].double(), A[i].double(), B[i].double()
            out[t: t + n] += s * (xd @ a.T @ b.T)
            mag[t: t + n] = abs(s) * (xd.abs() @ a.abs().T @ b.abs().T)
        t += n
    return out, BF * out.abs() + mag * ((x.shape[1] + A.shape[1]) * 2.0 ** -24 + 2.0 ** -16) + 1e-30


def turned(x, cos, sin):
    """x [n, heads, D] by the angles' rows [n, D / 2]: (value, bound)."""
    a, b = x.double().chunk(2, -1)
    c, s = cos.double()[:, None], sin.double()[:, None]
    y = torch.cat([a * c - b * s, b * c + a * s], -1)
    mag = torch.cat([(a * c).abs() + (b * s).abs()] * 2, -1) + torch.cat([(b * c).abs() + (a * s).abs()] * 2, -1)
    return y, BF * y.abs() + mag * 2.0 ** -22


def attention(q, k_pages, v_pages, table, new, kv, scale):
    """(out, bound).  Masked keys and memory past a sequence are not touched.  Bound: the output's rounding, the
    weights' rounding to bf16 (2^-8 of sum p |v|), and the scores' float32 error (it scales p)."""
    T, hq, d = q.shape
    hkv, page = k_pages.shape[1], k_pages.shape[2]
    g = hq // hkv
    out = torch.zeros((T, hq, d), dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    t = 0
    for i, (n, m) in enumerate(zip(new, kv)):
        if n == 0:
            continue
        ids = table[i, : max(0, -(-m // page))].long()
        K = k_pages[ids].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :m].double()
        V = v_pages[ids].permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :m].double()
        qs = q[t: t + n].double().permute(1, 0, 2).reshape(hkv, g * n, d)
        s = qs @ K.transpose(1, 2) * scale
        mags = (qs.abs() @ K.abs().transpose(1, 2) * abs(scale)).amax(-1, keepdim=True) if m else None
        pos = (m - n + torch.arange(n, device=q.device)).repeat(g)
        seen = torch.arange(m, device=q.device)[None] <= pos[:, None]
        some = seen.any(-1)
        p = torch.zeros_like(s)
        if m:
            p[:, some] = torch.softmax(s[:, some].masked_fill(~seen[some], -math.inf), -1)
        Vz = V.nan_to_num(0.0, 0.0, 0.0)
        o, a = p @ Vz, p @ Vz.abs()
        err = BF * o.abs() + a * (2.0 ** -8 + 2.0 ** -20) + 1e-7
        if m:
            err = err + a * 2 * mags * (d * 2.0 ** -24 + 2.0 ** -22)
        out[t: t + n] = o.reshape(hq, n, d).permute(1, 0, 2)
        bound[t: t + n] = err.reshape(hq, n, d).permute(1, 0, 2)
        t += n
    return out, bound


def assert_close(got, want, bound, what=""):
    err = (got.double() - want).abs()
    bad = ~(err <= bound)
    if bad.any():
        at = tuple(int(v) for v in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside the bound, first at {at}: "
                             f"{float(got[at])!r} for {float(want[at])!r} +- {float(bound[at])!r}")


def make_cache(gs, kv, hkv, d, page, seed, fill=float("nan"), spare=3, order="random"):
    """Pages in random order; slots that no sequence holds are `fill`; (cache, table on the device)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    need = [-(-max(0, v) // page) for v in kv]
    pages = sum(need) + spare
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    k = torch.full((pages, hkv, page, d), fill, dtype=torch.bfloat16, device="cuda")
    v = k.clone()
    table = torch.full((len(kv), max(1, max(need))), 2 ** 30, dtype=torch.int32, device="cuda")
    at = 0
    for i, m in enumerate(kv):
        table[i, : need[i]] = perm[at: at + need[i]]
        at += need[i]
        for dst in (k, v):
            rows = torch.randn((need[i] * page, hkv, d), generator=g, device="cuda").to(torch.bfloat16)
            rows[max(0, m):] = fill
            if need[i]:
                dst[table[i, : need[i]].long()] = rows.reshape(need[i], page, hkv, d).permute(0, 2, 1, 3)
    return gs.PagedCache(k, v), table


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return i32(at)
