"""Windowed attention and the 8-bit cache from their definitions, in 64 bits on the CPU, with how far a result may be off.

A product of 16-bit operands is exact in fp32 and sums are kept there (relative 2^-24 a term; with the logits of these tests,
which stay below 30, P's relative error from all of that is below 2^-10).  What counts are the roundings to 16 bits, half a step each
(`half`): P, dS and what is stored.  Every bound below is the sum of those over the terms they enter, element by element.
"""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -4}
FP32 = {torch.bfloat16: 2.0 ** -10, torch.float16: 2.0 ** -12}  # (logits of the fp16 tests are smaller: below 10)


def visible(nq, nk, left, right, sinks, unit):
    p = torch.arange(nq)[:, None] + (nk - nq)
    j = torch.arange(nk)[None, :]
    up, uj = torch.div(p, unit, rounding_mode="floor"), torch.div(j, unit, rounding_mode="floor")
    see = torch.ones(nq, nk, dtype=torch.bool)
    if right >= 0:
        see &= uj <= up + right
    if left >= 0:
        see &= (uj >= up - left) | (uj < sinks)
    return see


def attention(q, k, v, see, dout=None, scale=None, out_type=None):
    """q [nq,H,d], k, v [nk,Hkv,d] of any type.  Returns {name: (value, bound)} of out, lse and, with dout, dq, dk, dv."""
    t = out_type or q.dtype
    half, fp32 = HALF[t], FP32[t]
    nq, H, d = q.shape
    G = H // k.shape[1]
    scale = scale or d ** -0.5
    q, k, v = q.double().transpose(0, 1), k.double().transpose(0, 1), v.double().transpose(0, 1)
    kg, vg = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    s = (q @ kg.transpose(1, 2) * scale).masked_fill(~see, float("-inf"))
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse.isinf(), torch.zeros_like(lse), lse)[..., None])
    out = p @ vg
    out_off = (half + fp32) * (p @ vg.abs()) + half * out.abs()
    res = {"out": (out.transpose(0, 1), out_off.transpose(0, 1)), "lse": (lse, torch.full_like(lse, 2.0 ** -10))}
    if dout is None:
        return res
    do = dout.double().transpose(0, 1)
    dp = do @ vg.transpose(1, 2)
    delta = (do * out).sum(-1, keepdim=True)
    delta_off = (do.abs() * out_off).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    ds_off = half * ds.abs() + p * delta_off + fp32 * p * (dp.abs() + delta.abs())
    dv = p.transpose(1, 2) @ do
    dv_off = (half + fp32) * (p.transpose(1, 2) @ do.abs())
    dq, dq_off = scale * ds @ kg, scale * ds_off @ kg.abs()
    dk, dk_off = scale * ds.transpose(1, 2) @ q, scale * ds_off.transpose(1, 2) @ q.abs()
    group = lambda x: x.unflatten(0, (-1, G)).sum(1)
    dk, dk_off, dv, dv_off = group(dk), group(dk_off), group(dv), group(dv_off)
    for n, x, o in (("dq", dq, dq_off), ("dk", dk, dk_off), ("dv", dv, dv_off)):
        res[n] = (x.transpose(0, 1), (o + half * x.abs() + 2.0 ** -24).transpose(0, 1))
    return res


def check(got, want, name):
    value, off = want
    got = got.double().cpu()
    assert got.shape == value.shape, (name, got.shape, value.shape)
    same = (got == value) | (got.isnan() & value.isnan())
    bad = ~same & ~((got - value).abs() <= off)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {((got - value).abs() - off)[bad].max():.3e} beyond its bound, first at {bad.nonzero()[0].tolist()}"


def to_e4m3(x):
    """The nearest e4m3 value of |x| <= 448, ties to even (doubles)."""
    _, e = torch.frexp(x)
    step = torch.exp2(((e - 1).clamp(min=-6) - 3).double().round())
    return torch.round(x / step) * step


def page_scale(top):
    """The smallest power of two, at least 2^-60, that brings `top` to 448 or less."""
    s = 2.0 ** -60
    while top > 448 * s:
        s *= 2
    return s


def append(k8, v8, ks, vs, new_k, new_v, pages, start):
    """One sequence: k8 [pages,Hkv,64,d], v8 [pages,Hkv,d,64], ks, vs [pages,Hkv] in doubles, changed in place; new_k, new_v
    [n,Hkv,d].  `pages`: the sequence's page numbers (entries that name nothing: None)."""
    n, done = new_k.shape[0], 0
    while done < n:
        at, slot = (start + done) // 64, (start + done) % 64
        m = min(64 - slot, n - done)
        page = pages[at] if at < len(pages) else None
        for h in range(new_k.shape[1] if page is not None else 0):
            for new, pool, scales in ((new_k, k8[page, h], ks), (new_v, v8[page, h].t(), vs)):
                x = new[done:done + m, h].double()
                x = torch.where(x.isfinite(), x, torch.full_like(x, float("nan")))
                scale = page_scale(float(x.abs().nan_to_num(0.0).max()))
                if slot:
                    was = float(scales[page, h])
                    if was >= scale:
                        scale = was
                    else:
                        pool[:slot] = to_e4m3(pool[:slot] * (was / scale))
                pool[slot:slot + m] = to_e4m3(x / scale)
                scales[page, h] = scale
        done += m


def cached(k8, v8, ks, vs, pages, n):
    """Keys and values [n, Hkv, d] of a sequence, and which of them a page stands for."""
    Hkv, d = k8.shape[1], k8.shape[3]
    k, v, there = torch.zeros(n, Hkv, d, dtype=torch.float64), torch.zeros(n, Hkv, d, dtype=torch.float64), torch.zeros(n, dtype=torch.bool)
    for i in range(0, n, 64):
        page, m = pages[i // 64], min(64, n - i)
        if page is None:
            continue
        k[i:i + m] = (k8[page].double() * ks[page].double()[:, None, None]).transpose(0, 1)[:m]
        v[i:i + m] = (v8[page].double() * vs[page].double()[:, None, None]).permute(2, 0, 1)[:m]
        there[i:i + m] = True
    return k, v, there
