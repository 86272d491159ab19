"""What several query rows together are compared with: attention of a sequence's last tokens, and norms with rotary positions, in
64 bits from the definitions."""
import numpy as np
import torch

import kv_model as km


def held(cache, layer, s, begin, end):
    """Keys and values of tokens begin .. end of sequence s, in 64 bits."""
    page = cache.k.shape[2]
    table = cache.table[s].tolist()
    at = torch.tensor([[table[t // page] for t in range(begin, end)], [t % page for t in range(begin, end)]], device=cache.k.device)
    k, v = (x[layer].contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16)[at[0], at[1]].view(x.dtype).double()
            for x in (cache.k, cache.v))
    if cache.k_scale is not None:
        k, v = k * cache.k_scale[layer].double()[:, None], v * cache.v_scale[layer].double()[:, None]
    return k, v


def prompt(cache, layer, q, offsets, scale, seq=None, window=0):
    """(out, lse, spread, reach) of the rows that belong to a sequence (NaN elsewhere), as kv_model.attend."""
    q = q.double()
    rows, hq, dim = q.shape
    length, o = cache.length.tolist(), offsets.tolist()
    out, spread = torch.full_like(q, torch.nan), torch.full_like(q, torch.nan)
    lse, reach = torch.full((rows, hq), torch.nan, dtype=torch.float64, device=q.device), torch.zeros((rows, hq), dtype=torch.float64, device=q.device)
    group = hq // cache.heads
    for i, s in enumerate(range(len(o) - 1) if seq is None else seq.tolist()):
        a, b = o[i], o[i + 1]
        if a == b:
            continue
        first = length[s] - (b - a)
        begin = max(0, first + 1 - window) if window else 0
        k, v = held(cache, layer, s, begin, length[s])
        place, at = torch.arange(first, length[s], device=q.device)[:, None], torch.arange(begin, length[s], device=q.device)
        hidden = (at > place) | ((at <= place - window) if window else torch.zeros_like(at > place))
        for h in range(cache.heads):
            for m in range(h * group, (h + 1) * group):
                # (what a row does not see is taken out, whatever it is: infinities and NaN too)
                kh, vh = k[:, h], v[:, h]
                x = (scale * (q[a:b, m] @ kh.T)).masked_fill(hidden, -torch.inf)
                p = torch.softmax(x, 1)
                lse[a:b, m] = torch.logsumexp(x, 1)
                fine = torch.isfinite(vh).all(1)
                out[a:b, m], spread[a:b, m] = p[:, fine] @ vh[fine], p[:, fine] @ vh[fine].abs()
                for t in torch.nonzero(~fine)[:, 0].tolist():
                    sees = ~hidden[:, t]
                    out[a:b, m][sees] += p[sees, t, None] * vh[t]
                reach[a:b, m] = abs(scale) * (q[a:b, m].abs() @ kh.abs().T).masked_fill(hidden, 0).amax(1)
    return out, lse, spread, reach


def check(cache, layer, q, offsets, scale, got, seq=None, window=0):
    out, lse = got
    want, want_lse, spread, reach = prompt(cache, layer, q, offsets, scale, seq, window)
    kind = {torch.bfloat16: "bf16", torch.float16: "f16", torch.float8_e4m3fn: "e4m3"}[cache.k.dtype]
    off, off_lse = km.bounds(spread, reach, cache.dim, kind, "f16" if q.dtype == torch.float16 else "bf16")
    some = ~torch.isnan(want_lse)
    d, e = (out.double() - want)[some].abs(), off[some]
    assert bool((d <= e).all()), float((d / e).max())
    d, e = (lse.double() - want_lse)[some].abs(), off_lse[some]
    assert bool((d <= e).all()), float((d / e).max())


def rotated(x, pos, radians, amplitude, interleaved, weight=None, eps=1e-6):
    """(result, reach) in 64 bits: norm and rotation of rows x [tokens, heads, dim]; reach = sum of the magnitudes that a value is
    made of."""
    x = x.double().clone()
    if weight is not None:
        x = x * weight.double() / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    angle = pos.double()[:, None] * torch.from_numpy(np.ascontiguousarray(radians)).to(x.device)
    cos, sin = (amplitude * f(angle)[:, None] for f in (torch.cos, torch.sin))
    r = 2 * len(radians)
    first, second = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., first].clone(), x[..., second].clone()
    reach = x.abs()
    x[..., first], x[..., second] = a * cos - b * sin, a * sin + b * cos
    reach[..., first] = reach[..., second] = amplitude * (a.abs() + b.abs())
    return x, reach
