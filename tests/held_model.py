"""Pages held in 4 bits and attention over them, from their definition in plain torch on the CPU.  Nothing here is shared with the library."""
import math

import torch

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16}


def single(x):
    """A step of 32 bits, taken in 64 and rounded: for one +, -, *, / of 32-bit numbers that is the step itself."""
    return x.float().double()


def quantized(x):
    """x [..][D] of a 16-bit type -> codes (int64), scale and mn (64-bit, [..]); heads with a value that is not finite have scale NaN, codes 0."""
    dtype, y = x.dtype, x.double()
    wild = ~torch.isfinite(y).all(dim=-1)
    y = torch.where(wild[..., None], torch.zeros_like(y), y)
    mn, most = y.amin(dim=-1) + 0.0, y.amax(dim=-1)
    span = single(most - mn)
    step = single(span / 15)
    wild |= ~torch.isfinite(span)
    near = step.to(dtype)
    above = (near.view(torch.int16) + 1).view(dtype)  # the type's next number, of one that is not negative
    scale = torch.where(near.double() < step, above, near).double()
    inv = torch.where(scale == 0, torch.zeros_like(scale), single(1 / scale))
    code = torch.round(single(single(y - mn[..., None]) * inv[..., None])).clamp(max=15)
    code = torch.where(wild[..., None], torch.zeros_like(code), code).long()
    nan = torch.full_like(scale, math.nan)
    return code, torch.where(wild, nan, scale), torch.where(wild, torch.zeros_like(mn), mn)


def stands_for(code, scale, mn):
    return code.double() * scale[..., None] + mn[..., None]


def rounded(x, dtype):
    """What is read back."""
    x = x.float()  # (the definition's fma)
    most = torch.finfo(dtype).max
    return torch.where(x > most, torch.full_like(x, most), x).to(dtype)


def shift_of(element):
    return 4 * (element % 8 // 2) + 16 * (element % 2)


class Words:
    """A page's words: where a token's codes and its pair lie."""

    def __init__(self, H, D, block):
        self.H, self.D, self.block = H, D, block
        self.count = H * block * (D // 8) + H * block

    def word(self, head, slot, w):
        return ((head * (self.block // 4) + slot // 4) * (self.D // 8) + w) * 4 + slot % 4

    def pair(self, head, slot):
        return self.H * self.block * (self.D // 8) + head * self.block + slot

    def put(self, page, slot, x):
        """Writes a token x [H][D] into a page (int64 words of 32 bits, as a tensor)."""
        code, scale, mn = quantized(x)
        bits = lambda v: v.to(x.dtype).view(torch.int16).long() & 0xffff  # noqa: E731
        nan = 0x7e00 if x.dtype == torch.float16 else 0x7fc0
        pair = torch.where(torch.isnan(scale), torch.full_like(bits(scale), nan), bits(scale) | bits(mn) << 16)
        shifts = torch.tensor([shift_of(i) for i in range(8)])
        words = (code.view(self.H, self.D // 8, 8) << shifts).sum(dim=-1)
        for h in range(self.H):
            page[self.pair(h, slot)] = pair[h]
            page[[self.word(h, slot, w) for w in range(self.D // 8)]] = words[h]

    def get(self, pages, dtype):
        """pages [n][words] -> codes [n][block][H][D], scale, mn [n][block][H]."""
        pages = pages.long() & 0xffffffff
        H, D, b, W = self.H, self.D, self.block, self.D // 8
        at = torch.tensor([[[self.word(h, s, w) for w in range(W)] for h in range(H)] for s in range(b)])
        words = pages[:, at.flatten()].view(-1, b, H, W, 1)
        code = (words >> torch.tensor([shift_of(i) for i in range(8)]) & 15).reshape(-1, b, H, D)
        pair = pages[:, torch.tensor([[self.pair(h, s) for h in range(H)] for s in range(b)]).flatten()].view(-1, b, H)
        value = lambda v: (v - (v >= 0x8000).long() * 0x10000).to(torch.int16).view(dtype).double()  # noqa: E731
        return code, value(pair & 0xffff), value(pair >> 16)


def attention(q, keys, values, seen, scale, most=None):
    """One row of a table and one KV head, in 64 bits.  q [n][G][D]; keys and values (codes [tokens][D], scale, mn [tokens]); seen [n][tokens].
    -> out [n][G][D], lse [n][G] and the bounds of their rounding.

    u is half a step of the type, e = 2^-24 of 32-bit sums.  A score is s (q . (c - 8)) + (m + 8 s) sum(q): exact products, sums of D terms in 32 bits,
    and eight roundings more (sum, scale, two of the pair, factor, logarithm of the value's scale, shift, exp2's two steps): e (D + 8) (s |q| . |c - 8| +
    |m + 8 s| sum |q|) + 4 e, and the logarithm lv of the value's scale, which goes into the exponent with the weight, and the shift, that is near the largest of
    both, are rounded at their size: 4 e (|lv| + 10).  Elements of the query below 2^-34 of the largest one of all of the call's (of which `most` is told) lose
    what lies below 2^-38 of that, times codes of up to 8.
    Weights, numerator and denominator: twice that, and e for each of `tokens` terms summed and 24 for joining.
    w s is rounded to fp16 (2^-11), or twice (2^-21), which tells in the value itself; below 2^-14 of the largest w s, or 2^-22 where it is held 2^8 larger, by
    2^-25, or 2^-33, of that, times the value in steps of its scale.  What w s is multiplied with, codes of up to 15 + 8, and z s = m + 8 s, are summed in 32 bits."""
    dtype = q.dtype
    q = q.double()
    (kc, ks, km), (vc, vs, vm) = keys, values
    n, G, D = q.shape
    out, lse = torch.zeros_like(q), torch.full((n, G), -math.inf, dtype=torch.float64)
    off, lse_off = torch.zeros_like(q), torch.zeros_like(lse)
    u, e = torch.finfo(dtype).eps / 2, 2.0 ** -24
    fine, tiny = (2.0 ** -21, 2.0 ** -33) if dtype == torch.float16 else (2.0 ** -11, 2.0 ** -25)
    most = q.abs().amax() if most is None else most
    smallest = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134
    for i in range(n):
        at = seen[i]
        tokens = int(at.sum())
        if tokens == 0:
            off[i] = smallest
            continue
        k, v = stands_for(kc[at], ks[at], km[at]), stands_for(vc[at], vs[at], vm[at])
        s = q[i] @ k.T * scale
        top = s.amax(dim=-1, keepdim=True)
        w = torch.exp(s - top)
        total = w.sum(dim=-1, keepdim=True)
        w = w / total
        out[i], lse[i] = w @ v, (top + torch.log(total))[:, 0]
        a = q[i].abs()
        size = (a @ ((kc[at].double() - 8).abs() * ks[at][:, None]).T + a.sum(dim=-1, keepdim=True) * (km[at] + 8 * ks[at]).abs()).amax(dim=-1) * scale
        lost = D * 2.0 ** -38 * most * 8 * ks[at].amax() * scale
        steps = torch.where(vs[at] > 0, vs[at], vm[at].abs().clamp(min=2.0 ** -60))  # (a head of one value has a scale of its size)
        score = e * ((D + 8) * size + 4 * (11 + torch.log2(steps).abs().amax())) + lost
        share = (2 * score + (tokens + 24) * e)[:, None]
        sv = w * steps
        off[i] = (u * out[i].abs() + (share * (1 + u) + fine) * (w @ v.abs()) + tiny * sv.amax(dim=-1, keepdim=True) * (v.abs() / steps[:, None]).sum(dim=0)
                  + e * (tokens + 24) * (23 * sv.sum(dim=-1, keepdim=True) + (w @ (vm[at] + 8 * vs[at]).abs())[:, None]) + smallest)
        lse_off[i] = score + (tokens + 24) * e + 4 * e * lse[i].abs()
    return out, lse, off, lse_off
