"""Plain 64-bit statements of the 4-bit rows, the int8 cache and its attention, for the tests: CPU, numpy and torch."""
import numpy as np
import torch

MX4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_quantize(x):
    """bf16 CPU tensor [rows, cols] -> (codes, scales) of padded rows, by the definition: the nearest magnitude, a tie to the
    even code, the scale's exponent that of the largest magnitude less two."""
    rows, cols = x.shape
    v = np.zeros((rows, -(-cols // 128) * 128))
    v[:, :cols] = x.double().numpy()
    v = v.reshape(rows, -1, 32)
    top = np.abs(v).max(axis=-1)
    finite = np.isfinite(v).all(axis=-1)
    _, e = np.frexp(np.where(finite & (top > 0), top, 1.0))
    s = np.where(top > 0, np.maximum(e - 3, -127), -127)
    with np.errstate(invalid="ignore"):
        a = np.ldexp(np.abs(np.where(finite[..., None], v, 0.0)), -s[..., None])
    far = np.abs(a[..., None] - MX4)
    near = far.min(axis=-1, keepdims=True)
    ties = far == near
    even = ties & (np.arange(8) % 2 == 0)
    code = np.where(ties.sum(axis=-1) > 1, even.argmax(axis=-1), ties.argmax(axis=-1))
    code = np.where(a >= 6, 7, code) + 8 * (np.signbit(v) & finite[..., None])
    code = code.reshape(rows, -1)
    scales = np.where(finite, s + 127, 255).astype(np.uint8)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), scales


def mx4_values(codes, scales, cols):
    """float64 [rows, cols] that packed rows stand for; NaN where the scale byte is 255."""
    rows = codes.shape[0]
    code = np.stack((codes & 15, codes >> 4), axis=-1).reshape(rows, -1, 32).astype(np.int64)
    v = np.where(code >= 8, -1.0, 1.0) * MX4[code & 7]
    s = scales.astype(np.int64)
    v = np.where((s == 255)[..., None], np.nan, np.ldexp(v, (s - 127)[..., None]))
    return v.reshape(rows, -1)[:, :cols]


class CacheRef:
    """A cache as tensors of codes and scales by slot: [slots, heads, dim], [slots, heads, dim / block]."""

    def __init__(self, pages, heads, page, dim, block):
        self.pages, self.heads, self.page, self.dim, self.block = pages, heads, page, dim, block
        n = pages * page
        self.codes = [torch.zeros(n, heads, dim, dtype=torch.int8) for _ in "kv"]
        self.scales = [torch.zeros(n, heads, dim // block) for _ in "kv"]

    def write(self, k, v, slots):
        for i, x in enumerate((k, v)):
            w = x.double().reshape(*x.shape[:2], -1, self.block)
            top = w.abs().amax(-1, keepdim=True)
            alive = top >= 127 * 2.0 ** -126
            # every quotient and product of the definition rounded to fp32 where it says so
            inverse = torch.where(alive, 127.0 / torch.where(alive, top, 1.0), 0.0).float().double()
            code = torch.round((w * inverse).float()).clamp(-127, 127)
            scale = torch.where(alive, top / 127.0, 0.0).float()
            finite = torch.isfinite(w).all(-1, keepdim=True)
            code = torch.where(finite, code, torch.zeros_like(code))
            scale = torch.where(finite, scale, torch.full_like(scale, float("nan")))
            for t, slot in enumerate(slots.tolist()):
                if 0 <= slot < self.pages * self.page:
                    self.codes[i][slot] = code[t].reshape(self.heads, self.dim).to(torch.int8)
                    self.scales[i][slot] = scale[t].reshape(self.heads, -1)

    def device(self, where="cuda"):
        from paper_2506_17615_amd import binding as eq
        P, H, S, D = self.pages, self.heads, self.page, self.dim
        kc, vc = (c.view(P, S, H, D) for c in self.codes)
        ks, vs = (s.view(P, S, H, -1).permute(0, 2, 3, 1).contiguous().to(where) for s in self.scales)
        return eq.Cache(kc.permute(0, 2, 1, 3).contiguous().to(where), ks,
                        vc.view(P, S // 16, 16, H, D).permute(0, 3, 1, 4, 2).contiguous().to(where), vs)

    def values(self, i):
        """float64 keys (i = 0) or values by slot."""
        return self.codes[i].double() * self.scales[i].double().repeat_interleave(self.block, dim=-1)

    def slots_of(self, pages, length):
        """Slots of a sequence's tokens, -1 where its page does not exist."""
        t = torch.arange(length)
        p = torch.tensor(pages, dtype=torch.long)[t // self.page] if length else t
        return torch.where((p >= 0) & (p < self.pages), p * self.page + t % self.page, -1)


def attention(ref, q, pages, length, scale, causal, window):
    """One sequence: q [n, q_heads, dim] float64 at the end of `length` tokens.  Returns out, lse and what error bounds need:
    sum of p |v|, and the largest sum of |q k| * |scale| a row has."""
    n, q_heads, dim = q.shape
    group = q_heads // ref.heads
    slots = ref.slots_of(pages, length)
    t = torch.arange(length)
    there = slots >= 0
    K, V = ref.values(0)[slots.clamp(min=0)], ref.values(1)[slots.clamp(min=0)]
    out, mass, lse = torch.zeros(n, q_heads, dim, dtype=torch.float64), torch.zeros(n, q_heads, dim, dtype=torch.float64), \
        torch.full((n, q_heads), -np.inf, dtype=torch.float64)
    size = torch.zeros(n, q_heads, dtype=torch.float64)
    for i in range(n):
        at = length - n + i
        seen = there.clone()
        if causal:
            seen &= t <= at
            if window:
                seen &= t > at - window
        if not seen.any():
            continue
        k, v = K[seen], V[seen]
        for h in range(q_heads):
            s = scale * (k[:, h // group] @ q[i, h])
            lse[i, h] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[i, h])
            out[i, h] = p @ v[:, h // group]
            mass[i, h] = p @ v[:, h // group].abs()
            size[i, h] = abs(scale) * (k[:, h // group].abs() @ q[i, h].abs()).max()
    return out, lse, mass, size
