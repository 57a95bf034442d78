"""Plain fp64 forms of the operators on a paged cache, and caches to run them on (torch, any device)."""
import math

import torch

from paper_2605_29707_gb300 import binding as b

TORCH = {b.DOMINO_F32: torch.float32, b.DOMINO_BF16: torch.bfloat16, b.DOMINO_F16: torch.float16}


class Paged:
    """Keys and values of sequences of `kv` places in pages of any order; `fill` stands wherever nobody's place is.

    order: the storage order of (page, token, head), e.g. "pth" or "pht" (by head within the page); pad: elements behind
    every head's; layers: None or a leading dimension."""

    def __init__(self, kv, new, hkv, D, dtype, page, order="pth", pad=0, layers=None, seed=0, fill=float("nan"), std=1.0,
                 spare=2, device="cuda"):
        self.kv, self.new, self.hkv, self.D, self.dtype, self.page, self.layers = kv, new, hkv, D, dtype, page, layers
        self.B, self.device = len(kv), device
        g = torch.Generator(device=device).manual_seed(seed)
        need = [-(-n // page) for n in kv]
        self.pages, width = sum(need) + spare, max(max(need), 1)
        size = {"p": self.pages, "t": page, "h": hkv}
        L = layers or 1
        shape = [L] + [size[c] for c in order] + [D + pad]
        perm = [0] + [1 + order.index(c) for c in "pth"] + [4]
        self.k_store = torch.full(shape, fill, dtype=TORCH[dtype], device=device)
        self.v_store = torch.full(shape, fill, dtype=TORCH[dtype], device=device)
        self.k = self.k_store.permute(perm)[..., :D]  # [layer][page][token][head][D]
        self.v = self.v_store.permute(perm)[..., :D]
        ids = torch.randperm(self.pages, generator=torch.Generator().manual_seed(seed + 1)).tolist()
        self.table = torch.full((self.B, width + 1), -1, dtype=torch.int32)
        for i, n in enumerate(need):
            self.table[i, :n] = torch.tensor(ids[:n], dtype=torch.int32)
            del ids[:n]
        self.table = self.table.to(device)
        for i in range(self.B):
            at, off = self.slots(i, kv[i])
            for x in (self.k, self.v):
                x[:, at, off] = (torch.randn((L, kv[i], hkv, D), generator=g, device=device) * std).to(TORCH[dtype])
        start = [0]
        for n in new:
            start.append(start[-1] + n)
        self.start_host, self.tokens = start, start[-1]
        i32 = dict(dtype=torch.int32, device=device)
        self.kv_len, self.start = torch.tensor(kv, **i32), torch.tensor(start, **i32)
        s = self.k.stride()
        self.cache = b.make_cache(self.k_store, self.v_store, s[1], s[2], s[3], self.pages, page, hkv, D, dtype)
        self.batch = b.make_batch(self.table, self.table.stride(0), width, self.kv_len, self.start, self.B)
        self.layer_stride = s[0]

    def slots(self, i, n):
        t = torch.arange(n, device=self.device)
        return self.table[i, t // self.page].long(), t % self.page

    def read(self, which, i, layer=0):
        at, off = self.slots(i, self.kv[i])
        return which[layer][at, off]


def visible(mask, n, kv, parent=None):
    """[n, kv]: which places the new tokens of one sequence see; parent: its tree's, a list of N."""
    out = torch.zeros((n, kv), dtype=torch.bool)
    first = kv - n
    for i in range(n):
        if mask == b.DOMINO_MASK_FULL:
            out[i] = True
        elif mask == b.DOMINO_MASK_CAUSAL:
            out[i, :max(0, first + i + 1)] = True
        elif i <= len(parent):
            out[i, :max(first, 0)] = True
            a = i
            while a >= 0:
                if first + a >= 0:
                    out[i, first + a] = True
                if a == 0:
                    break
                up = parent[a - 1]
                a = (up if -1 <= up < a - 1 else -1) + 1
    return out


def attend(p, q, scale, mask, parents=None, tensor=True):
    """out, lse and their tolerances, fp64, of q [tokens][hq][D] over the cache p.

    The tolerances: with u the type's half step, A = sum_j w_j |v_j| and e the relative error of a weight,
      out: u A for the weights rounded to the type (tensor: the second product's operands), u |out| for the last
        rounding, e A for the scores;  fp16 weights below 2^-14 of the greatest are subnormal, off by 2^-25 each.
      e = 2 (D + 8) 2^-24 scale max_j sum_d |q_d k_jd| + 2^-20: D fp32 additions, the product by the scale, and the
        exponential's and the sums' own rounding; lse: half of it, and 2^-23 |lse|."""
    tokens, hq, D = q.shape
    G = hq // p.hkv
    out = torch.zeros((tokens, hq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((tokens, hq), -math.inf, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u = torch.finfo(q.dtype).eps / 2
    for i in range(p.B):
        n, kv, a = p.new[i], p.kv[i], p.start_host[i]
        if n == 0:
            continue
        see = visible(mask, n, kv, parents[i] if parents is not None else None).to(q.device)
        k, v = p.read(p.k, i).double(), p.read(p.v, i).double()
        for h in range(hq):
            x, kh, vh = q[a:a + n, h].double(), k[:, h // G], v[:, h // G]
            z = (scale * (x @ kh.T)).masked_fill(~see, -math.inf)
            l = torch.logsumexp(z, 1)
            some = see.any(1)
            w = torch.where(some[:, None], (z - l[:, None]).exp(), 0.0)
            o = w @ vh
            size = (scale * (x.abs() @ kh.abs().T)).masked_fill(~see, 0.0).amax(1) if kv else torch.zeros(n).to(x)
            e = 2 * (D + 8) * 2.0 ** -24 * size + 2.0 ** -20
            A = w @ vh.abs()
            t = u * o.abs() + (e[:, None] + (u if tensor and q.dtype != torch.float32 else 0.0)) * A
            if tensor and q.dtype == torch.float16:  # the weights as kept are at least e^(z - max): off by 2^-25
                top = torch.where(some, z.amax(1) - l, 0.0).exp() if kv else torch.zeros(n).to(x)
                t = t + 2.0 ** -25 * top[:, None] * (see.double() @ vh.abs())
            out[a:a + n, h], lse[a:a + n, h] = o, torch.where(some, l, -math.inf)
            tol[a:a + n, h], ltol[a:a + n, h] = t, e / 2 + 2.0 ** -23 * torch.where(some, l.abs(), 0.0)
    return out, lse, tol, ltol


def rotate(x, pos, freq, rot, layout, amplitude, back=False):
    """y and its tolerance, fp64, for x [tokens][heads][D].

    Tolerance: cos and sin (an angle good to 2^-25, a function good to 2^-23, the amplitude's rounding) are off by at
    most 3 2^-23 of the amplitude, the two products and their sum by 2 2^-24 of what they add: 4 2^-23 amplitude (|x0| + |x1|),
    and half a step of the type."""
    x64 = x.double()
    angle = pos.double()[:, None, None] * freq.double()
    co, si = angle.cos() * amplitude, angle.sin() * amplitude * (-1.0 if back else 1.0)
    y, size = x64.clone(), torch.zeros_like(x64)
    i = torch.arange(rot // 2, device=x.device)
    i0, i1 = (i, i + rot // 2) if layout == b.DOMINO_ROPE_HALF else (2 * i, 2 * i + 1)
    a, c = x64[..., i0], x64[..., i1]
    y[..., i0], y[..., i1] = a * co - c * si, c * co + a * si
    size[..., i0] = size[..., i1] = a.abs() + c.abs()
    return y, 4 * 2.0 ** -23 * abs(amplitude) * size + torch.finfo(x.dtype).eps / 2 * y.abs()


def random_trees(B, N, seed):
    """[B][N] parents, earlier nodes or -1, and depths."""
    g = torch.Generator().manual_seed(seed)
    parent = ((torch.rand(B, N, generator=g) * (torch.arange(N) + 1)).long() - 1).tolist()
    depth = [[0] * N for _ in range(B)]
    for t in range(B):
        for i in range(N):
            depth[t][i] = 1 if parent[t][i] < 0 else depth[t][parent[t][i]] + 1
    return parent, depth
