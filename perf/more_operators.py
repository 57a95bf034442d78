"""Operators on a target's paged cache of keys and values, as cases that can be timed and checked.

What a speculative-decoding user runs in every layer of the target (and of the draft's backbone) between a draft and
its verification:
- rotary positions of new tokens, their keys and values written into a paged cache (`domino_rope_append`), and the
  rotation alone with its gradient (`domino_rope`);
- attention of the new tokens over that cache: a single token, a chunk of a prompt, a draft block that sees all of
  itself, a drafted tree whose nodes see their ancestors (`domino_attend_paged`);
- after verification, the accepted nodes' keys and values moved to where the next step reads them, in all layers
  (`domino_cache_commit`).

Sizes: trees of 8 to 64 nodes and blocks of 16 draft positions, 1 to 64 sequences (the repository's
configurations), 32 query heads on 8 heads of keys with 128 elements and odd counts beside them, pages of 16 to 256
tokens in any order, contexts from some tokens to 32768.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------------------------- cases
def _attend(name, mask, B, new, kv, heads, D, dtype, page, ragged=True, by_head=False):
    """`new` tokens a sequence (at most, where chunks are ragged), `kv` keys at most; heads: of queries, of keys."""
    return dict(name=name, kind="attend", mask=mask, B=B, new=new, kv=kv, hq=heads[0], hkv=heads[1], D=D, dtype=dtype,
                page=page, ragged=ragged, by_head=by_head)


def _append(name, B, new, kv, heads, D, rot, dtype, page, layout, tree=False, factor=1.0, pad=0):
    return dict(name=name, kind="append", B=B, new=new, kv=kv, hq=heads[0], hkv=heads[1], D=D, rot=rot, dtype=dtype,
                page=page, layout=layout, tree=tree, factor=factor, pad=pad, ragged=False, by_head=False)


def _rope(name, tokens, heads, D, rot, dtype, layout, gradient, far, factor=1.0, pad=0):
    return dict(name=name, kind="rope", tokens=tokens, heads=heads, D=D, rot=rot, dtype=dtype, layout=layout,
                gradient=gradient, far=far, factor=factor, pad=pad)


def _commit(name, layers, B, N, kv, hkv, D, dtype, page, by_head=False):
    return dict(name=name, kind="commit", layers=layers, B=B, new=N + 1, kv=kv, hkv=hkv, D=D, dtype=dtype, page=page,
                ragged=True, by_head=by_head)


def listed():
    return [
        # one interactive user's next token after a short prompt: the smallest call, latency alone
        _attend("attend-b1-token", "causal", 1, 1, 1000, (16, 8), 128, "bf16", 16),
        # a serving batch that decodes a token each, contexts of very different lengths
        _attend("attend-b64-tokens", "causal", 64, 1, 8192, (32, 8), 128, "bf16", 64),
        # the draft backbone: one user's block of 16 positions; they see a long document's features and all of themselves
        _attend("attend-b1-block-long", "full", 1, 16, 30011, (32, 8), 128, "bf16", 16),
        # verification of a full batch's trees of 32 nodes, cache by head within the page
        _attend("attend-b64-tree-f16", "tree", 64, 33, 4096, (64, 8), 128, "f16", 32, by_head=True),
        # chunks of several users' prompts, odd heads and odd lengths
        _attend("attend-b7-chunks-odd", "causal", 7, 701, 5000, (14, 2), 80, "f16", 48),
        # the largest: a chunk of 4096 tokens at the end of a prompt of 32768
        _attend("attend-b1-chunk-long", "causal", 1, 4096, 32768, (32, 8), 128, "bf16", 64, ragged=False),
        # one tree's new tokens, positions by depth: latency alone
        _append("append-b1-tree", 1, 17, 2017, (32, 8), 128, 128, "bf16", 16, "half", tree=True),
        # a chunk of prompts, part of each head rotated in pairs, context stretched four times, padded rows
        _append("append-b3-chunk-f16", 3, 4001, 20000, (32, 8), 128, 64, "f16", 64, "pairs", factor=4.0, pad=64),
        # training: the gradient of rotated queries at far positions
        _rope("rope-gradient-m16384", 16384, 32, 128, 128, "bf16", "half", True, 1 << 20),
        # the rotation alone: fp32, odd counts, half of each head in pairs, stretched positions, padded rows
        _rope("rope-m3001-odd-f32", 3001, 14, 80, 40, "f32", "pairs", False, 1 << 17, 4.0, 24),
        # one user's accepted nodes in 28 layers: latency alone
        _commit("commit-b1", 28, 1, 16, 400, 8, 128, "bf16", 16),
        # a full batch's accepted nodes in 64 layers
        _commit("commit-b64-l64", 64, 64, 32, 120, 8, 128, "bf16", 32, by_head=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("token", "tree", "block", "chunk", "append", "rope", "commit"))
    dtype, page = rng.choice(("bf16", "f16")), rng.choice((16, 32, 48, 64, 128, 256))
    hkv, G, by_head = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 2, 3, 4, 5, 7, 8, 16)), rng.random() < 0.5
    D = rng.choice((64, 80, 96, 128))
    rot = rng.choice((D, D, D // 2))
    layout, factor = rng.choice(("half", "pairs")), rng.choice((1.0, 1.0, 4.0))
    pad = rng.choice((0, 0, 8 * rng.randint(1, 32)))
    heads = (hkv * G, hkv)
    if kind == "token":
        B = _log_int(rng, 1, 128)
        c = _attend("", "causal", B, 1, _log_int(rng, 2, min(32768, 400000 // B)), heads, D, dtype, page, True, by_head)
    elif kind == "tree":
        B, N = _log_int(rng, 1, 64), rng.randint(8, 64)
        c = _attend("", "tree", B, N + 1, N + 1 + _log_int(rng, 1, min(32768, 200000 // B)), heads, D, dtype, page, True,
                    by_head)
    elif kind == "block":
        B, K = _log_int(rng, 1, 64), rng.randint(4, 32)
        c = _attend("", "full", B, K, K + _log_int(rng, 1, min(32768, 200000 // B)), heads, D, dtype, page, True, by_head)
    elif kind == "chunk":
        B, new = _log_int(rng, 1, 8), _log_int(rng, 2, 2048)
        room = max(1, min(32768, (1 << 32) // (B * new * heads[0]) - new))
        c = _attend("", "causal", B, new, new + _log_int(rng, 1, room), heads, D, dtype, page, rng.random() < 0.7, by_head)
    elif kind == "append":
        B, tree = _log_int(rng, 1, 64), rng.random() < 0.5
        new = rng.randint(9, 65) if tree else _log_int(rng, 1, 16384 // B)
        c = _append("", B, new, new + _log_int(rng, 1, 65536 // B), heads, D, rot, dtype, page, layout, tree, factor, pad)
    elif kind == "rope":
        c = _rope("", _log_int(rng, 1, 16384), rng.randint(1, 32), D, rot, rng.choice(tuple(TYPES)), layout,
                  rng.random() < 0.5, _log_int(rng, 64, 1 << 20), factor, pad)
    else:
        N, B = rng.randint(8, 64), _log_int(rng, 1, 64)
        c = _commit("", rng.randint(1, 64), B, N, N + 1 + _log_int(rng, 1, 200), hkv, D, dtype, page, by_head)
    del c["name"]
    return c


def _lengths(c):
    """(keys, new tokens) of every sequence: lists, a case's own whatever the seed."""
    rng = random.Random(c["B"] * 1000003 + c["kv"] * 131 + c["new"])
    kv, new = [], []
    for b in range(c["B"]):
        n = c["new"]
        if c["kind"] == "attend" and c["mask"] == "causal" and c["ragged"] and b:  # the first sequence is the longest
            n = rng.randint(1, n)
        long = c["kv"] if b == 0 or not c["ragged"] else rng.randint(n, max(n, c["kv"]))
        kv.append(long)
        new.append(n)
    return kv, new


def _accepted(c):
    """(accepted nodes, how many of them, from the first on, lie where they belong already) of every sequence."""
    rng = random.Random(c["B"] * 7919 + c["kv"] * 31 + c["new"])
    n = [rng.randint(0 if b else 1, min(8, (c["new"] - 1) // 2)) for b in range(c["B"])]
    return n, [rng.randint(0, max(0, k - 1)) for k in n]


# ------------------------------------------------------------------------------------ inputs
def _gen(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + n)
    return g


def _randn(shape, dtype, g, std=1.0):
    out = torch.empty(shape, dtype=TYPES[dtype], device="cuda")
    flat, step = out.view(-1), 1 << 27
    for a in range(0, flat.numel(), step):  # in pieces: the fp32 draws of a whole cache would be large
        n = min(step, flat.numel() - a)
        flat[a:a + n] = torch.randn(n, generator=g, device="cuda").mul_(std)
    return out


def _cache(s, c, seed, layers=None):
    """Keys and values in pages that lie in any order, what earlier users left in the free ones, and the batch."""
    kv, new = _lengths(c)
    need = [-(-n // c["page"]) for n in kv]
    pages, wide = sum(need) + 3, max(need)
    shape = (pages, c["hkv"], c["page"], c["D"]) if c["by_head"] else (pages, c["page"], c["hkv"], c["D"])
    shape = shape if layers is None else (layers,) + shape
    g = _gen(seed, 1)
    s["k"], s["v"] = _randn(shape, c["dtype"], g), _randn(shape, c["dtype"], g)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(int(seed) * 64 + 2)).tolist()
    table = torch.zeros((c["B"], wide), dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor(order[:n])
        del order[:n]
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    s.update(kv_host=kv, new_host=new, start_host=start, tokens=start[-1], table=table.cuda(),
             kv_len=torch.tensor(kv, dtype=torch.int32, device="cuda"),
             start=torch.tensor(start, dtype=torch.int32, device="cuda"))


def _trees(B, N, seed):
    """Random trees, parents before children: parent [B, N] (-1: the anchor) and depth [B, N], on the host."""
    g = torch.Generator().manual_seed(int(seed) * 64 + 3)
    parent = (torch.rand(B, N, generator=g) * (torch.arange(N) + 1)).long() - 1
    depth = torch.ones(B, N, dtype=torch.long)
    for i in range(N):
        up = parent[:, i]
        depth[:, i] = torch.where(up < 0, 1, depth.gather(1, up.clamp(min=0)[:, None])[:, 0] + 1)
    return parent.int(), depth.int()


def _frequencies(c):
    """Turning speeds of the rotated pairs (radians a position), stretched `factor` times, and the amplitude."""
    half = c["rot"] // 2
    f = torch.tensor([1e6 ** (-i / half) / c["factor"] for i in range(half)], dtype=torch.float64)
    return f.float().cuda(), 0.1 * math.log(c["factor"]) + 1.0


def prepare(case, seed):
    c, s = dict(case), {}
    s["case"] = c
    g = _gen(seed, 4)
    if c["kind"] == "attend":
        _cache(s, c, seed)
        s["q"] = _randn((s["tokens"], c["hq"], c["D"]), c["dtype"], g, 2.0)  # scores of deviation 2: some keys matter
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["tokens"], c["hq"]), device="cuda")
        if c["mask"] == "tree":
            s["parent"] = _trees(c["B"], c["new"] - 1, seed)[0].cuda()
    elif c["kind"] == "append":
        _cache(s, c, seed)
        wide = (c["hq"] + 2 * c["hkv"]) * c["D"]
        s["qkv"] = _randn((s["tokens"], wide + c["pad"]), c["dtype"], g)  # one projection's output
        s["q_out"] = torch.empty((s["tokens"], c["hq"], c["D"]), dtype=TYPES[c["dtype"]], device="cuda")
        s["freq"], s["amplitude"] = _frequencies(c)
        s["depth"] = _trees(c["B"], c["new"] - 1, seed)[1].cuda() if c["tree"] else None
    elif c["kind"] == "rope":
        wide = c["heads"] * c["D"] + c["pad"]
        x = _randn((c["tokens"], wide), c["dtype"], g)
        s["x"] = x[:, :c["heads"] * c["D"]].unflatten(1, (c["heads"], c["D"]))
        s["y"] = torch.empty((c["tokens"], c["heads"], c["D"]), dtype=TYPES[c["dtype"]], device="cuda")
        s["pos"] = torch.randint(0, c["far"], (c["tokens"],), generator=g, device="cuda").int()
        s["freq"], s["amplitude"] = _frequencies(c)
    else:
        _cache(s, c, seed, c["layers"])
        N = c["new"] - 1
        count, kept = _accepted(c)
        rng = random.Random(int(seed))
        nodes = torch.full((c["B"], N), -1, dtype=torch.int32)
        for b in range(c["B"]):  # the first ones in place, the others from behind: the same however often it is called
            path = list(range(kept[b])) + sorted(rng.sample(range(count[b], N), count[b] - kept[b]))
            nodes[b, :count[b]] = torch.tensor(path, dtype=torch.int32)
        s["nodes"], s["count"] = nodes.cuda(), torch.tensor(count, dtype=torch.int32, device="cuda")
        s["new_len"] = torch.empty(c["B"], dtype=torch.int32, device="cuda")
    if own:  # what a program keeps: the descriptions of its cache and batch, and the workspace
        from paper_2605_29707_gb300 import binding as b
        s["type"] = {"f32": b.DOMINO_F32, "bf16": b.DOMINO_BF16, "f16": b.DOMINO_F16}[c["dtype"]]
        if c["kind"] != "rope":
            one = s["k"] if c["kind"] != "commit" else s["k"][0]
            page, x, y, _ = one.stride()
            token, head = (y, x) if c["by_head"] else (x, y)
            s["cache"] = b.make_cache(s["k"], s["v"], page, token, head, one.shape[0], c["page"], c["hkv"], c["D"],
                                      s["type"])
            s["batch"] = b.make_batch(s["table"], s["table"].stride(0), s["table"].shape[1], s["kv_len"], s["start"],
                                      c["B"])
        if c["kind"] == "attend":
            n = b.domino_attend_workspace_bytes(s["tokens"], c["hq"], s["cache"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return s


# --------------------------------------------------------------------------------- plain forms
def _slots(s, b, first, last):
    """(pages, places within them) of the positions first .. last - 1 of sequence b."""
    at = torch.arange(first, last, device="cuda")
    page = s["case"]["page"]
    return s["table"][b, at // page].long(), at % page


def _read(s, which, b, n):
    """The first n keys (or values) of sequence b: [n, heads, D]."""
    p, i = _slots(s, b, 0, n)
    return s[which][p, :, i] if s["case"]["by_head"] else s[which][p, i]


def _visible(s, b):
    """Which keys each new token of sequence b sees: [new, keys]."""
    kv, n, mask = s["kv_host"][b], s["new_host"][b], s["case"]["mask"]
    key = torch.arange(kv, device="cuda")
    at = torch.arange(n, device="cuda")
    if mask == "full":
        return torch.ones((n, kv), dtype=torch.bool, device="cuda")
    if mask == "causal":
        return key <= kv - n + at[:, None]
    path = torch.eye(n, device="cuda")  # a node sees itself and its parent, then, in doubling steps, what these see
    path[at[1:], s["parent"][b].long() + 1] = 1.0
    for _ in range(n.bit_length()):
        path = (path @ path).clamp(max=1.0)
    out = torch.ones((n, kv), dtype=torch.bool, device="cuda")
    out[:, kv - n:] = path > 0
    return out


def _plain_attend(s):
    c = s["case"]
    G, out, lse = c["hq"] // c["hkv"], [], []
    for b in range(c["B"]):
        kv, n = s["kv_host"][b], s["new_host"][b]
        q = s["q"][s["start_host"][b]:s["start_host"][b] + n].float()
        q = q.view(n, c["hkv"], G, c["D"]).permute(1, 0, 2, 3).reshape(c["hkv"], n * G, c["D"])
        z = q @ _read(s, "k", b, kv).float().permute(1, 2, 0)
        z *= c["D"] ** -0.5
        z.view(c["hkv"], n, G, kv).masked_fill_(~_visible(s, b)[:, None], -math.inf)
        top = z.amax(2, keepdim=True)
        z.sub_(top).exp_()
        mass = z.sum(2, keepdim=True)
        o = (z @ _read(s, "v", b, kv).float().transpose(0, 1)) / mass
        out.append(o.view(c["hkv"], n, G, c["D"]).permute(1, 0, 2, 3).reshape(n, c["hq"], c["D"]))
        lse.append((top + mass.log()).view(c["hkv"], n, G).permute(1, 0, 2).reshape(n, c["hq"]))
    return {"out": torch.cat(out).to(s["q"].dtype), "lse": torch.cat(lse)}


def _plain_rotate(x, pos, freq, rot, layout, amplitude, back=False):
    """x [tokens, heads, D]: the first rot elements turned by position times speed, or back."""
    angle = pos.double()[:, None, None] * freq.double()  # 64 bits: far positions turn thousands of times
    co, si = (angle.cos() * amplitude).float(), (angle.sin() * amplitude).float()
    si = -si if back else si
    y = x.float()
    a, b = (y[..., :rot // 2], y[..., rot // 2:rot]) if layout == "half" else (y[..., :rot:2], y[..., 1:rot:2])
    turned = (a * co - b * si, b * co + a * si)
    head = torch.cat(turned, 2) if layout == "half" else torch.stack(turned, 3).flatten(2)
    return torch.cat((head, y[..., rot:]), 2).to(x.dtype)


def _positions(s):
    """Places in the cache and positions of every new token, and its sequence."""
    c = s["case"]
    seq = torch.repeat_interleave(torch.arange(c["B"], device="cuda"), s["start"][1:] - s["start"][:-1],
                                  output_size=s["tokens"])
    i = torch.arange(s["tokens"], device="cuda") - s["start"][seq]
    place = s["kv_len"][seq] - c["new"] + i
    if s["depth"] is None:
        return seq, place, place
    depth = torch.cat((torch.zeros((c["B"], 1), dtype=torch.int32, device="cuda"), s["depth"]), 1)
    return seq, place, place - i + depth[seq, i]


def _split(s):
    c = s["case"]
    q, k, v, _ = s["qkv"].split((c["hq"] * c["D"], c["hkv"] * c["D"], c["hkv"] * c["D"], c["pad"]), 1)
    return tuple(t.unflatten(1, (-1, c["D"])) for t in (q, k, v))


def _plain_append(s):
    c = s["case"]
    q, k, v = _split(s)
    seq, place, pos = _positions(s)
    turn = (pos, s["freq"], c["rot"], c["layout"], s["amplitude"])
    page, i = s["table"][seq, place // c["page"]].long(), place % c["page"]
    s["k"][page, i], s["v"][page, i] = _plain_rotate(k, *turn), v
    return {"q": _plain_rotate(q, *turn), "k": s["k"], "v": s["v"]}


def _plain_commit(s):
    c = s["case"]
    N = c["new"] - 1
    j = torch.arange(N, device="cuda")
    first = (s["kv_len"] - N)[:, None]  # the place of node 0
    src = torch.where(j < s["count"][:, None], s["nodes"], j) + first
    dst = (j + first).expand_as(src)
    at = torch.arange(c["B"], device="cuda")[:, None]
    (p, i), (p2, i2) = (((s["table"][at, t // c["page"]]).long(), t % c["page"]) for t in (src, dst))
    for x in (s["k"], s["v"]):
        if c["by_head"]:
            x[:, p2, :, i2] = x[:, p, :, i]
        else:
            x[:, p2, i2] = x[:, p, i]
    return {"k": s["k"], "v": s["v"], "len": (s["kv_len"] - N + s["count"]).int()}


# ---------------------------------------------------------------------------------------- run
def run(state):
    s = state
    c = s["case"]
    if own:
        return _own(s, c)
    if c["kind"] == "attend":
        return _plain_attend(s)
    if c["kind"] == "append":
        return _plain_append(s)
    if c["kind"] == "rope":
        return {"y": _plain_rotate(s["x"], s["pos"], s["freq"], c["rot"], c["layout"], s["amplitude"], c["gradient"])}
    return _plain_commit(s)


def _own(s, c):
    from paper_2605_29707_gb300 import binding as b
    stream = torch.cuda.current_stream()
    if c["kind"] == "attend":
        mask = {"causal": b.DOMINO_MASK_CAUSAL, "full": b.DOMINO_MASK_FULL, "tree": b.DOMINO_MASK_TREE}[c["mask"]]
        tree = (s["parent"], c["new"] - 1) if c["mask"] == "tree" else (None, 0)
        rc = b.domino_attend_paged(s["q"], s["q"].stride(0), s["tokens"], c["hq"], s["cache"], s["batch"],
                                   c["D"] ** -0.5, mask, *tree, s["out"], s["out"].stride(0), s["lse"], s["ws"],
                                   s["ws"].numel(), stream)
        names = ("out", "lse")
        got = {n: s[n] for n in names}
    elif c["kind"] == "commit":
        rc = b.domino_cache_commit(s["cache"], s["batch"], c["layers"], s["k"].stride(0), s["nodes"], s["count"],
                                   c["new"] - 1, s["new_len"], stream)
        got = {"k": s["k"], "v": s["v"], "len": s["new_len"]}
    else:
        layout = b.DOMINO_ROPE_HALF if c["layout"] == "half" else b.DOMINO_ROPE_PAIRS
        if c["kind"] == "append":
            q, k, v = _split(s)
            wide = s["qkv"].stride(0)
            depth = (s["depth"], c["new"] - 1) if c["tree"] else (None, 0)
            rc = b.domino_rope_append(q, wide, k, wide, v, wide, None, *depth, s["freq"], s["amplitude"], layout,
                                      c["rot"], c["hq"], s["tokens"], s["q_out"], s["q_out"].stride(0), s["cache"],
                                      s["batch"], stream)
            got = {"q": s["q_out"], "k": s["k"], "v": s["v"]}
        else:
            rc = b.domino_rope(s["x"], s["type"], s["x"].stride(0), s["x"].stride(1), s["pos"], s["freq"],
                               s["amplitude"], layout, int(c["gradient"]), c["tokens"], c["heads"], c["D"], c["rot"],
                               s["y"], s["y"].stride(0), s["y"].stride(1), stream)
            got = {"y": s["y"]}
    if rc != b.DOMINO_OK:
        raise b.DominoError(rc, c["kind"])
    return got


# --------------------------------------------------------------------------------------- work
def work(case):
    """Every input read and every output written once; 4 D operations for each query and key that meet, six for each
    rotated pair."""
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "rope":
        n = c["tokens"] * c["heads"]
        return {"bytes": 2 * n * c["D"] * size + c["tokens"] * 4 + c["rot"] * 2, "flops": 3 * n * c["rot"]}
    kv, new = _lengths(c)
    if c["kind"] == "attend":
        if c["mask"] == "full":
            meet = sum(k * n for k, n in zip(kv, new))
        elif c["mask"] == "causal":
            meet = sum(n * (k - n) + n * (n + 1) // 2 for k, n in zip(kv, new))
        else:  # at the least: the context, the anchor and itself
            meet = sum(n * (k - n) + 2 * n - 1 for k, n in zip(kv, new))
        cache = 2 * sum(kv) * c["hkv"] * c["D"] * size
        return {"bytes": cache + sum(new) * c["hq"] * (2 * c["D"] * size + 4), "flops": 4 * c["D"] * c["hq"] * meet}
    if c["kind"] == "append":
        n = sum(new)
        return {"bytes": 2 * n * (c["hq"] + 2 * c["hkv"]) * c["D"] * size,
                "flops": 3 * n * (c["hq"] + c["hkv"]) * c["rot"]}
    count, kept = _accepted(c)
    moved = sum(count) - sum(kept)
    return {"bytes": 4 * moved * c["layers"] * c["hkv"] * c["D"] * size + 8 * c["B"], "flops": 0}


# -------------------------------------------------------------------------------------- exact
def exact(case, seed):
    """The definitions in 64 bits: a softmax over the keys that a token sees, a product of complex numbers, a copy."""
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] == "attend":
        return _exact_attend(s, c)
    if c["kind"] == "commit":
        k, v = s["k"].clone(), s["v"].clone()
        N, page = c["new"] - 1, c["page"]
        for b, n in enumerate(s["count"].tolist()):
            first = s["kv_host"][b] - N
            for j, node in enumerate(s["nodes"][b, :n].tolist()):  # in order: a place is read before it is written
                (p, i), (p2, i2) = ((int(s["table"][b, t // page]), t % page) for t in (first + node, first + j))
                for x in (k, v):
                    (x.transpose(2, 3) if c["by_head"] else x)[:, p2, i2] = \
                        (x.transpose(2, 3) if c["by_head"] else x)[:, p, i].clone()
        return {"k": k, "v": v, "len": torch.tensor([a - N + n for a, n in zip(s["kv_host"], s["count"].tolist())],
                                                    dtype=torch.int32, device="cuda")}

    def turn(x, pos, sign):
        x, r = x.double(), c["rot"]
        z = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) if c["layout"] == "pairs" else \
            torch.complex(x[..., :r // 2], x[..., r // 2:r])
        z = z * torch.polar(torch.full_like(z.real[:1], s["amplitude"]),
                            (sign * torch.outer(pos.double(), s["freq"].double()))[:, None])
        parts = torch.view_as_real(z)
        head = parts.flatten(-2) if c["layout"] == "pairs" else torch.cat(parts.unbind(-1), -1)
        return torch.cat((head, x[..., r:]), -1)

    if c["kind"] == "rope":
        return {"y": turn(s["x"], s["pos"], -1.0 if c["gradient"] else 1.0)}
    q, k, v = _split(s)
    kc, vc, pos, place = s["k"].double(), s["v"].double(), [], []
    for b in range(c["B"]):
        first = s["kv_host"][b] - c["new"]
        for i in range(c["new"]):
            place.append(int(first + i))
            pos.append(first + (i if s["depth"] is None else 0))
        if s["depth"] is not None:
            deep = s["depth"][b].tolist()
            pos[-c["new"]:] = [first] + [first + d for d in deep]
    pos = torch.tensor(pos, device="cuda")
    turned = turn(k, pos, 1.0)
    seq = torch.arange(c["B"], device="cuda").repeat_interleave(c["new"])
    place = torch.tensor(place, device="cuda")
    at = s["table"][seq, torch.div(place, c["page"], rounding_mode="floor")].long() * c["page"] + place % c["page"]
    kc.flatten(0, 1)[at], vc.flatten(0, 1)[at] = turned, v.double()
    return {"q": turn(q, pos, 1.0), "k": kc, "v": vc}


def _exact_attend(s, c):
    if 4 * c["D"] * c["hq"] * sum(k * n for k, n in zip(s["kv_host"], s["new_host"])) > 6e12:
        return None
    G = c["hq"] // c["hkv"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    k, v = ((x.transpose(1, 2) if c["by_head"] else x).flatten(0, 1) for x in (s["k"], s["v"]))
    for b in range(c["B"]):
        kv, n, a = s["kv_host"][b], s["new_host"][b], s["start_host"][b]
        places = (s["table"][b].long()[:, None] * c["page"] + torch.arange(c["page"], device="cuda")).flatten()[:kv]
        # seen[i]: of the new tokens, those that token i sees; all the keys before them are seen
        if c["mask"] == "tree":
            up, seen = [-1] + [p + 1 for p in s["parent"][b].tolist()], torch.zeros((n, n), dtype=torch.bool)
            for i in range(n):
                at = i
                while at >= 0:
                    seen[i, at] = True
                    at = up[at]
        else:
            seen = torch.ones((n, n), dtype=torch.bool)
            seen = seen.tril() if c["mask"] == "causal" else seen
        hidden = ~seen.cuda()
        for h in range(c["hkv"]):
            kh, vh = k[places, h].double(), v[places, h].double()
            for g in range(h * G, h * G + G):
                for i in range(0, n, 1024):
                    qg = s["q"][a + i:min(a + n, a + i + 1024), g].double()
                    z = torch.einsum("id,jd->ij", qg, kh) / math.sqrt(c["D"])
                    z[:, kv - n:].masked_fill_(hidden[i:i + 1024], -math.inf)
                    norm = torch.logsumexp(z, 1)
                    lse[a + i:a + i + z.shape[0], g] = norm
                    out[a + i:a + i + z.shape[0], g] = torch.einsum("ij,jd->id", (z - norm[:, None]).exp(), vh)
    return {"out": out, "lse": lse}
