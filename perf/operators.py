"""Operators on rows of vocabulary logits, as cases that can be timed and checked.

Three operators that a speculative-decoding user needs next to the draft step:
- drawing a token per row after temperature, top-k, top-p and min-p (`domino_sample_filtered`);
- checking drafted trees against a target that decodes with those filters (`domino_verify_tree_filtered`);
- distilling a teacher's top logits into the draft model: the loss of every row and its gradient
  (`domino_distill_loss`, `domino_distill_grad` and both in one pass, `domino_distill_loss_grad`).

Sizes: a vocabulary of 151936 (the repository's configurations), smaller and odd ones, rows stored with
a padded stride, 1 to 64 sequences, trees of 8 to 32 nodes, blocks of 16 draft positions.  Logits are
normal with deviation 5.1, about 3 nats of entropy over 151936 ids.
"""
import math

import torch

own = False

VOCAB = 151936
LOGIT_STD = 5.1
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
RENORM, TAIL = 0, 1  # what stands for the ids that the teacher's list leaves out: nothing, or one bucket
OFF_K, OFF_P, OFF_M = 0, 1.0, 0.0


# ------------------------------------------------------------------------------------- cases
def _sample(name, rows, V, dtype, rule, pad=0):
    return dict(name=name, kind="sample", rows=rows, V=V, dtype=dtype, rule=rule, pad=pad)


def _verify(name, B, N, V, dtype, rule, pad=0):
    return dict(name=name, kind="verify", B=B, N=N, V=V, dtype=dtype, rule=rule, pad=pad)


def _distill(name, part, rows, V, dtype, kt, mode, temperature=1.0, pad=0):
    return dict(name=name, kind="distill", part=part, rows=rows, V=V, dtype=dtype, kt=kt, mode=mode,
                temperature=temperature, pad=pad)


def listed():
    return [
        # one interactive user's next token, chat settings: the smallest call, latency alone
        _sample("sample-b1-chat", 1, VOCAB, "f32", "chat"),
        # a serving batch whose requests each bring their own settings, some of them greedy
        _sample("sample-b64-mixed-bf16", 64, VOCAB, "bf16", "mixed"),
        # an odd batch on a small odd vocabulary, rows padded to whole 128-byte lines, min-p alone
        _sample("sample-b37-minp-f16", 37, 49999, "f16", "minp", pad=17),
        # many parallel completions (reinforcement learning, best-of-n), nucleus sampling
        _sample("sample-r512-topp", 512, VOCAB, "f32", "topp"),
        # one interactive user's drafted tree against a target that decodes with chat settings
        _verify("verify-b1-chat", 1, 16, VOCAB, "f32", "chat"),
        # a few users on a small odd vocabulary with larger trees
        _verify("verify-b7-topp-v60001", 7, 21, 60001, "bf16", "topp"),
        # a full serving batch's trees, every sequence with its own settings
        _verify("verify-b64-mixed-bf16", 64, 16, VOCAB, "bf16", "mixed"),
        # held-out loss of one draft block
        _distill("distill-loss-m16", "loss", 16, VOCAB, "bf16", 8, TAIL),
        # held-out loss of a batch of blocks on an odd vocabulary at a raised temperature
        _distill("distill-loss-m1023-f16", "loss", 1023, 41511, "f16", 20, RENORM, 2.0),
        # the backward pass of a training step that keeps its logits
        _distill("distill-grad-m512-f32", "grad", 512, VOCAB, "f32", 32, TAIL, 1.5),
        # a small training step on an odd vocabulary, loss and gradient in one pass
        _distill("distill-both-m105-f32", "both", 105, 32003, "f32", 8, RENORM, pad=29),
        # the largest: a training step over 256 blocks of 16 draft positions
        _distill("distill-both-m4096", "both", 4096, VOCAB, "bf16", 8, TAIL),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("sample", "verify", "distill"))
    V = rng.choice((VOCAB, _log_int(rng, 4000, VOCAB)))
    dtype = rng.choice(tuple(TYPES))
    pad = rng.choice((0, 0, rng.randint(1, 64)))
    rule = rng.choice(("chat", "topk", "topp", "minp", "none", "mixed"))
    if kind == "sample":
        c = _sample("", _log_int(rng, 1, 700), V, dtype, rule, pad)
    elif kind == "verify":
        N = rng.randint(8, 32)
        c = _verify("", _log_int(rng, 1, 700 // (N + 1)), N, V, dtype, rule, pad)
    else:
        c = _distill("", rng.choice(("loss", "grad", "both")), _log_int(rng, 4, 2000), V, dtype, rng.randint(1, 64),
                     rng.choice((RENORM, TAIL)), rng.choice((1.0, round(rng.uniform(0.5, 4.0), 2))), pad)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------ inputs
def _gen(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 64 + n)
    return g


def _logits(rows, V, pad, dtype, g):
    """[rows, V] logits, row stride V + pad; the padding holds what a user's padding holds, anything."""
    out = torch.full((rows, V + pad), 1e4, dtype=TYPES[dtype], device="cuda")
    step = max(1, (1 << 26) // V)
    for a in range(0, rows, step):  # in pieces: the fp32 draws of a whole batch would be large
        b = min(rows, a + step)
        out[a:b, :V] = torch.randn((b - a, V), generator=g, device="cuda").mul_(LOGIT_STD)
    return out[:, :V]


def _settings(rule, n, g):
    """(temperature, top_k, top_p, min_p) of n requests, None where the whole batch leaves a filter off."""
    def pick(values):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), (n,), generator=g, device="cuda")]

    temperature = pick([0.6, 0.7, 0.8, 1.0])
    if rule == "chat":
        return temperature, pick([20, 40, 50]).int(), pick([0.8, 0.9, 0.95]), None
    if rule == "topk":
        return temperature, pick([5, 40, 100, 200]).int(), None, None
    if rule == "topp":
        return temperature, None, pick([0.8, 0.9, 0.95]), None
    if rule == "minp":
        return pick([0.8, 1.0, 1.3]), None, None, pick([0.02, 0.05, 0.1])
    if rule == "none":
        return pick([0.7, 1.0]), None, None, None
    return (pick([0.0, 0.6, 0.8, 1.0, 1.2]), pick([OFF_K, 1, 20, 50, 100]).int(), pick([OFF_P, 0.8, 0.95]),
            pick([OFF_M, 0.05, 0.1]))


def _trees(B, N, V, seed):
    """Random trees (parents before children): parent [B, N], token [B, N], on the host."""
    g = torch.Generator().manual_seed(int(seed) * 64 + 40)
    at = torch.arange(N).clamp(min=1)
    parent = (torch.rand(B, N, generator=g) * (at + 1)).long() - 1
    parent[:, 0] = -1
    return parent.clamp(max=N - 1), torch.randint(0, V, (B, N), generator=g)


def prepare(case, seed):
    c, s = dict(case), {}
    s["case"], dt = c, TYPES[c["dtype"]]
    if c["kind"] == "distill":
        M, V, kt, T = c["rows"], c["V"], c["kt"], c["temperature"]
        x = _logits(M, V, c["pad"], c["dtype"], _gen(seed, 1))
        ids = torch.empty((M, kt), dtype=torch.int32, device="cuda")
        score = torch.empty((M, kt), dtype=torch.float32, device="cuda")
        g, step = _gen(seed, 2), max(1, (1 << 26) // V)
        for a in range(0, M, step):  # the teacher: near the student, its best kt ids and their log-probabilities
            b = min(M, a + step)
            t = x[a:b].float() + torch.randn((b - a, V), generator=g, device="cuda")
            t = t / T if c["mode"] == TAIL else t
            v, i = torch.topk(t, kt, dim=1)
            if c["mode"] == TAIL:
                v = v - torch.logsumexp(t, 1, keepdim=True)
            ids[a:b], score[a:b] = i.int(), v
        short = torch.rand(M, generator=g, device="cuda") < 0.05  # lists that end early
        ids[short, kt // 2 + 1:] = -1
        pos = torch.arange(M, device="cuda") % 16
        weights = torch.exp(-pos / 8.0)  # nearer draft positions count more
        weights[torch.rand(M, generator=g, device="cuda") < 0.1] = 0.0  # rows of padding
        scale = 8192.0 if c["dtype"] == "f16" else 1.0  # the loss scale that training in fp16 needs
        s.update(x=x, ids=ids, score=score, weights=weights.float(),
                 up=torch.full((M,), scale / M, device="cuda"))
        s["loss"] = torch.empty(M, device="cuda")
        s["lse"] = torch.empty((M, 2), device="cuda")
        if c["part"] == "grad":  # what the forward pass left
            s["lse"] = torch.stack(_sums(s), 1).float().contiguous()
        if c["part"] != "loss":
            s["dx"] = torch.zeros((M, V + c["pad"]), dtype=dt, device="cuda")[:, :V]
        return s
    n = c["rows"] if c["kind"] == "sample" else c["B"]
    rows = n if c["kind"] == "sample" else n * (c["N"] + 1)
    s["x"] = _logits(rows, c["V"], c["pad"], c["dtype"], _gen(seed, 1))
    s["uniforms"] = torch.rand(rows, generator=_gen(seed, 3), device="cuda")
    s["set"] = _settings(c["rule"], n, _gen(seed, 4))
    s["tokens"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["logp"] = torch.empty(rows, device="cuda")
    if c["kind"] == "verify":
        B, N = c["B"], c["N"]
        parent, token = _trees(B, N, c["V"], seed)
        keep = torch.rand(B, N, generator=torch.Generator().manual_seed(int(seed) * 64 + 41)) < 0.7
        bb, ii = torch.nonzero(keep, as_tuple=True)  # after these nodes a child's token is the target's favourite
        at, top = (bb * (N + 1) + parent[bb, ii] + 1).cuda(), s["x"].amax(1).float()
        s["x"][at, token[bb, ii].cuda()] = (top[at] + 2.0 + 0.01 * ii.cuda()).to(dt)
        s["parent"], s["token"] = parent.int().cuda(), token.int().cuda()
        for name, shape in (("nodes", (B, N)), ("count", (B,)), ("bonus", (B,))):
            s[name] = torch.empty(shape, dtype=torch.int32, device="cuda")
    return s


# --------------------------------------------------------------------------------- plain forms
def _plain_draw(x, setting, u, per):
    """Row draws after temperature, top-k, top-p and min-p; `per` rows share a request's settings.  In 64 bits: a
    cumulative sum over a vocabulary decides which id a uniform next to a border names."""
    V = x.shape[1]
    T, k, p, m = (None if t is None else t.repeat_interleave(per)[:, None] for t in setting)
    greedy = ~(T > 0)
    k = torch.zeros_like(T).int() if k is None else k
    k = torch.where(greedy, 1, torch.where((k < 1) | (k > V), V, k))
    T = torch.where(greedy, 1.0, T).double()
    x = x.double()
    d = (x - x.amax(1, keepdim=True)) / T
    w, order = torch.sort(d, dim=1, descending=True, stable=True)  # equal values: the lower id first
    w = w.exp()
    keep = torch.arange(V, device=x.device) < k
    if p is not None:
        cum = (w * keep).cumsum(1)
        goal = torch.where(p < 1, p.double(), math.inf) * cum[:, -1:]
        keep &= cum - w < goal
    if m is not None:
        keep &= w.log() >= torch.where(m > 0, m.double(), 0.0).log()
    keep[:, 0] = True
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    cum = (d.exp() * kept).cumsum(1)
    token = (cum <= u.double()[:, None] * cum[:, -1:]).sum(1, keepdim=True).clamp(max=V - 1)
    return token[:, 0].int(), (d.gather(1, token) - cum[:, -1:].log())[:, 0].float()


def _plain_walk(parent, token, choice):
    """From the anchor: the child that carries the row's choice (the lowest such node), until there is none."""
    B, N = parent.shape
    cur = torch.full((B,), -1, device=parent.device)
    nodes = torch.full((B, N), -1, dtype=torch.int32, device=parent.device)
    count = torch.zeros(B, dtype=torch.int32, device=parent.device)
    live, at = torch.ones(B, dtype=torch.bool, device=parent.device), torch.arange(N, device=parent.device)
    for step in range(N):
        a = choice.gather(1, cur[:, None] + 1)
        hit = (parent == cur[:, None]) & (token == a) & live[:, None]
        child = torch.where(hit, at, N).amin(1)
        live = child < N
        nodes[:, step] = torch.where(live, child, -1).int()
        count += live.int()
        cur = torch.where(live, child, cur)
    return nodes, count, choice.gather(1, cur[:, None] + 1)[:, 0]


def _listed(s):
    """The teacher's lists: ids with 0 for an empty place, which places are filled, q of each and of the rest."""
    c, ok = s["case"], s["ids"] >= 0
    t = torch.where(ok, s["score"], -math.inf)
    if c["mode"] == TAIL:
        q = t.exp()
        return s["ids"].clamp(min=0).long(), ok, q, (1 - q.sum(1)).clamp(min=0)
    t = t / c["temperature"]
    q = (t - t.amax(1, keepdim=True)).exp()
    return s["ids"].clamp(min=0).long(), ok, q / q.sum(1, keepdim=True), torch.zeros_like(q[:, 0])


def _sums(s):
    """log of the sum of exp(logit / T) over every id, and over the ids that are not in the teacher's list."""
    z = s["x"].float() / s["case"]["temperature"]
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    idx = s["ids"].clamp(min=0).long()
    every = e.sum(1)
    e.scatter_(1, torch.where(s["ids"] >= 0, idx, idx[:, :1]), 0.0)
    return top[:, 0] + every.log(), top[:, 0] + e.sum(1).log()


def _plain_loss(s):
    idx, ok, q, rest = _listed(s)
    lse, lse_rest = _sums(s)
    logp = s["x"].gather(1, idx).float() / s["case"]["temperature"] - lse[:, None]
    loss = torch.where(ok & (q > 0), q * (q.log() - logp), 0.0).sum(1)
    loss = loss + torch.where(rest > 0, rest * (rest.log() - (lse_rest - lse)), 0.0)
    return torch.where(s["weights"] != 0, s["weights"] * loss, 0.0), torch.stack((lse, lse_rest), 1)


def _plain_grad(s, lse):
    idx, ok, q, rest = _listed(s)
    z = s["x"].float() / s["case"]["temperature"]
    g = (z - lse[:, :1]).exp()
    if s["case"]["mode"] == TAIL:
        at = g.gather(1, idx)
        g -= rest[:, None] * (z - lse[:, 1:]).exp()
        g.scatter_(1, torch.where(ok, idx, idx[:, :1]), torch.where(ok, at, at[:, :1]))
    g.scatter_add_(1, idx, torch.where(ok, -q, 0.0))
    scale = torch.where(s["weights"] != 0, s["weights"] * s["up"] / s["case"]["temperature"], 0.0)
    return (g * scale[:, None]).to(s["x"].dtype)


# ---------------------------------------------------------------------------------------- run
def run(state):
    s = state
    c = s["case"]
    if own:
        return _own(s, c)
    if c["kind"] == "sample":
        return dict(zip(("tokens", "logp"), _plain_draw(s["x"], s["set"], s["uniforms"], 1)))
    if c["kind"] == "verify":
        y, logp = _plain_draw(s["x"], s["set"], s["uniforms"], c["N"] + 1)
        walk = _plain_walk(s["parent"], s["token"], y.view(c["B"], -1))
        return dict(zip(("tokens", "logp", "nodes", "count", "bonus"), (y, logp) + walk))
    if c["part"] == "grad":
        return {"dx": _plain_grad(s, s["lse"])}
    loss, lse = _plain_loss(s)
    out = {"loss": loss, "lse": lse}
    if c["part"] == "both":
        out["dx"] = _plain_grad(s, lse)
    return out


def _own(s, c):
    from paper_2605_29707_gb300 import binding as b
    x, stream = s["x"], torch.cuda.current_stream()
    kind = {"f32": b.DOMINO_F32, "bf16": b.DOMINO_BF16, "f16": b.DOMINO_F16}[c["dtype"]]
    if c["kind"] == "sample":
        rc = b.domino_sample_filtered(x, kind, x.stride(0), *s["set"], s["uniforms"], c["rows"], c["V"], s["tokens"],
                                      s["logp"], stream)
        names = ("tokens", "logp")
    elif c["kind"] == "verify":
        rc = b.domino_verify_tree_filtered(x, kind, x.stride(0), s["parent"], s["token"], *s["set"], s["uniforms"],
                                           c["B"], c["N"], c["V"], s["tokens"], s["logp"], s["nodes"], s["count"],
                                           s["bonus"], stream)
        names = ("tokens", "logp", "nodes", "count", "bonus")
    else:
        mode = b.DOMINO_DISTILL_TAIL if c["mode"] == TAIL else b.DOMINO_DISTILL_RENORM
        teacher = (s["ids"], s["score"], s["weights"])
        sizes = (c["temperature"], mode, c["rows"], c["V"], c["kt"])
        if c["part"] == "loss":
            rc = b.domino_distill_loss(x, kind, x.stride(0), *teacher, *sizes, s["loss"], s["lse"], stream)
            names = ("loss", "lse")
        elif c["part"] == "grad":
            rc = b.domino_distill_grad(x, kind, x.stride(0), *teacher, s["up"], *sizes, s["lse"], s["dx"],
                                       s["dx"].stride(0), stream)
            names = ("dx",)
        else:
            rc = b.domino_distill_loss_grad(x, kind, x.stride(0), *teacher, s["up"], *sizes, s["loss"], s["lse"],
                                            s["dx"], s["dx"].stride(0), stream)
            names = ("loss", "lse", "dx")
    if rc != b.DOMINO_OK:
        raise b.DominoError(rc, c["kind"])
    return {n: s[n] for n in names}


# --------------------------------------------------------------------------------------- work
def work(case):
    """Every logit read once, every gradient written once, the small inputs and outputs once; per logit one comparison
    and one addition for a draw, an exponential and two more for a loss or a gradient."""
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "distill":
        n = c["rows"] * c["V"]
        passes = 2 if c["part"] != "loss" else 1
        return {"bytes": passes * n * size + c["rows"] * (8 * c["kt"] + 16), "flops": n * (8 if c["part"] == "both" else 4)}
    rows = c["rows"] if c["kind"] == "sample" else c["B"] * (c["N"] + 1)
    small = rows * 12 + (c["rows"] * 16 if c["kind"] == "sample" else c["B"] * (16 + 12 * c["N"] + 8))
    return {"bytes": rows * c["V"] * size + small, "flops": 2 * rows * c["V"]}


# -------------------------------------------------------------------------------------- exact
def _exact_draw(x, T, k, p, m, u):
    """One row's draw, from the definition: the ids in order of preference, cut three times, drawn in id order."""
    V, x = x.numel(), x.double()
    if not T > 0:
        T, k = 1.0, 1
    best = torch.argsort(x, descending=True, stable=True)
    if 1 <= k < V:
        best = best[:k]
    z = x[best] / T
    prob = torch.softmax(z, 0)
    n = best.numel()
    if p < 1:
        before = torch.cat((prob.new_zeros(1), prob.cumsum(0)[:-1]))
        n = max(1, int((before < p).sum()))
    if m > 0:
        n = min(n, max(1, int((z - z[0] >= math.log(m)).sum())))
    ids = best[:n].sort().values
    logp = torch.log_softmax(x[ids] / T, 0)
    at = min(n - 1, int(torch.searchsorted(logp.exp().cumsum(0), torch.tensor(u, dtype=torch.float64, device=x.device), right=True)))
    return int(ids[at]), float(logp[at])


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["kind"] != "distill":
        rows, n = s["x"].shape[0], s["set"][0].numel()
        host = [([off] * n if t is None else t.tolist()) for t, off in zip(s["set"], (1.0, OFF_K, OFF_P, OFF_M))]
        u = s["uniforms"].tolist()
        got = [_exact_draw(s["x"][r], *(t[r * n // rows] for t in host), u[r]) for r in range(rows)]
        out = {"tokens": torch.tensor([g[0] for g in got], dtype=torch.int32),
               "logp": torch.tensor([g[1] for g in got], dtype=torch.float64)}
        if c["kind"] == "verify":
            out.update(nodes=None, count=None, bonus=None)
        return out
    T, V, kt = c["temperature"], c["V"], c["kt"]
    out = {"loss": [], "lse": [], "dx": []}
    step = max(1, (1 << 26) // V)
    for a in range(0, c["rows"], step):
        x, ids = s["x"][a:a + step].double() / T, s["ids"][a:a + step].long()
        t, w = s["score"][a:a + step].double(), s["weights"][a:a + step].double()
        has = torch.zeros(x.shape[0], V + 1, dtype=torch.bool, device="cuda").scatter_(1, ids % (V + 1), True)[:, :V]
        q = torch.zeros(x.shape[0], V + 1, dtype=torch.float64, device="cuda")
        if c["mode"] == TAIL:
            q = q.scatter_(1, ids % (V + 1), t.exp())[:, :V]
            rest = (1 - q.sum(1)).clamp(min=0)
        else:
            q = torch.softmax(torch.full_like(q[:, :V], -math.inf).scatter_add_(
                1, ids.clamp(min=0), torch.zeros_like(t)).masked_scatter_(has, _by_id(ids, t / T)), 1)
            rest = torch.zeros_like(w)
        lse, lse_rest = torch.logsumexp(x, 1), torch.logsumexp(x.masked_fill(has, -math.inf), 1)
        if c["part"] == "grad":  # the given sums are what the forward pass left, rounded
            lse, lse_rest = s["lse"][a:a + step].double().unbind(1)
        loss = torch.special.xlogy(q, q).sum(1) - (q * (x - lse[:, None])).masked_fill(~has, 0).sum(1)
        loss += torch.special.xlogy(rest, rest) - rest * (lse_rest - lse)
        out["loss"].append((loss * w).masked_fill(w == 0, 0))
        out["lse"].append(torch.stack((lse, lse_rest), 1))
        if c["part"] != "loss":
            g = torch.exp(x - lse[:, None]) - q
            g -= (rest[:, None] * torch.exp(x - lse_rest[:, None])).masked_fill(has, 0) if c["mode"] == TAIL else 0
            out["dx"].append(g * (w * s["up"][a:a + step].double() / T)[:, None])
    out = {k: torch.cat(v) for k, v in out.items() if v}
    return {"dx": out["dx"]} if c["part"] == "grad" else out


def _by_id(ids, t):
    """The filled places of every row in id order, one after another (what masked_scatter_ takes)."""
    key = torch.where(ids >= 0, ids, 1 << 40)
    order = key.argsort(1)
    return t.gather(1, order)[key.gather(1, order) < 1 << 40]
