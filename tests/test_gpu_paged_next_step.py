"""A second step on what the first one left: lengths as the commit wrote them, the next tree behind the kept tokens, in the
same captured graph; against caches in which the same tokens were decoded one by one."""
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref
from tests.test_gpu_paged_together import D, DEV, HKV, HQ, LAYERS, N, PAGE, Server

pytestmark = pytest.mark.gpu


class Roomy(Server):
    """A server whose sequences have places for three steps; what no step has written yet is NaN."""

    def __init__(self, kv, seed):
        super().__init__([n + 2 * (N + 1) for n in kv], seed)
        self.context = list(kv)
        for i, n in enumerate(kv):
            at, off = self.p.slots(i, self.p.kv[i])
            self.p.k[:, at[n:], off[n:]] = float("nan")
            self.p.v[:, at[n:], off[n:]] = float("nan")
        self.p.kv = [n + N + 1 for n in kv]
        self.p.kv_len.copy_(torch.tensor(self.p.kv, dtype=torch.int32))


class Decoded:
    """The same contexts, to which one token after the other is appended."""

    def __init__(self, s):
        self.s, self.k, self.v = s, s.p.k.clone(), s.p.v.clone()
        self.len = list(s.context)

    def step(self, tokens):
        """tokens: for every sequence those that it decodes, in turn."""
        s, p, wide = self.s, self.s.p, (HQ + 2 * HKV) * D
        i32 = dict(dtype=torch.int32, device=DEV)
        q = torch.empty((1, HQ, D), dtype=torch.bfloat16, device=DEV)
        for i in range(p.B):
            for t in tokens[i]:
                self.len[i] += 1
                one = [torch.tensor(x, **i32) for x in ([self.len[i]], [0, 1])]
                batch = b.make_batch(p.table[i], p.table.stride(0), p.table.shape[1] - 1, *one, 1)
                for layer in range(LAYERS):
                    k, v = self.k[layer], self.v[layer]
                    cache = b.make_cache(k, v, *k.stride()[:3], p.pages, PAGE, HKV, D, b.DOMINO_BF16)
                    x = s.qkv[layer, t:t + 1]
                    parts = x.split((HQ * D, HKV * D, HKV * D), 1)
                    assert b.domino_rope_append(parts[0], wide, parts[1], wide, parts[2], wide, None, None, 0, s.freq, 1.0,
                                                b.DOMINO_ROPE_HALF, D, HQ, 1, q, HQ * D, cache, batch, torch.cuda.current_stream()) == 0
                torch.cuda.synchronize()

    def check(self, tokens):
        """The server's caches hold what was decoded, and its rows of the path (the last `tokens`) attend to it."""
        s, p = self.s, self.s.p
        for i in range(p.B):
            n, new = self.len[i], len(tokens[i])
            assert int(s.new_len[i]) == n
            at, off = p.slots(i, n)
            rows = [i * (N + 1)] + [i * (N + 1) + 1 + a for a in s.nodes[i, :new - 1].tolist()]
            for layer in range(LAYERS):
                assert torch.equal(p.k[layer][at, off], self.k[layer][at, off])
                assert torch.equal(p.v[layer][at, off], self.v[layer][at, off])
                own = ref.Paged([n], [new], HKV, D, b.DOMINO_BF16, PAGE, seed=1)
                a2, o2 = own.slots(0, n)
                own.k[0, a2, o2], own.v[0, a2, o2] = self.k[layer][at, off], self.v[layer][at, off]
                want, wl, tol, ltol = ref.attend(own, s.q[layer][rows], D ** -0.5, b.DOMINO_MASK_CAUSAL)
                assert bool(((s.out[layer][rows].double() - want).abs() <= tol).all())
                assert bool(((s.lse[layer][rows].double() - wl).abs() <= ltol).all())


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("kv", [[100, 3, 257], [16, 31], [1000]])
def test_steps_follow_each_other(kv, captured):
    s = Roomy(kv, seed=sum(kv))
    twin = Decoded(s)
    s.steer()
    graph = None
    if captured:
        k, v = s.p.k_store.clone(), s.p.v_store.clone()
        s.run()  # the libraries' first calls outside the capture
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        s.p.k_store.copy_(k)
        s.p.v_store.copy_(v)
    for step in range(2):
        anchor, was = s.anchor.tolist(), [n - N - 1 for n in s.p.kv_len.tolist()]
        graph.replay() if captured else s.run()
        torch.cuda.synchronize()
        assert b.domino_check_status(s.ws, None) == 0
        tokens = [[anchor[i]] + [int(s.token[i, a]) for a in s.nodes[i, :int(s.count[i])].tolist()] for i in range(s.B)]
        assert max(len(t) for t in tokens) >= 2
        twin.step(tokens)
        assert [a + len(t) for a, t in zip(was, tokens)] == twin.len
        twin.check(tokens)
        s.p.kv_len.copy_(s.new_len + (N + 1))  # on the device, as a captured server does it
        s.anchor.copy_(s.bonus)
