"""A target's layer around a verification, as a server runs it: the tree's new tokens turned and written into the paged
cache, attention with the tree's mask, greedy verification, the accepted nodes kept, and the next step on what they
left, on one stream and in one captured graph.  A sequence that decodes the accepted tokens one by one has the same
cache and the same attention."""
import pytest
import torch

from paper_2605_29707_gb300 import binding as b
from tests import paged_reference as ref
from tests.test_gpu_paged_rope import speeds

pytestmark = pytest.mark.gpu
DEV = "cuda"
HQ, HKV, D, LAYERS, N, V, PAGE = 8, 2, 64, 3, 12, 200, 16


class Server:
    """One cache of LAYERS layers; a layer's projections are rows of fixed tables, by token id."""

    def __init__(self, kv, seed=0):
        self.B = len(kv)
        self.p = ref.Paged([n + N + 1 for n in kv], [N + 1] * self.B, HKV, D, b.DOMINO_BF16, PAGE, layers=LAYERS, seed=seed)
        g = torch.Generator(device=DEV).manual_seed(seed + 1)
        self.qkv = torch.randn((LAYERS, V, (HQ + 2 * HKV) * D), generator=g, device=DEV).bfloat16()
        self.freq = speeds(D)
        rows = self.B * (N + 1)
        self.x = torch.empty((LAYERS, rows, (HQ + 2 * HKV) * D), dtype=torch.bfloat16, device=DEV)
        self.q = torch.empty((LAYERS, rows, HQ, D), dtype=torch.bfloat16, device=DEV)
        self.out, self.lse = torch.empty_like(self.q), torch.empty((LAYERS, rows, HQ), device=DEV)
        i32 = dict(dtype=torch.int32, device=DEV)
        parent, depth = ref.random_trees(self.B, N, seed + 2)
        self.parent_host = parent
        self.parent, self.depth = torch.tensor(parent, **i32), torch.tensor(depth, **i32)
        self.token = torch.randint(0, V, (self.B, N), generator=g, **i32)
        self.anchor = torch.randint(0, V, (self.B,), generator=g, **i32)
        self.logits = torch.randn((rows, V), generator=g, device=DEV)
        self.best, self.nodes = torch.empty((self.B, N + 1), **i32), torch.empty((self.B, N), **i32)
        self.count, self.bonus, self.new_len = (torch.empty(self.B, **i32) for _ in range(3))
        self.cache = [b.make_cache(self.p.k_store[i], self.p.v_store[i], *self.p.k.stride()[1:4], self.p.pages, PAGE, HKV, D,
                                   b.DOMINO_BF16) for i in range(LAYERS)]
        n = b.domino_attend_workspace_bytes(rows, HQ, self.cache[0])
        self.ws = torch.empty(n, dtype=torch.uint8, device=DEV)

    def run(self):
        s, rows, wide = torch.cuda.current_stream(), self.B * (N + 1), (HQ + 2 * HKV) * D
        ids = torch.cat((self.anchor[:, None], self.token), 1).flatten().long()
        for i in range(LAYERS):
            self.x[i] = self.qkv[i].index_select(0, ids)
            q, k, v = self.x[i].split((HQ * D, HKV * D, HKV * D), 1)
            assert b.domino_rope_append(q, wide, k, wide, v, wide, None, self.depth, N, self.freq, 1.0, b.DOMINO_ROPE_HALF, D, HQ, rows,
                                        self.q[i], HQ * D, self.cache[i], self.p.batch, s) == 0
            assert b.domino_attend_paged(self.q[i], HQ * D, rows, HQ, self.cache[i], self.p.batch, D ** -0.5, b.DOMINO_MASK_TREE,
                                         self.parent, N, self.out[i], HQ * D, self.lse[i], self.ws, self.ws.numel(), s) == 0
        assert b.domino_verify_tree_greedy(self.logits, self.parent, self.token, self.B, N, V, self.best, self.nodes, self.count,
                                           self.bonus, s) == 0
        assert b.domino_cache_commit(self.cache[0], self.p.batch, LAYERS, self.p.layer_stride, self.nodes, self.count, N, self.new_len,
                                     s) == 0

    def check(self):
        """Against the accepted tokens decoded one after the other on a cache of their own."""
        torch.cuda.synchronize()
        assert b.domino_check_status(self.ws, None) == 0
        for i in range(self.B):
            path = self.nodes[i, :int(self.count[i])].tolist()
            first = self.p.kv[i] - N - 1  # the anchor's place
            assert int(self.new_len[i]) == first + 1 + len(path)
            tokens = [int(self.anchor[i])] + [int(self.token[i, a]) for a in path]
            for layer in range(LAYERS):
                x = self.qkv[layer][tokens]
                q, k, v = (t.unflatten(1, (-1, D)) for t in x.split((HQ * D, HKV * D, HKV * D), 1))
                pos = torch.arange(first, first + len(tokens), device=DEV)
                kr, ktol = ref.rotate(k, pos, self.freq, D, b.DOMINO_ROPE_HALF, 1.0)
                at, off = self.p.slots(i, first + len(tokens))
                have = self.p.k[layer][at, off]
                assert bool(((have[first:].double() - kr).abs() <= ktol).all())
                assert torch.equal(self.p.v[layer][at, off][first:], v)
                # the attention of the path's nodes, on the keys as kept
                own = ref.Paged([first + len(tokens)], [len(tokens)], HKV, D, b.DOMINO_BF16, PAGE, seed=1)
                a2, o2 = own.slots(0, first + len(tokens))
                own.k[0, a2, o2], own.v[0, a2, o2] = have, self.p.v[layer][at, off]
                r = [i * (N + 1)] + [i * (N + 1) + 1 + a for a in path]
                want, wl, tol, ltol = ref.attend(own, self.q[layer][r], D ** -0.5, b.DOMINO_MASK_CAUSAL)
                assert bool(((self.out[layer][r].double() - want).abs() <= tol).all())
                assert bool(((self.lse[layer][r].double() - wl).abs() <= ltol).all())

    def steer(self):
        """Logits that accept a path: at each node the token of its last child."""
        for i in range(self.B):
            for node in range(-1, N):
                kids = [c for c in range(N) if self.parent_host[i][c] == node]
                if kids:
                    self.logits[i * (N + 1) + 1 + node, int(self.token[i, kids[-1]])] = 50.0


def test_a_step_of_every_layer():
    s = Server([100, 3, 257], seed=3)
    s.steer()
    s.run()
    s.check()
    assert int(s.count.max()) >= 2


def test_the_step_in_a_graph_and_the_next_one_on_what_it_left():
    s = Server([90, 31], seed=5)
    s.steer()
    s.run()  # the libraries' first calls outside the capture
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    other = Server([90, 31], seed=5)
    s.p.k_store.copy_(other.p.k_store)
    s.p.v_store.copy_(other.p.v_store)
    graph.replay()
    s.check()
    # the next step: its new tokens follow what was accepted (the table has room for them where pages do)
    done = s.new_len.clone()
    s.p.kv = [min(int(n) + N + 1, k) for n, k in zip(done, s.p.kv)]
    s.p.kv_len.copy_(torch.tensor(s.p.kv, dtype=torch.int32))
    s.anchor.copy_(s.bonus)
    graph.replay()
    s.check()


def test_timing_kinds_of_the_paged_operators():
    s = Server([40], seed=7)
    s.run()
    torch.cuda.synchronize()
    assert b.domino_timing_begin(64) == 0
    s.run()
    torch.cuda.synchronize()
    kinds = b.domino_timing_end()
    assert kinds["rope"][1] == LAYERS and kinds["attend"][1] == LAYERS and kinds["cache_commit"][1] == 1
    assert kinds["attend"][0] > 0
