"""The operators on rows of logits as a server and a trainer run them together, on the trees of a draft step: the
drafted tree is verified against a target that decodes with filters, the next token after the accepted path is drawn,
and the draft's logits are distilled towards the target's best tokens, on one stream and in one captured graph."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_29707_gb300 import binding as b, inputs
from paper_2605_29707_gb300.step import DraftStep
from tests import rows_reference as ref
from tests.test_gpu_distill import check as check_distill
from tests.test_gpu_sample_filtered import BORDER, DEV

pytestmark = pytest.mark.gpu

KT = 8


class Loop:
    """One sequence's cycle on fixed buffers: everything is enqueued by run() on the current stream."""

    def __init__(self, seed):
        self.wl = inputs.make_workload("tiny")
        c = self.c = self.wl.cfg
        self.step = DraftStep(self.wl.weights, c.B, c.K, c.H, c.V, c.k, c.N, Ds=c.Ds, R=c.R, device=DEV)
        self.hidden = torch.from_numpy(self.wl.hidden.view(np.int16)).view(torch.bfloat16).to(DEV)
        self.ids = torch.from_numpy(self.wl.prefix_ids).to(DEV)
        B, N, V, K = c.B, c.N, c.V, c.K
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.target = (torch.randn((B * (N + 1), V), generator=g, device=DEV) * 3).bfloat16()
        self.uniforms = torch.rand((B, N + 1), generator=g, device=DEV)
        self.next_u = torch.rand(B, generator=g, device=DEV)
        self.T, self.p = torch.full((B,), 0.8, device=DEV), torch.full((B,), 0.95, device=DEV)
        self.k = torch.full((B,), 50, dtype=torch.int32, device=DEV)
        w_lm = torch.from_numpy(self.wl.weights["w_lm"].view(np.int16)).view(torch.bfloat16).to(DEV)
        self.student = (self.hidden.reshape(B * K, -1).float() @ w_lm.float().t()).bfloat16()
        self.weights = torch.exp(-torch.arange(B * K, device=DEV) % K / 4.0)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.y, self.lp = torch.empty((B, N + 1), **i32), torch.empty((B, N + 1), device=DEV)
        self.nodes, self.count, self.bonus = torch.empty((B, N), **i32), torch.empty(B, **i32), torch.empty(B, **i32)
        self.next, self.loss = torch.empty(B, **i32), torch.empty(B * K, device=DEV)
        self.lse, self.grad = torch.empty((B * K, 2), device=DEV), torch.empty((B * K, V), dtype=torch.bfloat16, device=DEV)
        self.teacher_ids = torch.empty((B * K, KT), **i32)
        self.teacher_logp = torch.empty((B * K, KT), device=DEV)

    def run(self):
        c, st, s = self.c, self.step, torch.cuda.current_stream()
        V = c.V
        assert st.enqueue(self.hidden, self.ids) == 0
        assert b.domino_verify_tree_filtered(self.target, b.DOMINO_BF16, V, st.tree_parent, st.tree_token, self.T, self.k,
                                             self.p, None, self.uniforms, c.B, c.N, V, self.y, self.lp, self.nodes,
                                             self.count, self.bonus, s) == 0
        assert b.domino_sample_filtered(self.target, b.DOMINO_BF16, (c.N + 1) * V, self.T, self.k, self.p, None,
                                        self.next_u, c.B, V, self.next, None, s) == 0
        rows = c.B * c.K  # the target's best tokens after the anchor and the first nodes teach the block's positions
        lp, i = torch.log_softmax(self.target[:rows].float(), 1).topk(KT, dim=1)
        self.teacher_ids.copy_(i)
        self.teacher_logp.copy_(lp)
        assert b.domino_distill_loss_grad(self.student, b.DOMINO_BF16, V, self.teacher_ids, self.teacher_logp, self.weights,
                                          None, 1.0, b.DOMINO_DISTILL_TAIL, rows, V, KT, self.loss, self.lse, self.grad, V,
                                          s) == 0

    def check(self):
        torch.cuda.synchronize()
        c = self.c
        tree = self.step.outputs()
        x, u = self.target.double().cpu().numpy(), self.uniforms.cpu().numpy()
        T, p = float(np.float32(0.8)), float(np.float32(0.95))
        y = self.y.cpu().numpy()
        for r in range(c.N + 1):
            e, _, margin = ref.draw(x[r], u[0, r], T, 50, p)
            assert margin < BORDER or y[0, r] == e
        nodes, bonus = oracle.tree_walk(tree["tree_parent"][0], tree["tree_token"][0], y[0])
        assert int(self.count[0]) == len(nodes) and int(self.bonus[0]) == bonus
        assert self.nodes[0, :len(nodes)].tolist() == nodes.tolist()
        e, _, margin = ref.draw(x[0], float(self.next_u[0]), T, 50, p)
        assert margin < BORDER or int(self.next[0]) == e
        check_distill(self.student, b.DOMINO_BF16, self.teacher_ids.cpu(), self.teacher_logp.cpu(), 1.0,
                      b.DOMINO_DISTILL_TAIL, self.weights.cpu(), None, self.loss.cpu().double().numpy(), self.lse, self.grad)


def test_draft_verify_draw_and_distill():
    loop = Loop(5)
    # the target agrees with the draft at the first level: a child's token is its favourite
    loop.run()
    torch.cuda.synchronize()
    tree = loop.step.outputs()
    first = int(np.flatnonzero(tree["tree_parent"][0] == -1)[0])
    loop.target[0, int(tree["tree_token"][0][first])] = float(loop.target[0].amax()) + 8.0
    loop.run()
    loop.check()
    assert int(loop.count[0]) >= 1


def test_the_cycle_in_a_graph():
    loop = Loop(6)
    loop.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.run()
    other = Loop(7)
    loop.target.copy_(other.target)
    loop.uniforms.copy_(other.uniforms)
    loop.next_u.copy_(other.next_u)
    graph.replay()
    graph.replay()
    loop.check()


def test_timing_kinds_of_the_row_operators():
    """domino_timing_end reports the draws and the distillation under kinds of their own."""
    loop = Loop(8)
    loop.run()
    torch.cuda.synchronize()
    assert b.domino_timing_begin(64) == 0
    loop.run()
    torch.cuda.synchronize()
    kinds = b.domino_timing_end()
    assert kinds["sample_filtered"][1] == 2 and kinds["distill"][1] == 1
    assert kinds["sample_filtered"][0] > 0 and kinds["distill"][0] > 0
