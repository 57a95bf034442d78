"""Argument errors of the entry points on rows of logits come back before anything is enqueued (CPU)."""
import pytest

from paper_2605_29707_gb300 import binding as b

BAD, UNSUP = b.DOMINO_ERR_INVALID_ARG, b.DOMINO_ERR_UNSUPPORTED
P = 1 << 12  # an aligned non-null stand-in; never dereferenced because validation fails first
MAX_V = 1 << 19


def _sample(**kw):
    a = dict(logits=P, dtype=b.DOMINO_F32, row_stride=100, temperature=P, top_k=P, top_p=P, min_p=P, uniforms=P, rows=2,
             V=100, tokens=P, logp=P)
    a.update(kw)
    return b.domino_sample_filtered(**a)


def _verify(**kw):
    a = dict(target_logits=P, dtype=b.DOMINO_F32, row_stride=100, tree_parent=P, tree_token=P, temperature=P, top_k=P,
             top_p=P, min_p=P, uniforms=P, B=2, N=3, V=100, row_sample=P, row_logp=P, accepted_nodes=P,
             accepted_count=P, bonus_token=P)
    a.update(kw)
    return b.domino_verify_tree_filtered(**a)


def _distill(part, **kw):
    a = dict(logits=P, dtype=b.DOMINO_F32, row_stride=100, teacher_ids=P, teacher_scores=P, weights=P, temperature=1.0,
             mode=b.DOMINO_DISTILL_TAIL, rows=2, V=100, kt=4)
    if part != "grad":
        a["loss"] = P
    a["lse"] = P
    if part != "loss":
        a.update(grad_loss=P, dlogits=2 * P, grad_stride=100)
    a.update(kw)
    return {"loss": b.domino_distill_loss, "grad": b.domino_distill_grad, "both": b.domino_distill_loss_grad}[part](**a)


ROWS = [(dict(rows=0), BAD), (dict(rows=-1), BAD), (dict(V=0), BAD), (dict(row_stride=99), BAD),
        (dict(row_stride=-100), BAD), (dict(row_stride=(1 << 62)), BAD), (dict(rows=1 << 28), BAD),
        (dict(dtype=3), UNSUP), (dict(dtype=-1), UNSUP), (dict(V=MAX_V + 1, row_stride=MAX_V + 1), UNSUP)]


@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(logits=None), BAD), (dict(logits=P + 2), BAD), (dict(logits=P + 1, dtype=b.DOMINO_BF16), BAD),
    (dict(uniforms=None), BAD), (dict(tokens=None), BAD), (dict(tokens=P + 2), BAD), (dict(logp=P + 1), BAD),
    (dict(temperature=P + 2), BAD), (dict(top_k=P + 2), BAD), (dict(top_p=P + 2), BAD), (dict(min_p=P + 2), BAD),
    (dict(uniforms=P + 2), BAD)])
def test_sample_filtered_refusals(kw, code):
    assert _sample(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), BAD), (dict(N=-1), BAD), (dict(N=(1 << 20) + 1), BAD), (dict(V=0), BAD), (dict(row_stride=99), BAD),
    (dict(B=1 << 27, N=3), BAD), (dict(dtype=7), UNSUP), (dict(V=MAX_V + 1, row_stride=MAX_V + 1), UNSUP),
    (dict(target_logits=None), BAD), (dict(uniforms=None), BAD), (dict(row_sample=None), BAD),
    (dict(accepted_count=None), BAD), (dict(bonus_token=None), BAD), (dict(tree_parent=None), BAD),
    (dict(tree_token=None), BAD), (dict(accepted_nodes=None), BAD), (dict(tree_token=P + 2), BAD),
    (dict(row_logp=P + 2), BAD)])
def test_verify_filtered_refusals(kw, code):
    assert _verify(**kw) == code


@pytest.mark.parametrize("part", ["loss", "grad", "both"])
@pytest.mark.parametrize("kw,code", ROWS + [
    (dict(logits=None), BAD), (dict(logits=P + 2), BAD), (dict(teacher_ids=None), BAD), (dict(teacher_scores=None), BAD),
    (dict(kt=0), BAD), (dict(kt=257), UNSUP), (dict(mode=2), BAD), (dict(mode=-1), BAD), (dict(temperature=0.0), BAD),
    (dict(temperature=-1.0), BAD), (dict(temperature=float("nan")), BAD), (dict(temperature=float("inf")), BAD),
    (dict(temperature=1e-40), BAD), (dict(weights=P + 2), BAD), (dict(teacher_ids=P + 2), BAD)])
def test_distill_refusals(part, kw, code):
    assert _distill(part, **kw) == code


def test_distill_output_refusals():
    assert _distill("loss", loss=None) == BAD
    assert _distill("both", loss=None) == BAD
    for part in ("grad", "both"):
        assert _distill(part, dlogits=None) == BAD
        assert _distill(part, grad_stride=99) == BAD
        assert _distill(part, dlogits=P + 2) == BAD
        assert _distill(part, dlogits=P, grad_stride=104) == BAD  # in place, with another stride
    assert _distill("grad", lse=None) == BAD


@pytest.mark.parametrize("part", ["loss", "grad", "both"])
def test_distill_refuses_temperatures_whose_base_2_scale_overflows(part):
    """1 / 3.5e-39 is finite in fp32, log2(e) / 3.5e-39 is not."""
    assert _distill(part, temperature=3.5e-39) == BAD
