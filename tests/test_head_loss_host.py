"""The head's losses without a GPU: the oracle against closed forms and differences, and what the entry points refuse."""
import ctypes as C
import math

import pytest
import torch

import paper_2603_18464_amd as P
from oracle.loss_oracle import Loss, target
from paper_2603_18464_amd import binding as B


def small(T=5, d=8, V=11, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(T, d, generator=g, dtype=torch.float64), torch.randn(V, d, generator=g, dtype=torch.float64), g


# ---- the oracle -------------------------------------------------------------------------------------------------
def test_uniform_logits():
    h, W = torch.ones(2, 4, dtype=torch.float64), torch.full((7, 4), 0.25, dtype=torch.float64)
    o = Loss(h, W, target(7, labels=torch.tensor([3, -1])))
    assert abs(float(o.lse[0]) - 1.0 - math.log(7)) < 1e-12
    assert torch.allclose(o.loss, torch.tensor([math.log(7), 0.0], dtype=torch.float64))


def test_a_teacher_of_one_entry_is_a_label_and_equal_ids_add_up():
    h, W, _ = small()
    ids = torch.tensor([[4, -1, 4], [0, 10, 11], [2, 2, 3], [-5, 20, 11], [7, 7, 7]], dtype=torch.int32)
    logits = torch.tensor([[1.0, 9.0, 2.0], [0.5, -math.inf, 3.0], [1.0, 1.0, 1.0], [0.0, 0.0, 0.0], [1.0, 2.0, 3.0]])
    r = target(11, top_ids=ids, top_logits=logits)
    want = torch.zeros(5, 11, dtype=torch.float64)
    want[0, 4], want[1, 0], want[2, 2], want[2, 3], want[4, 7] = 1, 1, 2 / 3, 1 / 3, 1
    assert torch.allclose(r, want)
    one, two = Loss(h, W, r), Loss(h, W, target(11, labels=torch.tensor([4, 0, 2, -1, 7])))
    assert torch.allclose(one.loss[[0, 1, 4]], two.loss[[0, 1, 4]]) and one.loss[3] == 0


@pytest.mark.parametrize("tau", [1.0, 0.7])
def test_gradients_are_those_of_the_formula_by_differences(tau):
    h, W, gen = small()
    r = target(11, top_ids=torch.tensor([[1, 2], [3, 3], [-1, -1], [0, 10], [5, 6]]), top_logits=torch.randn(5, 2, generator=gen), tau=tau)
    g = torch.randn(5, generator=gen, dtype=torch.float64)

    def value(h, W):
        return float((Loss(h, W, r, tau).loss * g).sum())

    import oracle.loss_oracle as O
    O.OUT[torch.float64] = 0.0
    (gh, _), (gw, _) = Loss(h, W, r, tau).grad_bounds(g)
    del O.OUT[torch.float64]
    eps = 1e-6
    for x, grad, which in ((h, gh, 0), (W, gw, 1)):
        for i in range(x.shape[0]):
            for j in range(0, x.shape[1], 3):
                up, dn = x.clone(), x.clone()
                up[i, j] += eps
                dn[i, j] -= eps
                diff = (value(*((up, W) if which == 0 else (h, up))) - value(*((dn, W) if which == 0 else (h, dn)))) / (2 * eps)
                assert abs(diff - float(grad[i, j])) < 1e-8


# ---- refusals -----------------------------------------------------------------------------------------------------
def rows(**kw):
    a = dict(hidden=256, head=512, ld_hidden=64, ld_head=64, n_rows=3, d_model=64, vocab=100, dtype=B.VLA_BF16, temperature=0.0)
    a.update(kw)
    return B.vla_head_rows(**a)


def calls(r, work=4096, size=1 << 40, top=4, **null):
    """Status of the four calls.  Nothing is enqueued by a call that is refused, so any address does."""
    L = B.lib()
    p = lambda name: None if name in null else 1024   # noqa: E731
    ref = C.byref(r) if r is not None else None
    return [L.vla_token_loss(ref, p("target"), p("out"), p("out"), work, size, None),
            L.vla_token_loss_grad(ref, p("target"), p("lse"), p("lse"), p("out"), p("out"), work, size, None),
            L.vla_distill_loss(ref, p("target"), p("target"), top, p("out"), p("out"), work, size, None),
            L.vla_distill_loss_grad(ref, p("target"), p("target"), top, p("lse"), p("lse"), p("out"), p("out"), work, size, None)]


@pytest.mark.parametrize("bad,code", [
    (dict(n_rows=0), -3), (dict(n_rows=-1), -3), (dict(n_rows=(1 << 18) + 1), -3), (dict(vocab=0), -3), (dict(vocab=(1 << 20) + 1), -3),
    (dict(d_model=0), -3), (dict(d_model=60), -3), (dict(d_model=(1 << 15) + 8, ld_hidden=1 << 16, ld_head=1 << 16), -3),
    (dict(dtype=2), -2), (dict(dtype=-1), -2), (dict(temperature=-1.0), -3), (dict(temperature=math.nan), -3),
    (dict(temperature=math.inf), -3), (dict(temperature=1e-39), -3), (dict(temperature=2.0 ** -41), -3), (dict(temperature=2.0 ** 41), -3),
    (dict(hidden=None), -1), (dict(head=None), -1), (dict(ld_hidden=56), -3), (dict(ld_head=0), -3),
    (dict(ld_head=65), -3), (dict(ld_hidden=68), -3), (dict(hidden=258), -3), (dict(head=520), -3),
    (dict(dtype=B.VLA_F32, d_model=62), -3), (dict(dtype=B.VLA_F32, ld_head=66), -3),
])
def test_rows_that_are_refused(bad, code):
    assert calls(rows(**bad)) == [code] * 4


def test_other_refusals():
    ok = rows()
    assert calls(None) == [-1] * 4
    assert calls(ok, work=None) == [-1] * 4
    assert calls(ok, target=0) == [-1] * 4
    assert calls(ok, out=0) == [-1] * 4                                  # (of a gradient: both)
    assert calls(ok, lse=0)[1::2] == [-1] * 2
    assert calls(ok, work=4096 + 128) == [-3] * 4
    assert calls(ok, size=1000) == [-4] * 4
    assert calls(ok, top=0)[2:] == calls(ok, top=1025)[2:] == [-3] * 2
    L = B.lib()
    for grad in (0, 1):                                                  # one byte less than the size that is named
        n = C.c_size_t()
        assert L.vla_loss_workspace(C.byref(ok), 4, grad, C.byref(n)) == 0
        assert calls(ok, size=n.value - 1)[2 + grad] == -4
    assert L.vla_loss_workspace(C.byref(ok), 4, 0, None) == -1
    assert L.vla_loss_workspace(None, 4, 0, C.byref(n)) == -1
    assert L.vla_loss_workspace(C.byref(ok), -1, 0, C.byref(n)) == L.vla_loss_workspace(C.byref(ok), 1025, 0, C.byref(n)) == -3


def test_workspace_does_not_hold_the_logits_of_large_calls():
    big = rows(n_rows=1 << 16, d_model=64, vocab=1 << 17)
    assert P.vla_loss_workspace(big, 0, True) < (1 << 16) * (1 << 17) * 2 / 16


def test_tensors_that_are_refused():
    h, W, y = torch.zeros(3, 64), torch.zeros(10, 64), torch.zeros(3, dtype=torch.int32)
    for hh, ww, code in ((h.double(), W.double(), -2), (h, W.bfloat16(), -2), (h, W[:, :32], -3), (h[0], W, -3), (h, W, -3)):
        with pytest.raises(P.VlaError) as e:                             # (the last: not on a GPU)
            P.token_loss(hh, ww, y)
        assert e.value.code == code


def test_rows_of_a_context_without_a_call():
    import workloads as W
    wl = W.get_workload("C1")
    L = B.lib()
    assert L.vla_action_hidden(None, 1, 1, 256, None) == -1
    ctx = B.vla_create(B.make_config(wl.shape, 4, 64, 256))
    assert L.vla_action_hidden(ctx, 1, 1, 256, None) == -5               # nothing is bound
    B.vla_destroy(ctx)
