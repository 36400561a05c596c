"""The oracle of the LM head's other objectives, pinned to the plain cross-entropy's oracle, to a library's functions and their
differentiation, to finite differences and to closed forms."""
import numpy as np
import pytest
import torch

from oracle import lmhead_ce_oracle as ce
from oracle import objective_oracle as orc

S, D, V, K = 7, 16, 23, 5


def _inputs(seed=0, sigma=1.0):
    rng = np.random.default_rng(seed)
    H, W = rng.standard_normal((S, D)), rng.standard_normal((V, D)) * sigma / 4
    labels = rng.integers(0, V, S)
    labels[2] = -100
    index = np.argsort(-rng.standard_normal((S, V)), axis=1)[:, :K]
    index[1, 2] = -1
    index[4] = -1
    index[5, 4] = index[5, 0]                      # twice
    t = rng.standard_normal((S, V)) * 2
    logits = np.take_along_axis(t, np.maximum(index, 0), 1)
    return H, W, labels, index, logits, t, rng


def test_plain_cross_entropy():
    H, W, labels, *_ = _inputs()
    r, ref = orc.objective(H, W, labels, grad_loss=1.3), ce.lmhead_ce(H, W, labels, grad_loss=1.3)
    assert r["n"] == ref["n_valid"]
    np.testing.assert_allclose(r["loss"], ref["loss"], rtol=1e-13)
    np.testing.assert_allclose(r["dH"], ref["dH"], rtol=1e-11, atol=1e-15)
    np.testing.assert_allclose(r["dW"], ref["dW"], rtol=1e-11, atol=1e-15)


@pytest.mark.parametrize("cap,z_coef", [(0.0, 0.0), (0.7, 0.0), (3.0, 0.2)])
def test_weighted_capped_cross_entropy_against_a_library(cap, z_coef):
    H, W, labels, *_, rng = _inputs()
    w = rng.uniform(-1, 2, S)
    w[3] = 0
    r = orc.objective(H, W, labels, weights=w, softcap=cap, z_coef=z_coef, divisor=11)
    Ht, Wt = torch.tensor(H, requires_grad=True), torch.tensor(W, requires_grad=True)
    y = Ht @ Wt.t()
    y = cap * torch.tanh(y / cap) if cap else y
    nll = torch.nn.functional.cross_entropy(y, torch.tensor(labels), reduction="none", ignore_index=-100)
    valid = torch.tensor(labels != -100)
    loss = (torch.tensor(w) * (nll + z_coef * torch.logsumexp(y, 1) ** 2 * valid)).sum() / 11
    loss.backward()
    np.testing.assert_allclose(r["loss"], loss.item(), rtol=1e-12)
    np.testing.assert_allclose(r["nll"], nll.detach().numpy(), rtol=1e-12, atol=1e-14)
    np.testing.assert_allclose(r["dH"], Ht.grad.numpy(), rtol=1e-10, atol=1e-14)
    np.testing.assert_allclose(r["dW"], Wt.grad.numpy(), rtol=1e-10, atol=1e-14)


@pytest.mark.parametrize("T", [1.0, 2.5])
@pytest.mark.parametrize("tail", [False, True])
def test_all_entries_are_the_full_divergence(T, tail):
    H, W, *_ , t, _ = _inputs()
    index = np.tile(np.arange(V)[::-1], (S, 1))
    lse = np.array([orc._lse(x / T) for x in t]) if tail else None
    r = orc.objective(H, W, label_coef=0.0, teacher_index=index, teacher_logits=t[:, ::-1], teacher_lse=lse, teacher_coef=0.6, temperature=T)
    Ht = torch.tensor(H, requires_grad=True)
    p, q = torch.log_softmax(Ht @ torch.tensor(W).t() / T, 1), torch.log_softmax(torch.tensor(t) / T, 1)
    kd = torch.nn.functional.kl_div(p, q, reduction="none", log_target=True).sum(1)
    (0.6 * T * T * kd.mean()).backward()
    np.testing.assert_allclose(r["kd"], kd.detach().numpy(), rtol=1e-12)
    np.testing.assert_allclose(r["dH"], Ht.grad.numpy(), rtol=1e-10, atol=1e-14)


def test_rest_is_a_class_of_its_own():
    """With a rest the divergence is that of distributions over the entries and one class for all others."""
    H, W, _, index, _, t, _ = _inputs()
    T, s = 2.0, 0
    lse = np.array([orc._lse(x / T) for x in t])
    logits = np.take_along_axis(t, np.maximum(index, 0), 1)
    r = orc.objective(H, W, teacher_index=index, teacher_logits=logits, teacher_lse=lse, teacher_coef=1.0, temperature=T)
    p, q = np.exp(r["Z"][s] / T - orc._lse(r["Z"][s] / T)), np.exp(t[s] / T - lse[s])
    v = index[s]
    p5, q5 = np.append(p[v], 1 - p[v].sum()), np.append(q[v], 1 - q[v].sum())
    np.testing.assert_allclose(r["kd"][s], (q5 * np.log(q5 / p5)).sum(), rtol=1e-10)
    # and 0, without a gradient, where the student is the teacher
    r = orc.objective(H, W, teacher_index=index, teacher_logits=np.take_along_axis(r["Z"], np.maximum(index, 0), 1),
                      teacher_lse=np.array([orc._lse(x / T) for x in r["Z"]]), teacher_coef=1.0, temperature=T)
    assert np.abs(r["kd"]).max() < 1e-13 and np.abs(r["G"]).max() < 1e-13


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("cap", [0.0, 1.5])
def test_gradients_against_differences(tail, cap):
    H, W, labels, index, logits, t, rng = _inputs()
    T = 1.7
    kw = dict(weights=rng.uniform(0, 2, S), softcap=cap, label_coef=0.4, teacher_index=index, teacher_logits=logits,
              teacher_lse=np.array([orc._lse(x / T) for x in t]) if tail else None, teacher_coef=0.8, temperature=T, grad_loss=1.0)
    r = orc.objective(H, W, labels, **kw)
    assert r["n"] == S                              # row 2 has a teacher, row 4 a label
    e = 1e-5
    for X, g in ((H, r["dH"]), (W, r["dW"])):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in X.shape)
            keep = X[i]
            X[i] = keep + e
            up = orc.objective(H, W, labels, **kw)["loss"]
            X[i] = keep - e
            down = orc.objective(H, W, labels, **kw)["loss"]
            X[i] = keep
            np.testing.assert_allclose(g[i], (up - down) / (2 * e), rtol=1e-5, atol=1e-9)


def test_rows_that_do_not_count():
    H, W, labels, index, logits, *_ = _inputs()
    r = orc.objective(H, W, np.full(S, -100), teacher_index=np.full_like(index, -1), teacher_logits=logits, teacher_coef=1.0)
    assert r["n"] == 0 and r["loss"] == 0 and not r["dW"].any()
    logits[0] = -np.inf                              # a teacher that gives nothing to its entries
    r = orc.objective(H, W, None, label_coef=0.0, teacher_index=index, teacher_logits=logits, teacher_coef=1.0)
    assert r["n"] == S - 2 and not r["G"][0].any()
    with pytest.raises(ValueError):
        orc.objective(H, W, labels, teacher_index=np.where(index == index[0, 0], V, index), teacher_logits=logits, teacher_coef=1.0)


def test_an_index_that_comes_twice_counts_once():
    _, _, _, index, logits, _, _ = _inputs()
    v, t = orc.teacher_of_row(index[5], logits[5], V)
    assert list(v) == list(index[5, :4]) and list(t) == list(logits[5, :4])
