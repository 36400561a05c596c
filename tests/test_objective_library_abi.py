"""Host side of the LM head's other objectives: symbols, sizes, refusals.  No kernel is launched here."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, BAD_M, WORKSPACE, ALIGNMENT, NO_DEVICE, ARGUMENT = -1, -2, -3, -4, -5, -7, -8
S, D, V, K, M = 100, 64, 1000, 20, 2


@pytest.fixture(scope="module")
def lib():
    import paper_2407_15892_amd as m
    if not os.path.exists(m.binding.LIB_PATH):
        from paper_2407_15892_amd.build import build
        build()
    from paper_2407_15892_amd import objective_binding
    return objective_binding._lib()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mst_objective.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(mst_[a-z_]+)\s*\(", text))
    assert names == {"mst_objective_bytes", "mst_lmhead_wce_fwd", "mst_lmhead_wce_bwd", "mst_lmhead_distill_fwd", "mst_lmhead_distill_bwd"}
    assert all(hasattr(lib, n) for n in names)


def test_bytes(lib):
    import paper_2407_15892_amd as mst
    plain = mst.mst_workspace_bytes(8192, 4096, 128256, 8)
    fwd, bwd, saved = mst.mst_objective_bytes(8192, 4096, 128256, 8)
    assert bwd == plain[1] and plain[0] < fwd <= plain[0] + 8 * 8192 + 512 and saved <= 16 * 8192 + 512
    fwd, bwd, saved = mst.mst_objective_bytes(8192, 4096, 128256, 8, 64)
    assert bwd == plain[1] and fwd < bwd and saved <= (24 + 8 * 64) * 8192 + 2048
    # M is the largest number of mini-sequences: fewer where one of them is less than 512 MiB of fp32 logits
    assert mst.mst_objective_bytes(8192, 4096, 128256, 31, 64) == mst.mst_objective_bytes(8192, 4096, 128256, 8, 64)
    for S_, V_, M_, most in ((5003, 32003, 19, 2), (100, 1000, 50, 1), (16384, 256000, 16, 16), (16384, 256000, 2000, 32), (1 << 17, 32768, 64, 32)):
        c = -(-S_ // most)
        assert mst.mst_objective_bytes(S_, 64, V_, M_)[1] == c * (-(-V_ // 8) * 8) * 4
    # the next group of mini-sequences takes the room of the one before
    assert mst.mst_objective_bytes(1 << 17, 4096, 128256, 128, 64)[0] < 3 * mst.mst_objective_bytes(1 << 15, 4096, 128256, 32, 64)[0]
    for args, status in (((0, 64, 10, 1, 0), SHAPE), ((8, 63, 10, 1, 0), SHAPE), ((8, 64, 10, 9, 0), BAD_M), ((8, 64, 10, 1, 257), SHAPE),
                         ((8, 64, 10, 1, -1), SHAPE)):
        with pytest.raises(mst.MstError) as e:
            mst.mst_objective_bytes(*args)
        assert e.value.status == status


class Fwd:
    """Arguments of a forward call, with addresses that nothing reads: far apart and aligned."""
    names = ["H", "W", "labels", "weights", "index", "logits", "type", "lse", "S", "d", "V", "K", "ignore", "M", "cap", "alpha", "beta", "T", "divisor",
             "ws", "ws_bytes", "saved", "saved_bytes", "loss", "nll", "kd", "n", "stream"]

    def __init__(self, **over):
        import paper_2407_15892_amd as mst
        fwd, _, saved = mst.mst_objective_bytes(S, D, V, M, K)
        at = iter(range(1 << 30, 1 << 40, 1 << 28))
        self.a = dict(zip(self.names, [next(at) for _ in range(6)] + [1, next(at), S, D, V, K, -100, M, 0.0, 0.5, 0.5, 2.0, 0, next(at), fwd, next(at),
                                                                  saved] + [next(at) for _ in range(4)] + [None]))
        self.a.update(over)

    def distill(self, lib):
        return lib.mst_lmhead_distill_fwd(*(self.a[n] for n in self.names))

    def wce(self, lib):
        a = self.a
        return lib.mst_lmhead_wce_fwd(a["H"], a["W"], a["labels"], a["weights"], a["S"], a["d"], a["V"], a["ignore"], a["M"], a["cap"], a["alpha"],
                                      a["divisor"], a["ws"], a["ws_bytes"], a["saved"], a["saved_bytes"], a["loss"], a["nll"], a["kd"], a["n"], None)


NAN, INF = float("nan"), float("inf")
BOTH = [(dict(S=0), SHAPE), (dict(V=0), SHAPE), (dict(d=60), SHAPE), (dict(M=0), BAD_M), (dict(M=S + 1), BAD_M), (dict(H=None), NULL), (dict(W=None), NULL),
        (dict(loss=None), NULL), (dict(ws=None), WORKSPACE), (dict(ws_bytes=100), WORKSPACE), (dict(saved_bytes=100), WORKSPACE),
        (dict(H=(1 << 30) + 8), ALIGNMENT), (dict(ws=(1 << 33) + 16), ALIGNMENT), (dict(saved=(1 << 34) + 16), ALIGNMENT), (dict(weights=(1 << 34) + 2), ALIGNMENT),
        (dict(n=(1 << 35) + 4), ALIGNMENT), (dict(cap=-1.0), ARGUMENT), (dict(cap=NAN), ARGUMENT), (dict(cap=INF), ARGUMENT), (dict(cap=1e-6), ARGUMENT),
        (dict(alpha=NAN), ARGUMENT), (dict(alpha=INF), ARGUMENT), (dict(divisor=-1), ARGUMENT), (dict(nll=1 << 30), ARGUMENT),
        (dict(loss=(1 << 30) + 64), ARGUMENT), (dict(), "device"), (dict(saved=None, saved_bytes=0), "device"), (dict(weights=None, nll=None, kd=None, n=None), "device")]
DISTILL = [(dict(K=0), SHAPE), (dict(K=257), SHAPE), (dict(index=None), NULL), (dict(logits=None), NULL), (dict(type=2), ARGUMENT), (dict(T=0.0), ARGUMENT),
           (dict(T=NAN), ARGUMENT), (dict(T=1000.0), ARGUMENT), (dict(beta=INF), ARGUMENT), (dict(labels=None), ARGUMENT),
           (dict(labels=None, alpha=0.0), ARGUMENT), (dict(labels=None, alpha=0.0, nll=None), "device"), (dict(lse=(1 << 34) + 2), ALIGNMENT),
           (dict(logits=(1 << 34) + 2), ALIGNMENT), (dict(logits=(1 << 40) + 2, type=0), "device"), (dict(lse=None), "device")]


def _expected(status):
    import torch
    if status == "device":
        if torch.cuda.is_available():
            pytest.skip("would be launched")
        return NO_DEVICE
    return status


@pytest.mark.parametrize("over,status", BOTH + DISTILL, ids=str)
def test_distill_forward_refuses(lib, over, status):
    assert Fwd(**over).distill(lib) == _expected(status)


@pytest.mark.parametrize("over,status", BOTH + [(dict(labels=None), NULL)], ids=str)
def test_wce_forward_refuses(lib, over, status):
    assert Fwd(**over).wce(lib) == _expected(status)


BWD = [(dict(H=None), NULL), (dict(dW=None), NULL), (dict(saved=None), NULL), (dict(saved_bytes=1000), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE),
       (dict(ws=None), WORKSPACE), (dict(dH=(1 << 32) + 8), ALIGNMENT), (dict(dH=1 << 30), ARGUMENT), (dict(dW=(1 << 30) + 16), ARGUMENT), (dict(M=0), BAD_M),
       (dict(d=4), SHAPE), (dict(), "device")]


@pytest.mark.parametrize("k", [0, K])
@pytest.mark.parametrize("over,status", BWD, ids=str)
def test_backward_refuses(lib, k, over, status):
    import paper_2407_15892_amd as mst
    _, bwd, saved = mst.mst_objective_bytes(S, D, V, M, k)
    a = dict(H=1 << 30, W=1 << 31, S=S, d=D, V=V, M=M, saved=1 << 33, saved_bytes=saved, ws=1 << 34, ws_bytes=bwd, dH=1 << 35, dW=1 << 36)
    a.update(over)
    tail = (a["M"], 1.0, a["saved"], a["saved_bytes"], a["ws"], a["ws_bytes"], a["dH"], a["dW"], None)
    head = (a["H"], a["W"], a["S"], a["d"], a["V"])
    got = lib.mst_lmhead_distill_bwd(*head, k, *tail) if k else lib.mst_lmhead_wce_bwd(*head, *tail)
    assert got == _expected(status)


def test_backward_of_distillation_needs_entries(lib):
    assert lib.mst_lmhead_distill_bwd(1 << 30, 1 << 31, S, D, V, 0, M, 1.0, 1 << 33, 1 << 20, 1 << 34, 1 << 24, 1 << 35, 1 << 36, None) == SHAPE


def test_binding_refuses_tensors_of_another_kind():
    import torch
    import paper_2407_15892_amd as mst
    bf, f32 = torch.bfloat16, torch.float32
    t = dict(H=torch.zeros(S, D, dtype=bf), W=torch.zeros(V, D, dtype=bf), teacher_index=torch.zeros(S, K, dtype=torch.int32),
             teacher_logits=torch.zeros(S, K), M=M, workspace=torch.zeros(1 << 24, dtype=torch.uint8), loss=torch.zeros(1))
    bad = [(dict(H=t["H"].float()), ARGUMENT), (dict(W=torch.zeros(V, D + 8, dtype=bf)), SHAPE), (dict(H=t["H"].t()), ARGUMENT),
           (dict(H=torch.zeros(D, S, dtype=bf).t()), ARGUMENT), (dict(teacher_index=t["teacher_index"].long()), ARGUMENT),
           (dict(teacher_logits=torch.zeros(S, K + 1)), SHAPE), (dict(teacher_logits=torch.zeros(S, K, dtype=torch.float16)), ARGUMENT),
           (dict(labels=torch.zeros(S, dtype=torch.int64)), ARGUMENT), (dict(weights=torch.zeros(S, dtype=bf)), ARGUMENT),
           (dict(weights=torch.zeros(2 * S)[::2]), ARGUMENT), (dict(kd=torch.zeros(S + 1)), SHAPE), (dict(teacher_lse=torch.zeros(S, 1)), SHAPE),
           (dict(loss=None), NULL), (dict(loss=torch.zeros(2)), SHAPE), (dict(M=1 << 32), ARGUMENT), (dict(divisor=1 << 64), ARGUMENT),
           (dict(teacher_index=None), SHAPE), (dict(H=None), SHAPE), (dict(n_valid=torch.zeros(1, dtype=torch.int32)), ARGUMENT), (dict(), NO_DEVICE)]
    for over, status in bad:
        with pytest.raises(mst.MstError) as e:
            mst.mst_lmhead_distill_fwd(**{**t, **over})
        assert e.value.status == status, over
    dH, dW, saved = torch.zeros(S, D, dtype=bf), torch.zeros(V, D), torch.zeros(1 << 20, dtype=torch.uint8)
    for over, status in [(dict(dW=dW.to(bf)), ARGUMENT), (dict(dH=torch.zeros(S + 1, D, dtype=bf)), SHAPE), (dict(), NO_DEVICE)]:
        a = {**dict(dH=dH, dW=dW), **over}
        with pytest.raises(mst.MstError) as e:
            mst.mst_lmhead_wce_bwd(t["H"], t["W"], M, 1.0, saved, t["workspace"], a["dH"], a["dW"])
        assert e.value.status == status, over


@pytest.mark.parametrize("s,k,status", [(1 << 26, 1, SHAPE), ((1 << 26) - 1, 64, 0), (1 << 24, 256, SHAPE), ((1 << 24) - 1, 256, 0), (1 << 26, 0, 0)])
def test_entries_of_more_rows_than_a_launch_has_threads(lib, s, k, status):
    assert lib.mst_objective_bytes(s, 8, 8, 1, k, None, None, None) == status
