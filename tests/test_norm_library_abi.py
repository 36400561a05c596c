"""CPU-side checks of the norm library: symbols, workspace, and every refusal before anything is launched."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, SHAPE, WORKSPACE, ALIGNMENT, NO_DEVICE, ARGUMENT = -1, -2, -4, -5, -7, -8


@pytest.fixture(scope="module")
def mst():
    import paper_2407_15892_amd as m
    if not all(os.path.exists(p) for p in (m.norm_binding.NORM_LIB_PATH, m.binding.LIB_PATH)):
        from paper_2407_15892_amd.build import build
        build()
    m.load_norm_library()
    return m


def test_every_declared_symbol_is_exported(mst):
    text = open(os.path.join(ROOT, "include", "mst_norm.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(mst_[a-z_]+)\s*\(", text))
    assert len(names) == 12
    lib = mst.load_norm_library()
    for n in sorted(names):
        assert hasattr(lib, n), n
    assert "gfx950" in mst.mst_norm_version()
    for code in range(-8, 1):
        assert mst.mst_strerror(code) != "unknown status"


def test_workspace_and_rows_of_the_backward(mst):
    seen = set()
    for d in (8, 64, 512, 520, 4096, 8192, 8200, 16384):
        for S in (1, 2, 3, 63, 64, 1000, 8192, 131072, (1 << 30) - 1):
            if S * d > 1 << 36:
                continue
            one = mst.mst_norm_workspace_bytes(S, d)
            assert mst.mst_norm_workspace_bytes(S, d, S) == mst.mst_norm_workspace_bytes(S, d, S + 5) == one
            for L, prenorm in [(L, p) for L in sorted({0, 1, 2, 7, 100, S // 3 + 1, S - 1 or 1, S, S + 3}) for p in (False, True)]:
                info = mst.mst_norm_bwd_info(S, d, L, prenorm)
                teams, rows, groups, whole = (info[k] for k in ("teams", "rows", "workgroups", "whole"))
                length = min(L, S) if L else S
                gates = -(-S // length)
                assert info["threads"] % 64 == 0 and info["threads"] <= 1024
                assert info["threads"] // teams * 8 * (1 if d <= 8192 else 2) >= d
                if whole:                                # every row of the gate has a team
                    assert gates > 1 and rows % length == 0
                    assert teams * groups * (rows // length - 1) < gates <= teams * groups * (rows // length)
                    assert teams * length * d < 1 << 29  # offsets of a workgroup's rows at a time
                else:
                    assert groups % gates == 0           # as many workgroups each
                    share = groups // gates
                    assert teams * rows * (share - 1) < length <= teams * rows * share
                sums = -(-2 * groups * d * 4 // 256) * 256 if groups > 1 else 256
                other = mst.mst_norm_bwd_info(S, d, L, not prenorm)["workgroups"]
                bytes_ = mst.mst_norm_workspace_bytes(S, d, L)           # that of the call which needs most
                assert bytes_ == max(sums, -(-2 * other * d * 4 // 256) * 256 if other > 1 else 256)
                assert bytes_ <= 1 << 28
                seen.add((groups == 1, bool(whole)))
    assert seen == {(True, False), (False, False), (True, True), (False, True)}
    for S, d in ((0, 8), (-1, 8), (1, 0), (1, 12), (1, 16392), (1 << 30, 8), ((1 << 23) + 1, 8192)):
        with pytest.raises(mst.MstError) as e:
            mst.mst_norm_workspace_bytes(S, d)
        assert e.value.status == SHAPE
    with pytest.raises(mst.MstError) as e:
        mst.mst_norm_workspace_bytes(8, 8, -1)
    assert e.value.status == ARGUMENT


# Addresses that are never read: every call below is refused first.  Far apart, so that nothing overlaps.
def P(i):
    return 0x100000 * (i + 1)


S, D = 64, 40
EPS = 1e-5
WS = 1 << 20


def call(lib, name, **change):
    """The C call with good arguments, some of them changed; those good ones would get as far as the device."""
    good = {
        "ckpt_pack": dict(X=P(0), type=0, S=S, d=D, codes=P(1), exps=P(2)),
        "ckpt_unpack": dict(codes=P(1), exps=P(2), S=S, d=D, X=P(0), type=0),
        "prenorm_fwd": dict(X=P(0), type=0, w=P(1), offset=0.0, eps=EPS, S=S, d=D, H=P(2), codes=P(3), exps=P(4)),
        "prenorm_rebuild": dict(codes=P(3), exps=P(4), w=P(1), offset=0.0, eps=EPS, S=S, d=D, H=P(2)),
        "prenorm_bwd": dict(dH=P(0), X=None, codes=P(1), exps=P(2), dres=P(3), type=0, w=P(4), offset=0.0, eps=EPS, S=S, d=D, ws=P(5),
                            size=WS, dX=P(7), dw=P(8)),
        "residual_fwd": dict(O=P(0), X=P(1), type=0, normalize=1, w=P(2), offset=0.0, eps=EPS, gate=P(3), gate_rows=10, scale=1.0, S=S, d=D,
                             Y=P(4), codes=P(5), exps=P(6)),
        "residual_bwd": dict(dY=P(0), type=0, O=None, codes=P(1), exps=P(2), normalize=1, w=P(3), offset=0.0, eps=EPS, gate=P(4),
                             gate_rows=10, scale=1.0, S=S, d=D, ws=P(5), size=WS, dO=P(7), dw=P(8), dgate=P(9)),
        "residual_prenorm_fwd": dict(O=P(0), X=P(1), type=0, normalize=1, w_post=P(2), gate=P(3), gate_rows=10, scale=1.0, w=P(4), offset=0.0,
                                     eps=EPS, S=S, d=D, Y=P(5), H=P(6), codes_o=P(7), exps_o=P(8), codes=P(9), exps=P(10)),
        "residual_prenorm_bwd": dict(dH=P(0), dres=P(1), type=0, Y=None, codes_y=P(2), exps_y=P(3), O=None, codes=P(4), exps=P(5),
                                     normalize=1, w_post=P(6), gate=P(7), gate_rows=10, scale=1.0, w=P(8), offset=0.0, eps=EPS, S=S, d=D,
                                     ws=P(9), size=WS, dY=P(11), dO=P(12), dw=P(13), dw_post=P(14), dgate=P(15)),
    }[name]
    assert set(change) <= set(good), (name, change)
    return getattr(lib, "mst_" + name)(*{**good, **change}.values(), None)


ALL = ["ckpt_pack", "ckpt_unpack", "prenorm_fwd", "prenorm_rebuild", "prenorm_bwd", "residual_fwd", "residual_bwd",
       "residual_prenorm_fwd", "residual_prenorm_bwd"]
GATED, BACKWARD = ALL[5:], ["prenorm_bwd", "residual_bwd", "residual_prenorm_bwd"]


@pytest.mark.parametrize("name", ALL)
def test_shapes_are_refused(mst, name):
    lib = mst.load_norm_library()
    for bad in (dict(S=0), dict(S=-3), dict(S=1 << 30), dict(d=0), dict(d=4), dict(d=36), dict(d=16392), dict(d=-8)):
        assert call(lib, name, **bad) == SHAPE, bad


@pytest.mark.parametrize("name,required", [
    ("ckpt_pack", "X codes exps"), ("ckpt_unpack", "X codes exps"), ("prenorm_fwd", "X H"), ("prenorm_rebuild", "codes exps H"),
    ("prenorm_bwd", "dH dX dw"), ("residual_fwd", "O X Y"), ("residual_bwd", "dY dO dw dgate"),
    ("residual_prenorm_fwd", "O X Y H"), ("residual_prenorm_bwd", "dH dY dO dw dw_post dgate")])
def test_missing_pointers_are_refused(mst, name, required):
    lib = mst.load_norm_library()
    for n in required.split():
        assert call(lib, name, **{n: None}) == NULL, n
    if name in ("prenorm_bwd", "residual_bwd"):
        assert call(lib, name, codes=None, exps=None) == NULL               # neither a tensor nor its checkpoint
    if name == "residual_prenorm_bwd":
        assert call(lib, name, codes=None, exps=None) == NULL and call(lib, name, codes_y=None, exps_y=None) == NULL


@pytest.mark.parametrize("name", ALL)
def test_values_are_refused(mst, name):
    lib = mst.load_norm_library()
    nan, inf = float("nan"), float("inf")
    if "rebuild" not in name:
        assert call(lib, name, type=2) == ARGUMENT and call(lib, name, type=-1) == ARGUMENT
    if "ckpt" not in name:
        for eps in (0.0, -1.0, nan, inf, 1e-40, 2.0 ** -101):
            assert call(lib, name, eps=eps) == ARGUMENT, eps
        assert call(lib, name, offset=nan) == ARGUMENT
    if name in GATED:
        assert call(lib, name, scale=nan) == ARGUMENT and call(lib, name, scale=inf) == ARGUMENT
        assert call(lib, name, gate_rows=0) == ARGUMENT and call(lib, name, gate_rows=-1) == ARGUMENT
        without = dict(gate=None) if "fwd" in name else dict(gate=None, dgate=None)
        assert call(lib, name, **without) == ARGUMENT                       # rows of a gate that is not there


@pytest.mark.parametrize("name", ALL[2:])
def test_pointers_that_exclude_or_need_each_other(mst, name):
    lib = mst.load_norm_library()
    if "rebuild" not in name:
        assert call(lib, name, codes=None) == ARGUMENT and call(lib, name, exps=None) == ARGUMENT
    if "both" in name or name == "residual_prenorm_fwd":
        assert call(lib, name, codes_o=None) == ARGUMENT
    if name in BACKWARD:
        assert call(lib, name, **{"X" if name == "prenorm_bwd" else "O": P(20)}) == ARGUMENT      # tensor and checkpoint
    if name == "prenorm_bwd":
        assert call(lib, name, w=None) == ARGUMENT                          # a gradient of no weight
    if name == "residual_bwd":
        assert call(lib, name, w=None) == ARGUMENT and call(lib, name, gate=None, gate_rows=0) == ARGUMENT
    if name == "residual_prenorm_bwd":
        assert call(lib, name, w=None) == ARGUMENT and call(lib, name, w_post=None) == ARGUMENT
        assert call(lib, name, Y=P(20)) == ARGUMENT
    if name in GATED:
        assert call(lib, name, normalize=0) == ARGUMENT                     # the weight of no norm


@pytest.mark.parametrize("name", BACKWARD)
def test_workspace_is_checked(mst, name):
    lib = mst.load_norm_library()
    need = mst.mst_norm_workspace_bytes(S, D, 0 if name == "prenorm_bwd" else 10)
    assert call(lib, name, ws=None) == WORKSPACE and call(lib, name, size=need - 1) == WORKSPACE
    assert call(lib, name, ws=P(17) + 128) == ALIGNMENT


@pytest.mark.parametrize("name", ALL)
def test_alignment_and_overlap(mst, name):
    lib = mst.load_norm_library()
    import inspect
    source = inspect.getsource(call)
    line = source[source.index(f'"{name}"'):]
    tensors = [n for n in re.findall(r"(\w+)=P\(\d+\)", line[:line.index("),\n") if "),\n" in line else None]) if n not in ("exps", "exps_o", "exps_y")]
    for n in tensors:
        assert call(lib, name, **{n: P(30) + 8}) == ALIGNMENT, n
    outs = {"ckpt_pack": ["codes", "exps"], "ckpt_unpack": ["X"], "prenorm_fwd": ["H", "codes", "exps"], "prenorm_rebuild": ["H"],
            "prenorm_bwd": ["dX", "dw"], "residual_fwd": ["Y", "codes", "exps"], "residual_bwd": ["dO", "dw", "dgate"],
            "residual_prenorm_fwd": ["Y", "H", "codes_o", "codes"], "residual_prenorm_bwd": ["dY", "dO", "dw", "dw_post", "dgate"]}[name]
    for out in outs:
        for other in tensors:
            if other != out and other not in ("gate", "w", "w_post", "dw", "dw_post", "dgate"):
                assert call(lib, name, **{out: P(30) + 16, other: P(30)}) == ARGUMENT, (out, other)      # shifted
    for a in outs:
        for b in outs:
            if a != b:
                assert call(lib, name, **{a: P(30), b: P(30)}) == ARGUMENT, (a, b)
    if name == "prenorm_fwd":
        assert call(lib, name, type=1, H=P(0)) == ARGUMENT                  # bf16 in place of fp32
        assert call(lib, name, H=P(1)) == ARGUMENT                          # in place of the weight
        assert call(lib, name, codes=P(0)) == ARGUMENT


def test_the_binding_refuses_what_the_c_call_cannot_see(mst):
    """Wrong types, shapes, strides and devices: with tensors on the CPU the last check is the device's."""
    import torch
    bf, f32 = torch.bfloat16, torch.float32
    x, h, w = torch.zeros((S, D), dtype=bf), torch.zeros((S, D), dtype=bf), torch.zeros(D, dtype=bf)
    codes, exps = torch.zeros((S, D), dtype=torch.int8), torch.zeros((S, 2), dtype=torch.uint8)
    wide = torch.zeros((S, 2 * D), dtype=bf)

    def status(f, *args, **kw):
        with pytest.raises(mst.MstError) as e:
            f(*args, **kw)
        return e.value.status

    pre = lambda **kw: status(mst.mst_prenorm_fwd, **{**dict(X=x, w_pre=w, H=h, eps=EPS, codes=codes, exps=exps), **kw})  # noqa: E731
    assert pre() == NO_DEVICE
    assert pre(X=x.half()) == ARGUMENT and pre(H=h.float()) == ARGUMENT and pre(w_pre=w.float()) == ARGUMENT
    assert pre(X=wide[:, :D]) == ARGUMENT and pre(X=torch.zeros((D, S), dtype=bf).t()) == ARGUMENT
    assert pre(X=x[0]) == SHAPE and pre(H=h[1:]) == SHAPE and pre(w_pre=w[8:]) == SHAPE
    assert pre(exps=exps[:, :1]) == SHAPE and pre(codes=codes.to(torch.uint8)) == ARGUMENT
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    gate = torch.zeros((7, D), dtype=bf)
    good = dict(dY=x, dO=h, workspace=ws, w=w, dw=torch.zeros(D), gate=gate, gate_rows=10, dgate=torch.zeros((7, D)), codes=codes, exps=exps)
    res = lambda **kw: status(mst.mst_residual_bwd, **{**good, **kw})  # noqa: E731
    assert res() == NO_DEVICE
    assert res(gate_rows=11) == SHAPE and res(gate_rows=0) == ARGUMENT and res(dgate=torch.zeros((8, D))) == SHAPE
    assert res(dw=w) == ARGUMENT and res(dO=h.float()) == ARGUMENT and res(dY=x.double()) == ARGUMENT
    assert res(O=x.float(), codes=None, exps=None) == ARGUMENT
