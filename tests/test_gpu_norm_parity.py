"""Norms, residuals, their gradients and 8-bit checkpoints on the GPU against oracle/norm_oracle.py: small ragged shapes
element by element, every output guarded, every output rounded once (tolerances: tests/norm_gpu_harness.py)."""
import numpy as np
import pytest

from oracle import norm_oracle as orc
from tests.norm_gpu_harness import EPS, ROW_OPS, Case, Out, close, column_ops, f64, rounded

pytestmark = pytest.mark.gpu

# one token; a quad's end inside a wave; waves that are not full; rows that are no multiple of those held at a time; more rows
# than there are workgroups; two chunks per lane; the largest
SHAPES = [(1, 8), (1, 4096), (2, 32), (3, 40), (7, 200), (5, 264), (33, 512), (17, 520), (65, 1544), (4, 8192), (3, 8200), (2, 16384),
          (300, 256), (1025, 72), (2500, 136), (1300, 1032), (600, 4104)]


@pytest.fixture(scope="module")
def mst():
    import paper_2407_15892_amd as m
    return m


def gate_rows_of(S, kind):
    return {"none": 0, "one": S, "three": -(-S // 3), "token": 1, "five_rows": min(5, S), "more_than_all": S + 7}[kind]


def run_forward(mst, c, parts, checkpoints=True):
    """parts: "pre", "res" or "both".  The outputs as tensors, guards checked."""
    import torch
    H, Y = c.rows(torch.bfloat16), c.rows()
    (co, eo), (cy, ey) = c.checkpoint_room(), c.checkpoint_room()
    k = lambda **kw: {n: v.t for n, v in kw.items()} if checkpoints else {}  # noqa: E731
    branch = dict(gate=c.gpu("gate"), gate_rows=c.gate_rows, scale=c.scale, normalize=c.normalize, eps=EPS, w_offset=c.offset)
    if parts == "pre":
        mst.mst_prenorm_fwd(c.gpu("x"), c.gpu("w_pre"), H.t, EPS, c.offset, **k(codes=cy, exps=ey))
    elif parts == "res":
        mst.mst_residual_fwd(c.gpu("o"), c.gpu("x"), Y.t, w=c.gpu("w_post"), **k(codes=co, exps=eo), **branch)
    else:
        mst.mst_residual_prenorm_fwd(c.gpu("o"), c.gpu("x"), Y.t, H.t, c.gpu("w_pre"), w_post=c.gpu("w_post"),
                                     **k(codes_o=co, exps_o=eo, codes_y=cy, exps_y=ey), **branch)
    torch.cuda.synchronize()
    return {n: v.check() for n, v in dict(H=H, Y=Y, codes_o=co, exps_o=eo, codes_y=cy, exps_y=ey).items()}


def on_gpu(a):
    import torch
    return None if a is None else torch.from_numpy(a).cuda()


def run_backward(mst, c, parts, from_checkpoint, dres=True):
    import torch
    f32 = torch.float32
    dX, dO, ws = c.rows(), c.rows(torch.bfloat16), c.workspace()
    dwp, dwo = (Out((c.d,), f32) if w is not None else None for w in (c.w_pre, c.w_post))
    dg = Out(c.gate.shape, f32) if c.gate is not None else None
    t = lambda out: None if out is None else out.t  # noqa: E731
    (cy, ey), (co, eo) = (tuple(on_gpu(a) for a in orc.checkpoint(v)) for v in (c.y, c.o))
    branch = dict(gate=c.gpu("gate"), gate_rows=c.gate_rows, dgate=t(dg), scale=c.scale, normalize=c.normalize, eps=EPS, w_offset=c.offset)
    if parts == "pre":
        x = dict(codes=cy, exps=ey) if from_checkpoint else dict(X=c.gpu("y"))
        mst.mst_prenorm_bwd(c.gpu("dh"), c.gpu("w_pre"), dX.t, t(dwp), ws.t, EPS, c.offset, dres=c.gpu("dres") if dres else None, **x)
    elif parts == "res":
        o = dict(codes=co, exps=eo) if from_checkpoint else dict(O=c.gpu("o"))
        mst.mst_residual_bwd(c.gpu("dres"), dO.t, ws.t, w=c.gpu("w_post"), dw=t(dwo), **o, **branch)
    else:
        a = dict(codes_y=cy, exps_y=ey, codes_o=co, exps_o=eo) if from_checkpoint else dict(Y=c.gpu("y"), O=c.gpu("o"))
        mst.mst_residual_prenorm_bwd(c.gpu("dh"), c.gpu("dres") if dres else None, dX.t, dO.t, ws.t, c.gpu("w_pre"), t(dwp),
                                     w_post=c.gpu("w_post"), dw_post=t(dwo), **a, **branch)
    torch.cuda.synchronize()
    ws.check()
    return {n: None if v is None else v.check() for n, v in dict(dX=dX, dO=dO, dw_pre=dwp, dw_post=dwo, dgate=dg).items()}


def check_forward(c, parts, got, checkpoints=True):
    y, reach = c.x, np.abs(c.x)
    if parts != "pre":
        y, reach = orc.residual(c.o, c.x, c.normalize, c.w_post, c.offset, EPS, c.gate, c.gate_rows, c.scale)
        close(got["Y"], y, reach, ROW_OPS, c.stream)
        if checkpoints:
            codes, exps = orc.checkpoint(c.o)
            assert np.array_equal(got["codes_o"].cpu().numpy(), codes) and np.array_equal(got["exps_o"].cpu().numpy(), exps)
    if parts != "res":
        q = orc.rstd(y, EPS) * np.abs(orc.weight(c.w_pre, c.offset, c.d))
        # |y| itself enters H twice: in its place and through the mean, whose reach is that of the row
        close(got["H"], orc.prenorm(y, c.w_pre, c.offset, EPS), q * (reach + np.abs(y) * ((reach * np.abs(y)).mean(1, keepdims=True) /
              ((y * y).mean(1, keepdims=True) + EPS))), 2 * ROW_OPS)
        if checkpoints:
            stored = c.x if parts == "pre" else f64(got["Y"])
            codes, exps = orc.checkpoint(stored)
            assert np.array_equal(got["codes_y"].cpu().numpy(), codes) and np.array_equal(got["exps_y"].cpu().numpy(), exps)


def check_backward(c, parts, got, from_checkpoint, dres=True):
    y = orc.restore(*orc.checkpoint(c.y)) if from_checkpoint else c.y
    o = orc.restore(*orc.checkpoint(c.o)) if from_checkpoint else c.o
    cols = column_ops(c.S, c.d, c.gate_rows if parts != "pre" else 0, parts != "res")
    dy, reach, ops = c.dres, np.abs(c.dres), 0
    if parts != "res":
        dy, dw, reach, dw_reach = orc.norm_bwd(c.dh, y, c.w_pre, c.offset, EPS)
        if dres:
            dy, reach = dy + c.dres, reach + np.abs(c.dres)
        ops = 2 * ROW_OPS
        close(got["dX"], dy, reach, ops, c.stream)
        if c.w_pre is not None:
            close(got["dw_pre"], dw, dw_reach, cols + ROW_OPS, "fp32")
    if parts != "pre":
        want = orc.residual_bwd(dy, o, c.normalize, c.w_post, c.offset, EPS, c.gate, c.gate_rows, c.scale, reach)
        close(got["dO"], want["dO"], want["dO_reach"], ops + 2 * ROW_OPS)
        if c.w_post is not None:
            close(got["dw_post"], want["dw"], want["dw_reach"], ops + cols + ROW_OPS, "fp32")
        if c.gate is not None:
            close(got["dgate"], want["dgate"], want["dgate_reach"], ops + cols + ROW_OPS, "fp32")


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("S,d", SHAPES)
def test_checkpoint_and_back(mst, S, d, stream):
    import torch
    c = Case(S, d, stream)
    codes, exps = c.checkpoint_room()
    mst.mst_ckpt_pack(c.gpu("x"), codes.t, exps.t)
    want = orc.checkpoint(c.x)
    assert np.array_equal(codes.check().cpu().numpy(), want[0]) and np.array_equal(exps.check().cpu().numpy(), want[1])
    for dtype in (torch.bfloat16, torch.float32):
        back = c.rows(dtype)
        mst.mst_ckpt_unpack(codes.t, exps.t, back.t)
        assert np.array_equal(f64(back.check()), orc.restore(*want))


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_checkpoint_of_borders_ties_and_what_has_no_scale(mst, stream):
    import torch
    rows = np.zeros((14, 72))
    rows[0, :4] = 127.0, 0.5, 1.5, -2.5
    rows[1, 0], rows[1, 40] = 127.5, -127.5
    rows[2, 3], rows[2, 35] = np.inf, 1.0
    rows[3, 70], rows[3, 0] = np.nan, 2.0
    rows[4, 5] = -np.inf
    rows[5, 0], rows[5, 64] = 2.0 ** -126, 2.0 ** -120
    rows[6, :3] = 2.0 ** -127, 1.5 * 2.0 ** -127, -2.0 ** -127
    rows[7, 8], rows[7, 9] = 127.0 * 2.0 ** 121, -2.0 ** 120
    rows[8, 8] = 127.5 * 2.0 ** 121                    # stands for 2^128 otherwise
    rows[9, :] = -0.0
    rows[10, 33] = 2.0 ** -133
    rows[11, :] = 2.0 ** np.linspace(-20, 20, 72).round()
    rows[12, :] = np.linspace(-1, 1, 72)
    rows[13, 71] = 1e30
    c = Case(14, 72, stream)
    c.x = rounded(rows, stream)
    codes, exps = c.checkpoint_room()
    mst.mst_ckpt_pack(c.gpu("x"), codes.t, exps.t)
    want = orc.checkpoint(c.x)
    none = np.repeat(want[1] == 255, 32, axis=1)[:, :72]
    assert none.sum() == 32 + 8 + 32 + 32
    assert np.array_equal(exps.check().cpu().numpy(), want[1])
    assert np.array_equal(codes.check().cpu().numpy()[~none], want[0][~none])
    for dtype in (torch.bfloat16, torch.float32):
        back = c.rows(dtype)
        mst.mst_ckpt_unpack(codes.t, exps.t, back.t)
        assert np.array_equal(f64(back.check()), orc.restore(*want), equal_nan=True)
    # the same from the norm's forward, whose rows without a NaN are what they are without the others
    H = c.rows(torch.bfloat16)
    codes2, exps2 = c.checkpoint_room()
    mst.mst_prenorm_fwd(c.gpu("x"), None, H.t, EPS, codes=codes2.t, exps=exps2.t)
    assert torch.equal(exps2.check(), exps.t) and np.array_equal(codes2.check().cpu().numpy()[~none], want[0][~none])
    h = f64(H.check())
    assert np.isnan(h[3]).all()
    for r in (0, 1, 9, 11, 12):
        want_h = orc.prenorm(c.x[r:r + 1], None, 0.0, EPS)
        close(h[r:r + 1], want_h, np.abs(want_h), ROW_OPS)
    rebuilt = c.rows(torch.bfloat16)
    mst.mst_prenorm_rebuild(codes.t, exps.t, None, rebuilt.t, EPS)
    back = f64(rebuilt.check())
    assert np.isnan(back[[2, 3, 4, 8]]).all()           # a block of NaN makes its row one


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("S,d", SHAPES)
def test_prenorm(mst, S, d, stream):
    import torch
    for weights, offset in ((True, 0.0), (True, 1.0), (False, 0.25)):
        c = Case(S, d, stream, weights=weights, offset=offset)
        check_forward(c, "pre", run_forward(mst, c, "pre"))
        plain = run_forward(mst, c, "pre", checkpoints=False)
        assert torch.equal(plain["H"], run_forward(mst, c, "pre")["H"])
        for from_checkpoint, dres in ((True, True), (False, True), (True, False)):
            check_backward(c, "pre", run_backward(mst, c, "pre", from_checkpoint, dres), from_checkpoint, dres)


@pytest.mark.parametrize("S,d", SHAPES)
def test_rebuilt_input_is_the_norm_of_the_checkpoint(mst, S, d):
    c = Case(S, d, offset=1.0)
    import torch
    codes, exps = orc.checkpoint(c.x)
    H = c.rows(torch.bfloat16)
    mst.mst_prenorm_rebuild(on_gpu(codes), on_gpu(exps), c.gpu("w_pre"), H.t, EPS, 1.0)
    want = orc.prenorm(orc.restore(codes, exps), c.w_pre, 1.0, EPS)
    close(H.check(), want, np.abs(want), ROW_OPS)


@pytest.mark.parametrize("gate", ["none", "one", "three", "token", "five_rows", "more_than_all"])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("S,d", SHAPES)
def test_residual(mst, S, d, stream, gate):
    for normalize, weights, offset, scale in ((True, True, 1.0, 0.7), (False, True, 0.0, 1.0), (True, False, 0.0, -0.5)):
        c = Case(S, d, stream, gate_rows_of(S, gate), weights, normalize, offset, scale)
        check_forward(c, "res", run_forward(mst, c, "res"))
        for from_checkpoint in (True, False):
            check_backward(c, "res", run_backward(mst, c, "res", from_checkpoint), from_checkpoint)


@pytest.mark.parametrize("gate", ["none", "one", "three", "token", "five_rows", "more_than_all"])
@pytest.mark.parametrize("stream", ["bf16", "fp32"])
@pytest.mark.parametrize("S,d", SHAPES)
def test_residual_and_prenorm_in_one_pass(mst, S, d, stream, gate):
    import torch
    for normalize, weights, offset, scale in ((True, True, 0.0, 0.7), (False, True, 1.0, 1.0)):
        c = Case(S, d, stream, gate_rows_of(S, gate), weights, normalize, offset, scale)
        got = run_forward(mst, c, "both")
        check_forward(c, "both", got)
        assert torch.equal(got["Y"], run_forward(mst, c, "res")["Y"])            # the bits of the call by itself
        for from_checkpoint, dres in ((True, True), (False, False)):
            check_backward(c, "both", run_backward(mst, c, "both", from_checkpoint, dres), from_checkpoint, dres)


def test_repeated_calls_have_the_same_bits(mst):
    import torch
    c = Case(3001, 520, "bf16", 700, scale=0.5)
    first, second = (run_backward(mst, c, "both", True) for _ in range(2))
    for name, t in first.items():
        assert torch.equal(t, second[name]), name


def test_rows_of_zeros_and_a_tiny_eps(mst):
    """Nothing to divide by but eps: 0 in, 0 out, and gradients of their exact size."""
    import torch
    c = Case(6, 40)
    c.y[:] = 0
    c.o[:] = 0
    c.y[3] = rounded(np.random.default_rng(1).standard_normal(40))
    check_backward(c, "both", run_backward(mst, c, "both", True), True)
    H = c.rows(torch.bfloat16)
    mst.mst_prenorm_fwd(c.gpu("y"), None, H.t, 2.0 ** -100)
    h = f64(H.check())
    assert (h[[0, 1, 2, 4, 5]] == 0).all() and np.isfinite(h).all()


@pytest.mark.parametrize("stream", ["bf16", "fp32"])
def test_rows_of_far_apart_sizes(mst, stream):
    """Rows of 2^-50 to 2^50: their sums of squares fit, the third power of their root mean square does not."""
    c = Case(41, 264, stream)
    scale = 2.0 ** np.linspace(-50, 50, 41).round()[:, None]
    c.x, c.y, c.o = c.x * scale, c.y * scale, c.o * scale
    check_forward(c, "pre", run_forward(mst, c, "pre"))
    for parts in ("pre", "res", "both"):
        for from_checkpoint in (True, False):
            check_backward(c, parts, run_backward(mst, c, parts, from_checkpoint), from_checkpoint)


def test_gradients_of_rows_of_zeros_with_the_least_eps(mst):
    """rstd is 2^50 there; what it is multiplied with is 0 or a gradient."""
    import torch
    c = Case(3, 40)
    c.y[:] = 0
    dX, dw, ws = c.rows(), Out((40,), torch.float32), c.workspace()
    mst.mst_prenorm_bwd(c.gpu("dh"), c.gpu("w_pre"), dX.t, dw.t, ws.t, 2.0 ** -100, X=c.gpu("y"))
    want = c.dh * c.w_pre * 2.0 ** 50
    close(dX.check(), want, np.abs(want), ROW_OPS)
    assert (f64(dw.check()) == 0).all()


def test_outputs_in_place_of_inputs(mst):
    import torch
    for stream in ("bf16", "fp32"):
        c = Case(37, 264, stream, 10, scale=0.5)
        want = run_forward(mst, c, "both")
        x, o = c.gpu("x"), c.gpu("o")
        mst.mst_residual_prenorm_fwd(o, x, x, o, c.gpu("w_pre"), w_post=c.gpu("w_post"), gate=c.gpu("gate"), gate_rows=10, scale=0.5, eps=EPS)
        assert torch.equal(x, want["Y"]) and torch.equal(o, want["H"])
        want = run_backward(mst, c, "both", True)
        dh, dres, ws = c.gpu("dh"), c.gpu("dres"), c.workspace()
        (cy, ey), (co, eo) = (tuple(on_gpu(a) for a in orc.checkpoint(v)) for v in (c.y, c.o))
        dwp, dwo, dg = (torch.empty(s, device="cuda") for s in ((264,), (264,), c.gate.shape))
        mst.mst_residual_prenorm_bwd(dh, dres, dres, dh, ws.t, c.gpu("w_pre"), dwp, w_post=c.gpu("w_post"), dw_post=dwo, gate=c.gpu("gate"),
                                     gate_rows=10, dgate=dg, scale=0.5, eps=EPS, codes_y=cy, exps_y=ey, codes_o=co, exps_o=eo)
        for a, name in ((dres, "dX"), (dh, "dO"), (dwp, "dw_pre"), (dwo, "dw_post"), (dg, "dgate")):
            assert torch.equal(a, want[name]), name
    c = Case(37, 264)
    x = c.gpu("x")
    want = run_forward(mst, c, "pre")["H"]
    mst.mst_prenorm_fwd(x, c.gpu("w_pre"), x, EPS)
    assert torch.equal(x, want)


def test_captured_calls_replay_on_another_stream(mst):
    """Forward and backward captured once; replays see new inputs, with eager work between them."""
    import torch
    c, other = Case(700, 520, "bf16", 300, scale=0.5), Case(700, 520, "bf16", 300, scale=0.5, seed=1)
    args = {n: c.gpu(n) for n in ("o", "x", "dh", "dres", "w_pre", "w_post", "gate")}
    bf, f32 = torch.bfloat16, torch.float32
    Y, H, dY, dO = (c.rows(bf).t for _ in range(4))
    (co, eo), (cy, ey) = ((a.t, b.t) for a, b in (c.checkpoint_room(), c.checkpoint_room()))
    dwp, dwo, dg = Out((520,), f32).t, Out((520,), f32).t, Out(c.gate.shape, f32).t
    ws = c.workspace().t
    branch = dict(gate=args["gate"], gate_rows=300, scale=0.5, eps=EPS, codes_o=co, exps_o=eo, codes_y=cy, exps_y=ey)

    def step():
        mst.mst_residual_prenorm_fwd(args["o"], args["x"], Y, H, args["w_pre"], w_post=args["w_post"], **branch)
        mst.mst_residual_prenorm_bwd(args["dh"], args["dres"], dY, dO, ws, args["w_pre"], dwp, w_post=args["w_post"], dw_post=dwo,
                                     dgate=dg, **branch)

    outs = (Y, H, dY, dO, dwp, dwo, dg, co, eo, cy, ey)
    want = []
    for case in (c, other):
        for n, t in args.items():
            t.copy_(case.gpu(n))
        step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 0, 1):
        for n, t in args.items():
            t.copy_((c, other)[i].gpu(n))
        for t in outs:
            t.zero_()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        for a, b in zip(outs, want[i]):
            assert torch.equal(a, b)
    del graph


def test_two_streams_at_once_with_a_workspace_each(mst):
    import torch
    cases = [Case(900, 264, "bf16", 400, seed=s) for s in range(2)]
    want = [run_backward(mst, c, "both", False) for c in cases]
    runs, streams = [], [torch.cuda.Stream() for _ in cases]
    for c in cases:
        f32 = torch.float32
        runs.append(dict(dY=c.rows().t, dO=c.rows(torch.bfloat16).t, workspace=c.workspace().t, dw_pre=Out((264,), f32).t,
                         dw_post=Out((264,), f32).t, dgate=Out(c.gate.shape, f32).t, dH=c.gpu("dh"), dres=c.gpu("dres"), Y=c.gpu("y"),
                         O=c.gpu("o"), w_pre=c.gpu("w_pre"), w_post=c.gpu("w_post"), gate=c.gpu("gate"), gate_rows=400, eps=EPS))
    torch.cuda.synchronize()
    for _ in range(20):
        for r, s in zip(runs, streams):
            mst.mst_residual_prenorm_bwd(**r, stream=s)
    torch.cuda.synchronize()
    for r, w in zip(runs, want):
        for a, b in (("dY", "dX"), ("dO", "dO"), ("dw_pre", "dw_pre"), ("dw_post", "dw_post"), ("dgate", "dgate")):
            assert torch.equal(r[a], w[b]), a


def test_offsets_that_pass_32_bits(mst):
    """2^33 entries: the last rows of every call, against the oracle on these rows, and a sum over all."""
    import torch
    d, S = 8192, (1 << 20) + 3
    gen = torch.Generator(device="cuda").manual_seed(3)
    tile = torch.randn((64, d), generator=gen, device="cuda").to(torch.bfloat16)
    x = tile.repeat(-(-S // 64), 1)[:S]
    x[-3:] = torch.randn((3, d), generator=gen, device="cuda").to(torch.bfloat16)
    codes = torch.empty((S, d), dtype=torch.int8, device="cuda")
    exps = torch.empty((S, d // 32), dtype=torch.uint8, device="cuda")
    mst.mst_ckpt_pack(x, codes, exps)
    last = f64(x[-3:])
    want_codes, want_exps = orc.checkpoint(last)
    assert np.array_equal(codes[-3:].cpu().numpy(), want_codes) and np.array_equal(exps[-3:].cpu().numpy(), want_exps)
    H = torch.empty_like(x)
    mst.mst_prenorm_fwd(x, None, H, EPS)
    want = orc.prenorm(last, None, 0.0, EPS)
    close(H[-3:], want, np.abs(want), ROW_OPS)
    mst.mst_prenorm_rebuild(codes, exps, None, H, EPS)
    back = orc.restore(want_codes, want_exps)
    want = orc.prenorm(back, None, 0.0, EPS)
    close(H[-3:], want, np.abs(want), ROW_OPS)
    mst.mst_ckpt_unpack(codes, exps, H)
    assert np.array_equal(f64(H[-3:]), back)
    ws = torch.empty(mst.mst_norm_workspace_bytes(S, d), dtype=torch.uint8, device="cuda")
    w, dw = torch.ones(d, dtype=torch.bfloat16, device="cuda"), torch.empty(d, device="cuda")
    mst.mst_prenorm_bwd(x, w, H, dw, ws, EPS, codes=codes, exps=exps)
    dx, _, reach, _ = orc.norm_bwd(last, back, None, 0.0, EPS)
    close(H[-3:], dx, reach, 2 * ROW_OPS)
    tile64 = f64(tile)
    tile_back = orc.restore(*orc.checkpoint(tile64))
    of_row = tile64 * tile_back * orc.rstd(tile_back, EPS)        # row r of dw's sum, r % 64
    rest = (S - 3) % 64
    total = of_row.sum(0) * ((S - 3) // 64) + of_row[:rest].sum(0) + (last * back * orc.rstd(back, EPS)).sum(0)
    reach = np.abs(of_row).sum(0) * (S // 64 + 1)
    close(dw, total, reach, column_ops(S, d) + ROW_OPS, "fp32")
