"""The operators between the blocks: the norm before a block, the gated and scaled residual (with or without a norm) after
it, both of them in one pass, and 8-bit checkpoints of the activations that the backward passes read.

A *step* is a training program's forward and backward call of one operator: the forward leaves the 8-bit checkpoint of its
input, which takes the place of the 16 or 32 bit tensor, and the backward reads it.  The residual stream (X, Y and their
gradients) is bfloat16 or float32; what a block takes and gives (H, O and their gradients) is bfloat16, as are weights and
gates; gradients of weights and gates are float32.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5


def _case(name, kind, S, d, stream="bf16", normalize=True, gate_rows=0, scale=1.0, offset=0.0):
    """gate_rows: rows that share a row of the gate, 0 for no gate; offset: what is added to the norms' weights."""
    return {"name": name, "kind": kind, "S": S, "d": d, "stream": stream, "normalize": normalize, "gate_rows": gate_rows,
            "scale": scale, "offset": offset}


def listed():
    return [
        # one token through the norm before a block, at the hidden size of the 8B-shaped configurations: all latency
        _case("prenorm_fwd_token", "prenorm_fwd", 1, 4096),
        # the tiny configuration's training step
        _case("prenorm_step_tiny", "prenorm_step", 512, 256),
        # the 8B-shaped configuration at its ordinary training length
        _case("prenorm_step_8b", "prenorm_step", 8192, 4096),
        # a small model with nothing on a tile boundary, three packed sequences with a gate of their own each
        _case("residual_step_ragged", "residual_step", 5003, 1544, gate_rows=1668, scale=0.5),
        # the shape with norms on both sides of each block, whose weights are stored less one, at its training length
        _case("residual_step_large_vocab", "residual_step", 16384, 3584, offset=1.0),
        # a float32 residual stream whose eight sequences are gated apart
        _case("residual_step_fp32_gated", "residual_step", 8192, 4096, stream="fp32", gate_rows=1024),
        # a few tokens between two blocks without a norm behind the first
        _case("residual_prenorm_fwd_few", "residual_prenorm_fwd", 7, 4096, normalize=False),
        # an ordinary training length between two blocks with all there is: both norms, a learned gate, both checkpoints
        _case("residual_prenorm_fwd_8b", "residual_prenorm_fwd", 8192, 4096, gate_rows=8192, scale=0.7),
        # a short training sequence between two blocks
        _case("residual_prenorm_bwd_short", "residual_prenorm_bwd", 200, 4096, gate_rows=200),
        # the long-sequence configuration between two blocks
        _case("residual_prenorm_bwd_long", "residual_prenorm_bwd", 32768, 4096),
        # checkpoint of a float32 stream of ragged sizes, written and read back
        _case("checkpoint_ragged_fp32", "checkpoint", 3001, 1544, stream="fp32"),
        # checkpoint of the very long configuration, written and read back: the largest
        _case("checkpoint_very_long", "checkpoint", 131072, 4096),
    ]


KINDS = ("prenorm_fwd", "prenorm_step", "residual_step", "residual_prenorm_fwd", "residual_prenorm_bwd", "checkpoint")

# the most work a drawn case may have: that of the largest listed one
_MOST_BYTES = 131072 * 4096 * 6


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One token to 131072, hidden sizes 64 to 8192 (multiples of 8, half of them of 128); gates for the whole call, for
    each of a few sequences, for each token, or none; both types of the residual stream."""
    while True:
        kind = rng.choice(KINDS)
        S = _log_int(rng, 1, 131072)
        d = 8 * _log_int(rng, 8, 1024)
        if rng.random() < 0.5:
            d = max(128, d // 128 * 128)
        gate_rows = rng.choice([0, 0, S, -(-S // rng.randint(2, 9)), 1]) if kind.startswith("residual") else 0
        case = _case(None, kind, S, d, rng.choice(["bf16", "bf16", "fp32"]), rng.random() < 0.7 or not kind.startswith("residual"),
                     gate_rows, rng.choice([1.0, 1.0, 0.5, 0.125]), rng.choice([0.0, 0.0, 1.0]))
        del case["name"]
        if work(case)["bytes"] <= _MOST_BYTES:
            return case


def prepare(case, seed):
    S, d, L, kind = case["S"], case["d"], case["gate_rows"], case["kind"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    stream = torch.float32 if case["stream"] == "fp32" else torch.bfloat16
    bf16 = torch.bfloat16

    def normal(rows, dtype, std=1.0, by_channel=None):
        out = torch.empty((rows, d), dtype=dtype, device="cuda")
        block = max(1, (1 << 27) // d)
        for r in range(0, rows, block):
            x = torch.randn((min(block, rows - r), d), generator=gen, device="cuda").mul_(std)
            out[r:r + block] = x if by_channel is None else x.mul_(by_channel)
        return out

    def empty(*shape, dtype=bf16):
        return torch.empty(shape, dtype=dtype, device="cuda")

    # a residual stream: channels of different sizes, a few of them far larger than the rest
    size = torch.randn(d, generator=gen, device="cuda").mul_(0.5).exp_()
    size[torch.randint(0, d, (max(1, d // 512),), generator=gen, device="cuda")] *= 20
    around_one = lambda n: 1 - case["offset"] + 0.2 * torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    st = {"case": case}

    def pack_into(name, x):
        values, exps = _codes(x.float())
        st["codes_" + name], st["exps_" + name] = values.to(torch.int8), exps.to(torch.uint8)

    def room_for(name):
        st["codes_" + name] = empty(S, d, dtype=torch.int8)
        st["exps_" + name] = empty(S, -(-d // 32), dtype=torch.uint8)

    if kind == "checkpoint":
        st["X"], st["back"] = normal(S, stream, by_channel=size), empty(S, d, dtype=stream)
        room_for("x")
        return st
    if kind.startswith("prenorm"):
        st["X"] = normal(S, stream, by_channel=size)
        room_for("x")
    else:
        o = normal(S, bf16, 0.7)
        st["w_post"] = around_one(d).to(bf16) if case["normalize"] else None
        st["gate"] = torch.randn((-(-S // L), d), generator=gen, device="cuda").mul_(0.5).to(bf16) if L else None
        if kind == "residual_prenorm_bwd":
            pack_into("o", o)
            pack_into("y", normal(S, stream, by_channel=size))
        else:
            st["O"], st["X"] = o, normal(S, stream, by_channel=size)
            room_for("o")
            st["Y"] = empty(S, d, dtype=stream)
    if "prenorm" in kind:
        st["w_pre"] = around_one(d).to(bf16)
        st["H"] = empty(S, d)
    if kind == "residual_prenorm_fwd":
        room_for("y")
        st["back_o"], st["back_y"] = empty(S, d), empty(S, d)      # 7 bits fit bfloat16, whatever the stream
    if kind in ("prenorm_step", "residual_prenorm_bwd"):
        st.update(dH=normal(S, bf16, 1e-3), dres=normal(S, stream, 1e-3), dw_pre=empty(d, dtype=torch.float32))
        st["dX"] = empty(S, d, dtype=stream)
    if kind == "residual_step":
        st["dY"] = normal(S, stream, 1e-3)
    if kind in ("residual_step", "residual_prenorm_bwd"):
        st["dO"] = empty(S, d)
        st["dw_post"] = empty(d, dtype=torch.float32) if case["normalize"] else None
        st["dgate"] = empty(-(-S // L), d, dtype=torch.float32) if L else None
    return st


# ---------------------------------------------------------------- plain form

def _codes(x):
    """Codes (as float32) and exponent bytes of blocks of 32 columns of float32 x."""
    S, d = x.shape
    v = torch.nn.functional.pad(x, (0, -d % 32)).view(S, -1, 32)
    top = v.abs().amax(2).view(torch.int32)
    # the least power of two with which the largest value stays below 127.5: its own, or the next from 127.5 / 64 on
    byte = (((top + 0x10000) >> 23) - 6).clamp_(min=0)
    codes = torch.round(v * ((254 - byte) << 23).view(torch.float32)[:, :, None])
    return codes.view(S, -1)[:, :d], byte


def _values(codes, byte):
    """What codes (S x d) and exponent bytes stand for, float32."""
    S, d = codes.shape
    byte = byte.int()
    step = torch.where(byte == 0, 1 << 22, byte << 23).view(torch.float32)      # 2^(byte - 127), of 0 a subnormal
    v = torch.nn.functional.pad(codes.float(), (0, -d % 32)).view(S, -1, 32) * step[:, :, None]
    return v.view(S, -1)[:, :d]


def _rounded_trip(x):
    return _values(*_codes(x.float()))


def _rstd(x):
    return torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)


def _norm_bwd(dn, x, w):
    """Gradients of x and of w~ of x rstd(x) w~, dn being that of the result."""
    r = _rstd(x)
    n, a = x * r, dn * w
    return (a - n * (a * n).mean(1, keepdim=True)) * r, (dn * n).sum(0)


def _gate_rows(st):
    """The gate (times the scale) of each row, or the scale."""
    L, s = st["case"]["gate_rows"], st["case"]["scale"]
    if not L:
        return s
    return st["gate"].float().repeat_interleave(L, 0)[:st["case"]["S"]] * s


def _gate_sums(x, L):
    """Sums of L rows each."""
    S, d = x.shape
    return x if L == 1 else torch.nn.functional.pad(x, (0, 0, 0, -S % L)).view(-1, L, d).sum(1)


def _branch(st, o):
    if not st["case"]["normalize"]:
        return o
    return o * _rstd(o) * (st["w_post"].float() + st["case"]["offset"])


def _residual_bwd(st, dY, o):
    """(dO, dw_post, dgate) in float32, None where there is no such weight."""
    L, s, normalize = st["case"]["gate_rows"], st["case"]["scale"], st["case"]["normalize"]
    e = dY * _gate_rows(st)
    dgate = _gate_sums(dY * _branch(st, o) * s, L) if L else None
    if not normalize:
        return e, None, dgate
    dO, dw = _norm_bwd(e, o, st["w_post"].float() + st["case"]["offset"])
    return dO, dw, dgate


def _plain(st):
    case = st["case"]
    kind, bf16 = case["kind"], torch.bfloat16
    if kind == "checkpoint":
        return {"X": _rounded_trip(st["X"]).to(st["X"].dtype)}
    if kind.startswith("prenorm"):
        x, w = st["X"].float(), st["w_pre"].float() + case["offset"]
        out = {"H": (x * _rstd(x) * w).to(bf16)}
        if kind == "prenorm_step":
            dx, dw = _norm_bwd(st["dH"].float(), _rounded_trip(st["X"]), w)
            out.update(dX=(st["dres"].float() + dx).to(st["dres"].dtype), dw=dw)
        return out
    if kind == "residual_step":
        y = st["X"].float() + _gate_rows(st) * _branch(st, st["O"].float())
        dO, dw, dgate = _residual_bwd(st, st["dY"].float(), _rounded_trip(st["O"]))
        return {"Y": y.to(st["X"].dtype), "dO": dO.to(bf16), "dw": dw, "dgate": dgate}
    w = st["w_pre"].float() + case["offset"]
    if kind == "residual_prenorm_fwd":
        y = st["X"].float() + _gate_rows(st) * _branch(st, st["O"].float())
        stored = y.to(st["X"].dtype)
        return {"Y": stored, "H": (y * _rstd(y) * w).to(bf16), "O": _rounded_trip(st["O"]).to(bf16),
                "Y_checkpoint": _rounded_trip(stored).to(bf16)}
    dy, dw = _norm_bwd(st["dH"].float(), _values(st["codes_y"], st["exps_y"]), w)
    dy = dy + st["dres"].float()
    dO, dw_post, dgate = _residual_bwd(st, dy, _values(st["codes_o"], st["exps_o"]))
    return {"dY": dy.to(st["dres"].dtype), "dO": dO.to(bf16), "dw_pre": dw, "dw_post": dw_post, "dgate": dgate}


# ------------------------------------------------- the framework's own calls

def _framework(st):
    import paper_2407_15892_amd as mst
    case = st["case"]
    kind, off = case["kind"], case["offset"]
    if kind == "checkpoint":
        mst.mst_ckpt_pack(st["X"], st["codes_x"], st["exps_x"])
        mst.mst_ckpt_unpack(st["codes_x"], st["exps_x"], st["back"])
        return {"X": st["back"]}
    if kind == "prenorm_fwd":
        mst.mst_prenorm_fwd(st["X"], st["w_pre"], st["H"], eps=EPS, w_offset=off)
        return {"H": st["H"]}
    if kind != "residual_prenorm_fwd" and "ws" not in st:          # a program keeps its workspace
        st["ws"] = torch.empty(mst.mst_norm_workspace_bytes(case["S"], case["d"], case["gate_rows"]), dtype=torch.uint8, device="cuda")
    if kind == "prenorm_step":
        mst.mst_prenorm_fwd(st["X"], st["w_pre"], st["H"], eps=EPS, w_offset=off, codes=st["codes_x"], exps=st["exps_x"])
        mst.mst_prenorm_bwd(st["dH"], st["w_pre"], st["dX"], st["dw_pre"], st["ws"], eps=EPS, w_offset=off,
                            codes=st["codes_x"], exps=st["exps_x"], dres=st["dres"])
        return {"H": st["H"], "dX": st["dX"], "dw": st["dw_pre"]}
    branch = dict(gate=st["gate"], gate_rows=case["gate_rows"], scale=case["scale"], normalize=case["normalize"], eps=EPS, w_offset=off)
    if kind == "residual_step":
        mst.mst_residual_fwd(st["O"], st["X"], st["Y"], w=st["w_post"], codes=st["codes_o"], exps=st["exps_o"], **branch)
        mst.mst_residual_bwd(st["dY"], st["dO"], st["ws"], w=st["w_post"], dw=st["dw_post"], dgate=st["dgate"],
                             codes=st["codes_o"], exps=st["exps_o"], **branch)
        return {"Y": st["Y"], "dO": st["dO"], "dw": st["dw_post"], "dgate": st["dgate"]}
    checkpoints = dict(codes_o=st["codes_o"], exps_o=st["exps_o"], codes_y=st["codes_y"], exps_y=st["exps_y"])
    if kind == "residual_prenorm_fwd":
        mst.mst_residual_prenorm_fwd(st["O"], st["X"], st["Y"], st["H"], st["w_pre"], w_post=st["w_post"], **checkpoints, **branch)
        mst.mst_ckpt_unpack(st["codes_o"], st["exps_o"], st["back_o"])
        mst.mst_ckpt_unpack(st["codes_y"], st["exps_y"], st["back_y"])
        return {"Y": st["Y"], "H": st["H"], "O": st["back_o"], "Y_checkpoint": st["back_y"]}
    mst.mst_residual_prenorm_bwd(st["dH"], st["dres"], st["dX"], st["dO"], st["ws"], st["w_pre"], st["dw_pre"],
                                 w_post=st["w_post"], dw_post=st["dw_post"], dgate=st["dgate"], **checkpoints, **branch)
    return {"dY": st["dX"], "dO": st["dO"], "dw_pre": st["dw_pre"], "dw_post": st["dw_post"], "dgate": st["dgate"]}


def run(st):
    return _framework(st) if own else _plain(st)


def work(case):
    """Bytes: each tensor once for each call that it is an argument of (a checkpoint is written by the forward and read by
    the backward, which is what it is there for).  Operations: multiplications and additions of the formulas."""
    S, d, L, kind = case["S"], case["d"], case["gate_rows"], case["kind"]
    n, t = S * d, 4 if case["stream"] == "fp32" else 2
    ck = n + S * -(-d // 32)
    gate = 2 * d * -(-S // L) if L else 0
    w = 2 * d
    post = w if case["normalize"] else 0
    reads_o = case["normalize"] or L > 0            # whether the backward of the residual needs O at all
    grads = (2 * post if post else 0) + 2 * gate    # float32
    if kind == "checkpoint":
        return {"bytes": 2 * t * n + 2 * ck, "flops": 4 * n}
    if kind == "prenorm_fwd":
        return {"bytes": (t + 2) * n + w, "flops": 4 * n}
    if kind == "prenorm_step":
        return {"bytes": (t + 2) * n + ck + ck + (2 + 2 * t) * n + 2 * w + 2 * w, "flops": 20 * n}
    if kind == "residual_step":
        return {"bytes": (2 + 2 * t) * n + ck + (ck if reads_o else 0) + (t + 2) * n + 2 * post + 2 * gate + grads, "flops": 24 * n}
    if kind == "residual_prenorm_fwd":
        return {"bytes": (4 + 2 * t) * n + 2 * ck + 2 * ck + 4 * n + post + gate + w, "flops": 18 * n}
    return {"bytes": ck + (ck if reads_o else 0) + (4 + 2 * t) * n + post + gate + w + grads + 2 * w, "flops": 30 * n}


# ----------------------------------------------------- definition in 64 bits

def _power_of_two(k):
    """2^k from its bits: pow() need not be exact."""
    return ((k.long() + 1023) << 52).view(torch.float64)


def _exact_trip(x):
    """x after a checkpoint: every block of 32 columns to whole multiples of the least power of two of which its largest
    magnitude is less than 127.5 times."""
    rows = []
    for block in x.double().split(32, 1):
        m, e = torch.frexp(block.abs().amax(1, keepdim=True))
        k = torch.where(m * 128 < 127.5, e - 7, e - 6)
        k = torch.where(m == 0, torch.full_like(k, -127), k.clamp(min=-127))
        step = _power_of_two(k)
        rows.append(torch.round(block / step) * step)
    return torch.cat(rows, 1)


def _exact_unpack(codes, exps):
    k = exps.long().repeat_interleave(32, 1)[:, :codes.shape[1]] - 127
    return codes.double() * _power_of_two(k)


def exact(case, seed):
    st = prepare(case, seed)
    S, d, L, s, kind = case["S"], case["d"], case["gate_rows"], case["scale"], case["kind"]
    norm = lambda x: x / torch.sqrt((x * x).sum(1, keepdim=True) / d + EPS)  # noqa: E731
    weight = lambda name: st[name].double() + case["offset"]  # noqa: E731

    def through_norm(dn, x):
        """Gradient of x, dn being that of norm(x)."""
        q = (x * x).sum(1, keepdim=True) / d + EPS
        return dn / q.sqrt() - x * ((dn * x).sum(1, keepdim=True) / (d * q * q.sqrt()))

    if kind == "checkpoint":
        return {"X": _exact_trip(st["X"])}
    if kind.startswith("prenorm"):
        out = {"H": norm(st["X"].double()) * weight("w_pre")}
        if kind == "prenorm_step":
            x, dh = _exact_trip(st["X"]), st["dH"].double()
            out.update(dX=st["dres"].double() + through_norm(dh * weight("w_pre"), x), dw=(dh * norm(x)).sum(0))
        return out
    of_row = torch.arange(S, device="cuda") // L if L else None
    g = s * st["gate"].double()[of_row] if L else torch.tensor(s, dtype=torch.float64, device="cuda")
    branch = lambda o: norm(o) * weight("w_post") if case["normalize"] else o  # noqa: E731

    def residual_bwd(dY, o):
        dw = (dY * g * norm(o)).sum(0) if case["normalize"] else None
        dgate = None
        if L:
            dgate = torch.zeros(st["gate"].shape, dtype=torch.float64, device="cuda").index_add_(0, of_row, s * dY * branch(o))
        return through_norm(dY * g * weight("w_post"), o) if case["normalize"] else dY * g, dw, dgate

    if kind == "residual_step":
        dO, dw, dgate = residual_bwd(st["dY"].double(), _exact_trip(st["O"]))
        return {"Y": st["X"].double() + g * branch(st["O"].double()), "dO": dO, "dw": dw, "dgate": dgate}
    if kind == "residual_prenorm_fwd":
        y = st["X"].double() + g * branch(st["O"].double())
        # the checkpoint is one of the stored Y: next to a border its codes go by how Y was rounded, not by the definition
        return {"Y": y, "H": norm(y) * weight("w_pre"), "O": _exact_trip(st["O"]), "Y_checkpoint": None}
    y, dh = _exact_unpack(st["codes_y"], st["exps_y"]), st["dH"].double()
    dY = st["dres"].double() + through_norm(dh * weight("w_pre"), y)
    dO, dw, dgate = residual_bwd(dY, _exact_unpack(st["codes_o"], st["exps_o"]))
    return {"dY": dY, "dO": dO, "dw_pre": (dh * norm(y)).sum(0), "dw_post": dw, "dgate": dgate}
