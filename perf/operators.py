"""The grouped perceptron layers and the 8-bit checkpoints of their inputs: what they are timed on, and
what their results are compared with.

The rows of a layer's input are anchors in block order, block g of a scene owns the rows
offsets[g]..offsets[g+1] and a weight matrix of its own.  Sizes: the anchor decoder's perceptrons
(35 inputs, 3 x 32 hidden units side by side, 70 outputs) over the 300 000 anchors of the benchmark, single
listed anchors and a handful, wide layers in bfloat16, and odd sizes.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _layer(name, kind, rows, groups, k, n, dtype, relu=False, keep=False, gate=False, in_major=False, stride=0):
    """kind: forward | backward.  relu: the layer ends in a ReLU; keep: the forward pass keeps its input in
    8 bits; gate: the input is what a ReLU gave, the backward pass goes through it; in_major: weights [k][n];
    stride: columns between the rows of the input that belong to others (0: rows are packed)."""
    return dict(name=name, kind=kind, rows=rows, groups=groups, k=k, n=n, dtype=dtype, relu=relu, keep=keep,
                gate=gate, in_major=in_major, stride=stride)


def listed():
    return [
        # one anchor in view (one token of one request): latency of a launch and of one block's weights
        _layer("forward_one", "forward", 1, 8, 1024, 1024, "bf16", relu=True),
        # a handful of rows spread over many blocks: every row brings weights of its own
        _layer("forward_few", "forward", 24, 64, 1024, 2048, "bf16"),
        # first layers of the anchor decoder in training, three perceptrons side by side, a city in 24 blocks
        _layer("forward_anchors", "forward", 300_000, 24, 35, 96, "f32", relu=True, keep=True),
        # second layer of its covariance perceptron: a third of the hidden units, weights as the decoder has them
        _layer("forward_outputs", "forward", 300_000, 24, 32, 70, "f32", keep=True, in_major=True, stride=64),
        # odd sizes, ordinary number of rows
        _layer("forward_odd", "forward", 10_007, 7, 131, 257, "f32", relu=True, keep=True),
        # wide hidden layers: matrix products are all of it
        _layer("forward_wide", "forward", 65_536, 32, 1024, 1024, "bf16", relu=True, keep=True),
        # the gradients of the layers above
        _layer("backward_anchors", "backward", 300_000, 24, 35, 96, "f32"),
        _layer("backward_outputs", "backward", 300_000, 24, 32, 70, "f32", gate=True, in_major=True),
        _layer("backward_odd", "backward", 10_007, 7, 131, 257, "bf16"),
        _layer("backward_wide", "backward", 65_536, 32, 1024, 1024, "bf16", gate=True),
        # keeping and reading back the decoder's hidden units alone
        dict(name="checkpoint_hidden", kind="checkpoint", rows=300_000, k=96, dtype="f32"),
        # the same of a small crop, odd width, bfloat16
        dict(name="checkpoint_small", kind="checkpoint", rows=5_003, k=131, dtype="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16"])
    kind = rng.choice(["forward", "forward", "backward", "backward", "checkpoint"])
    if kind == "checkpoint":
        k = _log_uniform(rng, 8, 1024)
        return dict(kind=kind, rows=_log_uniform(rng, 1_000, min(600_000, 60_000_000 // k)), k=k, dtype=dtype)
    groups, k, n = _log_uniform(rng, 1, 128), _log_uniform(rng, 8, 2048), _log_uniform(rng, 8, 2048)
    if rng.random() < 0.4:          # some in whole tiles, as programs choose them
        k, n = (max(8, round(v / 64) * 64) for v in (k, n))
    groups = max(1, min(groups, 48_000_000 // (n * k)))
    products = 30_000_000_000 if dtype == "bf16" else 6_000_000_000
    rows = _log_uniform(rng, 1, max(2, min(300_000, 100_000_000 // (n + k), products // (n * k))))
    case = _layer(None, kind, rows, groups, k, n, dtype, in_major=rng.random() < 0.3)
    if kind == "forward":
        case.update(relu=rng.random() < 0.5, keep=rng.random() < 0.5, stride=rng.choice([0, 0, k, 7]))
    else:
        case.update(gate=rng.random() < 0.5)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------- inputs
def _gen(seed, salt=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + salt)
    return g


def _normal(g, shape, sigma=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).mul_(sigma)


def _sizes(case, seed):
    """Rows of each group: ragged, about half to twice the mean, every fifth group empty; the order is the seed's."""
    groups, rows = case["groups"], case["rows"]
    r = random.Random(groups * 1_000_003 + rows)
    share = [0.0 if g % 5 == 3 else math.exp(r.gauss(0.0, 0.4)) for g in range(groups)]
    total, cuts, run_ = sum(share), [], 0.0
    for s in share:
        run_ += s
        cuts.append(min(rows, int(round(rows * run_ / total))))
    sizes = [b - a for a, b in zip([0] + cuts[:-1], cuts)]
    random.Random(int(seed)).shuffle(sizes)
    return sizes


def _values(case, g, dtype):
    """The layer's input as [rows][k] of wider rows: features, or where `gate` or for hidden units alone what a ReLU left."""
    rows, k = case["rows"], case["k"]
    x = _normal(g, (rows, k + case.get("stride", 0)))
    if case.get("gate") or case["kind"] == "checkpoint":
        x.relu_()
    return x.to(dtype)[:, :k]


def _quantised(x):
    """Codes and scales of x as the library lays them out: rows of whole blocks of 32 codes, one byte of scale a block."""
    rows, k = x.shape
    blocks = (k + 31) // 32
    v = torch.zeros((rows, blocks * 32), dtype=torch.float32, device=x.device)
    v[:, :k] = x.float()
    v = v.reshape(rows, blocks, 32)
    bits = v.abs().amax(-1).view(torch.int32)
    scale = torch.clamp((bits >> 23) - 6 + ((bits & 0x7FFFFF) >= 0x7F0000).int(), min=1)
    scale = torch.where(bits == 0, torch.zeros_like(scale), torch.where(bits >= 0x7F800000, torch.full_like(scale, 255), scale))
    step = ((254 - scale.clamp(1, 253)) << 23).view(torch.float32)[..., None]
    code = torch.round(v * step).clamp(-127, 127)
    code = torch.where((code == 0) & (v != 0), torch.sign(v), code)
    code = torch.where((scale == 255)[..., None], torch.zeros_like(code), code)
    return code.to(torch.int8).reshape(rows, blocks * 32), scale.to(torch.uint8)


def _read_back(codes, scale, k):
    """What codes and scales stand for, float32 [rows][k]."""
    rows = codes.shape[0]
    step = (scale.int() << 23).view(torch.float32)[..., None]
    return (codes.reshape(rows, -1, 32).float() * step).reshape(rows, -1)[:, :k]


def prepare(case, seed):
    g, dtype, rows, k = _gen(seed), DTYPES[case["dtype"]], case["rows"], case["k"]
    s = SimpleNamespace(case=case, rows=rows, k=k)
    s.x = _values(case, g, dtype)
    blocks = (k + 31) // 32
    if case["kind"] == "checkpoint":
        s.codes = torch.empty((rows, blocks * 32), dtype=torch.int8, device=DEV)
        s.scale = torch.empty((rows, blocks), dtype=torch.uint8, device=DEV)
        s.back = torch.empty((rows, k), dtype=dtype, device=DEV)
        return s
    sizes, n, groups = _sizes(case, seed), case["n"], case["groups"]
    offsets = [0]
    for m in sizes:
        offsets.append(offsets[-1] + m)
    s.n, s.groups, s.longest = n, groups, max(sizes)
    s.offsets = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    s.w = _normal(g, (groups, k, n) if case["in_major"] else (groups, n, k), 1 / math.sqrt(k)).to(dtype)
    if case["kind"] == "forward":
        s.b = _normal(g, (groups, n), 0.1)
        s.y = torch.empty((rows, n), dtype=dtype, device=DEV)
        if case["keep"]:
            s.codes = torch.empty((rows, blocks * 32), dtype=torch.int8, device=DEV)
            s.scale = torch.empty((rows, blocks), dtype=torch.uint8, device=DEV)
            s.back = torch.empty((rows, k), dtype=dtype, device=DEV)
        return s
    s.codes, s.scale = _quantised(s.x)          # what the forward pass left
    del s.x
    s.dy = _normal(g, (rows, n), 1e-2).to(dtype)
    s.dx = torch.empty((rows, k), dtype=dtype, device=DEV)
    s.dw = torch.empty(s.w.shape, dtype=torch.float32, device=DEV)
    s.db = torch.empty((groups, n), dtype=torch.float32, device=DEV)
    return s


# ---------------------------------------------------------------------------------------- one pass
def _rows_of_groups(s):
    """[groups][longest] row numbers, and which of them are rows of the group."""
    at = s.offsets[:-1, None].long() + torch.arange(max(s.longest, 1), device=DEV)[None]
    there = at < s.offsets[1:, None]
    return at.clamp(max=s.rows - 1), there


def _padded(v, at, there):
    return torch.where(there[..., None], v.float()[at], torch.zeros((), device=DEV))


def _unpadded(v, s):
    """[groups][longest][m] back to [rows][m]."""
    row = torch.arange(s.rows, device=DEV)
    group = torch.searchsorted(s.offsets[1:].contiguous(), row.int(), right=True)
    return v[group, row - s.offsets[group].long()]


def _plain(s):
    c = s.case
    if c["kind"] == "checkpoint":
        return dict(x8=_read_back(*_quantised(s.x), s.k).to(s.x.dtype))
    at, there = _rows_of_groups(s)
    w = s.w.float() if c["in_major"] else s.w.float().transpose(1, 2).contiguous()          # [groups][k][n]
    if c["kind"] == "forward":
        y = _unpadded(torch.bmm(_padded(s.x, at, there), w), s)
        group = torch.searchsorted(s.offsets[1:].contiguous(), torch.arange(s.rows, device=DEV, dtype=torch.int32), right=True)
        y = y + s.b[group]
        out = dict(y=(torch.relu(y) if c["relu"] else y).to(s.x.dtype))
        if c["keep"]:
            out["x8"] = _read_back(*_quantised(s.x), s.k).to(s.x.dtype)
        return out
    x = _read_back(s.codes, s.scale, s.k)
    dy, xp = _padded(s.dy, at, there), _padded(x, at, there)
    dx = _unpadded(torch.bmm(dy, w.transpose(1, 2).contiguous()), s)
    if c["gate"]:
        dx = torch.where(x > 0, dx, torch.zeros_like(dx))
    dw = torch.bmm(xp.transpose(1, 2).contiguous(), dy) if c["in_major"] else torch.bmm(dy.transpose(1, 2).contiguous(), xp)
    return dict(dx=dx.to(s.dy.dtype), dw=dw, db=dy.sum(1))


def run(s):
    if not own:
        return _plain(s)
    from paper_2503_21364_amd import binding as B
    c = s.case
    if not hasattr(s, "kept"):          # handles and workspace, as a program keeps them
        s.kept = B.Checkpoint8(s.rows, s.k, codes=s.codes, scale=s.scale) if hasattr(s, "codes") else None
        if c["kind"] == "backward":
            s.work = torch.empty(B.grouped_linear_backward_bytes(s.rows, s.groups, s.n, s.k, s.dy.dtype), dtype=torch.uint8, device=DEV)
    if c["kind"] == "checkpoint":
        B.checkpoint8_pack(s.x, s.kept)
        B.checkpoint8_unpack(s.kept, s.back)
        return dict(x8=s.back)
    if c["kind"] == "forward":
        B.grouped_linear(s.x, s.w, s.offsets, s.y, bias=s.b, relu=c["relu"], in_major=c["in_major"], checkpoint=s.kept)
        if not c["keep"]:
            return dict(y=s.y)
        B.checkpoint8_unpack(s.kept, s.back)
        return dict(y=s.y, x8=s.back)
    B.grouped_linear_backward(s.dy, s.w, s.offsets, s.work, checkpoint=s.kept, gate=c["gate"], in_major=c["in_major"],
                              dx=s.dx, dw=s.dw, db=s.db)
    return dict(dx=s.dx, dw=s.dw, db=s.db)


def work(case):
    size, rows, k = (4 if case["dtype"] == "f32" else 2), case["rows"], case["k"]
    blocks = (k + 31) // 32
    kept = rows * blocks * 33
    if case["kind"] == "checkpoint":        # values in, codes and scales out and in again, values out
        return {"bytes": 2 * rows * k * size + 2 * kept, "flops": 0}
    n, groups = case["n"], case["groups"]
    used = sum(m > 0 for m in _sizes(case, 0))
    flops = 2 * rows * n * k
    if case["kind"] == "forward":
        b = rows * (k + n) * size + used * (n * k * size + 4 * n)
        if case["keep"]:
            b += 2 * kept + rows * k * size
        return {"bytes": b, "flops": flops}
    return {"bytes": rows * (k + n) * size + kept + used * n * k * size + groups * (n * k + n) * 4, "flops": 2 * flops}


# ---------------------------------------------------------------------------------------- 64 bits
def _power64(e):
    """2^e in 64 bits, from the bits of the number (a power function need not give it exactly)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _kept64(x):
    """What the 8-bit form of x stands for, from its definition: 32 values share the power of two 2^e, the least
    with |x| / 2^e below 127.5 (and not under 2^-126); whole multiples of it, never 0 for what is not 0."""
    rows, k = x.shape
    out = torch.empty((rows, k), dtype=torch.float64, device=x.device)
    for at in range(0, k, 32):
        v = x[:, at:at + 32].double()
        top = v.abs().amax(1, keepdim=True)
        m, p = torch.frexp(torch.where(top > 0, top, torch.ones_like(top)))     # top = m 2^p, 1/2 <= m < 1
        e = torch.where(m * 128 >= 127.5, p - 6, p - 7).clamp(min=-126)
        step = _power64(e)
        near = torch.floor(v.abs() / step)
        rest = v.abs() / step - near
        near = near + ((rest > 0.5) | ((rest == 0.5) & (near % 2 == 1)))        # ties to the even multiple
        out[:, at:at + 32] = torch.sign(v) * torch.where(v != 0, near.clamp(min=1), near) * step
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "checkpoint":
        return dict(x8=_kept64(s.x))
    edge = s.offsets.tolist()
    out = dict(y=torch.empty((s.rows, s.n), dtype=torch.float64, device=DEV)) if case["kind"] == "forward" else dict(
        dx=torch.empty((s.rows, s.k), dtype=torch.float64, device=DEV),
        dw=torch.zeros(s.w.shape, dtype=torch.float64, device=DEV),
        db=torch.zeros((s.groups, s.n), dtype=torch.float64, device=DEV))
    for g, (a, b) in enumerate(zip(edge, edge[1:])):
        if a == b:
            continue
        w = s.w[g].double().T if case["in_major"] else s.w[g].double()          # [n][k]
        if case["kind"] == "forward":
            y = s.x[a:b].double() @ w.T + s.b[g].double()
            out["y"][a:b] = y.clamp(min=0) if case["relu"] else y
            continue
        step = _power64(s.scale[a:b].int() - 127)
        x = (s.codes[a:b].double() * step.repeat_interleave(32, dim=1))[:, :s.k]
        dy = s.dy[a:b].double()
        dx = dy @ w
        out["dx"][a:b] = dx * (x > 0) if case["gate"] else dx
        dw = dy.T @ x
        out["dw"][g] = dw.T if case["in_major"] else dw
        out["db"][g] = dy.sum(0)
    if case.get("keep"):
        out["x8"] = _kept64(s.x)
    return out
