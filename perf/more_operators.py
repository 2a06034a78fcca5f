"""Operators of training and serving a learned hyper-encoder with gated layers, for timing: the gated feed-forward block,
its gradient, the block over 4-bit weights, and the clipping of many gradients by their common norm.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass through an
operator: with `own` false in elementary tensor operations, with `own` true through the library's binding.  `work` gives
the bytes and operations that a pass cannot do without, `exact` the results in 64 bits.

Rows are normalised activations, N(0, 1); weights N(0, 1 / fan-in); 4-bit weights are such weights, each group of columns
scaled to the largest of them.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # one row through the block of a small encoder: launches and latency
        dict(name="ffn_1_d1024", kind="ffn", rows=1, d=1024, f=2752, act="silu", residual=True),
        # the newest entries of 24 sequences, their real slots: bound by the weights' bytes
        dict(name="ffn_52_d4096", kind="ffn", rows=52, d=4096, f=10944, act="silu", residual=True),
        # the entries of a few prompts, a row count that no tile divides
        dict(name="ffn_1331_d3584", kind="ffn", rows=1331, d=3584, f=9600, act="gelu", residual=True),
        # all entries of a prefill batch's codebooks
        dict(name="ffn_35404_d4096", kind="ffn", rows=35404, d=4096, f=10944, act="silu", residual=False),
        # a training step on a few short sequences: forward and gradient
        dict(name="ffn_train_237_d1024", kind="train", rows=237, d=1024, f=2752, act="gelu"),
        # a training step on a batch
        dict(name="ffn_train_16411_d2048", kind="train", rows=16411, d=2048, f=5504, act="silu"),
        # a generation step's one new row over 4-bit weights
        dict(name="q4_1_d4096", kind="q4", rows=1, d=4096, f=10944, act="silu", group=64),
        # a serving batch's new rows
        dict(name="q4_24_d3584", kind="q4", rows=24, d=3584, f=9600, act="gelu", group=128),
        # a short prompt through the same weights
        dict(name="q4_300_d2048", kind="q4", rows=300, d=2048, f=5504, act="silu", group=32),
        # the vectors and matrices of a one-layer attention encoder, d = 256, and its slot positions
        dict(name="clip_small", kind="clip", set="small", d=256, f=0, layers=1, V=0, dtype="bf16"),
        # every gradient of a two-layer encoder: matrices bf16, vectors fp32
        dict(name="clip_encoder", kind="clip", set="encoder", d=4096, f=10944, layers=2, V=0, dtype="bf16"),
        # a whole training step's: the encoder's, the unembedding's (bf16) and the embedding's (fp32)
        dict(name="clip_step", kind="clip", set="step", d=4096, f=10944, layers=2, V=128256, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """Whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["ffn", "ffn", "train", "q4", "q4", "clip"])
    if kind == "clip":
        which = rng.choice(["small", "encoder", "step"])
        return dict(kind=kind, set=which, d=8 * _log(rng, 8, 512), f=8 * _log(rng, 16, 1368), layers=rng.randint(1, 4),
                    V=rng.choice([rng.randint(8000, 50257), 128256]) if which == "step" else 0, dtype=rng.choice(["bf16", "bf16", "f32"]))
    act = rng.choice(["silu", "gelu"])
    d = 64 * _log(rng, 4, 64)
    if kind == "q4":
        group = rng.choice([32, 64, 128])
        step = max(group, 64)
        d = step * max(1, d // step)
        return dict(kind=kind, rows=_log(rng, 1, 400), d=d, f=step * (int(d * rng.uniform(2, 4)) // step), act=act, group=group)
    f = 64 * max(1, int(d * rng.uniform(2, 4)) // 64)
    rows = _log(rng, 1, 32768 if kind == "ffn" else 16384)
    while rows * d * f > (1 << 40 if kind == "ffn" else 1 << 37):
        rows = rows // 2 + 1
    case = dict(kind=kind, rows=rows, d=d, f=f, act=act)
    return dict(case, residual=rng.random() < 0.7) if kind == "ffn" else case


# ---- inputs -----------------------------------------------------------------------------------------------------------------
def _normal(gen, shape, std, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


FOUR_BITS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def _to_four_bits(W, group):
    """W [rows, cols] -> words [rows / 16, blocks of 128 columns, 64, 4] int32 and scales [cols / group, rows] bf16.  Word m of lane 16 j + r
    holds columns 32 m + 8 j .. of row r of its block, the first in its lowest four bits; weights are the scale times one of FOUR_BITS."""
    rows, cols = W.shape
    w = W.float().reshape(rows, cols // group, group)
    scale = (w.abs().amax(dim=2) / 6).to(torch.bfloat16)
    x = w / scale.float()[:, :, None]
    y = x.abs()
    code = (y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)
    code = torch.where((code > 0) & (x < 0), code + 8, code)
    blocks = (cols + 127) // 128
    padded = torch.zeros((rows, blocks * 128), dtype=torch.int64, device="cuda")
    padded[:, :cols] = code.reshape(rows, cols)
    q = padded.reshape(rows // 16, 16, blocks, 4, 4, 8).permute(0, 2, 4, 1, 3, 5)      # tile, block, j, r, m, column of eight
    word = torch.zeros(q.shape[:-1], dtype=torch.int64, device="cuda")
    for i in range(8):
        word |= q[..., i] << (4 * i)
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).int()
    return word.reshape(rows // 16, blocks, 64, 4).contiguous(), scale.T.contiguous()


def _shapes(case):
    """Shapes and storage types of the gradients of a clip case."""
    d, f, V = case["d"], case["f"], case["V"]
    matrix = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    found = [((3, d), matrix)]
    for _ in range(case["layers"]):
        found += [((3 * d, d), matrix), ((d, d), matrix)] + [((n,), torch.float32) for n in (d, d, 3 * d, d)]
        if case["set"] != "small":
            found += [((2 * f, d), matrix), ((d, f), matrix)] + [((d,), torch.float32)] * 2
    if V:
        found += [((V, d), matrix), ((V, d), torch.float32)]
    return found


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * seed + 29)
    if case["kind"] == "clip":
        grads = [_normal(gen, shape, 10 ** (-2 - 2 * (i % 3) / 2), dtype) for i, (shape, dtype) in enumerate(_shapes(case))]
        st = dict(case=case, grads=grads, out=[torch.empty_like(g) for g in grads], max_norm=1e-3,
                  norm=torch.empty(2, dtype=torch.float32, device="cuda"))
        if own:
            from paper_2506_01084_amd import api

            st["ctx"] = api.Context(B=1, V=8, M=2, cap=0, d=64)
            st["list"] = api.Gradients(grads, st["out"])
        return st
    rows, d, f = case["rows"], case["d"], case["f"]
    st = dict(case=case, X=_normal(gen, (rows, d), 1.0), W1=_normal(gen, (2 * f, d), d ** -0.5), W2=_normal(gen, (d, f), f ** -0.5),
              Y=torch.empty((rows, d), dtype=torch.bfloat16, device="cuda"), residual=None, scale1=None, scale2=None)
    if case["kind"] != "ffn" or case["residual"]:
        st["residual"] = _normal(gen, (rows, d), 1.0)
    if case["kind"] == "q4":
        st["W1"], st["scale1"] = _to_four_bits(st["W1"], case["group"])
        st["W2"], st["scale2"] = _to_four_bits(st["W2"], case["group"])
    if case["kind"] == "train":
        st["dY"] = _normal(gen, (rows, d), 1e-2)
        st["kept"] = torch.empty((rows, 2 * f), dtype=torch.bfloat16, device="cuda")
        st["dX"], st["dW1"], st["dW2"] = torch.empty_like(st["X"]), torch.empty_like(st["W1"]), torch.empty_like(st["W2"])
    if own:
        from paper_2506_01084_amd import api

        st["ctx"] = api.Context(B=1, V=8, M=2, cap=0, d=d)
        st["block"] = api.GatedFFN(st["W1"], st["W2"], act=case["act"], scale_1=st["scale1"], scale_2=st["scale2"])
        if case["kind"] == "train":
            st["grad"] = api.GatedFFN(st["dW1"], st["dW2"], act=case["act"])
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(st):
    return dict(ffn=_run_ffn, train=_run_train, q4=_run_ffn, clip=_run_clip)[st["case"]["kind"]](st)


def _act(x, kind):
    return x / (1 + torch.exp(-x)) if kind == "silu" else 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))


def _slope(x, kind):
    if kind == "silu":
        s = 1 / (1 + torch.exp(-x))
        return s * (1 + x * (1 - s))
    return 0.5 * (1 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)


def _weights(W, scale, cols):
    """The matrix in 32 bits, out of 4 where there are scales."""
    if scale is None:
        return W.float()
    tiles, blocks = W.shape[:2]
    groups, rows = scale.shape
    q = W[:, :, :, :, None] >> torch.arange(0, 32, 4, dtype=torch.int32, device="cuda") & 15
    q = q.reshape(tiles, blocks, 4, 16, 4, 8).permute(0, 3, 1, 4, 2, 5).reshape(rows, blocks * 128)
    value = torch.tensor(FOUR_BITS, device="cuda")[q[:, :cols]]
    return (value.reshape(rows, groups, -1) * scale.T.float()[:, :, None]).reshape(rows, cols)


def _run_ffn(st):
    if own:
        st["ctx"].gated_ffn(st["X"], st["block"], st["Y"], residual=st["residual"])
        return st["Y"]
    d, f, act = st["case"]["d"], st["case"]["f"], st["case"]["act"]
    GU = st["X"].float() @ _weights(st["W1"], st["scale1"], d).T
    Y = (_act(GU[:, :f], act) * GU[:, f:]) @ _weights(st["W2"], st["scale2"], f).T
    return (Y if st["residual"] is None else Y + st["residual"].float()).to(st["Y"].dtype)


def _run_train(st):
    if own:
        st["ctx"].gated_ffn(st["X"], st["block"], st["Y"], residual=st["residual"], kept=st["kept"])
        st["ctx"].gated_ffn_backward(st["X"], st["block"], st["kept"], st["dY"], st["dX"], st["grad"])
        return st["Y"], st["dX"], st["dW1"], st["dW2"]
    f, act = st["case"]["f"], st["case"]["act"]
    X, W1, W2, dY = st["X"].float(), st["W1"].float(), st["W2"].float(), st["dY"].float()
    GU = X @ W1.T
    G, U = GU[:, :f], GU[:, f:]
    A = _act(G, act)
    F = A * U
    Y = F @ W2.T + st["residual"].float()
    dF = dY @ W2
    dGU = torch.cat([dF * U * _slope(G, act), dF * A], dim=1)
    dt = st["X"].dtype
    return Y.to(dt), (dGU @ W1).to(dt), (dGU.T @ X).to(dt), (dY.T @ F).to(dt)


def _run_clip(st):
    if own:
        st["ctx"].clip_gradients(st["list"], st["max_norm"], st["norm"])
        return (*st["out"], st["norm"])
    squares = torch.stack([(g.float() * g.float()).sum() for g in st["grads"]])
    norm = torch.sqrt(squares.sum())
    c = torch.clamp(st["max_norm"] / norm, max=1.0)
    return (*[(g.float() * c).to(g.dtype) for g in st["grads"]], torch.stack([norm, c]))


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "clip":
        by = sum(2 * math.prod(shape) * dtype.itemsize for shape, dtype in _shapes(case))
        return dict(bytes=int(by), flops=int(3 * sum(math.prod(shape) for shape, _ in _shapes(case))))
    rows, d, f = case["rows"], case["d"], case["f"]
    product = 2.0 * rows * d * f
    if case["kind"] == "train":
        # X, dY, the residual, both outputs; the weights and their gradients
        return dict(bytes=int(2 * 5 * rows * d + 2 * 2 * 3 * d * f), flops=int(9 * product))
    weights = 3 * d * f * (2.0 if case["kind"] == "ffn" else 0.5 + 2.0 / case["group"])
    return dict(bytes=int(2 * (3 if case.get("residual", True) else 2) * rows * d + weights), flops=int(3 * product))


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------------
def _decoded(words, scale, group):
    """4-bit weights in 64 bits, one place in a word at a time."""
    groups, rows = scale.shape
    W = torch.zeros((rows, words.shape[1] * 128), dtype=torch.float64, device="cuda")
    w = words.to(torch.int64).reshape(-1, words.shape[1], 4, 16, 4)
    for j in range(4):
        for m in range(4):
            for column in range(8):
                code = ((w[:, :, j, :, m] >> (4 * column)) & 15).permute(0, 2, 1).reshape(rows, -1)
                fraction, power = (code & 1).to(torch.float64), (code >> 1 & 3).to(torch.float64)
                size = torch.where(power == 0, fraction / 2, (1 + fraction / 2) * torch.exp2(power - 1))
                W[:, 32 * m + 8 * j + column::128] = torch.where(code >= 8, -size, size)
    W = W[:, :groups * group]
    return W * scale.to(torch.float64).repeat_interleave(group, dim=0).T


def exact(case, seed):
    st = prepare(case, seed)
    f64 = torch.float64
    if case["kind"] == "clip":
        total = sum(float(torch.linalg.vector_norm(g.to(f64))) ** 2 for g in st["grads"])
        norm = math.sqrt(total)
        c = min(1.0, st["max_norm"] / norm)
        return (*[g.to(f64) * c for g in st["grads"]], torch.tensor([norm, c], dtype=f64, device="cuda"))
    d, f = case["d"], case["f"]
    X = st["X"].to(f64)
    if case["kind"] == "q4":
        W1, W2 = (_decoded(st[w], st[s], case["group"]) for w, s in (("W1", "scale1"), ("W2", "scale2")))
    else:
        W1, W2 = st["W1"].to(f64), st["W2"].to(f64)
    gate, up = X @ W1[:f].T, X @ W1[f:].T
    if case["act"] == "silu":
        p = torch.sigmoid(gate)
        a, slope = gate * p, p + gate * p * (1 - p)
    else:
        p = 0.5 * torch.erfc(-gate / math.sqrt(2.0))
        a, slope = gate * p, p + gate * torch.exp(-gate * gate / 2) / math.sqrt(2 * math.pi)
    hidden = a * up
    Y = hidden @ W2.T
    if st["residual"] is not None:
        Y += st["residual"].to(f64)
    if case["kind"] != "train":
        return Y
    dY = st["dY"].to(f64)
    dhidden = dY @ W2
    dgate, dup = dhidden * up * slope, dhidden * a
    dX = dgate @ W1[:f] + dup @ W1[f:]
    return Y, dX, torch.cat([dgate.T @ X, dup.T @ X]), dY.T @ hidden
