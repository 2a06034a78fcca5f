"""Operators at the two ends of a model over the extended vocabulary, for timing: the lookup of codes and its gradient,
the loss against a teacher's top logits and its gradient, the pick of a beam search and the move of its codebooks.

A case is a dict of plain values.  `prepare` makes what a program holds before the call, `run` is one pass through an
operator: with `own` false in elementary tensor operations, with `own` true through the library's binding.  `work` gives
the bytes and operations that a pass cannot do without, `exact` the results in 64 bits.

Codebooks hold phrases of two base tokens, distinct within a sequence; codes and teachers' columns are spread evenly over
the logarithm of their rank (Zipf's law with exponent 1), weights N(0, 0.02), hidden rows N(0, 1) for the losses and
pointed at a dozen columns for the picks, as a trained model's are.
"""
from __future__ import annotations

import math

import torch

own = False


def listed():
    return [
        # the input of a generation step: one code for each of 64 sequences
        dict(name="lookup_64x1", kind="lookup", B=64, N=1, V=128256, d=4096, cap=1024, dtype="bf16", ragged=False),
        # a training batch's input rows, padded to the longest
        dict(name="lookup_8x4096", kind="lookup", B=8, N=4096, V=128256, d=4096, cap=2048, dtype="bf16", ragged=True),
        # a small model trained in fp32 on short ragged sequences: odd lengths, a width that no tile divides
        dict(name="lookup_grad_5x453_f32", kind="lookup_grad", B=5, N=453, V=32000, d=1000, cap=300, dtype="f32", ragged=True),
        # the gradient of a training batch's input rows
        dict(name="lookup_grad_8x4096", kind="lookup_grad", B=8, N=4096, V=128256, d=2048, cap=2048, dtype="bf16", ragged=True),
        # evaluation of a small fp32 student against a teacher's 20 best columns
        dict(name="distill_eval_3x117_f32", kind="distill", B=3, N=117, V=32000, d=256, cap=1000, K=20, T=1.0, dtype="f32", train=False),
        # a few short answers, teacher at a temperature, loss and gradient
        dict(name="distill_2x61", kind="distill", B=2, N=61, V=50257, d=1024, cap=700, K=33, T=2.0, dtype="bf16", train=True),
        # a distillation step's share of this path
        dict(name="distill_8x1024", kind="distill", B=8, N=1024, V=128256, d=4096, cap=2048, K=64, T=2.0, dtype="bf16", train=True),
        # one prompt searched with four beams on a small model
        dict(name="beam_1x4", kind="beam", P=1, beams=4, V=32000, d=1024, cap=512, picks=8, dtype="bf16"),
        # a serving batch: 16 prompts with four beams, twice as many candidates as beams
        dict(name="beam_16x4", kind="beam", P=16, beams=4, V=128256, d=4096, cap=1024, picks=8, dtype="bf16"),
        # many prompts and an odd number of beams, more rows than the decode kernels take in a pass
        dict(name="beam_27x5", kind="beam", P=27, beams=5, V=151936, d=3584, cap=512, picks=10, dtype="bf16"),
        # the beams' codebooks after a step: two of four die and are filled from the others, twice
        dict(name="reorder_1x4", kind="reorder", P=1, beams=4, V=32000, d=1024, cap=512, shared=300, grown=64, dtype="bf16"),
        # the same for a serving batch with long generations
        dict(name="reorder_16x4", kind="reorder", P=16, beams=4, V=128256, d=4096, cap=2048, shared=1400, grown=500, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    """Whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["lookup", "lookup_grad", "distill", "beam", "reorder"])
    V = rng.choice([rng.randint(8000, 50000), 32000, 50257, 128256, 151936])
    if kind in ("lookup", "lookup_grad"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = 8 * _log(rng, 8, 512) if dtype == "bf16" else 4 * _log(rng, 16, 512)
        if kind == "lookup_grad":
            V, d = min(V, 128256), min(d, 2048)
        B, N = _log(rng, 1, 64), _log(rng, 1, 4096)
        while B * N * d * (2 if dtype == "bf16" else 4) > (1 << 28 if kind == "lookup" else 1 << 27):
            N = N // 2 + 1
            if N <= 2:
                B = max(1, B // 2)
        return dict(kind=kind, B=B, N=N, V=V, d=d, cap=min(_log(rng, 16, 2048), 16384 // B), dtype=dtype, ragged=rng.random() < 0.6)
    if kind == "distill":
        if rng.random() < 0.3:
            return dict(kind=kind, B=_log(rng, 1, 6), N=_log(rng, 1, 200), V=rng.randint(8000, 32000), d=4 * _log(rng, 16, 256),
                        cap=_log(rng, 16, 1000), K=_log(rng, 1, 64), T=1.0, dtype="f32", train=False)
        d = 64 * _log(rng, 2, 64)
        B, N = _log(rng, 1, 16), _log(rng, 1, 1024)
        while B * N > 4096:
            N = N // 2 + 1
        return dict(kind=kind, B=B, N=N, V=V, d=d, cap=_log(rng, 16, 2048), K=_log(rng, 1, 128),
                    T=rng.choice([1.0, 1.5, 2.0, 4.0]), dtype="bf16", train=rng.random() < 0.75)
    beams = rng.randint(2, 8)
    P = _log(rng, 1, 24)
    if kind == "beam":
        return dict(kind=kind, P=P, beams=beams, V=V, d=128 * _log(rng, 2, 28), cap=min(_log(rng, 64, 1024), 65536 // (P * beams)), picks=rng.choice([beams, 2 * beams]), dtype="bf16")
    cap = _log(rng, 64, 2048)
    shared = rng.randint(0, cap // 2)
    return dict(kind=kind, P=min(P, 16), beams=max(beams, 3), V=V, d=128 * _log(rng, 2, 16), cap=cap, shared=shared,
                grown=rng.randint(1, cap - shared), dtype="bf16")


# ---- inputs -----------------------------------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _weights(gen, rows, d, dtype, std=0.02):
    return (torch.randn((rows, d), generator=gen, device="cuda") * std).to(dtype)


def _ranks(gen, shape, n):
    """Ranks in [0, n), even over the logarithm."""
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    return torch.clamp(torch.exp(u * math.log(n + 1)).long() - 1, 0, n - 1)


def _phrases(gen, n, V):
    """n distinct pairs of base tokens, [n, 2] int32."""
    first = _ranks(gen, (n,), V)
    step = torch.randint(0, V, (1,), generator=gen, device="cuda")
    second = (torch.arange(n, device="cuda") + step) % V           # distinct for up to V pairs
    return torch.stack([first, second], dim=1).int()


def _pooled(E, phrases):
    """The mean of a phrase's two embedding rows, rounded once."""
    a, b = E[phrases[..., 0].long()], E[phrases[..., 1].long()]
    return (a.float() * 0.5 + b.float() * 0.5).to(E.dtype)


def _context(case, B, phrases, sizes):
    """A context whose codebooks hold the first sizes[b] of phrases[b]."""
    from paper_2506_01084_amd import api

    ctx = api.Context(B=B, V=case["V"], M=2, cap=case["cap"], d=case["d"], dtype=case["dtype"], pool="mean")
    added = torch.empty(B, dtype=torch.int32, device="cuda")
    status = torch.empty(B, dtype=torch.int32, device="cuda")
    lens = torch.full(phrases.shape[:2], 2, dtype=torch.int32, device="cuda")
    ctx.codebook_prefill(phrases.contiguous(), lens, sizes, added, status, api.RESET)
    return ctx


def _books(gen, case, B, E):
    cap, V = case["cap"], case["V"]
    phrases = torch.stack([_phrases(gen, cap, V) for _ in range(B)])
    sizes = torch.randint(cap // 2, cap + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    W = _pooled(E, phrases)
    return phrases, sizes, W


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1_000_003 * seed + 17)
    return dict(lookup=_prepare_lookup, lookup_grad=_prepare_lookup, distill=_prepare_distill, beam=_prepare_beam,
                reorder=_prepare_reorder)[case["kind"]](gen, case)


def _lengths(gen, case):
    B, N = case["B"], case["N"]
    if not case.get("ragged", True):
        return torch.full((B,), N, dtype=torch.int32, device="cuda")
    lens = torch.randint(N // 2, N + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    lens[0] = N
    return lens


def _prepare_lookup(gen, case):
    B, N, V, d, cap, dt = case["B"], case["N"], case["V"], case["d"], case["cap"], _dtype(case)
    E = _weights(gen, V, d, dt)
    phrases, sizes, W = _books(gen, case, B, E)
    perm = torch.randperm(V, generator=gen, device="cuda")
    base = perm[_ranks(gen, (B, N), V)]
    entry = (torch.rand((B, N), generator=gen, device="cuda") * sizes[:, None]).long()
    hyper = torch.rand((B, N), generator=gen, device="cuda") < 0.3
    codes = torch.where(hyper & (sizes[:, None] > 0), V + entry, base).int()
    st = dict(case=case, E=E, W=W, sizes=sizes, codes=codes, lens=_lengths(gen, case), scale=math.sqrt(d))
    if case["kind"] == "lookup":
        st["X"] = torch.zeros((B, N, d), dtype=dt, device="cuda")
        st["status"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    else:
        st["dX"] = (torch.randn((B, N, d), generator=gen, device="cuda") * 1e-2).to(dt)
        st["dE"] = torch.zeros((V, d), dtype=torch.float32, device="cuda")
        st["dW"] = torch.zeros((B, cap, d), dtype=dt, device="cuda")
    if own:
        st["ctx"] = _context(case, B, phrases, sizes)
    return st


def _prepare_distill(gen, case):
    B, N, V, d, cap, K, dt = case["B"], case["N"], case["V"], case["d"], case["cap"], case["K"], _dtype(case)
    rows = B * N
    W_base = _weights(gen, V, d, dt)
    phrases, sizes, W = _books(gen, case, B, W_base)
    H = torch.randn((rows, d), generator=gen, device="cuda").to(dt)
    # a teacher's best columns: distinct, spread over the logarithm of their rank, hypertokens among them
    n = V + cap // 2
    perm = torch.randperm(n, generator=gen, device="cuda")
    u = torch.rand((rows, K), generator=gen, device="cuda", dtype=torch.float64)
    j = torch.arange(K, device="cuda")
    ranks = (torch.exp((j + u) / K * math.log(n - K)).long() - 1).clamp(0, n - K - 1) + j
    ids = perm[ranks].int()
    teacher = torch.sort(torch.randn((rows, K), generator=gen, device="cuda") * 2.0 + 8.0, dim=1, descending=True).values.contiguous()
    # some rows list fewer columns, padding behind a sequence's end lists none
    fewer = torch.rand((rows, 1), generator=gen, device="cuda") < 0.1
    ids = torch.where(fewer & (j >= (K + 1) // 2), torch.full_like(ids, -1), ids)
    lens = _lengths(gen, case)
    behind = (torch.arange(N, device="cuda")[None, :] >= lens[:, None]).reshape(rows, 1)
    ids = torch.where(behind, torch.full_like(ids, -1), ids).contiguous()
    st = dict(case=case, H=H, W_base=W_base, W=W, sizes=sizes, ids=ids, teacher=teacher,
              kl=torch.empty(rows, dtype=torch.float32, device="cuda"), lse=torch.empty(rows, dtype=torch.float32, device="cuda"),
              student=torch.empty((rows, K), dtype=torch.float32, device="cuda"))
    if case["train"]:
        # the usual T^2 / number of rows
        st["grad"] = torch.full((rows,), case["T"] ** 2 / rows, dtype=torch.float32, device="cuda")
        st["dH"], st["dW_base"], st["dW"] = torch.empty_like(H), torch.empty_like(W_base), torch.empty_like(W)
    if own:
        st["ctx"] = _context(case, B, phrases, sizes)
    return st


def _prepare_beam(gen, case):
    P, beams, V, d, cap, dt = case["P"], case["beams"], case["V"], case["d"], case["cap"], _dtype(case)
    B = P * beams
    W_base = _weights(gen, V, d, dt)
    phrases, sizes, W = _books(gen, case, B, W_base)
    # hidden rows point at a dozen columns, one of them a hypertoken; the rest of the vocabulary is noise
    H = torch.randn((B, d), generator=gen, device="cuda") * 0.2
    norm = 1.0 / (d * 0.02 ** 2)
    for i in range(12):
        want = 12.0 - 0.9 * i - 0.8 * torch.rand((B, 1), generator=gen, device="cuda")
        col = torch.randint(0, V, (B,), generator=gen, device="cuda")
        if i == 5:
            e = (torch.rand(B, generator=gen, device="cuda") * sizes).long()
            H += 2.0 * norm * want * W[torch.arange(B, device="cuda"), e].float()      # (the mean of two rows: half the square)
        else:
            H += norm * want * W_base[col].float()
    score = -torch.cumsum(torch.rand((P, beams), generator=gen, device="cuda") * 1.5, dim=1)
    fresh = torch.rand((P, 1), generator=gen, device="cuda") < 0.15                    # a prompt's first step: one beam lives
    score = torch.where(fresh & (torch.arange(beams, device="cuda") > 0), torch.full_like(score, -math.inf), score)
    st = dict(case=case, H=H.to(dt), W_base=W_base, W=W, sizes=sizes, score=score.reshape(B).contiguous(),
              parent=torch.empty((P, case["picks"]), dtype=torch.int32, device="cuda"),
              code=torch.empty((P, case["picks"]), dtype=torch.int32, device="cuda"),
              picked=torch.empty((P, case["picks"]), dtype=torch.float32, device="cuda"))
    if own:
        st["ctx"] = _context(case, B, phrases, sizes)
    return st


def _prepare_reorder(gen, case):
    P, beams, V, d, cap, dt = case["P"], case["beams"], case["V"], case["d"], case["cap"], _dtype(case)
    B, shared, grown = P * beams, case["shared"], case["grown"]
    E = _weights(gen, V, d, dt)
    # a prompt's beams share its entries and have grown their own since
    per_beam = torch.stack([_phrases(gen, cap, V) for _ in range(B)])
    prompt = per_beam[::beams].repeat_interleave(beams, dim=0)
    # (a beam's own pairs end in other tokens than the prompt's: no pair twice in a sequence)
    own_part = per_beam.clone()
    own_part[:, :, 1] = (prompt[:, :, 1] + cap + (torch.arange(B, device="cuda", dtype=torch.int32) % beams)[:, None] * 7) % V
    at = torch.arange(cap, device="cuda")[None, :, None]
    phrases = torch.where(at < shared, prompt, own_part).int()
    sizes = (shared + torch.randint((grown + 1) // 2, grown + 1, (B,), generator=gen, device="cuda")).int()
    live = torch.arange(cap, device="cuda")[None, :] < sizes[:, None]
    entries = torch.where(live[:, :, None], phrases, torch.full_like(phrases, -1)).contiguous()
    W = _pooled(E, phrases)
    # two beams live on, the others are filled from one of them, then from the other
    a = torch.randint(0, beams - 1, (P,), generator=gen, device="cuda")
    b = a + 1
    slot = torch.arange(beams, device="cuda")[None, :].expand(P, beams)
    keep = (slot == a[:, None]) | (slot == b[:, None])
    one = torch.where(keep, slot, torch.where(slot % 2 == 0, a[:, None], b[:, None])).reshape(B).int().contiguous()
    two = torch.where(keep, slot, torch.where(slot % 2 == 0, b[:, None], a[:, None])).reshape(B).int().contiguous()
    st = dict(case=case, E=E, W=W, sources=(one, two))
    if own:
        st["ctx"] = _context(case, B, phrases, sizes)
        st["book"] = st["ctx"].codebook()
    else:
        st["book"] = (entries, (live * 2).int(), sizes)
    return st


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(st):
    return dict(lookup=_run_lookup, lookup_grad=_run_lookup_grad, distill=_run_distill, beam=_run_beam,
                reorder=_run_reorder)[st["case"]["kind"]](st)


def _run_lookup(st):
    X, codes, lens = st["X"], st["codes"], st["lens"]
    if own:
        st["ctx"].embed_codes(codes, lens, st["E"], st["W"], X, st["status"], scale=st["scale"])
        return X, st["status"]
    V, cap = st["case"]["V"], st["case"]["cap"]
    N = codes.shape[1]
    c = codes.long()
    inside = torch.arange(N, device="cuda")[None, :] < lens[:, None]
    named = (c >= 0) & (c < V + st["sizes"][:, None])
    base = st["E"][c.clamp(0, V - 1)]
    b = torch.arange(c.shape[0], device="cuda")[:, None]
    hyper = st["W"][b, (c - V).clamp(0, cap - 1)]
    row = torch.where((c < V)[:, :, None], base, hyper).float() * st["scale"]
    row = torch.where(named[:, :, None], row, torch.zeros_like(row)).to(X.dtype)
    X.copy_(torch.where(inside[:, :, None], row, X))
    status = (2 * (inside & ~named).any(dim=1)).int()
    return X, status


def _run_lookup_grad(st):
    if own:
        st["ctx"].embed_codes_backward(st["codes"], st["lens"], st["dX"], st["dE"], st["dW"], scale=st["scale"])
        return st["dE"], st["dW"]
    case = st["case"]
    V, cap, d, B, N = case["V"], case["cap"], case["d"], case["B"], case["N"]
    c = st["codes"].long()
    inside = torch.arange(N, device="cuda")[None, :] < st["lens"][:, None]
    g = st["dX"].float() * st["scale"]
    to_base = (inside & (c >= 0) & (c < V)).reshape(-1)
    to_hyper = (inside & (c >= V) & (c < V + st["sizes"][:, None])).reshape(-1)
    g = g.reshape(B * N, d)
    dE = torch.zeros((V, d), device="cuda")
    dE.index_add_(0, c.reshape(-1)[to_base], g[to_base])
    dW = torch.zeros((B * cap, d), device="cuda")
    at = (torch.arange(B, device="cuda")[:, None] * cap + (c - V)).reshape(-1)
    dW.index_add_(0, at[to_hyper], g[to_hyper])
    return dE, dW.reshape(B, cap, d).to(st["dX"].dtype)


def _columns_exist(sizes, V, cap):
    """[B, V + cap] truth values: the columns that exist."""
    return torch.arange(V + cap, device="cuda")[None, :] < V + sizes[:, None]


def _joint_logits(H, W_base, W, sizes, N, kind):
    """[B, N, V + cap] logits in `kind`, -inf in columns that do not exist."""
    B, cap, d = W.shape
    V = W_base.shape[0]
    Hk = H.to(kind)
    z = torch.empty((B, N, V + cap), dtype=kind, device="cuda")
    z[:, :, :V] = (Hk @ W_base.to(kind).T).reshape(B, N, V)
    z[:, :, V:] = torch.bmm(Hk.reshape(B, N, d), W.to(kind).transpose(1, 2).contiguous())
    return z.masked_fill_(~_columns_exist(sizes, V, cap)[:, None, :], -math.inf)


def _run_distill(st):
    case = st["case"]
    N, T = case["N"], case["T"]
    if own:
        ctx = st["ctx"]
        ctx.extended_distill(st["H"], N, st["W_base"], st["W"], st["ids"], st["teacher"], st["kl"], st["lse"], st["student"], temperature=T)
        if not case["train"]:
            return st["kl"], st["lse"], st["student"]
        ctx.extended_distill_backward(st["H"], N, st["W_base"], st["W"], st["ids"], st["teacher"], st["lse"], st["student"],
                                      st["grad"], st["dH"], st["dW_base"], st["dW"], temperature=T)
        return st["kl"], st["lse"], st["student"], st["dH"], st["dW_base"], st["dW"]
    B, V, cap, d = case["B"], case["V"], case["cap"], case["d"]
    z = _joint_logits(st["H"], st["W_base"], st["W"], st["sizes"], N, torch.float32)
    z = z.reshape(B * N, V + cap)
    ids = st["ids"].long()
    used = ids >= 0
    student = torch.where(used, torch.gather(z, 1, ids.clamp(min=0)), torch.zeros(1, device="cuda"))
    z.div_(T)
    m = z.amax(dim=1, keepdim=True)
    lse = torch.log(torch.exp(z - m).sum(dim=1)) + m[:, 0]
    t = torch.where(used, st["teacher"] / T, torch.full_like(st["teacher"], -math.inf))
    tm = t.amax(dim=1, keepdim=True)
    some = used.any(dim=1)
    e = torch.where(used, torch.exp(t - torch.where(some[:, None], tm, torch.zeros_like(tm))), torch.zeros_like(t))
    s = torch.where(some, e.sum(dim=1), torch.ones_like(lse))
    q = e / s[:, None]
    diff = torch.where(used, t - tm - torch.log(s)[:, None] - student / T + lse[:, None], torch.zeros_like(t))
    kl = (q * diff).sum(dim=1)
    if not case["train"]:
        return kl, lse, student
    g = torch.where(some, st["grad"] / T, torch.zeros_like(lse))
    dz = z.sub_(lse[:, None]).exp_()                                # p
    dz.scatter_add_(1, ids.clamp(min=0), -q)
    dz.mul_(g[:, None])
    Hf = st["H"].float()
    dH = dz[:, :V] @ st["W_base"].float()
    dzh = dz.reshape(B, N, V + cap)[:, :, V:].contiguous()
    exist = torch.arange(cap, device="cuda")[None, :] < st["sizes"][:, None]
    dH += torch.bmm(dzh, torch.where(exist[:, :, None], st["W"].float(), torch.zeros(1, device="cuda"))).reshape(B * N, d)
    dW_base = dz[:, :V].T @ Hf
    dW = torch.bmm(dzh.transpose(1, 2).contiguous(), Hf.reshape(B, N, d))
    dt = st["H"].dtype
    return kl, lse, student, dH.to(dt), dW_base.to(dt), dW.to(dt)


def _run_beam(st):
    case = st["case"]
    P, beams, picks, V, cap = case["P"], case["beams"], case["picks"], case["V"], case["cap"]
    if own:
        st["ctx"].extended_beam(st["H"], beams, st["W_base"], st["W"], st["score"], st["parent"], st["code"], st["picked"])
        return st["parent"], st["code"], st["picked"]
    z = _joint_logits(st["H"], st["W_base"], st["W"], st["sizes"], 1, torch.float32).reshape(P * beams, V + cap)
    m = z.amax(dim=1, keepdim=True)
    lse = torch.log(torch.exp(z - m).sum(dim=1, keepdim=True)) + m
    cand = (z - lse + st["score"][:, None]).reshape(P, beams * (V + cap))
    best, at = torch.topk(cand, picks, dim=1)
    none = best == -math.inf
    parent = torch.where(none, torch.full_like(at, -1), at // (V + cap)).int()
    code = torch.where(none, torch.full_like(at, -1), at % (V + cap)).int()
    return parent, code, best


def _run_reorder(st):
    W = st["W"]
    if own:
        for source in st["sources"]:
            st["ctx"].codebook_reorder(st["case"]["beams"], source, W)
        return (*st["book"], W)
    entries, lens, sizes = st["book"]
    P, beams = st["case"]["P"], st["case"]["beams"]
    for source in st["sources"]:
        src = (torch.arange(P, device="cuda")[:, None] * beams + source.reshape(P, beams)).reshape(-1).long()
        from_lens = lens[src]
        W.copy_(torch.where((from_lens > 0)[:, :, None], W[src], W))
        entries.copy_(entries[src])
        lens.copy_(from_lens)
        sizes.copy_(sizes[src])
    return entries, lens, sizes, W


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------
def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    kind = case["kind"]
    if kind in ("lookup", "lookup_grad"):
        B, N, V, d, cap = case["B"], case["N"], case["V"], case["d"], case["cap"]
        rows = B * N * (0.75 if case["ragged"] and B > 1 else 1.0)
        if kind == "lookup":
            distinct = 0.3 * rows + min(0.7 * rows, V * (1 - math.exp(-0.7 * rows / V * 3)) / 3)
            return dict(bytes=int(rows * (d * size + 4) + distinct * d * size), flops=int(rows * d))
        return dict(bytes=int(rows * (d * size + 4) + V * d * 4 + B * cap * d * size), flops=int(2 * rows * d))
    if kind == "distill":
        B, N, V, d, cap, K = case["B"], case["N"], case["V"], case["d"], case["cap"], case["K"]
        rows, columns = B * N, V + 0.75 * cap
        weights = (V + 0.75 * cap * B) * d * size
        by = weights + rows * d * size + rows * K * 8 + rows * 8
        fl = 2.0 * rows * d * columns
        if case["train"]:
            by += weights + rows * d * size
            fl *= 4                                   # the logits once more or kept, and the two products
        return dict(bytes=int(by), flops=int(fl))
    B, d, cap = case["P"] * case["beams"], case["d"], case["cap"]
    if kind == "beam":
        return dict(bytes=int((case["V"] + 0.75 * cap * B) * d * size + B * d * size), flops=int(2.0 * B * d * (case["V"] + 0.75 * cap)))
    # the rows in which the moved beams differ from their sources, read and written, and their codebooks, twice
    moved = case["P"] * max(case["beams"] - 2, 0)
    return dict(bytes=int(2 * moved * 2 * (0.75 * case["grown"] * d * size + cap * 12)), flops=0)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "reorder":
        return None
    f64 = torch.float64
    if kind in ("lookup", "lookup_grad"):
        B, N, V, d, cap = case["B"], case["N"], case["V"], case["d"], case["cap"]
        if kind == "lookup":
            X = torch.zeros((B, N, d), dtype=f64, device="cuda")
            for b in range(B):
                n = int(st["lens"][b])
                table = torch.cat([st["E"], st["W"][b]])
                X[b, :n] = table[st["codes"][b, :n].long()].to(f64) * st["scale"]
            return X, torch.zeros(B, dtype=torch.int32, device="cuda")
        dE = torch.zeros((V, d), dtype=f64, device="cuda")
        dW = torch.zeros((B, cap, d), dtype=f64, device="cuda")
        for b in range(B):
            n = int(st["lens"][b])
            code, rows = st["codes"][b, :n].long(), st["dX"][b, :n].to(f64) * st["scale"]
            both = torch.zeros((V + cap, d), dtype=f64, device="cuda")
            both.index_add_(0, code, rows)
            dE += both[:V]
            dW[b] = both[V:]
        return dE, dW
    if kind == "beam":
        P, beams, V, cap, picks = case["P"], case["beams"], case["V"], case["cap"], case["picks"]
        parent, code, picked = [], [], []
        Wb = st["W_base"].to(f64)
        for p in range(P):
            cand = torch.full((beams, V + cap), -math.inf, dtype=f64, device="cuda")
            for k in range(beams):
                b = p * beams + k
                n = int(st["sizes"][b])
                h = st["H"][b].to(f64)
                z = torch.cat([Wb @ h, st["W"][b, :n].to(f64) @ h])
                cand[k, :V + n] = st["score"][b].to(f64) + z - torch.logsumexp(z, 0)
            best, at = torch.topk(cand.reshape(-1), picks)
            picked.append(best)
            parent.append((at // (V + cap)).int())
            code.append((at % (V + cap)).int())
        return torch.stack(parent), torch.stack(code), torch.stack(picked)
    B, N, V, d, cap, T = case["B"], case["N"], case["V"], case["d"], case["cap"], case["T"]
    kl = torch.zeros(B * N, dtype=f64, device="cuda")
    lse = torch.zeros(B * N, dtype=f64, device="cuda")
    student = torch.zeros((B * N, case["K"]), dtype=f64, device="cuda")
    if case["train"]:
        dH = torch.zeros((B * N, d), dtype=f64, device="cuda")
        dWb = torch.zeros((V, d), dtype=f64, device="cuda")
        dW = torch.zeros((B, cap, d), dtype=f64, device="cuda")
    Wb = st["W_base"].to(f64)
    for b in range(B):
        n = int(st["sizes"][b])
        table = torch.cat([Wb, st["W"][b, :n].to(f64)])
        sl = slice(b * N, (b + 1) * N)
        h = st["H"][sl].to(f64)
        logits = h @ table.T
        ids = st["ids"][sl].long()
        used = ids >= 0
        student[sl] = torch.where(used, torch.gather(logits, 1, ids.clamp(min=0)), torch.zeros(1, dtype=f64, device="cuda"))
        lse[sl] = torch.logsumexp(logits / T, dim=1)
        logp = torch.log_softmax(logits / T, dim=1)
        del logits
        t = torch.where(used, st["teacher"][sl].to(f64) / T, torch.tensor(-math.inf, dtype=f64, device="cuda"))
        some = used.any(dim=1)
        t = torch.where(some[:, None], t, torch.zeros_like(t))
        logq = torch.log_softmax(t, dim=1)
        q = torch.where(used, logq.exp(), torch.zeros_like(logq))
        term = torch.where(used, logq - torch.gather(logp, 1, ids.clamp(min=0)), torch.zeros_like(logq))
        kl[sl] = (q * term).sum(dim=1)
        if case["train"]:
            dz = logp.exp()
            dz.scatter_add_(1, ids.clamp(min=0), -q)
            dz *= torch.where(some, st["grad"][sl].to(f64) / T, torch.zeros(1, dtype=f64, device="cuda"))[:, None]
            dH[sl] = dz @ table
            dt = dz.T @ h
            dWb += dt[:V]
            dW[b, :n] = dt[V:]
            del dz, dt
        del table, logp
    return (kl, lse, student, dH, dWb, dW) if case["train"] else (kl, lse, student)
