"""GPU parity: extended_distill (the loss of section 2.4 against a teacher's top logits) and its backward pass through the C ABI against the float64
oracle.

Bars.  A logit is an fp32 sum of d products: off by at most (d + 2) 2^-24 of the sum of their magnitudes, z_tol; the log-sum-exp
moves by z_tol / T, its sums of positive terms in parts and the hardware exponentials by 2^-18, and every exponent x / T log2 e is
rounded once (2^-24 of up to |x| / T).  kl adds K products of fp32 values of the size of |ln q| + |ln p|.  dZ is that p (relative error of the
exponent's absolute one), minus q (2^-20); in columns that are not listed it is rounded to bf16 once (2^-8), the listed ones stay fp32.  dH, dW
are sums of products of it, in fp32; the dense part is rounded to bf16 (2^-8 of what stands there) before the listed rows are added, the whole once
more.  A row's error is bounded by the products of the magnitudes.
"""
import math

import numpy as np
import pytest

import oracle
from paper_2506_01084_amd import workloads as wl

from helpers import gpu_encode, oracle_encode_batch, storage_to_host, torch_storage

pytestmark = pytest.mark.gpu


def _setup(dtype, B, N, V, d, M, cap, K, seed):
    import torch
    from paper_2506_01084_amd import api

    cfg = dict(name="distill", B=B, N=max(N, 200), V=V, d=d, dtype=dtype, M=M, cap=cap, zipf_s=1.2, copy_frac=0.4, span=(2, 6), mode="motif",
               pool="mean", seed=seed)
    tokens = wl.make_tokens(cfg)
    lens = wl.make_lens(cfg, ragged=True)
    E, H = wl.make_embeddings(cfg), wl.make_hidden(cfg, B * N)
    ctx = api.Context(B=B, V=V, M=M, cap=cap, d=d, dtype=dtype)
    gpu_encode(ctx, tokens, lens)
    ref = oracle_encode_batch(tokens, lens, V, M, cap)
    d_E = torch_storage(E, dtype)
    d_W = torch.zeros((B, cap, d), dtype=ctx.torch_dtype, device="cuda")
    ctx.hyper_embed(d_E, d_W)
    d_W[torch.arange(cap, device="cuda")[None] >= ctx.codebook()[2][:, None]] = math.nan    # rows that are no columns
    rng = np.random.default_rng(seed)
    ids = np.full((B, N, K), -1, dtype=np.int32)
    t = (rng.normal(size=(B, N, K)) * 3).astype(np.float32)
    for b in range(B):
        n = V + len(ref[b][1])
        for i in range(N):
            ids[b, i] = rng.permutation(n)[:K] if K <= n else rng.integers(0, n, size=K)
            if len(ref[b][1]) and i % 3 == 0:
                ids[b, i, rng.integers(0, K)] = V + rng.integers(0, len(ref[b][1]))
            kind = rng.integers(0, 12)
            if kind == 0:
                ids[b, i] = rng.choice([-1, -2 ** 31], size=K)       # nothing, with anything beside it
                t[b, i] = rng.choice([math.nan, math.inf, 0.0], size=K)
            elif kind == 1:
                ids[b, i, K // 2:] = -1                              # a shorter list
                t[b, i, K // 2:] = math.nan
            elif kind == 2:
                ids[b, i, rng.integers(0, K)] = ids[b, i, 0]         # twice
            elif kind == 3:
                ids[b, i, K - 1] = n                                 # mass where no column is
            elif kind == 4:
                ids[b, i, K - 1], t[b, i, K - 1] = 2 ** 31 - 1, -math.inf
            elif kind == 5:
                t[b, i, ::2] = np.float32(-3.4028235e38)             # the type's lowest value
            elif kind == 6:
                t[b, i] = -math.inf if i % 2 else np.float32(-3.4028235e38)
    return ctx, ref, E, H, d_E, d_W, ids.reshape(B * N, K), t.reshape(B * N, K), rng


def _bars(E, W, H, d, dtype, T):
    u = 2.0 ** -24
    mass = np.abs(oracle.to_f64(H, dtype)) @ np.abs(np.concatenate([oracle.to_f64(E, dtype), W])).T
    z = (d + 2) * u * mass.max(axis=1)
    return z, z / T + 2.0 ** -18 + 8 * u * mass.max(axis=1) / T


SHAPES = [
    # dtype, B, N, V, d, M, cap, K, T
    ("bf16", 3, 1, 3000, 128, 3, 100, 8, 1.0),        # one row per sequence
    ("bf16", 3, 1, 3000, 128, 3, 100, 8, 2.0),
    ("bf16", 70, 1, 30000, 128, 3, 50, 5, 4.0),
    ("bf16", 300, 1, 600, 64, 3, 20, 3, 2.0),         # more rows than the streaming kernel takes, one per sequence
    ("bf16", 4, 5, 2000, 256, 4, 300, 33, 1.0),       # a few rows
    ("bf16", 4, 5, 2000, 256, 4, 300, 33, 0.0625),
    ("bf16", 2, 61, 5003, 192, 3, 200, 64, 2.0),      # the streaming kernel
    ("bf16", 2, 45, 33000, 64, 3, 60, 9, 2.0),        # 90 and 140 rows of it, tiles of 256 and of 128 columns
    ("bf16", 2, 70, 700, 128, 3, 300, 11, 2.0),
    ("bf16", 2, 150, 2100, 64, 3, 300, 65, 1.5),      # the tile kernel
    ("bf16", 3, 301, 700, 320, 3, 120, 256, 1024.0),
    ("bf16", 2, 40, 300, 64, 3, 0, 1, 1.0),           # no codebook, one column
    ("bf16", 2, 23, 40, 1024, 3, 30, 2, 3.0),
    ("f32", 3, 39, 1200, 100, 3, 200, 20, 1.0),
    ("f32", 2, 7, 130, 4, 3, 60, 100, 2.0),
    ("bf16", 2, 33, 500, 72, 3, 90, 7, 2.0),          # a width of the general kernel
    ("f32", 1, 1, 1, 4, 1, 0, 1, 1.0),
]


@pytest.mark.parametrize("dtype,B,N,V,d,M,cap,K,T", SHAPES)
def test_loss_matches_oracle(dtype, B, N, V, d, M, cap, K, T):
    import torch

    print(f"[case] distill {dtype} B={B} N={N} V={V} d={d} cap={cap} K={K} T={T}", flush=True)
    ctx, ref, E, H, d_E, d_W, ids, t, rng = _setup(dtype, B, N, V, d, M, cap, K, 50 + V + N)
    kl, lse = (torch.full((B * N,), 7.0, device="cuda") for _ in range(2))
    student = torch.full((B * N, K), 7.0, device="cuda")
    ctx.extended_distill(torch_storage(H, dtype), N, d_E, d_W, torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), kl, lse, student, temperature=T)
    torch.cuda.synchronize()
    got_kl, got_lse, got_z = (x.cpu().numpy().astype(np.float64) for x in (kl, lse, student))
    W_host = storage_to_host(d_W, dtype)
    for b in range(B):
        sl = slice(b * N, (b + 1) * N)
        C = len(ref[b][1])
        r = oracle.extended_distill(H[sl], E, W_host[b][:C], C, dtype, ids[sl], t[sl], T)
        z_tol, lse_tol = _bars(E, oracle.to_f64(W_host[b][:C], dtype), H[sl], d, dtype, T)
        assert (np.abs(got_lse[sl] - r["lse"]) <= lse_tol).all(), f"lse seq {b}: {np.abs(got_lse[sl] - r['lse']).max()} {lse_tol.min()}"
        assert (np.abs(got_z[sl] - r["student"]) <= z_tol[:, None]).all()
        absent = (ids[sl] < 0) | (ids[sl] >= V + C)
        assert (got_z[sl][absent] == 0).all()
        inf = np.isinf(r["kl"])
        assert (np.isposinf(got_kl[sl]) == inf).all()
        size = np.abs(r["logits"]).max(axis=1) / T + np.abs(r["lse"]) + 60.0
        bar = z_tol / T + lse_tol + (K + 16) * 2.0 ** -24 * size
        assert (np.abs(got_kl[sl][~inf] - r["kl"][~inf]) <= bar[~inf]).all(), f"kl seq {b}"
        nothing = np.array([len(oracle.loss.teacher_distribution(ids[i], t[i], T, V + C)[0]) == 0 for i in range(sl.start, sl.stop)])
        assert (got_kl[sl][nothing] == 0).all()
    ctx.close()


@pytest.mark.parametrize("chunk", [0, 1])
@pytest.mark.parametrize("dtype,B,N,V,d,M,cap,K,T", [s for s in SHAPES if s[0] == "bf16" and s[4] % 64 == 0])
def test_gradients_match_oracle(dtype, B, N, V, d, M, cap, K, T, chunk):
    import torch
    from paper_2506_01084_amd import api

    print(f"[case] distill backward B={B} N={N} V={V} d={d} cap={cap} K={K} T={T} chunk={chunk}", flush=True)
    ctx, ref, E, H, d_E, d_W, ids, t, rng = _setup(dtype, B, N, V, d, M, cap, K, 90 + V + N)
    d_W = torch.nan_to_num(d_W.float()).bfloat16()          # (the products read whole codebooks)
    kl, lse = (torch.empty(B * N, device="cuda") for _ in range(2))
    student = torch.empty((B * N, K), device="cuda")
    d_H, d_ids, d_t = torch_storage(H, dtype), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    g = rng.uniform(0.25, 2.0, size=B * N).astype(np.float32)
    g[rng.random(B * N) < 0.1] = 0.0
    use_g = K != 64
    ctx.extended_distill(d_H, N, d_E, d_W, d_ids, d_t, kl, lse, student, temperature=T)
    dH, dWb, dWh = torch.full_like(d_H, 9.0), torch.full_like(d_E, 9.0), torch.full_like(d_W, 9.0)
    ctx.set_option(api.OPT_BACKWARD_CHUNK, chunk)
    ctx.extended_distill_backward(d_H, N, d_E, d_W, d_ids, d_t, lse, student, torch.from_numpy(g).cuda() if use_g else None, dH, dWb, dWh, temperature=T)
    torch.cuda.synchronize()
    dH_h, dWb_h, dWh_h, W_host = (oracle.to_f64(storage_to_host(x, dtype), dtype) for x in (dH, dWb, dWh, d_W))
    W_bits = storage_to_host(d_W, dtype)
    half = 2.0 ** -8 * 1.01
    want_Wb, dense_Wb, bar_Wb = np.zeros((V, d)), np.zeros((V, d)), np.zeros((V, d))
    for b in range(B):
        sl = slice(b * N, (b + 1) * N)
        C = len(ref[b][1])
        gr = g[sl] if use_g else np.ones(N)
        r = oracle.extended_distill_backward(H[sl], E, W_bits[b], C, dtype, ids[sl], t[sl], T, gr)
        z_tol, lse_tol = _bars(E, W_host[b][:C], H[sl], d, dtype, T)
        listed = np.zeros(r["dZ"].shape, dtype=bool)
        for i in range(N):
            listed[i, ids[sl][i][(ids[sl][i] >= 0) & (ids[sl][i] < V + C)]] = True
        dense, size = np.where(listed, 0.0, r["dZ"]), np.abs(r["dZ"])
        # listed columns: fp32 throughout.  The others: rounded to bf16 once
        off = (z_tol / T + lse_tol + 2.0 ** -18)[:, None] * r["P"] + 2.0 ** -20 * (size + r["P"]) + (half + 2.0 ** -16) * np.abs(dense)
        off += (V + cap + N + K) * 2.0 ** -24 * size                    # (and the products' own fp32 sums)
        W = np.concatenate([oracle.to_f64(E, dtype), W_host[b][:C]])
        # dH: the dense base product, that with the hyper product, and that with the listed rows are each rounded to bf16: half a step of each
        base = dense[:, :V] @ W[:V]
        bar = off @ np.abs(W) + half * (np.abs(base) + np.abs(base + dense[:, V:] @ W[V:]) + np.abs(r["dH"])) + 1e-30
        assert (np.abs(dH_h[sl] - r["dH"]) <= bar).all(), f"dH seq {b}"
        # dW: the dense product (with the earlier passes', one at a time), and that with the listed rows
        h = oracle.to_f64(H[sl], dtype)
        got, want = dWh_h[b], r["dW_hyper"]
        bar = np.zeros_like(want)
        bar[:C] = off[:, V:].T @ np.abs(h) + half * np.abs(dense[:, V:].T @ h)
        assert (np.abs(got - want) <= bar + half * np.abs(want)).all(), f"dW_hyper seq {b}"
        assert (got[C:] == 0).all()
        want_Wb += r["dW_base"]
        dense_Wb += dense[:, :V].T @ h
        bar_Wb += off[:, :V].T @ np.abs(h)
        if chunk or b + 1 == B:
            bar_Wb += half * np.abs(dense_Wb)
    assert (np.abs(dWb_h - want_Wb) <= bar_Wb * 1.02 + half * np.abs(want_Wb)).all(), "dW_base"
    ctx.close()


def test_one_column_is_the_target_of_the_loss():
    """K = 1 at T = 1: extended_nll and its backward pass, bit for bit where the arithmetic is the same and within its bars elsewhere."""
    import torch

    print("[case] distill, one column", flush=True)
    ctx, ref, E, H, d_E, d_W, ids, t, rng = _setup("bf16", 3, 70, 900, 128, 3, 100, 1, 5)
    d_W = torch.nan_to_num(d_W.float()).bfloat16()
    rows = 210
    t[:] = np.where(np.isfinite(t), t, 0.5)                  # (a logit that lists nothing is no target)
    d_H, d_ids, d_t = torch_storage(H, "bf16"), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    kl, lse, nll, lse2 = (torch.empty(rows, device="cuda") for _ in range(4))
    student = torch.empty((rows, 1), device="cuda")
    ctx.extended_distill(d_H, 70, d_E, d_W, d_ids, d_t, kl, lse, student)
    ctx.extended_nll(d_H, 70, d_E, d_W, d_ids.reshape(-1), nll, lse2)
    torch.cuda.synchronize()
    assert torch.equal(lse, lse2)
    same = torch.isinf(kl) == torch.isinf(nll)
    assert same.all() and torch.allclose(kl[torch.isfinite(kl)], nll[torch.isfinite(nll)], atol=2e-6, rtol=2e-6)
    out = []
    for fn in (lambda *o: ctx.extended_distill_backward(d_H, 70, d_E, d_W, d_ids, d_t, lse, student, None, *o),
               lambda *o: ctx.extended_nll_backward(d_H, 70, d_E, d_W, d_ids.reshape(-1), lse, None, *o)):
        o = (torch.empty_like(d_H), torch.empty_like(d_E), torch.empty_like(d_W))
        fn(*o)
        out.append(o)
    torch.cuda.synchronize()
    for a, b in zip(*out):
        scale = b.float().abs().amax(dim=-1, keepdim=True)
        assert ((a.float() - b.float()).abs() <= 2.0 ** -7 * scale).all()
    ctx.close()


def test_a_teacher_that_is_not_finite_makes_its_row_nan_and_no_other():
    import torch

    print("[case] distill, NaN", flush=True)
    ctx, ref, E, H, d_E, d_W, ids, t, rng = _setup("bf16", 1, 20, 500, 64, 3, 20, 5, 6)
    ids[:] = rng.integers(0, 500, size=ids.shape)
    t[:] = 1.0
    t[3, 2], t[4, 1] = math.nan, math.inf
    args = (torch_storage(H, "bf16"), 20, d_E, torch.nan_to_num(d_W.float()).bfloat16(), torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda())
    kl, lse, student = torch.empty(20, device="cuda"), torch.empty(20, device="cuda"), torch.empty((20, 5), device="cuda")
    ctx.extended_distill(*args, kl, lse, student, temperature=2.0)
    dH, dWb, dWh = torch.empty_like(args[0]), torch.empty_like(d_E), torch.empty_like(args[3])
    ctx.extended_distill_backward(*args, lse, student, None, dH, dWb, dWh, temperature=2.0)
    torch.cuda.synchronize()
    bad = torch.tensor([3, 4], device="cuda")
    assert torch.isnan(kl).sum() == 2 and torch.isnan(kl[bad]).all() and torch.isfinite(lse).all()
    assert torch.isnan(dH[bad]).all() and torch.isnan(dH).any(dim=1).sum() == 2
    ctx.close()


def test_a_training_step_runs_eagerly_captured_and_beside_another():
    """Lookup, loss, its gradient, the lookup's gradient and the pooling's: as a program trains with them.  dE against the oracle's chain on the
    kernels' own roundings; a captured step replays on new inputs with the eager bits (but for the pooling's float atomics); two contexts on
    two streams at once; larger eager work between the replays."""
    import torch
    from paper_2506_01084_amd import api

    print("[case] a distillation step", flush=True)
    B, N, V, d, M, cap, K, T = 3, 90, 900, 128, 3, 120, 16, 2.0

    def state():
        ctx, ref, E, H, d_E, d_W, ids, t, rng = _setup("bf16", B, N, V, d, M, cap, K, 21)
        codes = torch.from_numpy(np.stack([rng.integers(0, V + len(ref[b][1]), size=N) for b in range(B)]).astype(np.int32)).cuda()
        z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")
        return dict(ctx=ctx, ref=ref, E=d_E, W=torch.nan_to_num(d_W.float()).bfloat16(), codes=codes, ids=torch.from_numpy(ids).cuda(),
                    t=torch.from_numpy(t).cuda(), X=z(B, N, d, dt=torch.bfloat16), st=z(B, dt=torch.int32), kl=z(B * N), lse=z(B * N),
                    z=z(B * N, K), g=torch.full((B * N,), 0.5, device="cuda"), dX=z(B * N, d, dt=torch.bfloat16), dWb=z(V, d, dt=torch.bfloat16),
                    dWh=z(B, cap, d, dt=torch.bfloat16), dWin=z(B, cap, d, dt=torch.bfloat16), dE=z(V, d))

    def step(s, pool=True):
        c = s["ctx"]
        c.embed_codes(s["codes"], None, s["E"], s["W"], s["X"], s["st"], scale=5.0)
        H = s["X"].reshape(B * N, d)
        c.extended_distill(H, N, s["E"], s["W"], s["ids"], s["t"], s["kl"], s["lse"], s["z"], temperature=T)
        c.extended_distill_backward(H, N, s["E"], s["W"], s["ids"], s["t"], s["lse"], s["z"], s["g"], s["dX"], s["dWb"], s["dWh"], temperature=T)
        c.embed_codes_backward(s["codes"], None, s["dX"].reshape(B, N, d), s["dE"], s["dWin"], scale=5.0)
        c.embed_codes_backward(s["codes"], None, s["dX"].reshape(B, N, d), torch.zeros_like(s["dE"]), s["dWh"], scale=5.0, add=True)
        if pool:
            c.hyper_embed_backward(s["dWh"], s["dE"])

    s = state()
    step(s)
    torch.cuda.synchronize()
    # the chain behind dX and dWh, from the values the kernels left
    want = np.zeros((V, d))
    size = np.zeros((V, d))
    dX, dWh = storage_to_host(s["dX"], "bf16").reshape(B, N, d), oracle.bf16_bits_to_f64(storage_to_host(s["dWh"], "bf16"))
    for b in range(B):
        r = oracle.embed_codes_backward(s["codes"][b].cpu().numpy(), dX[b], V, len(s["ref"][b][1]), cap, "bf16", 5.0)
        want += r["dE"] + oracle.hyper_embed_backward(dWh[b], s["ref"][b][1], V, "mean", ())
        size += r["mass"][:V] + oracle.hyper_embed_backward(np.abs(dWh[b]), s["ref"][b][1], V, "mean", ())
    terms = B * (N + cap)
    assert (np.abs(s["dE"].cpu().numpy() - want) <= (terms + 4) * 2.0 ** -24 * size + 1e-30).all()

    graphed = state()
    step(graphed, pool=False)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed, pool=False)
    outputs = ("X", "kl", "lse", "z", "dX", "dWb", "dWh", "dWin", "dE")
    gen = torch.Generator(device="cuda").manual_seed(3)
    for turn in range(4):
        s["codes"].copy_(torch.randint(0, V, (B, N), generator=gen, device="cuda", dtype=torch.int32))
        s["t"].copy_(torch.randn((B * N, K), generator=gen, device="cuda"))
        for k in ("codes", "t"):
            graphed[k].copy_(s[k])
        graph.replay()
        step(s, pool=False)
        torch.cuda.synchronize()
        for k in outputs:
            a, b = s[k].float(), graphed[k].float()
            assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)), (turn, k)
        rows = 700 + 100 * turn                              # more than the graph's buffers hold
        big = torch.randn((B * rows, d), generator=gen, device="cuda").bfloat16()
        f = [torch.empty(B * rows, device="cuda") for _ in range(2)]
        bi, bt = graphed["ids"][:1].repeat(B * rows, 1).contiguous(), graphed["t"][:1].repeat(B * rows, 1).contiguous()
        bz = torch.empty((B * rows, K), device="cuda")
        graphed["ctx"].extended_distill(big, rows, s["E"], s["W"], bi, bt, *f, bz, temperature=T)
        graphed["ctx"].extended_distill_backward(big, rows, s["E"], s["W"], bi, bt, f[1], bz, None, torch.empty_like(big), graphed["dWb"].clone(),
                                                 graphed["dWh"].clone(), temperature=T)
        torch.cuda.synchronize()
    # both at once, on streams of their own
    want = {k: s[k].clone() for k in outputs}
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(s1):
            step(s, pool=False)
        with torch.cuda.stream(s2):
            step(graphed, pool=False)
    torch.cuda.synchronize()
    for k in outputs:
        for x in (s, graphed):
            assert torch.equal(torch.nan_to_num(want[k].float()), torch.nan_to_num(x[k].float())), k
    s["ctx"].close()
    graphed["ctx"].close()
