"""GPU: the gradient of extended_distill where the sums of its parts cancel.  A row of dZ sums to zero, so what all rows of W have in common meets the
listed columns with one sign and the others with the other; the same holds for a column of dZ and the rows of H where the student is as sure of a
column as its teachers are.  Each gradient is rounded once, from an fp32 sum of all of its parts.

Bars, on the root mean square of a tensor's error.  A rounding is off by up to half a step h = 2^-8 2^floor(log2 |x|) either way, h^2 / 3 on average
over its square; dZ is rounded where nothing is listed, the outputs once.  Those errors are independent of each other: the squares add up,
weighted by the squares of what they are multiplied with (15 % for what their mean may be off by over a few hundred rows).  The exponent's error of p,
the same for a whole row, and the fp32 sums move a value by at most their share of the magnitudes; that is added as it is."""
import numpy as np
import pytest

import oracle
from paper_2506_01084_amd import workloads as wl

from helpers import gpu_encode, oracle_encode_batch, storage_to_host, torch_storage

pytestmark = pytest.mark.gpu


def _step2(x):
    """The mean square of bf16's rounding error of x."""
    a = np.abs(x)
    h = np.where(a > 0, 2.0 ** (np.floor(np.log2(np.where(a > 0, a, 1.0))) - 8), 0.0)
    return h * h / 3


@pytest.mark.parametrize("common_w,common_h", [(4.0, 0.0), (1.0, 2.0), (0.0, 4.0)])
@pytest.mark.parametrize("B,N,V,d,cap,K,T,chunk", [
    (2, 61, 3000, 128, 200, 33, 2.0, 0),             # the streaming kernel; dH's base product in parts
    (3, 100, 900, 192, 60, 8, 1.0, 0),               # the tile kernel, products whole
    (2, 60, 1200, 64, 0, 200, 4.0, 0),               # no codebook: dH is the base product's
    (2, 1100, 500, 64, 40, 5, 2.0, 0),               # more positions than one workgroup sorts; dW_base in parts
    (3, 100, 900, 192, 60, 8, 1.0, 1),               # a sequence at a time
    (1, 1, 300, 64, 20, 30, 1.0, 0),
])
def test_gradients_are_rounded_once(B, N, V, d, cap, K, T, chunk, common_w, common_h):
    import torch
    from paper_2506_01084_amd import api

    print(f"[case] distill sums B={B} N={N} V={V} d={d} cap={cap} K={K} T={T} chunk={chunk} common {common_w} {common_h}", flush=True)
    cfg = dict(name="sums", B=B, N=max(N, 200), V=V, d=d, dtype="bf16", M=3, cap=cap, zipf_s=1.2, copy_frac=0.4, span=(2, 6), mode="motif", pool="mean",
               seed=V + N)
    rng = np.random.default_rng(V + d)
    tokens, lens = wl.make_tokens(cfg), wl.make_lens(cfg)
    E = oracle.round_to_storage(0.02 * (rng.normal(size=(V, d)) + common_w * rng.normal(size=d)), "bf16")
    H = oracle.round_to_storage(rng.normal(size=(B * N, d)) + common_h * rng.normal(size=d), "bf16")
    ctx = api.Context(B=B, V=V, M=3, cap=cap, d=d, dtype="bf16")
    gpu_encode(ctx, tokens, lens)
    sizes = [len(x[1]) for x in oracle_encode_batch(tokens, lens, V, 3, cap)]
    d_E, d_H = torch_storage(E, "bf16"), torch_storage(H, "bf16")
    d_W = torch.zeros((B, cap, d), dtype=torch.bfloat16, device="cuda")
    ctx.hyper_embed(d_E, d_W)
    ids = np.stack([rng.permutation(V + sizes[r // N])[:K] for r in range(B * N)]).astype(np.int32)
    t = (2 * rng.normal(size=(B * N, K))).astype(np.float32)
    d_ids, d_t = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    kl, lse, student = torch.empty(B * N, device="cuda"), torch.empty(B * N, device="cuda"), torch.empty((B * N, K), device="cuda")
    dH, dWb, dWh = (torch.full_like(x, 9.0) for x in (d_H, d_E, d_W))
    ctx.set_option(api.OPT_BACKWARD_CHUNK, chunk)
    ctx.extended_distill(d_H, N, d_E, d_W, d_ids, d_t, kl, lse, student, temperature=T)
    ctx.extended_distill_backward(d_H, N, d_E, d_W, d_ids, d_t, lse, student, None, dH, dWb, dWh, temperature=T)
    torch.cuda.synchronize()
    got_H, got_Wb, got_Wh, W_host = (oracle.to_f64(storage_to_host(x, "bf16"), "bf16") for x in (dH, dWb, dWh, d_W))
    W_bits = storage_to_host(d_W, "bf16")
    u = 2.0 ** -24
    sums = {"dW_base": [np.zeros((V, d)) for _ in range(3)]}           # value, mean square, share of the magnitudes
    err = {}
    E64 = oracle.to_f64(E, "bf16")
    for b in range(B):
        sl, C = slice(b * N, (b + 1) * N), sizes[b]
        r = oracle.extended_distill_backward(H[sl], E, W_bits[b], C, "bf16", ids[sl], t[sl], T, np.ones(N))
        W, h = np.concatenate([E64, W_host[b][:C]]), oracle.to_f64(H[sl], "bf16")
        listed = np.zeros(r["dZ"].shape, dtype=bool)
        np.put_along_axis(listed, ids[sl].astype(np.int64), True, axis=1)
        dense = _step2(np.where(listed, 0.0, r["dZ"]))
        mass = (np.abs(h) @ np.abs(W).T).max(axis=1)
        z = (d + 2) * u * mass
        off = (2 * z / T + 2.0 ** -18 + 8 * u * mass / T)[:, None]     # of p's exponent
        row = off * (np.where(listed, 0.0, r["P"]) @ W) , off * (np.where(listed, r["P"], 0.0) @ np.abs(W))
        sums[f"dH {b}"] = [r["dH"], dense @ W ** 2, np.abs(row[0]) + row[1] + (V + cap + K) * u * (np.abs(r["dZ"]) @ np.abs(W))]
        err[f"dH {b}"] = got_H[sl] - r["dH"]
        P = r["P"] * off
        share = np.abs(P.T @ h) + (N + K) * u * (np.abs(r["dZ"]).T @ np.abs(h))
        if C:
            sums[f"dW_hyper {b}"] = [r["dW_hyper"][:C], dense[:, V:].T @ h ** 2, share[V:]]
            err[f"dW_hyper {b}"] = got_Wh[b][:C] - r["dW_hyper"][:C]
        assert (got_Wh[b][C:] == 0).all()
        for a, x in zip(sums["dW_base"], (r["dW_base"], dense[:, :V].T @ h ** 2, share[:V])):
            a += x
    err["dW_base"] = got_Wb - sums["dW_base"][0]
    if chunk:
        del err["dW_base"]                                             # (one more rounding per pass over the sequences)
    for k, e in err.items():
        want, square, share = sums[k]
        bar = np.sqrt(1.15 * (square + _step2(want)).mean()) + np.sqrt((share ** 2).mean())
        rms = np.sqrt((e ** 2).mean())
        print(f"{k}: {rms / np.sqrt((want ** 2).mean()):.3e} of {bar / np.sqrt((want ** 2).mean()):.3e}", flush=True)
        assert rms <= bar, k
    ctx.close()
