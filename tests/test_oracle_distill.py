"""Pins of the oracle's loss against a teacher's top logits and its gradient (CPU)."""
import numpy as np
import pytest
import torch

import oracle


def _inputs(seed, rows=7, V=11, C=3, cap=5, d=4, K=6):
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.normal(size=s).astype(np.float32)
    ids = np.stack([rng.permutation(V + C)[:K] for _ in range(rows)]).astype(np.int32)
    return rng, f(rows, d), f(V, d), f(cap, d), C, ids, f(rows, K) * 2


@pytest.mark.parametrize("T", [1.0, 2.0, 0.5])
def test_full_lists_are_the_librarys_divergence_and_its_gradient(T):
    """K = all columns: the library's kl_div of the two softmaxes, and its reverse-mode gradient."""
    rng, H, Wb, Wh, C, ids, t = _inputs(1, K=14)
    logits = lambda h, wb, wh: h @ torch.cat([wb, wh[:C]]).T
    h, wb, wh = (torch.tensor(x.astype(np.float64), requires_grad=True) for x in (H, Wb, Wh))
    full = np.zeros((7, 14))
    np.put_along_axis(full, ids.astype(np.int64), t.astype(np.float64), axis=1)
    g = rng.uniform(0.5, 2.0, size=7)
    lp = torch.log_softmax(logits(h, wb, wh) / T, dim=1)
    kl = torch.nn.functional.kl_div(lp, torch.log_softmax(torch.tensor(full) / T, dim=1), log_target=True, reduction="none").sum(dim=1)
    r = oracle.extended_distill(H, Wb, Wh, C, "f32", ids, t, T)
    assert np.allclose(r["kl"], kl.detach().numpy(), atol=1e-12) and (r["kl"] >= 0).all()
    (kl * torch.tensor(g)).sum().backward()
    b = oracle.extended_distill_backward(H, Wb, Wh, C, "f32", ids, t, T, g)
    for got, want in ((b["dH"], h.grad), (b["dW_base"], wb.grad), (b["dW_hyper"], wh.grad)):
        assert np.allclose(got, want.numpy(), atol=1e-12)
    assert np.allclose(b["dZ"].sum(axis=1), 0, atol=1e-14)


def test_gradient_against_differences_with_short_lists_and_special_rows():
    rng, H, Wb, Wh, C, ids, t = _inputs(2)
    ids[0, 3:] = -1
    t[0, 3:] = np.nan                                        # not read
    ids[1] = -1                                              # lists nothing
    ids[2, 1], t[2, 1] = 14, 5.0                             # mass on a column that does not exist
    ids[3, 1], t[3, 1] = 14, -np.inf                         # no mass there
    ids[4, 1] = ids[4, 0]                                    # twice
    T, g = 1.5, rng.uniform(0.5, 2.0, size=7)
    f = lambda h, wb, wh: oracle.extended_distill(h.astype(np.float64).astype(np.float32), wb, wh, C, "f32", ids, t, T)
    r = f(H, Wb, Wh)
    assert r["kl"][1] == 0 and r["kl"][2] == np.inf and np.isfinite(r["kl"][[0, 3, 4, 5, 6]]).all()
    b = oracle.extended_distill_backward(H, Wb, Wh, C, "f32", ids, t, T, g)
    assert (b["dH"][[1, 2]] == 0).all()
    finite = np.isfinite(r["kl"])

    def loss(h, wb, wh):                                     # in float64 throughout
        W = np.concatenate([wb, wh[:C]])
        total = 0.0
        for i in np.nonzero(finite)[0]:
            z = h[i] @ W.T / T
            lp = z - z.max() - np.log(np.exp(z - z.max()).sum())
            use = [(c, x) for c, x in zip(ids[i], t[i]) if c >= 0 and x > -np.inf]
            if use:
                x = np.array([v for _, v in use], dtype=np.float64) / T
                q = np.exp(x - x.max()) / np.exp(x - x.max()).sum()
                total += g[i] * sum(qq * (np.log(qq) - lp[c]) for (c, _), qq in zip(use, q))
        return total

    base = [x.astype(np.float64) for x in (H, Wb, Wh)]
    for which, grad in enumerate((b["dH"], b["dW_base"], b["dW_hyper"])):
        for _ in range(6):
            D, eps = rng.normal(size=grad.shape), 1e-5
            up, down = [x.copy() for x in base], [x.copy() for x in base]
            up[which] += eps * D
            down[which] -= eps * D
            num = (loss(*up) - loss(*down)) / (2 * eps)
            assert abs(num - (grad * D).sum()) < 1e-6 * max(1.0, abs(num))


def test_one_column_at_temperature_one_is_the_negative_log_likelihood():
    _, H, Wb, Wh, C, ids, t = _inputs(3, K=1)
    ids[2, 0], ids[3, 0] = -1, 14
    r = oracle.extended_distill(H, Wb, Wh, C, "f32", ids, t, 1.0)
    n = oracle.extended_nll(H, Wb, Wh, C, "f32", ids[:, 0])
    assert np.allclose(r["kl"], n["nll"], atol=1e-12) and np.allclose(r["lse"], n["lse"], atol=1e-12)


def test_a_student_that_agrees_has_no_loss():
    _, H, Wb, Wh, C, ids, _ = _inputs(4, K=14)
    z = oracle.extended_logits(H, Wb, Wh, C, "f32", return_logits=True)["logits"]
    t = np.take_along_axis(z, ids.astype(np.int64), axis=1)
    for T in (0.5, 1.0, 3.0):
        assert np.abs(oracle.extended_distill(H, Wb, Wh, C, "f32", ids, t, T)["kl"]).max() < 1e-12
