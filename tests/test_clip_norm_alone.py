"""Gradients that count for the common norm alone: nothing is launched for them behind the norm, and their values stay."""
import pytest

from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_launches(without_a_device):
    without_a_device("""
h = context(B=1, V=8, M=2, cap=0, d=8)
N, A, O = P + (1 << 50), P + (1 << 32), P + (3 << 40)
def clip(*tensors):
    arr = (api.GradientDesc * len(tensors))()
    for a, t in zip(arr, tensors):
        a.data, a.out, a.n, a.dtype = t
    assert lib.z2z_clip_gradients(h, arr, len(tensors), 1.0, N, None) == 0
    return [g for n, g in launches() if "clip_scale" in n]
alone = [(A + (i << 20), None, 1 << 16, api.BF16) for i in range(400)]
assert clip(*alone[:1]) == [1] and clip(*alone[:96]) == [1]
assert clip(*alone) == [1]                                    # (one launch writes the norm, whatever the number of lists)
# chunks of 32 KiB of what is written, and of nothing else
some = [(d, O + (i << 20) if i % 100 == 5 else None, n, t) for i, (d, _, n, t) in enumerate(alone)]
assert clip(*some[:96]) == [4] and clip(*some) == [4, 4, 4, 4]
assert clip(*some[:100], *alone[100:]) == [4]
assert clip(*alone[:96], *some[96:192]) == [1, 4]
clean()
""")


@pytest.mark.gpu
def test_the_norm_alone_costs_less_than_clipping():
    torch = pytest.importorskip("torch")
    from paper_2506_01084_amd import api

    ctx = api.Context(B=1, V=8, M=2, cap=0, d=64)
    whole = torch.randn(1 << 29, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    tensors, out, norm = list(whole.split(1 << 26)), torch.empty_like(whole), torch.empty(2, device="cuda")
    lists = [api.Gradients(tensors, [None] * len(tensors)), api.Gradients(tensors, list(out.split(1 << 26)))]

    def took(g):
        ctx.clip_gradients(g, 1.0, norm)
        start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(3):
            ctx.clip_gradients(g, 1.0, norm)
        end.record()
        torch.cuda.synchronize()
        return start.elapsed_time(end)

    before = whole.clone()
    times = [took(g) for g in lists]
    # (reads 1 GiB; the other reads it twice and writes it)
    assert times[0] < times[1], times
    assert torch.equal(before, whole)


@pytest.mark.gpu
def test_some_of_many_are_written():
    torch = pytest.importorskip("torch")
    from paper_2506_01084_amd import api

    ctx = api.Context(B=1, V=8, M=2, cap=0, d=64)
    gen = torch.Generator().manual_seed(4)
    tensors = [torch.randn(1 + (7919 * i) % 40000, generator=gen).to(torch.bfloat16 if i % 2 else torch.float32).cuda() for i in range(250)]
    for which in (lambda i: False, lambda i: i in (3, 249), lambda i: 96 <= i < 192, lambda i: i % 3 == 0):
        host = [t.double() for t in tensors]
        kept = [t.clone() for t in tensors]
        out = [t if which(i) and i % 4 else torch.full_like(t, 7.0) if which(i) else None for i, t in enumerate(tensors)]
        norm = torch.empty(2, device="cuda")
        ctx.clip_gradients(api.Gradients(tensors, out), 2.0, norm)
        want = float(torch.sqrt(sum((h * h).sum() for h in host)))
        # (a square and at most 64 of them added up in 32 bits, halved by the root; one rounding of the norm, one of the coefficient)
        assert abs(float(norm[0]) - want) <= want * 35 * 2.0 ** -24 and abs(float(norm[1]) - 2.0 / want) <= 2.0 / want * 36 * 2.0 ** -24
        for t, h, k, o in zip(tensors, host, kept, out):
            if o is not t:
                assert torch.equal(t, k)
            if o is not None:
                step = 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24
                assert torch.all((o.double() - h * (2.0 / want)).abs() <= h.abs() * (2.0 / want) * (step + 40 * 2.0 ** -24) + 2.0 ** -133)
        for t, k in zip(tensors, kept):
            t.copy_(k)
