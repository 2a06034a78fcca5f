"""GPU: the lookup of more positions, and the move of more entries, than one launch has threads for (2^26 waves of 64)."""
import pytest

pytestmark = pytest.mark.gpu


def test_a_lookup_of_more_than_2_to_the_26_positions():
    import torch
    from paper_2506_01084_amd import api

    N, V, d = (1 << 26) + 1001, 1000, 8
    print(f"[case] lookup of {N} positions", flush=True)
    ctx = api.Context(B=1, V=V, M=2, cap=0, d=d, dtype="bf16")
    E = (torch.arange(V * d, device="cuda").reshape(V, d) % 251).bfloat16()
    W = torch.empty((1, 0, d), dtype=torch.bfloat16, device="cuda")
    codes = (torch.arange(N, device="cuda", dtype=torch.int32) % V)[None].contiguous()
    codes[0, -5] = V
    X = torch.full((1, N, d), 7.0, dtype=torch.bfloat16, device="cuda")
    st = torch.full((1,), -7, dtype=torch.int32, device="cuda")
    ctx.embed_codes(codes, None, E, W, X, st, scale=2.0)
    torch.cuda.synchronize()
    assert st.item() == 2
    want = E * 2
    for i0 in range(0, N, 1 << 24):
        c = codes[0, i0:i0 + (1 << 24)].long()
        same = torch.where((c < V)[:, None], want[c.clamp(max=V - 1)], torch.zeros(1, dtype=torch.bfloat16, device="cuda")) == X[0, i0:i0 + (1 << 24)]
        assert same.all(), i0
    ctx.close()


def test_a_move_of_more_than_2_to_the_26_entries():
    import torch
    from paper_2506_01084_amd import api

    B, cap, V, d = 2064, 65535, 1000, 8
    print(f"[case] move of {B // 2} x {cap} entries", flush=True)
    ctx = api.Context(B=B, V=V, M=2, cap=cap, d=d, dtype="bf16")
    n = 5
    phrases = torch.zeros((B, n, 2), dtype=torch.int32, device="cuda")
    phrases[:, :, 0] = torch.arange(B, device="cuda", dtype=torch.int32)[:, None] % V
    phrases[:, :, 1] = torch.arange(n, device="cuda", dtype=torch.int32)
    counts = 2 + torch.arange(B, device="cuda", dtype=torch.int32) % 4
    added, st = torch.empty_like(counts), torch.empty_like(counts)
    ctx.codebook_prefill(phrases, torch.full((B, n), 2, dtype=torch.int32, device="cuda"), counts, added, st, api.RESET)
    assert torch.equal(added, counts)
    entries, lens, size = ctx.codebook()
    source = torch.tensor([1, 1], dtype=torch.int32, device="cuda").repeat(B // 2)
    ctx.codebook_reorder(2, source)
    torch.cuda.synchronize()
    want = torch.arange(1, B, 2, device="cuda").repeat_interleave(2)
    assert torch.equal(size, counts[want])
    at = torch.arange(n, device="cuda")[None] < counts[want][:, None]
    assert torch.equal(lens[:, :n], at.int() * 2) and torch.equal(torch.where(at[:, :, None], entries[:, :n], 0), torch.where(at[:, :, None], phrases[want], 0))
    # the tables have moved, too: a phrase that beam 0 had not known is found in them
    codes = torch.empty((B, 2), dtype=torch.int32, device="cuda")
    n_codes = torch.empty(B, dtype=torch.int32, device="cuda")
    tokens = torch.stack([want.int() % V, torch.zeros_like(want).int()], dim=1).contiguous()
    ctx.lzw_encode(tokens, None, codes, n_codes, st, api.APPEND)
    torch.cuda.synchronize()
    assert (n_codes == 1).all() and (codes[:, 0] == V).all()
    ctx.close()
