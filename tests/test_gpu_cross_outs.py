"""Outs of attention over states that go out by bulk copies (heads of 128, two query
tiles a CTA), where a CTA takes over the work of others: a warp stages the rows of
one piece of work while copies of the piece before may still read its place. Pieces
with rows alternate here with query tiles, and warps of a tile, that have none (an
odd number of tiles, a partial last one) and with sequences without states, whose
rows are ready at once. The same sequence alone is no more work than the device
holds, so that nothing is taken over: every bit must be the same, each time."""
import pytest

from test_gpu_prompt import cfg_of, check_cross, ints, mods, qkv, run_cross

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("S,T,heads,KV,N", [
    (16, 300, 32, 32, 64),      # three tiles of a head
    (8, 4160, 32, 32, 120),     # 33, the last one of 64 tokens
    (40, 100, 24, 8, 64),       # three heads a group, a tile each
    (16, 257, 32, 32, 64),      # a last tile of one token
    (24, 130, 32, 32, 120),     # two tiles, the second of two tokens
])
def test_rows_stay_while_work_without_rows_follows(S, T, heads, KV, N, ragged):
    torch, H = mods()
    D = 128
    q, k, v = qkv(torch, S, T, heads, KV, N, D, "bf16")
    klens = [N - (i * N) // (2 * S) for i in range(S)] if ragged else None
    if ragged:
        klens[1::3] = [0] * len(klens[1::3])
    want = torch.empty_like(q)
    wlse = torch.empty(S, heads, T, device="cuda")
    for s in range(S):
        o, lse = run_cross(H, torch, q[s:s + 1], k[s:s + 1], v[s:s + 1], klens=klens and klens[s:s + 1])
        want[s], wlse[s] = o[0], lse[0]
    check_cross(q[:1], k[:1], v[:1], want[:1], wlse[:1], klens=klens and klens[:1], heads=[0, heads - 1])
    cfg = cfg_of(H, S, heads, D, "bf16")
    tok, st = H.make_tokens(T), H.make_states(k, v, None if klens is None else ints(klens))
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty_like(wlse)
    rows, outs = H.make_rows(q), H.make_rows(out)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    bits = want.view(torch.int16)
    for _ in range(300):
        out.fill_(3.0)
        H.hkv_cross_attention(cfg, st, tok, rows, outs, lse, ws, n)
        wrong += (out.view(torch.int16) != bits).sum()
    assert int(wrong) == 0 and torch.equal(lse, wlse)
