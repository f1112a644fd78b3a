"""Attention over states whose queries and keys hold infinite elements: a key whose
score is -inf weighs nothing, a query that has no other keys gets zeros and -inf, and
one with a score of +inf or NaN gets numbers that are not finite. The same on every
kernel, whatever the number of query rows. Tolerances as in test_gpu_prompt.py, over
the keys that weigh something."""
import math

import numpy as np
import pytest

from oracle import prompt as P
from test_gpu_prompt import close, host, mods, qkv, run_cross

pytestmark = pytest.mark.gpu

INF = float("inf")


def check(torch, q, k, v, out, lse):
    S, T, heads, D = q.shape
    half = out.dtype != lse.dtype
    parts = 2.0 ** -9 if half else 2.0 ** -24
    q, k, v, out, lse = (host(x) for x in (q, k, v, out, lse))
    seen = set()
    for h in range(heads):
        with np.errstate(invalid="ignore"):
            scores = q[0, :, h] @ k[0, h].T / math.sqrt(D)
        for t in range(T):
            x = scores[t]
            if np.isnan(x).any() or (x == INF).any():
                assert not np.isfinite(out[0, t, h]).any() and not np.isfinite(lse[0, h, t]), (t, h)
                seen.add("not finite")
                continue
            keep = x > -1e30    # (an fp32 score below may be -inf; its weight is zero either way)
            K, V = k[0, h, keep], v[0, h, keep]
            want, wlse = P.cross(q[0, t:t + 1, h], K, V)
            if not keep.any():
                assert (out[0, t, h] == 0).all() and lse[0, h, t] == -INF, (t, h)
                seen.add("nothing")
                continue
            # (infinite elements of a query meet none but keys that weigh nothing or all)
            A = float((np.abs(q[0, t, h]) * np.abs(K)).sum(-1).max()) / math.sqrt(D)
            eps, vmax = 2.0 ** -19 * A, float(np.abs(V).max())
            close(out[0, t, h], want[0], np.full(D, (2 * eps + 2.0 ** -19 + parts) * vmax), "bf16" if half else "fp32")
            assert abs(lse[0, h, t] - wlse[0]) <= eps + 2.0 ** -17
            seen.add("some" if not keep.all() else "all")
    return seen


@pytest.mark.parametrize("T", [1, 2, 16, 17, 100, 200])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "fp32")])
def test_infinite_elements(dtype, out, D, T):
    torch, H = mods()
    heads, N = 4, 150
    q, k, v = qkv(torch, 1, T, heads, heads, N, D, dtype, seed=T)
    q[0, :, :, 3] = q[0, :, :, 3].abs() + 1
    q[0, 1::2, :, 3] *= -1
    # head 0: keys of either infinity, queries of one sign and the other: -inf beside
    # finite scores, or +inf
    k[0, 0, 70, 3] = -INF
    k[0, 0, 149, 3] = -INF
    # head 1: every key, so that half of the queries have none left
    k[0, 1, :, 3] = -INF
    # head 2: an infinite query over keys of both signs, and one over keys of one
    k[0, 2, :, 5] = -k[0, 2, :, 5].abs() - 1
    q[0, 0, 2, 5] = INF
    q[0, T // 2, 2, 7] = -INF
    # head 3: a query element of zero beside an infinite key
    k[0, 3, 11, 9] = INF
    q[0, :, 3, 9] = q[0, :, 3, 9].abs() * -1 - 1
    q[0, T - 1, 3, 9] = 0.0
    o, lse = run_cross(H, torch, q, k, v, out_dtype=torch.float32 if out == "fp32" else None)
    seen = check(torch, q, k, v, o, lse)
    assert {"not finite", "some", "nothing"} <= seen or T == 1


@pytest.mark.parametrize("T", [1, 16, 17, 100, 200])
@pytest.mark.parametrize("D", [64, 128])
def test_products_past_the_largest_number(D, T):
    """fp32 elements whose product overflows: a score of -inf, however it is put
    together from parts."""
    torch, H = mods()
    heads, N = 3, 150
    q, k, v = qkv(torch, 1, T, heads, heads, N, D, "fp32", seed=T)
    rng = np.random.default_rng(D)
    for h, size in enumerate((1e20, 1.7e5, 3e37)):
        q[0, :, h, 3] = torch.from_numpy(rng.uniform(1, 1.1, T) * size).float().cuda()
        k[0, h, :, 3] = 0.0
        k[0, h, 5::7, 3] = -torch.from_numpy(rng.uniform(3.0e38, 3.4e38, len(range(5, N, 7)))).float().cuda()
    o, lse = run_cross(H, torch, q, k, v)
    assert check(torch, q, k, v, o, lse) == {"some"}


@pytest.mark.parametrize("T", [16, 17, 200])
def test_infinite_elements_of_ranges_and_padded_rows(T):
    """In ranges of keys, grouped heads, queries and states of unequal length whose rest
    is infinite or NaN: the same rows as without the keys of -inf."""
    torch, H = mods()
    S, heads, KV, D, N = 2, 4, 2, 64, 3000
    q, k, v = qkv(torch, S, T, heads, KV, N, D, "fp32", seed=3)
    q[..., 3] = q[..., 3].abs() + 1
    ql, kl = [T, T // 2], [N - 700, N]
    drop = torch.arange(4, N, 9, device="cuda")
    k[:, :, drop, 3] = -INF
    # the same scores with a large finite number in the infinity's place
    plain = k.clone()
    plain[:, :, drop, 3] = -1e30
    for s in range(S):
        q[s, ql[s]:], k[s, :, kl[s]:], v[s, :, kl[s]:] = float("nan"), INF, float("nan")
    got = run_cross(H, torch, q, k, v, qlens=ql, klens=kl)
    want = run_cross(H, torch, q, plain, v, qlens=ql, klens=kl)
    assert torch.isfinite(got[0]).all()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
