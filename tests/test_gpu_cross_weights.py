"""The weights' precision in attention over states with bf16 outs. Values of both signs
whose sum over the keys is near zero, and weights that are nearly the same, leave outs
so small that rounding them hides nothing: weights in two bf16 parts (up to 128 query
rows of a key head) are off by 2^-18, one part's 2^-9 is far outside the tolerance.

Tolerance: two parts, 2^-18 of a weight, the sums 2^-19, both of max|v|; the logits as in
test_gpu_prompt.py, 2^-19 A, twice; rounding the out to bf16, 2^-8 of it."""
import math

import numpy as np
import pytest

from oracle import prompt as P
from test_gpu_prompt import host, mods, run_cross, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group,T,N", [(1, 1, 40), (4, 4, 33), (1, 17, 40), (1, 128, 65), (2, 64, 200), (4, 5, 1100),
                                       (1, 100, 1500)])
def test_two_parts_up_to_128_rows(group, T, N, D):
    torch, H = mods()
    rng = np.random.default_rng(T)
    S, KV = 3, 2
    heads = KV * group
    q = tensor(rng.normal(size=(S, T, heads, D)) * 0.2, "bf16")
    k = tensor(rng.normal(size=(S, KV, N, D)), "bf16")
    v = rng.uniform(1, 1.5, size=(S, KV, N, D))
    v[:, :, 1::2] = -v[:, :, :N - N % 2:2]
    v[:, :, N - N % 2:] = 0.0
    v = tensor(v[:, :, rng.permutation(N)], "bf16")
    out, _ = run_cross(H, torch, q, k, v)
    q, k, v, out = (host(x) for x in (q, k, v, out))
    one_part = 0.0
    for s in range(S):
        for h in range(heads):
            Q, K, V = q[s, :, h], k[s, h // group], v[s, h // group]
            want, lse = P.cross(Q, K, V)
            A = float((np.abs(Q) @ np.abs(K).T).max()) / math.sqrt(D)
            tol = (2 * 2.0 ** -19 * A + 2.0 ** -19 + 2.0 ** -18) * np.abs(V).max() + np.abs(want) * 2.0 ** -8
            bad = np.abs(out[s, :, h] - want) > tol
            assert not bad.any(), (s, h, np.argwhere(bad)[:3], (np.abs(out[s, :, h] - want) / tol).max())
            # what rounding the weights once would give
            x = Q @ K.T / math.sqrt(D)
            e = np.exp(x - x.max(-1, keepdims=True))
            w = torch.from_numpy(e).bfloat16().double().numpy()
            one_part = max(one_part, float((np.abs(w @ V / e.sum(-1, keepdims=True) - want) / tol).max()))
    assert one_part > 2, one_part
