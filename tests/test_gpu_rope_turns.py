"""A rotation whose frequencies the caller fills in: a ramp over the pairs' numbers, and a
factor for each pair."""
import math

import numpy as np
import pytest

from oracle import prompt as P
from test_gpu_prompt import U, cfg_of, close, host, ints, mods, rotation_error, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("kind", ["ramp", "factors"])
def test_frequencies_of_the_caller(kind, layout):
    torch, H = mods()
    S, T, heads, D = 2, 50, 5, 64
    rng = np.random.default_rng(4)
    f = P.frequencies(D, (D // 2,))
    if kind == "ramp":
        g = np.clip((np.arange(D // 2) - 5) / 14, 0, 1)
        f = f * (1 - g) + f / 8 * g
    else:
        f = f / rng.uniform(1, 30, D // 2)
    rope = H.hkv_make_rope(head_dim=D, layout=["half", "pairs"].index(layout))
    for i in range(D // 2):
        rope.turns[i] = int(f[i] / (2 * math.pi) * 2.0 ** 64)
    pos = rng.integers(0, 100000, size=(1, S, T))
    x = tensor(rng.normal(size=(S, T, heads, D)), "fp32")
    out = torch.empty_like(x)
    H.hkv_rope_rotate(cfg_of(H, S, heads, D, "fp32"), rope, H.make_tokens(T, None, ints(pos)), H.make_rows(x),
                      H.make_rows(out))
    a = np.broadcast_to(P.angles_of(pos, f, (D // 2,))[:, :, None], (S, T, heads, D // 2))
    want = P.rotate(host(x), a, layout)
    close(host(out), want, rotation_error(host(x), a, layout, 1.0) + 2 * U * np.abs(want), "fp32")
