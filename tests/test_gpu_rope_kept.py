"""Channels behind a rotation's part of the head: without a norm they are the
input's bits, whatever those say, in both layouts; with one they are the norm's
result, untouched by the rotation. The channels that turn are as they were."""
import numpy as np
import pytest

from oracle import prompt as P
from test_gpu_prompt import U, cfg_of, close, host, ints, mods, norm_error, tensor

pytestmark = pytest.mark.gpu

ODD = [float("nan"), float("inf"), -float("inf"), -0.0, 0.0, 1e-40]   # 1e-40: below the normal numbers


def bits(torch, x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def odd_rows(torch, shape, rot, dtype):
    """Normal numbers where channels turn; behind them one value or another of ODD, and
    NaN of other bits."""
    x = torch.randn(*shape, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    n = shape[-1] - rot
    pick = torch.randint(0, len(ODD) + 2, shape[:-1] + (n,), device="cuda")
    for i, value in enumerate(ODD):
        x[..., rot:][pick == i] = value
    raw = bits(torch, x)
    raw[..., rot:][pick == len(ODD)] = 0x7F81 if dtype == "bf16" else 0x7F800001
    return raw.view(x.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("D,rot", [(64, 2), (64, 10), (64, 24), (64, 32), (128, 2), (128, 24), (128, 42),
                                   (128, 64), (128, 126), (64, 64)])
def test_rotation_keeps_the_bits_behind_it(D, rot, layout, dtype):
    torch, H = mods()
    torch.manual_seed(rot)
    # (several heads a thread, and rows that a thread has at a time)
    for S, T, heads in ((2, 7, 3), (1, 700, 40)):
        x = odd_rows(torch, (S, T, heads, D), rot, dtype)
        cfg = cfg_of(H, S, heads, D, dtype)
        pos = ints(np.arange(T)[None] * 3 + 1)
        rope = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=["half", "pairs"].index(layout), amplitude=1.5)
        tok = H.make_tokens(T, None, pos)
        fine = x.clone()
        fine[..., rot:] = 1.0
        want, out = torch.empty_like(x), torch.empty_like(x)
        H.hkv_rope_rotate(cfg, rope, tok, H.make_rows(fine), H.make_rows(want))
        H.hkv_rope_rotate(cfg, rope, tok, H.make_rows(x), H.make_rows(out))
        assert torch.equal(bits(torch, out[..., rot:]), bits(torch, x[..., rot:]))
        assert torch.equal(bits(torch, out[..., :rot]), bits(torch, want[..., :rot]))
        # as a set of a prepared projection without a norm, in place
        mine = x.clone()
        rows = H.make_rows(mine)
        H.hkv_qk_norm_rope(cfg, None, rope, tok, rows, None, None, rows, None, None)
        assert torch.equal(bits(torch, mine), bits(torch, out))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("D,rot", [(64, 10), (64, 24), (128, 42), (128, 64)])
def test_normed_channels_behind_the_rotation(D, rot, kind, dtype):
    """The interleaved layout: a weight that is infinite, or -0, behind the rotation
    makes its own channel infinite, or -0, and no neighbour NaN."""
    torch, H = mods()
    S, T, heads = 2, 9, 5
    rng = np.random.default_rng(rot)
    x = tensor(rng.normal(size=(S, T, heads, D)), dtype)
    w = 1 + 0.3 * rng.normal(size=D)
    w = tensor(w, dtype)
    w[rot + 1::4] = float("inf")
    w[rot + 2::4] = 0.0
    cfg = cfg_of(H, S, heads, D, dtype)
    norm = H.make_norm(H.HKV_NORM_RMS if kind == "rms" else H.HKV_NORM_LAYER, 1e-5, w)
    rope = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=H.HKV_ROPE_PAIRS)
    out = torch.empty_like(x)
    H.hkv_qk_norm_rope(cfg, norm, rope, H.make_tokens(T, None, ints(np.arange(T)[None])), H.make_rows(x), None, None,
                       H.make_rows(out), None, None)
    eps = float(np.float32(1e-5))
    plain = P.norm(host(x), kind, eps, None)[..., rot:]
    got, weight = host(out)[..., rot:], host(w)[rot:]
    open_, zero = np.isinf(weight), weight == 0
    assert np.array_equal(np.isinf(got), np.broadcast_to(open_, got.shape)) and not np.isnan(got).any()
    assert np.array_equal(np.sign(got[..., open_]), np.sign(plain[..., open_]))
    # (a zero has the sign of what it was multiplied with)
    assert (got[..., zero] == 0).all() and np.array_equal(np.signbit(got[..., zero]), np.signbit(plain[..., zero]))
    rest = ~open_ & ~zero
    tol = norm_error(host(x), kind, eps, None)[..., rot:][..., rest] * np.abs(weight[rest])
    want = plain[..., rest] * weight[rest]
    close(got[..., rest], want, tol + 2 * U * np.abs(want), dtype)
