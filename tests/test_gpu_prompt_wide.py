"""Rows far apart: every axis of every operand with its last row 2^31 elements behind
its first, on every kernel of include/hkv_prompt.h. The same bits as from rows side by
side, which are compared with the oracle."""
import numpy as np
import pytest

from test_gpu_prompt import cfg_of, check_cross, ints, mods, qkv, run_cross, tensor

pytestmark = pytest.mark.gpu

FAR = 1 << 31   # elements


def spread(torch, x, axis, buffer, shift=0):
    """A copy of x [4 axes, the last of neighbours] in `buffer`, its axis' rows FAR apart
    altogether; shift: places of the same kind behind."""
    n = x.shape[axis]
    step = -(-FAR // (n - 1) // 64) * 64
    rest = [i for i in range(3) if i != axis]
    inner = x.shape[rest[1]] * x.shape[3]
    block = x.shape[rest[0]] * inner
    assert n > 1 and (shift + 1) * block <= step
    strides = [0, 0, 0, 1]
    strides[axis], strides[rest[0]], strides[rest[1]] = step, inner, x.shape[3]
    y = buffer.as_strided(x.shape, strides, storage_offset=shift * block)
    y.copy_(x)
    return y


@pytest.fixture(scope="module")
def buffers():
    import torch
    made = {}

    def get(dtype):
        if dtype not in made:
            made[dtype] = torch.empty(FAR + (1 << 24), dtype=dtype, device="cuda")
        return made[dtype]
    yield get
    made.clear()
    torch.cuda.empty_cache()


@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("operand", ["q", "out", "states"])
@pytest.mark.parametrize("dtype,out,D,T,N", [
    ("bf16", "bf16", 64, 2, 9), ("bf16", "fp32", 128, 3, 700),                  # few rows, in ranges
    ("bf16", "bf16", 128, 100, 70), ("bf16", "bf16", 64, 90, 1100),             # one query tile a CTA
    ("bf16", "bf16", 128, 300, 90), ("bf16", "bf16", 64, 300, 90),              # two
    ("fp32", "fp32", 64, 2, 9), ("fp32", "fp32", 128, 4, 1100),
    ("fp32", "fp32", 64, 40, 90), ("fp32", "fp32", 128, 200, 700), ("bf16", "fp32", 128, 40, 90)])
def test_attention_of_rows_far_apart(buffers, dtype, out, D, T, N, operand, axis):
    torch, H = mods()
    S, heads, KV = 2, 4, 2
    odt = torch.float32 if out == "fp32" else torch.bfloat16
    q, k, v = qkv(torch, S, T, heads, KV, N, D, dtype)
    want, wlse = run_cross(H, torch, q, k, v, out_dtype=odt)
    check_cross(q, k, v, want, wlse)
    got = torch.full_like(want, 3.0)
    if operand == "q":
        q = spread(torch, q, axis, buffers(q.dtype))
    elif operand == "out":
        got = spread(torch, got, axis, buffers(odt))
    else:
        k, v = (spread(torch, x.contiguous(), axis, buffers(x.dtype), i) for i, x in enumerate((k, v)))
    cfg = cfg_of(H, S, heads, D, dtype)
    tok, st = H.make_tokens(T), H.make_states(k, v)
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    ws, lse = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty_like(wlse)
    H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(got), lse, ws, n)
    assert torch.equal(got, want) and torch.equal(lse, wlse)


@pytest.mark.parametrize("axis", [0, 1, 2])
@pytest.mark.parametrize("far", ["in", "out"])
@pytest.mark.parametrize("kind", [None, "rms", "layer"])
@pytest.mark.parametrize("dtype,D,rot,layout", [("bf16", 128, 128, 0), ("fp32", 64, 64, 1), ("bf16", 64, 24, 0),
                                                ("fp32", 128, 10, 0)])
def test_rotation_and_norms_of_rows_far_apart(buffers, dtype, D, rot, layout, kind, far, axis):
    torch, H = mods()
    S, T, heads = 3, 37, 6
    rng = np.random.default_rng(rot)
    x = tensor(rng.normal(size=(S, T, heads, D)), dtype)
    w = tensor(1 + 0.2 * rng.normal(size=(heads, D)), dtype)
    cfg = cfg_of(H, S, heads, D, dtype)
    rope = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=layout)
    norm = kind and H.make_norm(H.HKV_NORM_RMS if kind == "rms" else H.HKV_NORM_LAYER, 1e-5, None, w)
    tok = H.make_tokens(T, ints([T, 5, T - 1]), ints(np.arange(T)[None]))

    def run(src, to):
        # as keys, so that their weights of each head are used
        H.hkv_qk_norm_rope(cfg, norm, rope, tok, None, H.make_rows(src), None, None, H.make_rows(to), None)
        return to
    want = run(x, torch.full_like(x, 3.0))
    if far == "in":
        got = run(spread(torch, x, axis, buffers(x.dtype)), torch.full_like(x, 3.0))
    else:
        got = run(x, spread(torch, torch.full_like(x, 3.0), axis, buffers(x.dtype)))
    assert torch.equal(got, want)
