"""Rotary positions, norms of queries and keys, and attention over other states
on the GPU, each against the fp64 oracle (oracle/prompt.py).

Tolerances, u = 2^-24 (half a step of fp32).
Rotation of (x, y), amplitude A: the angle's fraction of a turn is cut at 2^-32
turns (2^-29 rad) and rounded to fp32 (pi u), sincospi is off by 2 ulp, the
amplitude, its product, the two products and their sum round once each: 10 u A
(|x| + |y|) covers it (3.2 + 4 + 2.x u). The oracle's own angle, a product in
fp64, and the table's frequency are off by 2^-52 of the angle each.
Norms: sums of D numbers in chains of at most 16 and 4 shuffles, 20 u of the
numbers' mean magnitude; a root and a quotient, 3 u; the products and the bias,
3 u: 30 u of |weight| (|x - mean| + mean |x|) / sigma and 2 u of the result.
Attention: a logit x = sum q_i k_i / sqrt(D) is off by at most 2^-19 A with A =
sum |q_i k_i| / sqrt(D), as chained sums in the tensor core truncate. Weights
off by eps each move an output by at most 2 eps max|v|, the sums over the keys
add 2^-19 max|v|, and weights in two bf16 parts (2^-18) or one (2^-9) as much
of max|v|.
Rounding to bf16 is off by at most 2^-8 of the value.
"""
import math

import numpy as np
import pytest

from oracle import prompt as P

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def cfg_of(H, seqs, heads, D, dtype, **kw):
    base = dict(n_layers=1, n_seqs=seqs, n_heads=heads, head_dim=D, dtype=dtype, n_cond=0, n_image=1,
                row_len=1, recent_w=1, local_w=1, period=1, group_at=1, global_budget=1)
    base.update(kw)
    return H.make_config(**base)


def mods():
    import torch
    from paper_2605_20600_gb300 import hkv as H
    return torch, H


def tensor(x, dtype):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32))
    return (t.bfloat16() if dtype == "bf16" else t).cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def ints(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rotation_error(x, angles, layout, amp):
    """|x| + |y| of every rotated channel's pair, times 10 u, and the oracle's angle."""
    n = angles.shape[-1]
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    e = np.zeros(x.shape)
    both = np.abs(x[..., a]) + np.abs(x[..., b])
    e[..., a] = e[..., b] = abs(amp) * both * (10 * U + np.abs(angles) * 2.0 ** -51)
    return e


def close(got, want, tol, dtype):
    if dtype == "bf16":
        tol = tol + np.abs(want) * 2.0 ** -8 + tol * 2.0 ** -8
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - want)[bad][:4], np.broadcast_to(tol, bad.shape)[bad][:4])


ROTATIONS = [
    # dtype, D, rot, layout, sections, joint, scaling, seqs, tokens, heads, start
    ("bf16", 128, 128, "half", None, False, "plain", 1, 1, 8, 0),
    ("fp32", 64, 64, "half", None, False, "plain", 1, 1, 8, 77),
    ("bf16", 64, 64, "pairs", (16, 16), False, "plain", 3, 37, 20, 0),
    ("fp32", 128, 32, "half", None, False, "parts", 2, 65, 11, 900000),
    ("bf16", 128, 48, "half", None, False, "base", 2, 9, 3, 5000),
    ("bf16", 64, 24, "half", None, False, "linear", 2, 9, 3, 5000),      # pieces of 8 do not fall together
    ("fp32", 64, 6, "half", (1, 2), False, "plain", 2, 5, 3, 40),
    ("fp32", 128, 10, "pairs", None, False, "plain", 2, 5, 3, 40),
    ("bf16", 128, 128, "half", (16, 24, 24), True, "plain", 4, 33, 7, 3),
    ("bf16", 128, 2, "pairs", None, False, "plain", 1, 300, 1, 2 ** 31 - 301),
    ("fp32", 128, 2, "half", None, False, "plain", 1, 3, 130, -5),
    ("bf16", 128, 128, "half", None, False, "plain", 2, 700, 40, 1000),   # several heads a thread
    ("bf16", 64, 64, "half", None, False, "plain", 1, 2, 600, 1000),      # more heads than a block's slots
]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("case", ROTATIONS, ids=lambda c: "-".join(str(x) for x in c))
def test_rotation(case, back):
    dtype, D, rot, layout, sections, joint, scaling, S, T, heads, start = case
    torch, H = mods()
    rng = np.random.default_rng(1)
    kw = {} if scaling == "plain" else dict(factor=8.0)
    if scaling == "parts":
        kw.update(original=4096.0, low=1.0, high=32.0)
    amp = 1.0 if scaling == "plain" else 1.2
    rope = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=["half", "pairs"].index(layout), sections=sections,
                           joint=joint, scaling=["plain", "linear", "base", "parts"].index(scaling),
                           amplitude=amp, **kw)
    sec = sections or (rot // 2,)
    freq = P.frequencies(rot, sec, joint=joint, scaling=scaling, **kw)
    pos = start + rng.permuted(np.tile(np.arange(T), (len(sec), S, 1)), axis=2)
    lens = np.array([T - (i * T) // S for i in range(S)])
    if S > 2:
        lens[1] = 0
    x = tensor(rng.normal(size=(S, T, heads, D)), dtype)
    want = P.rotate(host(x), P.angles_of(pos, freq, sec)[:, :, None] * (-1 if back else 1), layout, float(np.float32(amp)))
    tol = rotation_error(host(x), np.broadcast_to(P.angles_of(pos, freq, sec)[:, :, None], (S, T, heads, rot // 2)),
                         layout, amp) + 2 * U * np.abs(want)
    live = np.arange(T)[None] < lens[:, None]
    cfg = cfg_of(H, S, heads, D, dtype)
    tok = H.make_tokens(T, ints(lens), ints(pos))
    flags = H.HKV_ROPE_BACK if back else 0
    # into rows by heads, past the last token left alone
    out = torch.full((S, heads, T + 1, D), 7.0, dtype=x.dtype, device="cuda")
    H.hkv_rope_rotate(cfg, rope, tok, H.make_rows(x), H.make_rows(out[:, :, :T].transpose(1, 2)), flags)
    got = host(out[:, :, :T].transpose(1, 2))
    close(got[live], want[live], tol[live], dtype)
    assert (got[~live] == 7.0).all() and (host(out[:, :, T]) == 7.0).all()
    # channels that do not turn are the input's bits
    assert np.array_equal(got[live][..., rot:], host(x)[live][..., rot:])
    # a slice of a fused projection, in place: the same bits
    fused = torch.randn(S, T, heads + 3, D, device="cuda").to(x.dtype)
    fused[:, :, 2:2 + heads] = x
    rest = fused.clone()
    mine = fused[:, :, 2:2 + heads]
    H.hkv_rope_rotate(cfg, rope, tok, H.make_rows(mine), H.make_rows(mine), flags)
    assert np.array_equal(host(mine)[live], got[live]) and np.array_equal(host(mine)[~live], host(x)[~live])
    assert torch.equal(fused[:, :, :2], rest[:, :, :2]) and torch.equal(fused[:, :, 2 + heads:], rest[:, :, 2 + heads:])


def test_rotation_back_is_the_gradient_and_the_way_back():
    """A rotation's gradient against differences, and forth and back."""
    torch, H = mods()
    rng = np.random.default_rng(3)
    S, T, heads, D, rot = 2, 5, 3, 64, 48
    rope = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=1, amplitude=1.5)
    cfg = cfg_of(H, S, heads, D, "fp32")
    tok = H.make_tokens(T, None, ints(rng.integers(0, 3000, size=(1, S, T))))

    def f(x, flags=0, rope=rope):
        out = torch.empty_like(x)
        H.hkv_rope_rotate(cfg, rope, tok, H.make_rows(x), H.make_rows(out), flags)
        return out
    x, g, d = (tensor(rng.normal(size=(S, T, heads, D)), "fp32") for _ in range(3))
    grad = f(g, H.HKV_ROPE_BACK)
    # linear: g . (f(x + d) - f(x)) = grad . d up to rounding of the sums' parts
    left = float((host(g) * (host(f(x + d)) - host(f(x)))).sum())
    right = float((host(grad) * host(d)).sum())
    size = float((np.abs(host(g)) * (np.abs(host(x)) + np.abs(host(d)))).sum())
    assert abs(left - right) <= 64 * U * size
    plain = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=1)
    there = f(f(x, 0, plain), H.HKV_ROPE_BACK, plain)
    close(host(there), host(x), 44 * U * np.abs(host(x)).max() * np.ones(x.shape), "fp32")


NORMS = [
    # dtype, D, kind, weights per head, seqs, tokens, q heads, kv heads, rope
    ("bf16", 128, "layer", True, 8, 1, 32, 32, "half"),
    ("bf16", 128, "rms", False, 3, 70, 14, 2, "half"),
    ("fp32", 64, "layer", False, 3, 33, 6, 3, "pairs"),
    ("fp32", 128, "rms", True, 2, 5, 7, 1, None),
    ("bf16", 64, "rms", None, 2, 41, 5, 5, "part"),
    ("bf16", 64, "layer", True, 2, 9, 3, 3, "apart"),      # a warp per row
    ("fp32", 64, "rms", False, 1, 1, 1, 1, "apart"),
    ("bf16", 128, None, None, 2, 130, 9, 9, "half"),
]


def norm_error(x, kind, eps, w):
    mean = x.mean(-1, keepdims=True) if kind == "layer" else 0.0
    sigma = np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    e = 30 * U * (np.abs(x - mean) + (np.abs(x).mean(-1, keepdims=True) if kind == "layer" else 0.0)) / sigma
    return e * (1.0 if w is None else np.abs(w))


@pytest.mark.parametrize("case", NORMS, ids=lambda c: "-".join(str(x) for x in c))
def test_norms_with_the_rotation(case):
    dtype, D, kind, per_head, S, T, HQ, KV, rope_kind = case
    torch, H = mods()
    rng = np.random.default_rng(5)
    rope, rot, layout = None, 0, "half"
    if rope_kind:
        rot = {"half": D, "pairs": D, "part": D // 2, "apart": 24 if dtype == "bf16" else 20}[rope_kind]
        rot = 10 if rope_kind == "apart" and dtype == "fp32" else rot
        layout = "pairs" if rope_kind == "pairs" else "half"
        rope = H.hkv_make_rope(head_dim=D, rot_dim=rot, layout=["half", "pairs"].index(layout))
    freq = P.frequencies(rot, (rot // 2,)) if rope else None
    pos = rng.integers(0, 5000, size=(1, S, T))
    lens = np.array([T] + [max(0, T - 3 * (i + 1)) for i in range(S - 1)])
    x = tensor(rng.normal(size=(S, T, HQ + 2 * KV, D)) * 2 + 0.5, dtype)
    shape = {None: None, False: (D,), True: "heads"}[per_head]

    def weights(n):
        return None if shape is None else tensor(1 + 0.3 * rng.normal(size=(n, D) if shape == "heads" else (D,)), dtype)
    qw, kw = weights(HQ), weights(KV)
    qb, kb = (weights(HQ), weights(KV)) if kind == "layer" else (None, None)
    norm = None if kind is None else H.make_norm(H.HKV_NORM_RMS if kind == "rms" else H.HKV_NORM_LAYER, 1e-5, qw, kw, qb, kb)
    cfg = cfg_of(H, S, HQ, D, dtype)
    tok = H.make_tokens(T, ints(lens), ints(pos) if rope else None)
    parts = (x[:, :, :HQ], x[:, :, HQ:HQ + KV], x[:, :, HQ + KV:])
    outs = [torch.full((S, T, HQ, D), 7.0, dtype=x.dtype, device="cuda"),
            torch.full((S, KV, T, D), 7.0, dtype=x.dtype, device="cuda"),
            torch.full((S, KV, T, D), 7.0, dtype=x.dtype, device="cuda")]
    views = [outs[0], outs[1].transpose(1, 2), outs[2].transpose(1, 2)]
    H.hkv_qk_norm_rope(cfg, norm, rope, tok, *(H.make_rows(p) for p in parts), *(H.make_rows(v) for v in views))
    live = np.arange(T)[None] < lens[:, None]
    for got, xin, w, b in zip(views[:2], parts[:2], (qw, kw), (qb, kb)):
        xin = host(xin)
        w64, b64 = (None if y is None else host(y) for y in (w, b))
        want, tol = xin, np.zeros(xin.shape)
        eps = float(np.float32(1e-5))
        if kind:
            want = P.norm(xin, kind, eps, w64, b64)
            tol = norm_error(xin, kind, eps, w64) + 2 * U * np.abs(want)
        if rope:
            a = np.broadcast_to(P.angles_of(pos, freq, (rot // 2,))[:, :, None], want.shape[:3] + (rot // 2,))
            # the input's error is turned with it: at most the sum of the pair's
            turned = rotation_error(want, a, layout, 1.0)
            both = rotation_error(tol, np.zeros(a.shape), layout, 1.0) / (10 * U)
            tol = np.where(both > 0, both, tol) + turned
            want = P.rotate(want, a, layout)
        close(host(got)[live], want[live], (tol + 2 * U * np.abs(want))[live], dtype)
    assert np.array_equal(host(views[2])[live], host(parts[2])[live])
    for v in views:
        assert (host(v)[~live] == 7.0).all()
    # each set alone, and in place, gives the same bits
    alone = x.clone()
    ins = (alone[:, :, :HQ], alone[:, :, HQ:HQ + KV])
    for i in range(2):
        rows = [H.make_rows(ins[i]) if j == i else None for j in range(2)]
        H.hkv_qk_norm_rope(cfg, norm, rope, tok, *rows, None, *rows, None)
        assert np.array_equal(host(ins[i])[live], host(views[i])[live])
        assert np.array_equal(host(ins[i])[~live], host(parts[i])[~live])


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("dtype,D,HQ,KV", [("bf16", 64, 40, 8), ("fp32", 128, 24, 24)])
def test_norms_of_long_padded_batches(dtype, D, HQ, KV, kind):
    """Many rows a thread: tokens there are as in a full batch, those behind left alone."""
    torch, H = mods()
    S, T = 5, 900
    cfg = cfg_of(H, S, HQ, D, dtype)
    x = torch.randn(S, T, HQ + 2 * KV, D, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    rope, norm = H.hkv_make_rope(head_dim=D), H.make_norm(H.HKV_NORM_RMS if kind == "rms" else H.HKV_NORM_LAYER, 1e-5)
    pos, parts = ints(np.arange(T)[None]), (x[:, :, :HQ], x[:, :, HQ:HQ + KV], x[:, :, HQ + KV:])
    got = []
    for lens in (None, [T, 0, 1, 450, T - 1]):
        out = torch.full_like(x, 7.0)
        outs = (out[:, :, :HQ], out[:, :, HQ:HQ + KV], out[:, :, HQ + KV:])
        tok = H.make_tokens(T, None if lens is None else ints(lens), pos)
        H.hkv_qk_norm_rope(cfg, norm, rope, tok, *(H.make_rows(p) for p in parts), *(H.make_rows(o) for o in outs))
        got.append(out)
    full, padded = got
    live = torch.arange(T, device="cuda")[None] < ints(lens)[:, None]
    assert torch.equal(padded[live], full[live]) and (padded[~live] == 7.0).all()
    xin = host(x[3, 440:460, :HQ])
    want = P.norm(xin, kind, float(np.float32(1e-5)), None, None)
    tol = norm_error(xin, kind, float(np.float32(1e-5)), None) + 2 * U * np.abs(want)
    freq = P.frequencies(D, (D // 2,))
    a = np.broadcast_to(P.angles_of(np.arange(440, 460)[None, None], freq, (D // 2,))[0][:, None], (20, HQ, D // 2))
    turned = rotation_error(want, a, "half", 1.0)
    tol = rotation_error(tol, np.zeros(a.shape), "half", 1.0) / (10 * U) + turned
    want = P.rotate(want, a, "half")
    close(host(full[3, 440:460, :HQ]), want, tol + 2 * U * np.abs(want), dtype)


def test_rows_of_extremes():
    """Zeros, infinities and NaN stay in their row; eps carries a row of zeros."""
    torch, H = mods()
    S, T, heads, D = 1, 4, 4, 64
    x = torch.randn(S, T, heads, D, device="cuda")
    x[0, 1, 2] = 0.0
    x[0, 2, 0, 5] = float("nan")
    x[0, 3, 3, 9] = float("inf")
    cfg = cfg_of(H, S, heads, D, "fp32")
    rope = H.hkv_make_rope(head_dim=D)
    tok = H.make_tokens(T, None, ints(np.arange(T)[None]))
    out = torch.empty_like(x)
    for kind in (H.HKV_NORM_RMS, H.HKV_NORM_LAYER):
        H.hkv_qk_norm_rope(cfg, H.make_norm(kind, 1e-6), rope, tok, H.make_rows(x), None, None, H.make_rows(out), None, None)
        fine = torch.isfinite(out).all(-1).cpu().numpy()
        want = np.ones((S, T, heads), bool)
        want[0, 2, 0] = want[0, 3, 3] = False
        assert np.array_equal(fine, want)
        assert (out[0, 1, 2] == 0).all() and not torch.isfinite(out[0, 2, 0]).any()


@pytest.mark.parametrize("bad", [-1, 6, 2 ** 31 - 1])
def test_lengths_out_of_range(bad):
    torch, H = mods()
    S, T, heads, D = 3, 5, 2, 64
    cfg = cfg_of(H, S, heads, D, "bf16")
    x = torch.randn(S, T, heads, D, device="cuda").bfloat16()
    for rot in (64, 24):
        err = ints([0])
        out = torch.full_like(x, 3.0)
        tok = H.make_tokens(T, ints([T, bad, T]), ints(np.zeros((1, 1, T))), err)
        H.hkv_rope_rotate(cfg, H.hkv_make_rope(head_dim=D, rot_dim=rot), tok, H.make_rows(x), H.make_rows(out))
        assert int(err) == H.HKV_ERR_BOUNDS
        assert (out[1] == 3.0).all() and torch.equal(out[0], x[0]) and torch.equal(out[2], x[2])


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
@pytest.mark.parametrize("which", ["queries", "states"])
@pytest.mark.parametrize("dtype,out,S,T,N", [("bf16", "bf16", 3, 5, 9), ("bf16", "bf16", 3, 5, 4000),
                                             ("fp32", "fp32", 3, 5, 9), ("bf16", "bf16", 3, 100, 70),
                                             ("bf16", "bf16", 3, 300, 70), ("bf16", "bf16", 3, 300, 3000),
                                             ("bf16", "bf16", 400, 300, 70), ("fp32", "fp32", 3, 100, 70),
                                             ("bf16", "fp32", 3, 100, 2000)])
def test_attention_lengths_out_of_range(dtype, out, S, T, N, which, bad):
    """A bad number of queries leaves the sequence's outputs, one of states gives
    NaN; the error word says so, also where most sequences are empty."""
    torch, H = mods()
    heads, D = 2, 64
    cfg = cfg_of(H, S, heads, D, dtype)
    q, k, v = qkv(torch, S, T, heads, heads, N, D, dtype)
    err = ints([0])
    ql, kl = [T] + [0] * (S - 2) + [max(1, T // 2)], [N] * (S - 1) + [N // 2]
    (ql if which == "queries" else kl)[1] = bad
    if which == "states":
        ql[1] = T
    tok, st = H.make_tokens(T, ints(ql), None, err), H.make_states(k, v, ints(kl), err)
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    o = torch.full(q.shape, 3.0, dtype=torch.float32 if out == "fp32" else torch.bfloat16, device="cuda")
    lse = torch.full((S, heads, T), 3.0, device="cuda")
    H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(o), lse, ws, n)
    assert int(err) == H.HKV_ERR_BOUNDS
    if which == "queries":
        assert (o[1] == 3.0).all() and (lse[1] == 3.0).all()
    else:
        assert torch.isnan(o[1]).all() and torch.isnan(lse[1]).all()
    keep = [0] + list(range(2, min(S, 4))) + ([S - 1] if S > 4 else [])
    ql[1] = kl[1] = 0
    check_cross(q[keep], k[keep], v[keep], o[keep], lse[keep], qlens=[ql[i] for i in keep],
                klens=[kl[i] for i in keep])


# attention over states ------------------------------------------------------
def run_cross(H, torch, q, k, v, *, qlens=None, klens=None, causal=False, out_dtype=None, cfg=None):
    """q [S, T, heads, D], k and v [S, KV, N, D] tensors -> out, lse (3.0 where nothing is written)."""
    S, T, heads, D = q.shape
    dtype = "bf16" if q.dtype == torch.bfloat16 else "fp32"
    cfg = cfg or cfg_of(H, S, heads, D, dtype)
    tok = H.make_tokens(T, None if qlens is None else ints(qlens))
    st = H.make_states(k, v, None if klens is None else ints(klens))
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")   # it may hold anything
    out = torch.full((S, T, heads, D), 3.0, dtype=out_dtype or q.dtype, device="cuda")
    lse = torch.full((S, heads, T), 3.0, device="cuda")
    H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(out), lse, ws, n,
                          H.HKV_ATTN_CAUSAL if causal else 0)
    return out, lse


def check_cross(q, k, v, out, lse, *, qlens=None, klens=None, causal=False, heads=None):
    """Outputs of (some) heads of every sequence against the oracle."""
    S, T, HQ, D = q.shape
    N, group = k.shape[2], HQ // k.shape[1]
    half = out.dtype != lse.dtype
    # weights of bf16 outs enter in two parts, or (batches of many queries) in one
    parts = 2.0 ** -9 if half else 2.0 ** -24
    q, k, v, out, lse = (host(x) for x in (q, k, v, out, lse))
    for s in range(S):
        n, m = (T if qlens is None else qlens[s]), (N if klens is None else klens[s])
        for h in heads or range(HQ):
            K, V = k[s, h // group, :m], v[s, h // group, :m]
            want, wlse = P.cross(q[s, :n, h], K, V, causal)
            A = float((np.abs(q[s, :n, h]) @ np.abs(K).T).max(initial=0.0)) / math.sqrt(D)
            eps, vmax = 2.0 ** -19 * A, float(np.abs(V).max(initial=0.0))
            tol = np.full(want.shape, (2 * eps + 2.0 ** -19 + parts) * vmax)
            close(out[s, :n, h], want, tol, "bf16" if half else "fp32")
            empty = np.isneginf(wlse)
            assert np.array_equal(np.isneginf(lse[s, h, :n]), empty)
            assert (out[s, :n, h][empty] == 0).all()
            assert (np.abs(lse[s, h, :n][~empty] - wlse[~empty]) <= eps + 2.0 ** -20 * 8).all()
            assert (out[s, n:, h] == 3.0).all() and (lse[s, h, n:] == 3.0).all()


def qkv(torch, S, T, heads, KV, N, D, dtype, seed=0, slack=0):
    rng = np.random.default_rng(seed)
    q = tensor(rng.normal(size=(S, T, heads, D)) * 1.5, dtype)
    k = tensor(rng.normal(size=(S, KV, N + slack, D)), dtype)[:, :, :N]
    v = tensor(rng.normal(size=(S, KV, N + slack, D)) + 0.3, dtype)[:, :, :N]
    return q, k, v


CROSS = [
    # dtype, out, D, S, heads, KV, T, N
    ("bf16", "bf16", 64, 1, 1, 1, 1, 1),
    ("bf16", "fp32", 128, 3, 4, 4, 1, 65),
    ("bf16", "fp32", 64, 2, 6, 2, 1, 1000),        # grouped heads side by side, ranges joined
    ("bf16", "bf16", 128, 1, 8, 2, 5, 3001),       # 20 rows of a key head
    ("bf16", "fp32", 128, 2, 2, 1, 40, 129),       # fp32 outs of more rows
    ("fp32", "fp32", 64, 2, 3, 3, 1, 63),
    ("fp32", "fp32", 128, 2, 2, 1, 37, 200),
    ("fp32", "fp32", 64, 1, 8, 4, 130, 777),
    ("fp32", "fp32", 128, 2, 4, 4, 1, 333),        # no tensor core: 1, 4, 16 rows
    ("fp32", "fp32", 64, 2, 6, 2, 1, 2100),
    ("fp32", "fp32", 128, 2, 4, 2, 8, 1500),
    ("fp32", "fp32", 64, 1, 4, 2, 7, 31),
    ("fp32", "fp32", 128, 2, 2, 2, 300, 400),      # three query tiles, several key tiles
    ("bf16", "fp32", 64, 2, 4, 2, 200, 500),
    ("bf16", "fp32", 64, 1, 2, 1, 9, 1300),
    ("fp32", "fp32", 64, 1, 2, 1, 20, 9001),       # many key tiles, several ranges
    ("bf16", "bf16", 64, 2, 16, 2, 17, 300),       # seven heads a query tile, eight a group
    ("bf16", "bf16", 64, 3, 64, 64, 300, 300),     # more work than CTAs at a time
    ("bf16", "bf16", 64, 2, 4, 2, 100, 64),
    ("bf16", "bf16", 128, 2, 3, 3, 257, 300),
    ("bf16", "bf16", 64, 3, 4, 1, 130, 513),
    ("bf16", "bf16", 128, 1, 2, 2, 1000, 1000),
    ("bf16", "bf16", 64, 1, 2, 1, 700, 127),
    ("bf16", "bf16", 128, 2, 1, 1, 300, 5000),     # few CTAs: ranges joined
    ("bf16", "bf16", 64, 1, 1, 1, 2049, 1),
    ("bf16", "bf16", 128, 170, 2, 2, 100, 700),    # one query tile a CTA, many key tiles
    ("bf16", "bf16", 64, 2, 160, 160, 128, 900),
    ("bf16", "bf16", 64, 1, 160, 160, 256, 1500),  # two
]


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("case", CROSS, ids=lambda c: "-".join(str(x) for x in c))
def test_attention_over_states(case, ragged, causal):
    torch, H = mods()
    dtype, out, D, S, heads, KV, T, N = case
    q, k, v = qkv(torch, S, T, heads, KV, N, D, dtype, slack=2)
    lens = {}
    if ragged:
        lens = dict(qlens=[max(0, T - 5 * i) for i in range(S)], klens=[max(0, (N * (i + 1)) // S - i) for i in range(S)])
        if S > 1:
            lens["klens"][0] = 0 if not causal else max(0, lens["qlens"][0] - 2)
            lens["klens"][0] = min(N, lens["klens"][0])
        # rows that do not count hold anything
        for s in range(S):
            q[s, lens["qlens"][s]:] = float("nan")
            k[s, :, lens["klens"][s]:] = float("inf")
            v[s, :, lens["klens"][s]:] = float("nan")
    o, lse = run_cross(H, torch, q, k, v, causal=causal, out_dtype=torch.float32 if out == "fp32" else None, **lens)
    check_cross(q, k, v, o, lse, causal=causal, heads=range(0, heads, max(1, S * heads // 16)), **lens)


@pytest.mark.parametrize("which", ["both", "queries", "states", "bad"])
@pytest.mark.parametrize("dtype,out,D,S,heads,KV,T,N", [
    ("bf16", "bf16", 64, 16, 20, 4, 300, 200), ("bf16", "bf16", 128, 32, 24, 6, 40, 100),
    ("bf16", "bf16", 64, 31, 12, 12, 100, 90), ("bf16", "bf16", 64, 33, 12, 12, 100, 90),
    ("fp32", "fp32", 64, 7, 11, 11, 300, 300), ("fp32", "fp32", 128, 9, 20, 4, 130, 257),
    ("bf16", "fp32", 64, 5, 16, 16, 257, 600),
    # in ranges of keys
    ("bf16", "fp32", 64, 21, 12, 12, 1, 1200), ("bf16", "bf16", 128, 32, 16, 8, 3, 1100),
    ("fp32", "fp32", 128, 20, 24, 12, 3, 1100), ("fp32", "fp32", 64, 7, 22, 11, 18, 1600),
    ("bf16", "bf16", 64, 10, 10, 10, 200, 4000)])
def test_more_work_than_the_device_holds_of_unequal_sequences(dtype, out, D, S, heads, KV, T, N, which):
    """Up to 32 sequences are worked on by length; equal ones, empty ones, lengths that
    are out of range and batches with one kind of lengths only."""
    torch, H = mods()
    q, k, v = qkv(torch, S, T, heads, KV, N, D, dtype)
    rng = np.random.default_rng(S)
    ql, kl = ([int(x) for x in rng.integers(1, most + 1, S)] for most in (T, N))
    ql[0], kl[1], ql[2], kl[3], kl[4] = T, N, 0, 0, kl[1]
    if which == "queries":
        kl = None
    if which == "states":
        ql = None
    tok_err, st_err = ints([0]), ints([0])
    given = list(ql or []), list(kl or [])
    if which == "bad":
        given[0][0], given[1][1] = T + 1, -1
    tok = H.make_tokens(T, ints(given[0]) if ql else None, None, tok_err)
    st = H.make_states(k, v, ints(given[1]) if kl else None, st_err)
    cfg = cfg_of(H, S, heads, D, dtype)
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    o = torch.full(q.shape, 3.0, dtype=torch.float32 if out == "fp32" else torch.bfloat16, device="cuda")
    lse = torch.full((S, heads, T), 3.0, device="cuda")
    for causal in (0, H.HKV_ATTN_CAUSAL):
        o.fill_(3.0), lse.fill_(3.0)
        H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(o), lse, ws, n, causal)
        first = 0
        if which == "bad":
            assert int(tok_err) == int(st_err) == H.HKV_ERR_BOUNDS
            assert (o[0] == 3.0).all() and (lse[0] == 3.0).all()
            assert torch.isnan(o[1, :ql[1]]).all() and torch.isnan(lse[1, :, :ql[1]]).all()
            assert (o[1, ql[1]:] == 3.0).all() and (lse[1, :, ql[1]:] == 3.0).all()
            first = 2
        check_cross(q[first:], k[first:], v[first:], o[first:], lse[first:], causal=bool(causal),
                    qlens=ql and ql[first:], klens=kl and kl[first:],
                    heads=range(0, heads, max(1, S * heads // 16)))
        # the same rows whatever the batch
        if which == "both":
            a, b = run_cross(H, torch, q.flip(0), k.flip(0), v.flip(0), qlens=ql[::-1], klens=kl[::-1],
                             causal=bool(causal), out_dtype=o.dtype)
            assert torch.equal(a.flip(0), o) and torch.equal(b.flip(0), lse)


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("S,T,heads,KV", [(2, 100, 3, 3), (2, 300, 3, 3), (1, 257, 4, 2), (2, 60, 6, 1)])
def test_outs_between_other_rows(S, T, heads, KV, ragged):
    """Views of outs leave the tokens, heads and sequences around them as they are."""
    torch, H = mods()
    D, N = 128, 90
    q, k, v = qkv(torch, S, T, heads, KV, N, D, "bf16")
    ql = [T - 37] + [T] * (S - 1) if ragged else None
    want, wlse = run_cross(H, torch, q, k, v, qlens=ql)
    check_cross(q, k, v, want, wlse, qlens=ql)
    around = torch.full((S + 1, T + 5, heads + 2, D + 8), 3.0, dtype=q.dtype, device="cuda")
    out = around[:S, 2:T + 2, 1:heads + 1, :D]
    cfg = cfg_of(H, S, heads, D, "bf16")
    tok, st = H.make_tokens(T, None if ql is None else ints(ql)), H.make_states(k, v)
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(out), None, ws, n)
    assert torch.equal(out, want)
    out.fill_(3.0)
    assert (around == 3.0).all()


def test_no_lse_and_strided_views():
    """Queries and outs by heads, states by tokens (slices of one projection), no lse."""
    torch, H = mods()
    for dtype, T, N in (("bf16", 200, 150), ("bf16", 3, 150), ("fp32", 20, 70)):
        S, heads, KV, D = 2, 4, 2, 64
        q, k, v = qkv(torch, S, T, heads, KV, N, D, dtype)
        want, _ = run_cross(H, torch, q, k, v)
        qh = torch.zeros(S, heads, T + 3, D, dtype=q.dtype, device="cuda")
        qh[:, :, 1:T + 1] = q.transpose(1, 2)
        kv = torch.zeros(S, N, 2 * KV + 1, D, dtype=q.dtype, device="cuda")
        kv[:, :, :KV], kv[:, :, KV:2 * KV] = k.transpose(1, 2), v.transpose(1, 2)
        out = torch.full((S, heads, T + 1, D), 3.0, dtype=q.dtype, device="cuda")
        cfg = cfg_of(H, S, heads, D, dtype)
        st = H.make_states(kv[:, :, :KV].transpose(1, 2), kv[:, :, KV:2 * KV].transpose(1, 2))
        tok = H.make_tokens(T)
        n = H.hkv_cross_workspace_size(cfg, st, tok)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        H.hkv_cross_attention(cfg, st, tok, H.make_rows(qh[:, :, 1:T + 1].transpose(1, 2)),
                              H.make_rows(out[:, :, :T].transpose(1, 2)), None, ws, n)
        assert torch.equal(out[:, :, :T].transpose(1, 2), want) and (out[:, :, T] == 3.0).all()


@pytest.mark.parametrize("T", [1, 300])
def test_offsets_past_32_bits(T):
    """A head and a token whose elements lie more than 2^32 bytes, and 2^31 elements, apart."""
    torch, H = mods()
    D, N = 64, 9
    big = torch.empty((1 << 31) + (1 << 20), dtype=torch.bfloat16, device="cuda")
    q = torch.randn(1, T, 2, D, device="cuda").bfloat16()
    k, v = torch.randn(2, 1, 2, N, D, device="cuda").bfloat16()
    # keys of head 0 at the start, of head 1 2^31 elements on; values in the rows between
    far = big.as_strided((1, 2, N, D), (1 << 31, 1 << 31, 2 * D, 1))
    far_v = big.as_strided((1, 2, N, D), (1 << 31, 1 << 31, 2 * D, 1), storage_offset=D)
    far.copy_(k)
    far_v.copy_(v)
    out, lse = run_cross(H, torch, q, far, far_v)
    check_cross(q, k, v, out, lse)


def test_elements_that_are_not_finite():
    torch, H = mods()
    for T in (2, 200):
        q, k, v = qkv(torch, 1, T, 2, 2, 100, 64, "bf16")
        k[0, 0, 50] = float("nan")
        v[0, 1, 70, 3] = float("inf")
        q[0, 1, 1] = float("nan")
        out, lse = run_cross(H, torch, q, k, v)
        fine = torch.isfinite(out[0]).cpu().numpy()
        want = np.ones(fine.shape, bool)
        want[:, 0] = False
        want[:, 1, 3] = False
        want[1, 1] = False
        assert np.array_equal(fine, want)


def test_scores_of_minus_infinity_weigh_nothing():
    """The lowest numbers of the type as keys: scores of -inf beside others, and alone."""
    torch, H = mods()
    for T in (1, 200):
        q = torch.full((1, T, 1, 64), 2.0, dtype=torch.bfloat16, device="cuda")
        k = torch.zeros(1, 1, 40, 64, dtype=torch.bfloat16, device="cuda")
        v = torch.randn(1, 1, 40, 64, device="cuda").bfloat16()
        k[0, 0, :39] = torch.finfo(torch.bfloat16).min
        out, lse = run_cross(H, torch, q, k, v)
        assert torch.equal(out[0, :, 0], v[0, 0, 39].expand(T, 64)) and (lse == 0).all()


def test_streams_graphs_and_two_calls_at_once():
    """Calls captured and replayed on new data, and two streams with a workspace each."""
    torch, H = mods()
    S, T, heads, KV, N, D = 1, 2, 4, 2, 2000, 64     # ranges joined through the workspace
    cfg = cfg_of(H, S, heads, D, "bf16")
    rope = H.hkv_make_rope(head_dim=D)
    q, k, v = qkv(torch, S, T, heads, KV, N, D, "bf16")
    tok = H.make_tokens(T, None, ints(np.arange(T)[None]))
    st = H.make_states(k, v)
    n = H.hkv_cross_workspace_size(cfg, st, tok)
    assert n > 256
    runs = []
    for i in range(2):
        runs.append(dict(stream=torch.cuda.Stream(), x=torch.zeros_like(q), q=torch.zeros_like(q), out=torch.zeros_like(q),
                         ws=torch.zeros(n, dtype=torch.uint8, device="cuda")))

    def calls(r, stream):
        H.hkv_rope_rotate(cfg, rope, tok, H.make_rows(r["x"]), H.make_rows(r["q"]), stream=stream)
        H.hkv_cross_attention(cfg, st, tok, H.make_rows(r["q"]), H.make_rows(r["out"]), None, r["ws"], n, stream=stream)
    torch.cuda.synchronize()
    graphs = []
    for r in runs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=r["stream"]):
            calls(r, torch.cuda.current_stream().cuda_stream)
        graphs.append(g)
    xs = [tensor(np.random.default_rng(7 + i).normal(size=q.shape), "bf16") for i in range(6)]
    want = []
    for x in xs:
        r = dict(x=x, q=torch.zeros_like(q), out=torch.zeros_like(q), ws=torch.zeros(n, dtype=torch.uint8, device="cuda"))
        calls(r, torch.cuda.current_stream().cuda_stream)
        want.append(r["out"])
    torch.cuda.synchronize()
    for i in range(0, 6, 2):
        for j, r in enumerate(runs):
            with torch.cuda.stream(r["stream"]):
                r["x"].copy_(xs[i + j])
                graphs[j].replay()
        torch.cuda.synchronize()
        for j, r in enumerate(runs):
            assert torch.equal(r["out"], want[i + j])


def test_attention_joins_a_quantised_cache():
    """One query over an encoder's states, as the prior of a cache in 8 bits."""
    torch, H = mods()
    from oracle import serve as OS
    from test_gpu_serve import QCache
    heads, D, N = 3, 64, 77
    c = QCache([50, 1, 0], D, 8, "bf16")
    q, k, v = qkv(torch, 1, 1, heads, heads, N, D, "bf16")
    cfg = c.cfg
    out, lse = run_cross(H, torch, q, k, v, out_dtype=torch.float32, cfg=cfg)
    n = H.hkv_quant_workspace_size(cfg)
    both, both_lse = torch.zeros(heads, D, device="cuda"), torch.zeros(heads, device="cuda")
    H.hkv_quant_attention(cfg, c.c, 0, q, both, torch.zeros(n, dtype=torch.uint8, device="cuda"), n,
                          prior=(out, lse), lse=both_lse)
    for h in range(heads):
        rows = slice(c.off[h], c.off[h] + c.lens[h])
        K = np.concatenate([host(k)[0, h], OS.values(c.k_codes[rows], c.k_scales[rows])])
        V = np.concatenate([host(v)[0, h], OS.values(c.v_codes[rows], c.v_scales[rows])])
        want, wlse = OS.attention_lse(host(q)[0, 0, h], K, V)
        A = float((np.abs(K) @ np.abs(host(q)[0, 0, h])).max()) / math.sqrt(D)
        assert np.abs(host(both)[h] - want).max() <= (2.0 ** -18 * A + 2.0 ** -18) * np.abs(V).max()
        assert abs(float(both_lse[h]) - wlse) <= 2.0 ** -19 * A + 2.0 ** -16


@pytest.mark.parametrize("fmt", [None, 8])
def test_from_projections_to_the_cache(fmt):
    """Projections normed, rotated and generated with: the run prepares what a
    provider of ready queries and keys gives, and every output is the same."""
    torch, H = mods()
    from paper_2605_20600_gb300.engine import Engine, Heads
    from paper_2605_20600_gb300.runner import generate
    L, S, HQ, D, C, N, W = 2, 2, 3, 64, 5, 40, 8
    cfg = cfg_of(H, S, HQ, D, "bf16", n_layers=L, n_cond=C, n_image=N, row_len=8, recent_w=16, local_w=16,
                 period=8, group_at=20, global_budget=24)
    rng = np.random.default_rng(11)
    cond = tensor(rng.normal(size=(L, 2, S, HQ, C, D)), "bf16")
    image = tensor(rng.normal(size=(N, 3, L, S, HQ, D)), "bf16")
    weights = tensor(1 + 0.2 * rng.normal(size=(L, 2, D)), "bf16")
    norms = [H.make_norm(H.HKV_NORM_LAYER, 1e-5, weights[i, 0], weights[i, 1]) for i in range(L)]
    # conditioning tokens on the diagonal, image tokens on a grid of W columns
    grid = np.arange(N)
    pos = ints(np.stack([np.r_[np.arange(C), C + grid // W], np.r_[np.arange(C), C + grid % W]])[:, None])
    rope = H.hkv_make_rope(head_dim=D, layout=H.HKV_ROPE_PAIRS, sections=(16, 16))
    heads = Heads(cfg, rope=rope, norms=norms, positions=pos)

    class Raw:
        def cond(self, kc, vc, layer, stream):
            kc.copy_(cond[layer, 0]), vc.copy_(cond[layer, 1])

        def image(self, q, k, v, l0, nl, t0, nt, stream):
            for x, y in zip((q, k, v), image[t0]):
                x.copy_(y)

    # the same by plain torch in fp64, rounded once
    freq = P.frequencies(D, (16, 16))

    def ready(x, layer, which, places):
        """x [..., places, D] fp64"""
        a = P.angles_of(pos.cpu().numpy()[:, 0, places], freq, (16, 16))
        return P.rotate(P.norm(x, "layer", float(np.float32(1e-5)), host(weights[layer, which])), a, "pairs")

    def close_bits(got, want):
        close(host(got), want, np.full(want.shape, 2.0 ** -16), "bf16")

    seen = {}

    class Ready(Raw):
        def cond(self, kc, vc, layer, stream):
            super().cond(kc, vc, layer, stream)
            eng.prepare(heads, layer, None, kc.transpose(1, 2), 0)
            close_bits(kc, ready(host(cond[layer, 0]), layer, 1, slice(0, C)))

        def image(self, q, k, v, l0, nl, t0, nt, stream):
            super().image(q, k, v, l0, nl, t0, nt, stream)
            for layer in range(L):
                eng.prepare(heads, layer, q[layer], k[layer], C + t0)
                for which, x in enumerate((q, k)):
                    want = ready(host(image[t0, which, layer])[..., None, :], layer, which, slice(C + t0, C + t0 + 1))
                    close_bits(x[layer], want[..., 0, :])

    outs = []
    for provider, h in ((Raw(), heads), (Ready(), None)):
        eng = Engine(cfg)
        got = []
        generate(eng, provider, on_step=lambda t, out: got.append(out.clone()), cache_format=fmt, heads=h)
        eng.check()
        outs.append(torch.stack(got))
    assert torch.equal(outs[0], outs[1]) and torch.isfinite(outs[0]).all()


def test_a_prompt_from_the_projection_to_the_first_step():
    """Norms and rotation into the cache's layouts, the prompt's own causal
    attention, prefill, and the first step over the cache, as a model runs them."""
    torch, H = mods()
    from paper_2605_20600_gb300.engine import Engine
    S, HQ, D, C = 2, 4, 64, 70
    cfg = cfg_of(H, S, HQ, D, "bf16", n_cond=C, n_image=16, row_len=4, recent_w=8, local_w=8, period=4,
                 group_at=8, global_budget=8)
    eng = Engine(cfg)
    rng = np.random.default_rng(2)
    x = tensor(rng.normal(size=(S, C + 1, 3 * HQ, D)), "bf16")
    rope = H.hkv_make_rope(head_dim=D)
    norm = H.make_norm(H.HKV_NORM_RMS, 1e-6)
    q = torch.empty(S, C, HQ, D, dtype=x.dtype, device="cuda")
    kc, vc = (torch.empty(S, HQ, C, D, dtype=x.dtype, device="cuda") for _ in range(2))
    step = torch.empty(3, S, HQ, D, dtype=x.dtype, device="cuda")
    every = ints(np.arange(C + 1)[None])

    def prepare(tokens, first, outs):
        rows = [H.make_rows(x[:, first:first + tokens, i * HQ:(i + 1) * HQ]) for i in range(3)]
        H.hkv_qk_norm_rope(cfg, norm, rope, H.make_tokens(tokens, None, every[:, first:first + tokens]), *rows,
                           *(H.make_rows(o) for o in outs))
    prepare(C, 0, (q, kc.transpose(1, 2), vc.transpose(1, 2)))
    out, lse = run_cross(H, torch, q, kc, vc, causal=True, cfg=cfg)
    check_cross(q, kc, vc, out, lse, causal=True)
    eng.prefill(0, kc, vc)
    prepare(1, C, step)
    got = torch.empty(S, HQ, D, device="cuda")
    eng.step(0, step[0], step[1], step[2], got)
    eng.check()
    freq = P.frequencies(D, (D // 2,))
    full = host(x)
    for i, name in ((0, "q"), (1, "k")):
        y = P.norm(full[:, :, i * HQ:(i + 1) * HQ], "rms", float(np.float32(1e-6)))
        y = P.rotate(y, (np.arange(C + 1)[:, None] * freq)[:, None], "half")
        mine = host(q) if name == "q" else host(kc).transpose(0, 2, 1, 3)
        close(mine, y[:, :C], np.full(mine.shape, 2.0 ** -17), "bf16")
    keys, values = torch.cat([kc, step[1][:, :, None]], 2), torch.cat([vc, step[2][:, :, None]], 2)
    check_cross(step[0][:, None], keys, values, got[:, None], torch.from_numpy(np.stack([
        [[P.cross(host(step[0])[s, h][None], host(keys)[s, h], host(values)[s, h])[1][0]] for h in range(HQ)]
        for s in range(S)])).float())
