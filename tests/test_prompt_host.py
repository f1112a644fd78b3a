"""Rotary positions, norms of heads and attention over other states without a
GPU: exported symbols, host-side checks, the rotation's table, the oracle."""
import ctypes
import math
import os
import re

import numpy as np
import pytest

from conftest import ROOT

from oracle import prompt as P

HEADER = os.path.join(ROOT, "include", "hkv_prompt.h")


@pytest.fixture(scope="module")
def H():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2605_20600_gb300 import hkv
    hkv.lib()
    return hkv


def cfg_of(H, **kw):
    base = dict(n_layers=1, n_seqs=3, n_heads=6, head_dim=64, dtype="bf16", n_cond=0, n_image=8,
                row_len=1, recent_w=1, local_w=1, period=1, group_at=1, global_budget=1)
    base.update(kw)
    return H.make_config(**base)


def views(H):
    # aligned host addresses: never dereferenced by the checks tested here
    buf = ctypes.create_string_buffer(8192)
    a = (ctypes.addressof(buf) + 255) & ~255
    rows = H.hkv_rows(a, 5 * 6 * 64, 6 * 64, 64, 6, H.HKV_BF16)
    other = H.hkv_rows(a + 1024, 5 * 6 * 64, 6 * 64, 64, 6, H.HKV_BF16)
    tokens = H.hkv_tokens(5, 0, a, a, 15, 5, a)
    states = H.hkv_states(a, a, a, a, 2 * 50 * 64, 50 * 64, 64, 2, 50)
    return buf, a, rows, other, tokens, states


def change(base, **kw):
    x = type(base).from_buffer_copy(base)
    for k, v in kw.items():
        setattr(x, k, v)
    return x


def test_every_declared_symbol_is_exported(H):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(hkv_[a-z_]+)\s*\(", text))
    assert names == {"hkv_make_rope", "hkv_rope_rotate", "hkv_qk_norm_rope",
                     "hkv_cross_workspace_size", "hkv_cross_attention"}
    for n in names:
        assert hasattr(H.lib(), n) and hasattr(H, n), n


def test_struct_sizes(H):
    assert ctypes.sizeof(H.hkv_rope_params) == 40 + 48
    assert ctypes.sizeof(H.hkv_rope) == 32 + 512
    assert ctypes.sizeof(H.hkv_rows) == 40 and ctypes.sizeof(H.hkv_tokens) == 48
    assert ctypes.sizeof(H.hkv_norm) == 56 and ctypes.sizeof(H.hkv_states) == 64


SCALINGS = [("plain", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
            ("parts", dict(factor=32.0, original=2048, low=1.0, high=4.0))]


@pytest.mark.parametrize("scaling,kw", SCALINGS)
@pytest.mark.parametrize("rot,sections,joint", [(128, None, False), (32, None, False), (6, None, False),
                                                (2, None, False), (64, (16, 16), False),
                                                (48, (4, 12, 8), True), (48, (12, 12), False)])
def test_the_table_holds_the_frequencies(H, scaling, kw, rot, sections, joint):
    rope = H.hkv_make_rope(head_dim=128, rot_dim=rot, sections=sections, joint=joint, base=500000.0,
                           scaling=["plain", "linear", "base", "parts"].index(scaling), amplitude=1.25, **kw)
    want = P.frequencies(rot, sections or (rot // 2,), joint=joint, base=500000.0, scaling=scaling, **kw)
    got = np.array([rope.turns[i] for i in range(rot // 2)], dtype=np.float64) * (2 * math.pi / 2.0 ** 64)
    # (no angle above one turn a position for base > 1); the table cuts at 2^-64 turns
    np.testing.assert_allclose(got, want, rtol=1e-13, atol=2 * math.pi * 2.0 ** -64)
    assert list(rope.section)[:rope.n_axes] == list(sections or (rot // 2,))
    assert rope.amplitude == 1.25 and rope.rot_dim == rot
    assert all(rope.turns[i] == 0 for i in range(rot // 2, 64))


def test_make_rope_refuses(H):
    def status(**kw):
        base = dict(head_dim=64, rot_dim=64)
        base.update(kw)
        try:
            H.hkv_make_rope(**base)
        except H.HkvError as e:
            return e.status
        return 0
    assert status() == 0
    for kw in (dict(head_dim=96), dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=0), dict(rot_dim=-2),
               dict(sections=(16, 15)), dict(sections=(32, 0)), dict(sections=(33, -1)),
               dict(sections=(8, 8, 8, 8))):
        assert status(**kw) == 2, kw
    for kw in (dict(layout=2), dict(scaling=4), dict(scaling=-1), dict(base=0.0), dict(base=math.nan),
               dict(base=math.inf), dict(amplitude=math.nan), dict(scaling=1, factor=0.5),
               dict(scaling=1, factor=math.nan), dict(scaling=3, factor=2.0, original=0.0),
               dict(scaling=3, factor=2.0, original=8.0, low=4.0, high=4.0),
               dict(scaling=3, factor=2.0, original=8.0, low=-1.0)):
        assert status(**kw) == 1, kw
    p = H.hkv_rope_params()
    assert H.lib().hkv_make_rope(None, ctypes.byref(H.hkv_rope())) == 1
    assert H.lib().hkv_make_rope(ctypes.byref(p), None) == 1


def common_refusals(H, call, cfg, a, rows, tokens):
    """call(cfg, tokens, in, out) -> status; what every call on rows refuses."""
    assert call(cfg=cfg_of(H, head_dim=96)) == 2
    assert call(tokens=change(tokens, n_tokens=0)) == 2 and call(tokens=change(tokens, n_tokens=1 << 25)) == 2
    assert call(tokens=change(tokens, reserved=1)) == 1 and call(tokens=change(tokens, len=a + 2)) == 8
    for side in ("x", "out"):
        r = rows[side]
        assert call(**{side: change(r, data=None)}) == 1
        assert call(**{side: change(r, data=a + 8)}) == 8
        assert call(**{side: change(r, dtype=7)}) == 1
        assert call(**{side: change(r, n_heads=0)}) == 2
        assert call(**{side: change(r, n_heads=5)}) == 2      # not the other side's
        for s in ("seq_stride", "token_stride", "head_stride"):
            for bad in (0, -64, 63, 68, 56, (1 << 40) + 8):
                assert call(**{side: change(r, **{s: bad})}) == 2, (side, s, bad)


def test_rotate_and_norm_refuse(H):
    buf, a, rows, other, tokens, states = views(H)
    cfg, R, lib = cfg_of(H), ctypes.byref, H.lib()
    rope = H.hkv_make_rope(head_dim=64)

    def rotate(cfg=cfg, rope=rope, tokens=tokens, x=rows, out=other, flags=0):
        return lib.hkv_rope_rotate(R(cfg), R(rope) if rope else None, R(tokens), R(x), R(out), flags, None)

    def prepare(cfg=cfg, norm=None, rope=rope, tokens=tokens, x=rows, out=other):
        n = R(norm) if norm else None
        return lib.hkv_qk_norm_rope(R(cfg), n, R(rope) if rope else None, R(tokens), R(x), None, None,
                                    R(out), None, None, None)

    for call in (rotate, prepare):
        common_refusals(H, call, cfg, a, {"x": rows, "out": other}, tokens)
        assert call(out=change(other, dtype=H.HKV_FP32)) == 2
        assert call(out=change(rows, token_stride=7 * 64)) == 1     # in place, other rows
        assert call(tokens=change(tokens, pos=None)) == 1 and call(tokens=change(tokens, pos=a + 1)) == 8
        assert call(tokens=change(tokens, pos_seq_stride=-1)) == 2
        assert call(rope=change(rope, head_dim=128)) == 2 and call(rope=change(rope, rot_dim=62)) == 2
        assert call(rope=change(rope, n_axes=0)) == 2 and call(rope=change(rope, n_axes=4)) == 2
        assert call(rope=change(rope, layout=3)) == 1 and call(rope=change(rope, amplitude=math.nan)) == 1
        assert call(rope=change(rope, section=(ctypes.c_int32 * 3)(31, 1, 0))) == 2
    assert rotate(rope=None) == 1 and rotate(flags=2) == 1
    norm = H.make_norm(H.HKV_NORM_LAYER, 1e-5)
    assert prepare(norm=change(norm, kind=0)) == 1 and prepare(norm=change(norm, kind=3)) == 1
    assert prepare(norm=change(norm, eps=-1.0)) == 1 and prepare(norm=change(norm, eps=math.nan)) == 1
    for f in ("q_weight", "q_bias", "k_weight", "k_bias"):
        assert prepare(norm=change(norm, **{f: a + 8})) == 8, f
    for bad in (4, 60, 68, -64):
        assert prepare(norm=change(norm, q_head_stride=bad)) == 2, bad
    assert prepare(norm=change(norm, kind=H.HKV_NORM_RMS, q_bias=a)) == 1

    def sets(q=None, k=None, v=None, qo=None, ko=None, vo=None):
        return lib.hkv_qk_norm_rope(R(cfg), None, R(rope), R(tokens),
                                    *(R(x) if x else None for x in (q, k, v, qo, ko, vo)), None)
    assert sets() == 1 and sets(q=rows) == 1 and sets(qo=rows) == 1 and sets(k=rows, vo=other) == 1
    assert sets(q=change(rows, n_heads=2), qo=change(other, n_heads=2)) == 2    # not the config's


def test_cross_refuses(H):
    buf, a, rows, other, tokens, states = views(H)
    cfg, R, lib = cfg_of(H), ctypes.byref, H.lib()

    def cross(cfg=cfg, states=states, tokens=tokens, x=rows, out=other, lse=a, ws=a, n=1 << 40, flags=0):
        return lib.hkv_cross_attention(R(cfg), R(states), R(tokens), R(x), R(out), lse, ws, n, flags, None)

    common_refusals(H, cross, cfg, a, {"x": rows, "out": other}, tokens)
    assert cross(x=change(rows, dtype=H.HKV_FP32)) == 2
    f32 = cfg_of(H, dtype="fp32")
    assert cross(cfg=f32, x=change(rows, dtype=H.HKV_FP32), out=other) == 2    # a bf16 out of fp32
    assert cross(out=change(other, data=rows.data)) == 1
    assert cross(ws=None) == 1 and cross(ws=a + 8) == 8 and cross(lse=a + 2) == 8 and cross(flags=2) == 1
    for f in ("k", "v"):
        assert cross(states=change(states, **{f: None})) == 1 and cross(states=change(states, **{f: a + 8})) == 8
    assert cross(states=change(states, n_heads=4)) == 2 and cross(states=change(states, n_heads=0)) == 2
    assert cross(states=change(states, max_len=0)) == 2 and cross(states=change(states, max_len=1 << 25)) == 2
    assert cross(states=change(states, len=a + 1)) == 8
    for s in ("seq_stride", "head_stride", "token_stride"):
        for bad in (0, -64, 56, 68):
            assert cross(states=change(states, **{s: bad})) == 2, (s, bad)
    # more partial results than the workspace holds
    long = change(states, max_len=5000)
    need = H.hkv_cross_workspace_size(cfg, long, tokens)
    assert need > 256 and cross(states=long, n=64) == 3
    # too many queries, lse elements past an int
    many = cfg_of(H, n_seqs=1 << 14, n_heads=1 << 6)
    assert H.hkv_cross_workspace_size(many, change(states, n_heads=1 << 6), change(tokens, n_tokens=1 << 11)) == 0
    assert H.hkv_cross_workspace_size(cfg, change(states, n_heads=5), tokens) == 0
    assert H.hkv_cross_workspace_size(cfg_of(H, head_dim=32), states, tokens) == 0


def test_views_of_tensors(H):
    import torch
    x = torch.zeros(3, 5, 6, 64, dtype=torch.bfloat16)
    cfg = cfg_of(H)
    rope = H.hkv_make_rope(head_dim=64)
    pos = torch.zeros(1, 3, 5, dtype=torch.int32)
    tok = H.make_tokens(5, None, pos)

    def refused(f, *args, status=2, **kw):
        with pytest.raises(H.HkvError) as e:
            f(*args, **kw)
        assert e.value.status == status
    refused(H.make_rows, x.transpose(2, 3))
    refused(H.make_rows, x.half())
    refused(H.make_rows, x[0, 0])
    refused(H.make_tokens, 5, torch.zeros(3, dtype=torch.int64))
    refused(H.make_tokens, 5, None, pos[:, :, :4])
    refused(H.make_tokens, 5, None, pos.long())
    refused(H.make_states, x, x.float())
    refused(H.make_states, x, x, torch.zeros(2, dtype=torch.int32))
    refused(H.make_states, x, x[:, :, ::2])
    refused(H.make_norm, 1, 1e-5, torch.zeros(64), torch.zeros(32))
    refused(H.make_norm, 1, 1e-5, torch.zeros(64), torch.zeros(64).bfloat16())
    refused(H.make_norm, 2, 1e-5, torch.zeros(6, 64), None, torch.zeros(64))
    refused(H.make_norm, 1, 1e-5, torch.zeros(64, dtype=torch.float16))
    # sizes of the call: sequences, tokens, channels, axes, sequences of lengths and positions
    r = H.make_rows(x)
    refused(H.hkv_rope_rotate, cfg, rope, tok, H.make_rows(x[:2]), r)
    refused(H.hkv_rope_rotate, cfg, rope, tok, r, H.make_rows(x[:, :4]))
    refused(H.hkv_rope_rotate, cfg, rope, tok, H.make_rows(x[..., :32]), r)
    refused(H.hkv_rope_rotate, cfg, H.hkv_make_rope(head_dim=64, sections=(16, 16)), tok, r, r)
    refused(H.hkv_rope_rotate, cfg, rope, H.make_tokens(5, None, pos[:, :2]), r, r)
    refused(H.hkv_rope_rotate, cfg, rope, H.make_tokens(5, torch.zeros(2, dtype=torch.int32), pos), r, r)
    refused(H.hkv_qk_norm_rope, cfg, H.make_norm(1, 1e-5, torch.zeros(64)), rope, tok, r, None, None, r, None, None)
    refused(H.hkv_qk_norm_rope, cfg, H.make_norm(1, 1e-5, x[0, 0, :5].contiguous()), rope, tok, r, None, None, r,
            None, None)
    st = H.make_states(x[:2], x[:2])
    assert H.hkv_cross_workspace_size(cfg, st, tok) == 0
    refused(H.hkv_cross_attention, cfg, st, tok, r, r, None, 256, 1 << 20)


@pytest.mark.parametrize("name", ["make_rope", "rope_rotate", "qk_norm_rope", "cross_attention"])
def test_fault_injection(H, name, monkeypatch):
    buf, a, rows, other, tokens, states = views(H)
    cfg, rope = cfg_of(H), H.hkv_make_rope(head_dim=64)
    monkeypatch.setenv("HKV_FAULT_INJECT", f"{name}:6")
    calls = {
        "make_rope": lambda: H.hkv_make_rope(head_dim=64),
        "rope_rotate": lambda: H.hkv_rope_rotate(cfg, rope, tokens, rows, other),
        "qk_norm_rope": lambda: H.hkv_qk_norm_rope(cfg, None, rope, tokens, rows, None, None, other, None, None),
        "cross_attention": lambda: H.hkv_cross_attention(cfg, states, tokens, rows, other, a, a, 1 << 40),
    }
    with pytest.raises(H.HkvError) as e:
        calls[name]()
    assert e.value.status == 6


# the oracle -----------------------------------------------------------------
def test_oracle_rotation_turns_pairs():
    x = np.arange(1.0, 9.0)
    quarter = np.array([math.pi / 2, 0.0])
    np.testing.assert_allclose(P.rotate(x, quarter, "half"), [-3, 2, 1, 4, 5, 6, 7, 8], atol=1e-15)
    np.testing.assert_allclose(P.rotate(x, quarter, "pairs", 2.0), [-4, 2, 6, 8, 5, 6, 7, 8], atol=1e-15)
    a = np.array([0.3, -1.1])
    np.testing.assert_allclose(P.rotate(P.rotate(x, a, "half"), -a, "half"), x, atol=1e-14)
    # scores depend on the distance alone
    f = P.frequencies(8, (4,))
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(2, 8))

    def score(p, r):
        return P.rotate(q, p * f, "pairs") @ P.rotate(k, r * f, "pairs")
    assert abs(score(100, 93) - score(7, 0)) < 1e-12
    np.testing.assert_array_equal(P.angles_of([[2], [3]], np.array([1.0, 0.5, 1.0]), (2, 1)), [[2, 1, 3]])


def test_oracle_frequencies():
    np.testing.assert_allclose(P.frequencies(4, (2,), base=100.0), [1, 0.1])
    np.testing.assert_allclose(P.frequencies(8, (2, 2), base=100.0), [1, 0.1, 1, 0.1])
    np.testing.assert_allclose(P.frequencies(4, (1, 1), base=100.0, joint=True), [1, 0.1])
    np.testing.assert_allclose(P.frequencies(4, (2,), base=100.0, scaling="base", factor=10.0), [1, 0.01])
    # fast pairs keep their frequency, slow ones are divided
    f = P.frequencies(4, (2,), base=1e6, scaling="parts", factor=8.0, original=1000.0, low=1.0, high=32.0)
    np.testing.assert_allclose(f, [1, 1e-3 / 8])


def test_oracle_norms():
    x = np.array([3.0, 1.0, -1.0, 1.0])
    np.testing.assert_allclose(P.norm(x, "rms", 1.0), x / 2)
    np.testing.assert_allclose(P.norm(x, "layer", 2.0, [2, 2, 2, 2], [1, 0, 0, 0]), np.array([2, 0, -2, 0]) + [1, 0, 0, 0])


def test_oracle_attention():
    q = np.zeros((3, 4))
    V = np.arange(8.0).reshape(2, 4)
    out, lse = P.cross(q, np.ones((2, 4)), V, causal=True)      # query 0 sees nothing
    np.testing.assert_allclose(out, [[0] * 4, V[0], V.mean(0)])
    np.testing.assert_allclose(lse, [-math.inf, 0, math.log(2)])
    out, lse = P.cross(q, np.ones((0, 4)), np.ones((0, 4)))
    assert (out == 0).all() and np.isneginf(lse).all()
