"""The serving cache without a GPU: the library exports what the header
declares, its host-side checks answer before any CUDA call, and the oracle's
row format holds what it promises."""
import ctypes
import os
import re

import numpy as np
import pytest

from conftest import ROOT

from oracle import serve as S

HEADER = os.path.join(ROOT, "include", "hkv_serve.h")


@pytest.fixture(scope="module")
def H():
    import __graft_entry__
    __graft_entry__.build()
    from paper_2605_20600_gb300 import hkv
    hkv.lib()
    return hkv


def cfg_of(H, **kw):
    base = dict(n_layers=2, n_seqs=4, n_heads=4, head_dim=64, dtype="bf16", n_cond=8, n_image=64,
                row_len=8, recent_w=16, local_w=16, period=8, group_at=16, global_budget=24)
    base.update(kw)
    return H.make_config(**base)


def caches(H):
    # aligned host addresses: never dereferenced by the checks tested here
    buf = ctypes.create_string_buffer(8192)
    a = (ctypes.addressof(buf) + 255) & ~255
    plain = H.hkv_cache(a, a, a, a, a, a, a, a, a, a, a, 1000)
    quant = H.hkv_qcache(a, a, a, a, a, a, a, a, a, a, a, a, a, 1000, 8, 0)
    prefix = H.hkv_prefix(a, a, a, None, 4 * 50 * 64, 50 * 64, 64, 2, 50)
    return buf, a, plain, quant, prefix


def test_every_declared_symbol_is_exported(H):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(hkv_[a-z_]+)\s*\(", text))
    assert names == {"hkv_quant_pack", "hkv_quant_unpack", "hkv_quant_workspace_size",
                     "hkv_quant_attention", "hkv_quant_step", "hkv_quant_evict",
                     "hkv_quant_evict_all", "hkv_quant_check", "hkv_prefix_workspace_size", "hkv_prefix_attention"}
    for n in names:
        assert hasattr(H.lib(), n) and hasattr(H, n), n


def test_struct_sizes(H):
    assert ctypes.sizeof(H.hkv_qcache) == 14 * 8 + 8
    assert ctypes.sizeof(H.hkv_prefix) == 7 * 8 + 8


def status(f, *args):
    return f(*args)


def test_refusals(H):
    buf, a, plain, quant, prefix = caches(H)
    lib, R = H.lib(), ctypes.byref
    cfg = cfg_of(H)
    big = 1 << 30

    def change(base, **kw):
        x = type(base).from_buffer_copy(base)
        for k, v in kw.items():
            setattr(x, k, v)
        return x

    def attention(cfg=cfg, c=quant, layer=0, q=a, po=None, pl=None, out=a, ws=a, n=big):
        return lib.hkv_quant_attention(R(cfg), R(c), layer, q, po, pl, out, None, ws, n, None)

    assert attention(q=None) == 1 and attention(out=None) == 1 and attention(ws=None) == 1
    assert attention(layer=2) == 1 and attention(layer=-1) == 1
    assert attention(po=a) == 1 and attention(pl=a) == 1
    assert attention(q=a + 8) == 8 and attention(out=a + 4) == 8 and attention(po=a + 8, pl=a) == 8
    assert attention(n=8) == 3
    assert attention(cfg=cfg_of(H, head_dim=96)) == 2
    for field in ("k", "v", "ks", "vs", "pos", "off", "cap", "len", "nbuf", "ntok", "label", "qbuf", "err"):
        assert attention(c=change(quant, **{field: None})) == 1, field
    for field in ("k", "v", "ks", "vs", "qbuf"):
        assert attention(c=change(quant, **{field: a + 8})) == 8, field
    assert attention(c=change(quant, format=6)) == 1 and attention(c=change(quant, reserved=1)) == 1
    assert attention(c=change(quant, capacity_tokens=0)) == 3
    assert lib.hkv_quant_attention(R(cfg), None, 0, a, None, None, a, None, a, big, None) == 1

    def step(k=a, v=a, flags=0, n=big):
        return lib.hkv_quant_step(R(cfg), R(quant), 0, a, k, v, None, None, a, None, a, n, flags, None)

    assert step(k=None) == 1 and step(v=None) == 1 and step(flags=2) == 1
    assert step(k=a + 8) == 8 and step(n=16) == 3

    assert lib.hkv_quant_pack(R(cfg), R(plain), R(quant), 2, 0, None) == 1
    assert lib.hkv_quant_pack(R(cfg), R(plain), R(quant), -2, 0, None) == 1
    assert lib.hkv_quant_pack(R(cfg), R(plain), R(quant), 0, 2, None) == 1
    assert lib.hkv_quant_pack(R(cfg), R(plain), R(change(quant, qbuf=a + 256)), 0, 0, None) == 1
    assert lib.hkv_quant_pack(R(cfg), None, R(quant), 0, 0, None) == 1
    assert lib.hkv_quant_unpack(R(cfg), R(change(quant, qbuf=a + 256)), R(plain), 0, None) == 1
    assert lib.hkv_quant_unpack(R(cfg), R(quant), None, 0, None) == 1
    assert lib.hkv_quant_evict(R(cfg), R(quant), -1, None) == 1
    assert lib.hkv_quant_evict(R(cfg), R(quant), 2, None) == 1
    assert lib.hkv_quant_evict_all(R(cfg), None, None) == 1
    assert lib.hkv_quant_check(None, None) == 1
    assert lib.hkv_quant_check(R(change(quant, err=None)), None) == 1
    # a ring that does not fit shared memory
    assert lib.hkv_quant_evict_all(R(cfg_of(H, n_image=4000, period=2000, group_at=2000)), R(quant), None) == 3

    def prefix_call(cfg=cfg, p=prefix, q=a, out=a, lse=a, ws=a, n=big):
        return lib.hkv_prefix_attention(R(cfg), R(p), q, out, lse, ws, n, None)

    assert prefix_call(q=None) == 1 and prefix_call(out=None) == 1 and prefix_call(lse=None) == 1
    assert prefix_call(ws=None) == 1 and prefix_call(n=4) == 3
    assert prefix_call(q=a + 2) == 8 and prefix_call(p=change(prefix, k=a + 8)) == 8
    assert prefix_call(p=change(prefix, len=None)) == 1 and prefix_call(p=change(prefix, v=None)) == 1
    assert prefix_call(p=change(prefix, n_groups=3)) == 2 and prefix_call(p=change(prefix, n_groups=0)) == 2
    assert prefix_call(p=change(prefix, max_len=0)) == 2
    for s in ("group_stride", "head_stride", "token_stride"):
        assert prefix_call(p=change(prefix, **{s: 68})) == 2, s
        assert prefix_call(p=change(prefix, **{s: 0})) == 2, s
    assert H.hkv_prefix_workspace_size(cfg, change(prefix, n_groups=3)) == 0
    assert H.hkv_quant_workspace_size(cfg_of(H, head_dim=32)) == 0
    assert H.hkv_prefix_workspace_size(cfg, prefix) > 0 and H.hkv_quant_workspace_size(cfg) > 0


@pytest.mark.parametrize("name", ["quant_pack", "quant_unpack", "quant_attention", "quant_step",
                                  "quant_evict", "quant_evict_all", "quant_check",
                                  "prefix_attention"])
def test_fault_injection(H, name, monkeypatch):
    monkeypatch.setenv("HKV_FAULT_INJECT", f"{name}:6")
    buf, a, plain, quant, prefix = caches(H)
    cfg = cfg_of(H)
    calls = {
        "quant_pack": lambda: H.hkv_quant_pack(cfg, plain, quant, 0),
        "quant_unpack": lambda: H.hkv_quant_unpack(cfg, quant, plain, 0),
        "quant_attention": lambda: H.hkv_quant_attention(cfg, quant, 0, a, a, a, 1 << 30),
        "quant_step": lambda: H.hkv_quant_step(cfg, quant, 0, a, a, a, a, a, 1 << 30),
        "quant_evict": lambda: H.hkv_quant_evict(cfg, quant, 0),
        "quant_evict_all": lambda: H.hkv_quant_evict_all(cfg, quant),
        "quant_check": lambda: H.hkv_quant_check(quant),
        "prefix_attention": lambda: H.hkv_prefix_attention(cfg, prefix, a, a, a, a, 1 << 30),
    }
    with pytest.raises(H.HkvError) as e:
        calls[name]()
    assert e.value.status == 6


def test_make_prefix_refuses(H):
    import torch
    k = torch.zeros(2, 3, 10, 64)
    n = torch.zeros(2, dtype=torch.int32)
    H.make_prefix(k, torch.zeros(2, 3, 10, 64), n)
    for bad in (lambda: H.make_prefix(k[0], k[0], n), lambda: H.make_prefix(k, k[:, :2], n),
                lambda: H.make_prefix(k.transpose(2, 3), k.transpose(2, 3), n),
                lambda: H.make_prefix(k, k.transpose(1, 2).contiguous().transpose(1, 2), n),
                lambda: H.make_prefix(k, k, n[:1])):
        with pytest.raises(H.HkvError):
            bad()


def test_runner_refuses_what_it_cannot_run(H):
    from paper_2605_20600_gb300.runner import generate

    class Fake:
        cfg = cfg_of(H)

    with pytest.raises(ValueError):
        generate(Fake(), None, fused=False, cache_format=8)
    with pytest.raises(ValueError):
        generate(Fake(), None, shared_prompt=True)
    Fake.cfg = cfg_of(H, n_cond=0)
    with pytest.raises(ValueError):
        generate(Fake(), None, cache_format=8, shared_prompt=True)


@pytest.mark.parametrize("bits", [8, 4])
def test_oracle_row_format(bits):
    """What a row stands for is within half a step (and the rounding of the
    scale) of the row; storing and reading the codes is exact."""
    rng = np.random.default_rng(0)
    x = (rng.normal(size=(200, 128)) * np.exp(rng.normal(size=(200, 1)) * 5)).astype(np.float32)
    c, s = S.quantise(x, bits)
    M = 127 if bits == 8 else 7
    assert np.abs(c).max() == M
    assert np.array_equal(S.unpacked(S.packed(c, bits), bits), c)
    err = np.abs(S.values(c, s) - x).reshape(200, 4, 32)
    # half a step, or what the clamp cuts where the scale was rounded down
    assert (err <= s[..., None] * (0.5 + M * 2.0 ** -8)).all()
    z, sz = S.quantise(np.zeros((1, 32), np.float32), bits)
    assert (z == 0).all() and (sz == 0).all()
    bad = np.zeros((2, 32), np.float32)
    bad[0, 1], bad[1, 2] = np.inf, np.nan
    c, s = S.quantise(bad, bits)
    assert np.isnan(s).all() and (c == 0).all()


def test_make_prefix_refuses_types_the_kernel_would_misread(H):
    import torch
    bf, n = torch.bfloat16, torch.zeros(2, dtype=torch.int32)
    k = torch.zeros(2, 3, 10, 64, dtype=bf)
    H.make_prefix(k, k, n)
    for bad in (lambda: H.make_prefix(k, k, n.long()), lambda: H.make_prefix(k, k, n.float()),
                lambda: H.make_prefix(k, k, torch.zeros(4, dtype=torch.int32)[::2]),
                lambda: H.make_prefix(k, k.float(), n), lambda: H.make_prefix(k.half(), k.half(), n),
                lambda: H.make_prefix(k, k.to("meta"), n), lambda: H.make_prefix(k, k, n.to("meta"))):
        with pytest.raises(H.HkvError):
            bad()


def test_a_prompt_of_another_type_than_the_config_is_refused(H):
    """bf16 rows read as fp32 would be read past their end."""
    import torch
    buf, a, _, _, _ = caches(H)
    n = torch.zeros(2, dtype=torch.int32)
    for dtype, other in (("fp32", torch.bfloat16), ("bf16", torch.float32)):
        cfg = cfg_of(H, dtype=dtype)
        k = torch.zeros(2, 4, 10, 64, dtype=other)
        pre = H.make_prefix(k, k, n)
        assert H.hkv_prefix_workspace_size(cfg, pre) == 0
        with pytest.raises(H.HkvError) as e:
            H.hkv_prefix_attention(cfg, pre, a, a, a, a, 1 << 30)
        assert e.value.status == 2
        k = k.to(torch.float32 if dtype == "fp32" else torch.bfloat16)
        assert H.hkv_prefix_workspace_size(cfg, H.make_prefix(k, k, n)) > 0


def test_engine_refuses_a_prompt_before_it_changes_anything(H):
    import torch
    from paper_2605_20600_gb300.engine import Engine
    cfg = cfg_of(H)                                       # 2 layers, 4 sequences, 4 heads, C = 8
    good = torch.zeros(2, 2, 4, 8, 64, dtype=torch.bfloat16)
    wide = torch.zeros(2, 2, 4, 8, 65, dtype=torch.bfloat16)[..., :64]
    for k, v in ((good[:, :1].expand(2, 3, 4, 8, 64), None),      # 3 groups of 4 sequences
                 (good[:, :0], None), (good[:1], None), (good[:, 0], None), (good[:, :, :, :7], None),
                 (good.float(), None), (good, good.float()), (good.half(), None), (good, good[:, :1]),
                 (good.to("meta"), None)):
        eng = Engine.__new__(Engine)
        eng.cfg, eng.device, eng.quant, eng.prompt = cfg, torch.device("cpu"), None, None
        eng.ragged, eng.labels = object(), torch.zeros(32, dtype=torch.uint8)
        eng.off, eng.cap, eng.total_tokens = object(), object(), 5
        before = dict(vars(eng))
        with pytest.raises(H.HkvError) as e:
            eng.quantise(8, (k, k if v is None else v))
        assert e.value.status in (H.HKV_ERR_SHAPE, H.HKV_ERR_INVALID_ARG)
        assert vars(eng) == before
    # what the strides would make the attention refuse is known to the workspace query
    pre = H.make_prefix(wide[0], wide[0], torch.zeros(2, dtype=torch.int32))
    assert H.hkv_prefix_workspace_size(cfg, pre) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_runner_takes_only_prompts_that_are_shared(H, dtype):
    """The conditioning tokens of every run of sequences are looked at before
    they are prefilled; without image tokens nothing else runs."""
    import torch
    from paper_2605_20600_gb300.runner import generate

    class Fake:
        cfg = cfg_of(H, dtype=dtype)      # 4 sequences
        device, quant = torch.device("cpu"), None

        def __init__(self):
            self.filled = []

        def stream(self):
            return 0

        def prefill(self, layer, kc, vc):
            self.filled.append(layer)

    class Provider:
        def __init__(self, runs, odd=None):
            self.runs, self.odd = runs, odd

        def cond(self, kc, vc, layer, st):
            for x, sign in ((kc, 1.0), (vc, -1.0)):
                for s in range(4):
                    x[s] = sign * (1 + layer + s * self.runs // 4)
            if self.odd == "v" and layer == 1:
                vc[3, 2, 5, 7] += 1.0
            elif self.odd == "zero":       # other bits, equal as numbers
                kc[:] = 0.0
                kc[2] = -0.0
            elif self.odd == "nan":        # the same bits
                kc[:] = float("nan")

    def run(prompts, provider):
        f = Fake()
        generate(f, provider, last_step=-1, cache_format=8, shared_prompt=prompts)
        return f.filled

    assert run(True, Provider(1)) == [0, 1] and run(2, Provider(2)) == [0, 1] and run(4, Provider(4)) == [0, 1]
    assert run(1, Provider(1, "nan")) == [0, 1]
    for prompts, provider in ((True, Provider(2)), (True, Provider(4)), (2, Provider(4)),
                              (1, Provider(1, "v")), (1, Provider(1, "zero")), (3, Provider(1)),
                              (8, Provider(1)), (-1, Provider(1))):
        with pytest.raises(ValueError):
            run(prompts, provider)


def test_runner_quantises_a_cache_it_continues_with(H):
    import torch
    from paper_2605_20600_gb300.engine import Engine
    from paper_2605_20600_gb300.runner import generate

    class Fake:
        cfg = cfg_of(H)                    # E = 16, N = 64
        device = torch.device("cpu")

        def __init__(self, fmt=None):
            self.calls, self.quant = [], None
            if fmt is not None:
                self.quantise(fmt)
                self.calls.clear()

        def stream(self):
            return 0

        def quantise(self, fmt, prompt=None):
            self.calls.append((fmt, prompt))
            self.quant = type("Q", (), {"c": H.hkv_qcache(format=fmt)})

    def run(f, first, **kw):               # no token left: only what comes before the first
        generate(f, None, first_step=first, last_step=first - 1, **kw)
        return f.calls

    for first in (16, 17, 40):
        assert run(Fake(), first, cache_format=4) == [(4, None)]
    assert run(Fake(), 15, cache_format=4) == [] and run(Fake(), 40) == []
    assert run(Fake(8), 40) == [] and run(Fake(8), 40, cache_format=8) == []
    for kw in (dict(cache_format=4), dict(fused=False)):
        with pytest.raises(ValueError):
            run(Fake(8), 40, **kw)
    eng = Engine.__new__(Engine)           # calls that the codes have no form of
    eng.quant = object()
    for call in (lambda: eng.append(0, 1, 1, 1), lambda: eng.attend(0, 1, 1),
                 lambda: eng.step_identify(0, 1, 1, 1, 1)):
        with pytest.raises(H.HkvError) as e:
            call()
        assert e.value.status == H.HKV_ERR_STATE


def test_many_long_heads_are_not_refused(H):
    """Tiles are counted per head: heads times tiles past 31 bits is no fault.
    Without a GPU the call gets as far as asking for the device."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not the device's")
    buf, a, _, quant, _ = caches(H)
    cfg = cfg_of(H, n_seqs=256, n_heads=32, n_image=1 << 23, group_at=1 << 23)
    st = H.lib().hkv_quant_attention(ctypes.byref(cfg), ctypes.byref(quant), 0, a, None, None, a, None, a,
                                     1 << 30, None)
    assert st == H.HKV_ERR_CUDA


def test_updates_that_just_do_not_fit_shared_memory(H):
    """Segments whose work area fits 227 KB only without the kernels' own
    432 bytes: a capacity error, with the longest that fits beside it."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not the device's")
    buf, a, plain, quant, _ = caches(H)
    room = 227 * 1024 - 4 * 64 - 2544

    def cfg(stage, over):              # n_cond = 8; 16 bytes a token
        n = (room - stage) // 16 + over
        return cfg_of(H, n_image=20000, row_len=100, group_at=n - 8)

    for call in (lambda c: H.hkv_quant_evict_all(c, quant), lambda c: H.hkv_quant_evict(c, quant, 0)):
        for over, want in ((0, H.HKV_ERR_CUDA), (1, H.HKV_ERR_CAPACITY), (26, H.HKV_ERR_CAPACITY),
                           (28, H.HKV_ERR_CAPACITY)):   # the first fits, but there is no device
            with pytest.raises(H.HkvError) as e:
                call(cfg(32 * 64 * 8, over))
            assert e.value.status == want, over


def test_pack_without_the_conditioning_rows_wants_lengths_of_its_own(H):
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not the device's")
    buf, a, plain, quant, _ = caches(H)
    cfg, call = cfg_of(H), H.lib().hkv_quant_pack

    def pack(flags, cfg=cfg, **kw):
        q = H.hkv_qcache.from_buffer_copy(quant)
        for k, v in kw.items():
            setattr(q, k, v)
        return call(ctypes.byref(cfg), ctypes.byref(plain), ctypes.byref(q), 0, flags, None)

    assert pack(H.HKV_PACK_SKIP_COND, len=a + 256) == H.HKV_ERR_INVALID_ARG
    assert pack(H.HKV_PACK_SKIP_COND, pos=a + 256) == H.HKV_ERR_INVALID_ARG
    # accepted, up to the launch: own arrays, or no rows left out
    for st in (pack(H.HKV_PACK_SKIP_COND, len=a + 256, pos=a + 512), pack(0),
               pack(H.HKV_PACK_SKIP_COND, cfg=cfg_of(H, n_cond=0))):
        assert st == H.HKV_ERR_CUDA


def test_a_prompt_of_other_heads_than_the_config_is_refused(H):
    """Heads that the prompt does not have would be read past its end."""
    import torch
    buf, a, _, _, _ = caches(H)
    cfg = cfg_of(H)                                       # 4 heads of 64, bf16
    n = torch.zeros(2, dtype=torch.int32)
    for heads, dim, ok in ((4, 64, True), (3, 64, False), (5, 64, False), (4, 128, False), (2, 128, False)):
        k = torch.zeros(2, heads, 10, dim, dtype=torch.bfloat16)
        pre = H.make_prefix(k, k, n)
        assert (H.hkv_prefix_workspace_size(cfg, pre) > 0) == ok
        if not ok:
            with pytest.raises(H.HkvError) as e:
                H.hkv_prefix_attention(cfg, pre, a, a, a, a, 1 << 30)
            assert e.value.status == H.HKV_ERR_SHAPE
