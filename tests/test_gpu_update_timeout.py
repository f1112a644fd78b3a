"""A bounded wait of the periodic update that runs out. A test build of the
library (-D HKV_UPD_TEST_STALL) makes one warp of every global head's CTA wait,
after the buffered queries have arrived, for a barrier phase that nothing
completes, with the limit shortened to 50 ms (-D HKV_WAIT_TIMEOUT_NS); which
warp goes round with the heads. Such a head must be left exactly as it is, the
local heads must be updated as ever, and the error word must say
HKV_ERR_TIMEOUT, for plain and quantised caches."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def _stall_main(lib_path):
    import torch
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import CacheBuffers, QuantCacheBuffers
    H.LIB_PATH = lib_path
    C, P, w, B, D, n = 5, 8, 16, 40, 64, 16
    cfg = H.make_config(n_layers=1, n_seqs=1, n_heads=n, head_dim=D, dtype="bf16", n_cond=C, n_image=200,
                        row_len=1, recent_w=w, local_w=w, period=P, group_at=100, global_budget=B)
    cap, ntok = C + B + P, 120
    q = torch.randn(n, D, device="cuda").bfloat16()
    glob = torch.arange(n, device="cuda") % 4 != 3

    def cache(plain):
        g = torch.Generator(device="cuda").manual_seed(0)
        c = CacheBuffers(cfg, n * cap, "cuda")
        c.k.normal_(generator=g)
        c.v.normal_(generator=g)
        c.qbuf.normal_(generator=g)
        c.off.copy_(torch.arange(n) * cap)
        c.cap.fill_(cap)
        c.label.copy_(glob)                       # HKV_GLOBAL = 1, HKV_LOCAL = 0
        c.len.fill_(cap)
        c.nbuf.fill_(P)
        c.ntok.fill_(ntok)
        img = torch.cat([torch.arange(B + P - w) * 2, torch.arange(ntok - w, ntok)]) + C
        c.pos.copy_(torch.cat([torch.arange(C), img]).repeat(n))
        if plain:
            return c
        x = QuantCacheBuffers(cfg, 8, n * cap, "cuda", qbuf=c.qbuf, label=c.label, off=c.off, cap=c.cap)
        H.hkv_quant_pack(cfg, c.c, x.c, 0)
        return x

    for plain, call in ((True, lambda c: H.hkv_evict(cfg, c.c, 0)), (True, lambda c: H.hkv_evict_all(cfg, c.c)),
                        (True, lambda c: H.hkv_append_evict(cfg, c.c, 0, q, q, q)),
                        (False, lambda c: H.hkv_quant_evict(cfg, c.c, 0)),
                        (False, lambda c: H.hkv_quant_evict_all(cfg, c.c))):
        c = cache(plain)
        arrays = [c.k, c.v, c.pos] + ([] if plain else [c.ks, c.vs])
        before = [x.clone() for x in arrays]
        counters = [x.clone() for x in (c.len, c.nbuf, c.ntok)]
        ring = c.qbuf.clone()
        call(c)
        with pytest.raises(H.HkvError) as e:
            (H.hkv_check if plain else H.hkv_quant_check)(c.c)
        assert e.value.status == H.HKV_ERR_TIMEOUT
        rows = glob.repeat_interleave(cap)
        for x, y in zip(arrays, before):
            assert torch.equal(x[rows], y[rows])
        for x, y in zip((c.len, c.nbuf, c.ntok), counters):
            assert torch.equal(x[glob], y[glob])
        assert torch.equal(c.qbuf[glob], ring[glob])
        assert bool((c.len[~glob] <= C + w + 1).all()) and bool((c.nbuf[~glob] <= 1).all())

    # the first update, out of place from the uncompressed cache
    dense = cache(True)
    ragged = CacheBuffers(cfg, n * cap, "cuda", qbuf=dense.qbuf, label=dense.label.clone(), off=dense.off,
                          cap=dense.cap)
    dense.label.fill_(H.HKV_DENSE)
    ragged.len.fill_(3)
    H.hkv_repack(cfg, dense.c, ragged.c, 0)
    with pytest.raises(H.HkvError) as e:
        H.hkv_check(ragged.c)
    assert e.value.status == H.HKV_ERR_TIMEOUT
    assert bool((ragged.len[glob] == 3).all()) and bool((ragged.len[~glob] == C + w).all())
    # the context is still usable
    x = torch.arange(1000, device="cuda", dtype=torch.float32)
    assert float(x.sum().item()) == 499500.0
    print("timeout ok")


def test_an_update_whose_wait_runs_out_leaves_the_head_alone(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import build as B
    lib = str(tmp_path / "libheadkv_stall.so")
    B.build(force=True, extra_flags=["-DHKV_UPD_TEST_STALL", "-DHKV_WAIT_TIMEOUT_NS=50000000ull"],
            lib_path=lib, build_dir=str(tmp_path / "obj"))
    code = (f"import sys; sys.path.insert(0, {ROOT!r}); sys.path.insert(0, {HERE!r}); "
            f"import test_gpu_update_timeout as t; t._stall_main({lib!r})")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "timeout ok" in r.stdout
