"""Bounded waits of the tcgen05 kernels of attention over states that run out. A
test build of the library (-D HKV_CROSS_TEST_STALL) makes one warp of every CTA
wait, at the second key tile of a query tile, for a barrier that nothing completes
before its limit, shortened to 50 ms (-D HKV_WAIT_TIMEOUT_NS); which warp goes
round with the CTA. The products that were issued are complete by then. The error
word must say HKV_ERR_TIMEOUT, the queries of the stalled query tile must come out
as NaN, all others as NaN or right, and the context must stay usable."""
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
    good_lib = H.LIB_PATH
    g = torch.Generator(device="cuda").manual_seed(0)
    cases = []
    # one and two query tiles a CTA, one range of keys and several, more work than
    # CTAs; fp32 and bf16 parts. Every range has two key tiles at least.
    for dtype, out_dtype, D, S, heads, T, N in (
            ("bf16", "bf16", 64, 2, 4, 128, 300), ("bf16", "bf16", 128, 1, 3, 300, 1300),
            ("bf16", "bf16", 128, 2, 170, 256, 200), ("bf16", "bf16", 64, 1, 320, 100, 300),
            ("fp32", "fp32", 64, 2, 90, 200, 200), ("fp32", "fp32", 128, 1, 2, 40, 700),
            ("bf16", "fp32", 128, 1, 3, 100, 300)):
        cfg = H.make_config(n_layers=1, n_seqs=S, n_heads=heads, head_dim=D, dtype=dtype, n_cond=0,
                            n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                            global_budget=1)
        dt = torch.float32 if dtype == "fp32" else torch.bfloat16
        q = torch.randn(S, T, heads, D, generator=g, device="cuda").to(dt)
        k, v = (torch.randn(S, heads, N, D, generator=g, device="cuda").to(dt) for _ in range(2))
        cases.append((cfg, q, k, v, torch.float32 if out_dtype == "fp32" else torch.bfloat16))

    def run(case):
        cfg, q, k, v, odt = case
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        st, tok = H.make_states(k, v, None, err), H.make_tokens(q.shape[1])
        n = H.hkv_cross_workspace_size(cfg, st, tok)
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        out = torch.full(q.shape, 3.0, dtype=odt, device="cuda")
        lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 3.0, device="cuda")
        H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(out), lse, ws, n)
        torch.cuda.synchronize()
        return out, lse, int(err)

    want = [run(c) for c in cases]
    assert all(e == 0 for _, _, e in want)
    H.LIB_PATH, H._lib = lib_path, None
    for case, (out0, lse0, _) in zip(cases, want):
        out, lse, err = run(case)
        T = case[1].shape[1]
        assert err == H.HKV_ERR_TIMEOUT, case[0].head_dim
        nan = torch.isnan(out).all(-1)
        assert torch.equal(nan, torch.isnan(out).any(-1)), "a row is NaN or not"
        assert torch.equal(nan, torch.isnan(lse).transpose(1, 2)), "with its lse"
        assert nan[:, :min(T, 128)].all(), "the stalled tile, which holds every head's first queries or is all"
        same = (out == out0).all(-1)
        assert (nan | same).all()
    H.LIB_PATH, H._lib = good_lib, None
    for case, (out0, lse0, _) in zip(cases, want):   # the context is still usable
        out, lse, err = run(case)
        assert err == 0 and torch.equal(out, out0) and torch.equal(lse, lse0)
    print("timeout ok")


def test_a_wait_that_runs_out_fails_its_queries(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import build as B
    lib = str(tmp_path / "libheadkv_stall.so")
    B.build(force=True, extra_flags=["-DHKV_CROSS_TEST_STALL", "-DHKV_WAIT_TIMEOUT_NS=50000000ull"],
            lib_path=lib, build_dir=str(tmp_path / "obj"))
    code = (f"import sys; sys.path.insert(0, {ROOT!r}); sys.path.insert(0, {HERE!r}); "
            f"import test_gpu_cross_timeout as t; t._stall_main({lib!r})")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "timeout ok" in r.stdout
