"""Bounded waits that run out in a CTA that has taken over the work of others. In
the test build of test_gpu_cross_timeout.py (one warp waits for what nothing
completes) the work that stalls is one long sequence's, which comes first; behind it
come sequences with queries and no states, whose work needs no products and so is
handed on at once. Whatever a CTA has taken over it has to write, before the wait runs
out or after: every row is NaN or right, with its lse, and none is what it was."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


def _items_main(lib_path):
    import torch
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import hkv as H
    good_lib = H.LIB_PATH
    g = torch.Generator(device="cuda").manual_seed(0)
    cases = []
    # two query tiles a CTA and one, one range of keys and several
    for D, S, heads, T, N in ((128, 16, 24, 300, 330), (64, 24, 40, 256, 330), (128, 24, 40, 100, 330),
                              (64, 32, 40, 60, 450), (64, 10, 12, 200, 4000), (128, 12, 12, 200, 4000),
                              (64, 20, 12, 100, 4000)):
        cfg = H.make_config(n_layers=1, n_seqs=S, n_heads=heads, head_dim=D, dtype="bf16", n_cond=0,
                            n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                            global_budget=1)
        q = torch.randn(S, T, heads, D, generator=g, device="cuda").bfloat16()
        k, v = (torch.randn(S, heads, N, D, generator=g, device="cuda").bfloat16() for _ in range(2))
        klens = torch.zeros(S, dtype=torch.int32, device="cuda")
        klens[S // 2] = N - 7
        cases.append((cfg, q, k, v, klens))

    def run(case):
        cfg, q, k, v, klens = case
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        st, tok = H.make_states(k, v, klens, err), H.make_tokens(q.shape[1])
        n = H.hkv_cross_workspace_size(cfg, st, tok)
        # partial results that a call before might have left: sums that count
        ws = torch.full((n // 4,), 3.0, device="cuda")
        out = torch.full(q.shape, 3.0, dtype=q.dtype, device="cuda")
        lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 3.0, device="cuda")
        H.hkv_cross_attention(cfg, st, tok, H.make_rows(q), H.make_rows(out), lse, ws, n)
        torch.cuda.synchronize()
        return out, lse, int(err)

    want = [run(c) for c in cases]
    assert all(e == 0 for _, _, e in want)
    H.LIB_PATH, H._lib = lib_path, None
    for i, (case, (out0, lse0, _)) in enumerate(zip(cases, want)):
        out, lse, err = run(case)
        assert err == H.HKV_ERR_TIMEOUT, i
        nan = torch.isnan(out).all(-1)
        assert torch.equal(nan, torch.isnan(out).any(-1)) and torch.equal(nan, torch.isnan(lse).transpose(1, 2)), i
        assert not (out == 3.0).all(-1).any() and not (lse == 3.0).any(), (i, int((lse == 3.0).sum()))
        same = (out == out0).all(-1) & (lse == lse0).transpose(1, 2)
        assert (nan | same).all(), (i, int((~(nan | same)).sum()))
        assert nan[case[0].n_seqs // 2].any()
    H.LIB_PATH, H._lib = good_lib, None
    for case, (out0, lse0, _) in zip(cases, want):   # the context is still usable
        out, lse, err = run(case)
        assert err == 0 and torch.equal(out, out0) and torch.equal(lse, lse0)
    print("items ok")


def test_work_that_was_taken_over_is_written(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import build as B
    lib = str(tmp_path / "libheadkv_stall.so")
    B.build(force=True, extra_flags=["-DHKV_CROSS_TEST_STALL", "-DHKV_WAIT_TIMEOUT_NS=50000000ull"],
            lib_path=lib, build_dir=str(tmp_path / "obj"))
    code = (f"import sys; sys.path.insert(0, {ROOT!r}); sys.path.insert(0, {HERE!r}); "
            f"import test_gpu_cross_timeout_items as t; t._items_main({lib!r})")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "items ok" in r.stdout
