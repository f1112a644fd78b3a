"""A bounded wait of the shared-prompt kernel on tcgen05 that runs out. A test
build of the library (-D HKV_PREFIX_TEST_STALL) makes one warp of every CTA
wait, at the second tile of its keys, for a barrier that nothing arrives at,
with the limit shortened to 50 ms (-D HKV_WAIT_TIMEOUT_NS); which warp goes
round with the CTA. The products themselves are complete by then. Every query
of such a CTA must come out as NaN, in every row and channel, and the error
word must say HKV_ERR_TIMEOUT, leaving the context usable."""
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
    H.LIB_PATH = lib_path
    g = torch.Generator(device="cuda").manual_seed(0)
    # up to 64 queries and more of them; one range of keys and several. Ranges
    # of one tile do not stall, so every prompt has two tiles a range at least.
    for D, seqs, heads, T, splits in ((64, 40, 160, 300, False), (128, 64, 20, 1025, True),
                                      (128, 100, 160, 130, False), (64, 128, 20, 1500, True)):
        cfg = H.make_config(n_layers=1, n_seqs=seqs, n_heads=heads, head_dim=D, dtype="bf16",
                            n_cond=0, n_image=8, row_len=1, recent_w=1, local_w=1, period=1,
                            group_at=8, global_budget=1)
        k, v, q = (torch.randn(*s, D, generator=g, device="cuda").bfloat16()
                   for s in ((1, heads, T), (1, heads, T), (seqs, heads)))
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        pre = H.make_prefix(k, v, torch.tensor([T], dtype=torch.int32, device="cuda"), err)
        n = H.hkv_prefix_workspace_size(cfg, pre)
        assert (n > 256) == splits
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        out = torch.full((seqs, heads, D), 3.0, device="cuda")
        lse = torch.full((seqs, heads), 3.0, device="cuda")
        H.hkv_prefix_attention(cfg, pre, q, out, lse, ws, n)
        torch.cuda.synchronize()
        assert int(err) == H.HKV_ERR_TIMEOUT, (D, seqs)
        assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all()), (D, seqs)
    # the context is still usable
    x = torch.arange(1000, device="cuda", dtype=torch.float32)
    assert float(x.sum().item()) == 499500.0
    print("timeout ok")


def test_a_wait_that_runs_out_in_one_warp_fails_the_whole_cta(tmp_path):
    sys.path.insert(0, ROOT)
    from paper_2605_20600_gb300 import build as B
    lib = str(tmp_path / "libheadkv_stall.so")
    B.build(force=True, extra_flags=["-DHKV_PREFIX_TEST_STALL", "-DHKV_WAIT_TIMEOUT_NS=50000000ull"],
            lib_path=lib, build_dir=str(tmp_path / "obj"))
    code = (f"import sys; sys.path.insert(0, {ROOT!r}); sys.path.insert(0, {HERE!r}); "
            f"import test_gpu_prefix_timeout as t; t._stall_main({lib!r})")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "timeout ok" in r.stdout
