"""The serving cache on the GPU: rows in 8 and 4 bits written, read back,
attended over and trimmed, and attention over shared prompts, each against the
fp64 oracle (oracle/serve.py, oracle/headkv.py).

Tolerances. A logit x = sum q_i k_i / sqrt(D) is off by at most 2^-19 A with
A = sum |q_i k_i| / sqrt(D): operands in two 11-bit parts (2^-22) and at most
D / 16 = 8 chained sums whose rounding may truncate (8 x 2^-23). Weights off
by eps each move an output by at most 2 eps max|v|, and the sums over the
rows add 2^-19 max|v| (at most 16 chained sums between fp32 additions, and the
base-2 exponential's 2 ulp). Codes, scales, positions and counters are exact.
"""
import math

import numpy as np
import pytest

from oracle import headkv as O
from oracle import serve as S
from synth import configs, gen

from _gpu_util import cfg_of, flat

pytestmark = pytest.mark.gpu

FMT = [8, 4]


def tolerances(q, K, V):
    A = float((np.abs(K) @ np.abs(q)).max()) / math.sqrt(q.shape[0]) if len(K) else 0.0
    eps = 2.0 ** -19 * A
    vmax = float(np.abs(V).max()) if len(V) else 0.0
    return (2 * eps + 2.0 ** -19) * vmax, eps + 2.0 ** -20 * 8


def to_torch(x, dtype, device="cuda"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(
        torch.bfloat16 if dtype == "bf16" else torch.float32).to(device)


def rounded(x, dtype):
    return gen.round_bf16(np.asarray(x, np.float32)) if dtype == "bf16" else np.asarray(x, np.float32)


class QCache:
    """A quantised cache with heads of given lengths; rows past a head's
    length hold NaN scales and arbitrary codes."""

    def __init__(self, lens, D, bits, dtype, seed=0, slack=3, period=4, label=255, n_seqs=1,
                 max_len=None, lead=0):
        import torch
        from paper_2605_20600_gb300 import hkv as H
        rng = np.random.default_rng(seed)
        self.H, self.D, self.bits, self.dtype = H, D, bits, dtype
        self.lens = np.asarray(lens, dtype=np.int64)
        n = self.lens.size
        self.n = n
        caps = self.lens + slack
        self.off = lead + np.cumsum(caps) - caps
        tokens = int(lead + caps.sum())
        self.tokens = tokens
        most = int(max_len or caps.max() + 1)
        self.cfg = H.make_config(n_layers=1, n_seqs=n_seqs, n_heads=n // n_seqs, head_dim=D,
                                 dtype=dtype, n_cond=0, n_image=most + period, row_len=1, recent_w=1,
                                 local_w=1, period=period, group_at=max(most, period),
                                 global_budget=1)
        gain = np.exp(0.7 * rng.normal(size=D))
        self.k_codes, self.k_scales = S.quantise(rng.normal(size=(tokens, D)) * gain, bits)
        self.v_codes, self.v_scales = S.quantise(rng.normal(size=(tokens, D)), bits)
        live = np.zeros(tokens, bool)
        for o, ln in zip(self.off, self.lens):
            live[o:o + ln] = True
        ks, vs = self.k_scales.copy(), self.v_scales.copy()
        ks[~live] = np.nan
        vs[~live] = np.nan
        dev = "cuda"
        self.ck = torch.from_numpy(S.packed(self.k_codes, bits)).to(dev)
        self.cv = torch.from_numpy(S.packed(self.v_codes, bits)).to(dev)
        self.sk, self.sv = to_torch(ks, "bf16"), to_torch(vs, "bf16")
        self.pos = torch.full((tokens,), -7, dtype=torch.int32, device=dev)
        self.toff = torch.from_numpy(self.off).to(dev)
        self.cap = torch.from_numpy(caps.astype(np.int32)).to(dev)
        self.len = torch.from_numpy(self.lens.astype(np.int32)).to(dev)
        self.nbuf = torch.zeros(n, dtype=torch.int32, device=dev)
        self.ntok = torch.from_numpy(self.lens.astype(np.int32)).to(dev)
        self.label = torch.full((n,), label, dtype=torch.uint8, device=dev)
        self.qbuf = torch.zeros(n, period, D, device=dev,
                                dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)
        self.c = H.make_qcache(bits, self.ck, self.cv, self.sk, self.sv, self.pos, self.toff, self.cap,
                               self.len, self.nbuf, self.ntok, self.label, self.qbuf, self.err, tokens)
        self.ws_bytes = H.hkv_quant_workspace_size(self.cfg)
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=dev)
        self.q = rounded(rng.normal(size=(n, D)) * 1.5, dtype)
        self.k_new = rounded(rng.normal(size=(n, D)) * gain, dtype)
        self.v_new = rounded(rng.normal(size=(n, D)), dtype)

    def rows(self, h, step=False):
        a = slice(self.off[h], self.off[h] + self.lens[h])
        K = S.values(self.k_codes[a], self.k_scales[a])
        V = S.values(self.v_codes[a], self.v_scales[a])
        if step:
            K = np.concatenate([K, S.stored(self.k_new[h:h + 1], self.bits)])
            V = np.concatenate([V, S.stored(self.v_new[h:h + 1], self.bits)])
        return K, V


def joined(o1, l1, o2, l2):
    both = np.logaddexp(l1, l2)
    if both == -np.inf:
        return np.zeros_like(o1), both
    return math.exp(l1 - both) * o1 + math.exp(l2 - both) * o2, both


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300, 511, 513, 1000,
        1025, 2049]


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("prior", [False, True])
def test_attention_over_codes(bits, D, dtype, prior):
    import torch
    c = QCache(LENS, D, bits, dtype, seed=1 + bits + D, lead=5)
    H, rng = c.H, np.random.default_rng(99)
    q = to_torch(c.q, dtype)
    out = torch.full((c.n, D), -1.0, device="cuda")
    lse = torch.full((c.n,), -1.0, device="cuda")
    pr = None
    if prior:
        po = rng.normal(size=(c.n, D)).astype(np.float32)
        pl = (rng.normal(size=c.n) * 4).astype(np.float32)
        pl[[0, 3, 7]] = -np.inf       # an empty prior: its outputs are not looked at
        po[[0, 3, 7]] = np.nan
        pr = (to_torch(po, "fp32"), to_torch(pl, "fp32"))
    for _ in range(2):                # the workspace is left ready for the next call
        H.hkv_quant_attention(c.cfg, c.c, 0, q, out, c.ws, c.ws_bytes, prior=pr, lse=lse)
    H.hkv_quant_check(c.c)
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    for h in range(c.n):
        K, V = c.rows(h)
        o, l = S.attention_lse(c.q[h], K, V)
        to, tl = tolerances(c.q[h], K, V)
        if prior:
            if pl[h] != -np.inf:
                to += 2.0 ** -19 * np.abs(po[h]).max() + 2 * tl * np.abs(po[h]).max()
                o, l = joined(o, l, po[h].astype(np.float64), float(pl[h]))
        assert np.abs(got[h] - o).max() <= to, (h, c.lens[h], np.abs(got[h] - o).max(), to)
        assert gl[h] == l or abs(gl[h] - l) <= tl, (h, gl[h], l, tl)
    assert int(c.ws[:4 * (c.n + 2)].sum()) == 0


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("label", [255, 0])
def test_step_appends_and_attends(bits, D, dtype, label):
    import torch
    c = QCache(LENS, D, bits, dtype, seed=5 + bits + D, label=label)
    H = c.H
    before = [x.clone() for x in (c.ck, c.cv, c.sk, c.sv)]
    q, k, v = (to_torch(x, dtype) for x in (c.q, c.k_new, c.v_new))
    out = torch.empty(c.n, D, device="cuda")
    lse = torch.empty(c.n, device="cuda")
    H.hkv_quant_step(c.cfg, c.c, 0, q, k, v, out, c.ws, c.ws_bytes, lse=lse)
    H.hkv_quant_check(c.c)
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    rows = c.off + c.lens
    for x, codes, scales in ((c.k_new, c.ck, c.sk), (c.v_new, c.cv, c.sv)):
        cc, ss = S.quantise(x, bits)
        assert np.array_equal(codes.cpu().numpy()[rows], S.packed(cc, bits))
        assert np.array_equal(scales.float().cpu().numpy()[rows], ss)
    other = np.setdiff1d(np.arange(c.tokens), rows)
    for a, b in zip(before, (c.ck, c.cv, c.sk, c.sv)):   # nothing else moved
        assert torch.equal(a.view(torch.uint8)[other], b.view(torch.uint8)[other])
    assert np.array_equal(c.len.cpu().numpy(), c.lens + 1)
    assert np.array_equal(c.ntok.cpu().numpy(), c.lens + 1)
    assert np.array_equal(c.nbuf.cpu().numpy(), np.full(c.n, 0 if label == 255 else 1))
    pos = c.pos.cpu().numpy()
    assert np.array_equal(pos[rows], c.lens) and (pos[other] == -7).all()
    ring = c.qbuf.float().cpu().numpy()
    for h in range(c.n):
        assert np.array_equal(ring[h, c.lens[h] % 4], c.q[h])
        K, V = c.rows(h, step=True)
        o, l = S.attention_lse(c.q[h], K, V)
        to, tl = tolerances(c.q[h], K, V)
        assert np.abs(got[h] - o).max() <= to, (h, np.abs(got[h] - o).max(), to)
        assert abs(gl[h] - l) <= tl


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[40003], [20000, 3, 256, 0, 257, 9000]])
def test_long_heads_cut_into_many_parts(bits, D, lens):
    """Heads cut between CTAs, next to heads too short for it: attention, then
    steps over one workspace, each bit-identical when it is run again."""
    import torch
    c = QCache(lens, D, bits, "bf16", seed=31 + bits + D, lead=3)
    H = c.H
    q, k, v = (to_torch(x, "bf16") for x in (c.q, c.k_new, c.v_new))
    outs = [torch.full((c.n, D), -1.0, device="cuda") for _ in range(2)]
    for o in outs:
        H.hkv_quant_attention(c.cfg, c.c, 0, q, o, c.ws, c.ws_bytes)
    assert torch.equal(*outs)
    state = (c.ck, c.cv, c.sk, c.sv, c.pos, c.len, c.nbuf, c.ntok, c.qbuf)
    before = [x.clone() for x in state]
    steps = []
    for o in outs:
        for x, b in zip(state, before):
            x.copy_(b)
        H.hkv_quant_step(c.cfg, c.c, 0, q, k, v, o, c.ws, c.ws_bytes)
        steps.append([x.clone().view(torch.uint8) for x in state])
    H.hkv_quant_check(c.c)
    assert torch.equal(*outs) and all(torch.equal(a, b) for a, b in zip(*steps))
    assert np.array_equal(c.len.cpu().numpy(), c.lens + 1)
    got = outs[0].cpu().numpy()
    for h in range(c.n):
        K, V = c.rows(h, step=True)
        o, _ = S.attention_lse(c.q[h], K, V)
        to, _ = tolerances(c.q[h], K, V)
        assert np.abs(got[h] - o).max() <= to, (h, np.abs(got[h] - o).max(), to)
    assert int(c.ws[:4 * c.n].sum()) == 0


@pytest.mark.parametrize("bits", FMT)
def test_every_bf16_quotient_rounds_as_defined(bits):
    """Groups whose largest value has each bf16 significand, holding every bf16
    value from it down to where all codes are 0, both signs: exact codes."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import QuantCacheBuffers
    D, M = 128, 127 if bits == 8 else 7
    steps = int(math.ceil(math.log2(4 * M)))
    groups = []
    for i in range(128):
        top = 1 + i / 128
        x = np.array([(1 + j / 128) * 2.0 ** -e for e in range(steps) for j in range(128)])
        x = x[x <= top]
        x = np.concatenate([x, -x])
        x = np.concatenate([x, np.zeros(-len(x) % 31)]).reshape(-1, 31)
        groups.append(np.concatenate([np.full((len(x), 1), top), x], 1))
    g = np.concatenate(groups)
    g = np.concatenate([g, np.zeros((-len(g) % 4, 32))]).reshape(-1, D).astype(np.float32)
    v = g[::-1].copy()
    n = len(g)
    cfg = H.make_config(n_layers=1, n_seqs=1, n_heads=1, head_dim=D, dtype="bf16", n_cond=0,
                        n_image=n, row_len=1, recent_w=1, local_w=1, period=1, group_at=n,
                        global_budget=1)
    src = plain_cache(H, cfg, [n], [n], "bf16", g, v)
    dst = QuantCacheBuffers(cfg, bits, n, "cuda", qbuf=src.qbuf, label=src.label, off=src.off,
                            cap=src.cap)
    H.hkv_quant_pack(cfg, src.c, dst.c, 0, 0, 0)
    H.hkv_quant_check(dst.c)
    for x, codes, scales in ((g, dst.k, dst.ks), (v, dst.v, dst.vs)):
        cc, ss = S.quantise(x, bits)
        assert np.array_equal(scales.float().cpu().numpy(), ss)
        assert np.array_equal(codes.cpu().numpy(), S.packed(cc, bits))


def test_step_refuses_per_head_through_the_error_word():
    import torch
    for what, code in (("full", 3), ("buffer", 4), ("outside", 5)):
        c = QCache([40, 41, 300, 7], 64, 8, "bf16", label=1)
        if what == "full":
            c.cap[1] = 41
        elif what == "buffer":
            c.nbuf[1] = 4
        else:
            c.toff[1] = c.tokens
        q, k, v = (to_torch(x, "bf16") for x in (c.q, c.k_new, c.v_new))
        out = torch.full((4, 64), 9.0, device="cuda")
        c.H.hkv_quant_step(c.cfg, c.c, 0, q, k, v, out, c.ws, c.ws_bytes)
        with pytest.raises(c.H.HkvError) as e:
            c.H.hkv_quant_check(c.c)
        assert e.value.status == code
        assert c.len.tolist() == [41, 41, 301, 8] and c.ntok.tolist() == [41, 41, 301, 8]
        got = out.cpu().numpy()
        assert (got[1] == 9.0).all() and (got[[0, 2, 3]] != 9.0).all()


def test_segment_longer_than_the_config_is_a_capacity_error():
    import torch
    c = QCache([40, 2000], 64, 4, "bf16", max_len=100)
    q = to_torch(c.q, "bf16")
    out = torch.full((2, 64), 9.0, device="cuda")
    c.H.hkv_quant_attention(c.cfg, c.c, 0, q, out, c.ws, c.ws_bytes)
    with pytest.raises(c.H.HkvError) as e:
        c.H.hkv_quant_check(c.c)
    assert e.value.status == 3
    assert (out[1] == 9.0).all() and (out[0] != 9.0).all()


@pytest.mark.parametrize("bits", FMT)
def test_attention_with_extreme_rows(bits):
    """Groups of zeros, very large and very small scales, one row that takes
    all the weight, and a NaN row that reaches only its own head."""
    import torch
    D = 128
    c = QCache([70, 70, 70, 70], D, bits, "fp32", seed=3)
    rng = np.random.default_rng(8)
    ks, vs = c.k_scales.copy(), c.v_scales.copy()
    o = c.off
    ks[o[0]:o[0] + 70, 1] = 0.0                                   # a group of zeros
    vs[o[0] + 5:o[0] + 20] = 0.0
    vs[o[1]:o[1] + 70] = S.round_bf16((2.0 ** rng.uniform(-60, 60, size=(70, 4))).astype(np.float32))
    ks[o[2] + 33] = S.round_bf16(np.full(4, 300.0, np.float32))     # a logit far above the others
    vs[o[3] + 69, 2] = np.nan
    for x, t in ((ks, c.sk), (vs, c.sv)):
        for h in range(4):
            t[o[h]:o[h] + 70] = to_torch(x[o[h]:o[h] + 70], "bf16")
    c.k_scales, c.v_scales = ks, vs
    out = torch.empty(4, D, device="cuda")
    c.H.hkv_quant_attention(c.cfg, c.c, 0, to_torch(c.q, "fp32"), out, c.ws, c.ws_bytes)
    got = out.cpu().numpy()
    for h in range(4):
        K, V = c.rows(h)
        if h == 3:
            assert np.isnan(got[h, 64:96]).all()
            keep = np.r_[0:64, 96:128]
            got_h, V = got[h, keep], V[:, keep]
        else:
            got_h = got[h]
        want, _ = S.attention_lse(c.q[h], K, V)
        A = float((np.abs(K) @ np.abs(c.q[h])).max()) / math.sqrt(D)
        # each channel against the largest magnitude of its own group
        vmax = np.repeat(np.abs(V).reshape(70, -1, 32).max((0, 2)), 32)
        assert (np.abs(got_h - want) <= (2 * 2.0 ** -19 * A + 2.0 ** -19) * vmax).all(), h


@pytest.mark.parametrize("bits", FMT)
def test_offsets_past_32_bits(bits):
    """A head whose rows start beyond 2^32 bytes of the arena."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    D, rb = 128, 128 * bits // 8
    lead = (1 << 32) // rb + 11
    c = QCache([77, 301], D, bits, "bf16", seed=4)
    tokens = lead + c.tokens
    big = [torch.empty(tokens, w, dtype=t.dtype, device="cuda")
           for t, w in ((c.ck, rb), (c.cv, rb), (c.sk, 4), (c.sv, 4))]
    for b, t in zip(big, (c.ck, c.cv, c.sk, c.sv)):
        b[lead:] = t
    pos = torch.zeros(tokens, dtype=torch.int32, device="cuda")
    off = c.toff + lead
    qc = H.make_qcache(bits, *big, pos, off, c.cap, c.len, c.nbuf, c.ntok, c.label, c.qbuf, c.err, tokens)
    q, k, v = (to_torch(x, "bf16") for x in (c.q, c.k_new, c.v_new))
    out = torch.empty(2, D, device="cuda")
    H.hkv_quant_step(c.cfg, qc, 0, q, k, v, out, c.ws, c.ws_bytes)
    H.hkv_quant_check(qc)
    for h in range(2):
        K, V = c.rows(h, step=True)
        o, _ = S.attention_lse(c.q[h], K, V)
        assert np.abs(out[h].cpu().numpy() - o).max() <= tolerances(c.q[h], K, V)[0]
        cc, _ = S.quantise(c.k_new[h], bits)
        assert np.array_equal(big[0][lead + int(c.off[h] + c.lens[h])].cpu().numpy(), S.packed(cc, bits))


def plain_cache(H, cfg, lens, caps, dtype, k, v, device="cuda"):
    """CacheBuffers holding rows k, v [tokens, D] (segments back to back)."""
    import torch
    from paper_2605_20600_gb300.engine import CacheBuffers
    cb = CacheBuffers(cfg, int(np.sum(caps)), device)
    cb.k.copy_(to_torch(k, dtype))
    cb.v.copy_(to_torch(v, dtype))
    cb.off.copy_(torch.from_numpy((np.cumsum(caps) - caps).astype(np.int64)))
    cb.cap.copy_(torch.from_numpy(np.asarray(caps, np.int32)))
    cb.len.copy_(torch.from_numpy(np.asarray(lens, np.int32)))
    cb.pos.copy_(torch.arange(int(np.sum(caps)), dtype=torch.int32))
    return cb


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("skip", [0, 5])
def test_pack_and_unpack(bits, D, dtype, skip):
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import CacheBuffers, QuantCacheBuffers
    rng = np.random.default_rng(17)
    lens = np.array([5, 6, 63, 64, 65, 130, 200, 7] if skip else [0, 1, 63, 64, 65, 130, 200, 7])
    caps = lens + 2
    n, tokens = lens.size, int(caps.sum())
    cfg = H.make_config(n_layers=2, n_seqs=2, n_heads=2, head_dim=D, dtype=dtype, n_cond=5,
                        n_image=300, row_len=1, recent_w=1, local_w=1, period=4, group_at=300,
                        global_budget=1)
    k = rounded(rng.normal(size=(tokens, D)) * np.exp(rng.normal(size=D)), dtype)
    v = rounded(rng.normal(size=(tokens, D)), dtype)
    off = np.cumsum(caps) - caps
    # groups of zeros, exact ties, tiny (the scale underflows), huge, infinite, NaN
    r = int(off[5]) + 6
    k[r, :32] = 0.0
    k[r + 1, :32] = rounded(np.arange(32) * 0.5 + 111.5, dtype)
    k[r + 2, :32] = 1e-41 if dtype == "fp32" else 0.0
    k[r + 3, :32] = rounded(np.float32(3e38) * np.linspace(-1, 1, 32), dtype)
    k[r + 4, 3], k[r + 5, 40] = np.inf, np.nan
    k[r + 6, :32] = rounded(np.float32(2.0 ** -126) * np.linspace(-1, 1, 32), dtype)
    src = plain_cache(H, cfg, lens, caps, dtype, k, v)
    src.nbuf.copy_(torch.arange(n))
    src.ntok.copy_(torch.arange(n) + 100)
    qc = QuantCacheBuffers(cfg, bits, tokens, "cuda", qbuf=src.qbuf, label=src.label, off=src.off,
                           cap=src.cap)
    for t in (qc.k, qc.v, qc.ks, qc.vs):
        t.view(torch.uint8).fill_(0x5A)
    H.hkv_quant_pack(cfg, src.c, qc.c, H.HKV_ALL_LAYERS, H.HKV_PACK_SKIP_COND if skip else 0)
    H.hkv_quant_check(qc.c)
    assert np.array_equal(qc.len.cpu().numpy(), lens - skip)
    assert torch.equal(qc.nbuf, src.nbuf) and torch.equal(qc.ntok, src.ntok)
    got = [t.cpu() for t in (qc.k, qc.v, qc.ks, qc.vs, qc.pos)]
    live = np.zeros(tokens, bool)
    for h in range(n):
        o, ln = int(off[h]), int(lens[h]) - skip
        live[o:o + ln] = True
        for x, codes, scales in ((k, got[0], got[2]), (v, got[1], got[3])):
            cc, ss = S.quantise(x[o + skip:o + skip + ln], bits)
            assert np.array_equal(codes[o:o + ln].numpy(), S.packed(cc, bits)), h
            assert np.array_equal(scales[o:o + ln].float().numpy(), ss, equal_nan=True), h
        assert np.array_equal(got[4][o:o + ln].numpy(), np.arange(o, o + ln))
    for t in (qc.k, qc.v, qc.ks, qc.vs):      # rows past a head's length are left alone
        assert (t.view(torch.uint8).cpu().numpy()[~live] == 0x5A).all()
    back = CacheBuffers(cfg, tokens, "cuda", qbuf=src.qbuf, label=src.label, off=src.off, cap=src.cap)
    back.k.fill_(77.0)
    H.hkv_quant_unpack(cfg, qc.c, back.c, H.HKV_ALL_LAYERS)
    H.hkv_check(back.c)
    bk, bv = back.k.float().cpu().numpy(), back.v.float().cpu().numpy()
    assert (bk[~live] == 77.0).all()
    for h in range(n):
        o, ln = int(off[h]), int(lens[h]) - skip
        for x, y in ((k, bk), (v, bv)):
            want = rounded(S.stored(x[o + skip:o + skip + ln], bits).astype(np.float32), dtype)
            assert np.array_equal(y[o:o + ln], want, equal_nan=True), h
    assert torch.equal(back.len, qc.len)
    # one layer alone: the other layer's heads are left alone
    qc.len.fill_(-5)
    H.hkv_quant_pack(cfg, src.c, qc.c, 1, H.HKV_PACK_SKIP_COND if skip else 0)
    assert np.array_equal(qc.len.cpu().numpy(), np.r_[np.full(4, -5), lens[4:] - skip])


def test_pack_reports_heads_that_do_not_fit():
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import QuantCacheBuffers
    cfg = H.make_config(n_layers=1, n_seqs=1, n_heads=3, head_dim=64, dtype="bf16", n_cond=9,
                        n_image=64, row_len=1, recent_w=1, local_w=1, period=4, group_at=64,
                        global_budget=1)
    rows = np.ones((60, 64), np.float32)
    for what, code in (("room", 3), ("cond", 4), ("outside", 5)):
        src = plain_cache(H, cfg, [10, 20, 15], [20, 20, 20], "bf16", rows, rows)
        cap, off = src.cap.clone(), src.off.clone()
        if what == "room":
            cap[1] = 19
        elif what == "cond":
            src.len[1] = 8
        else:
            off[1] = 41
        qc = QuantCacheBuffers(cfg, 8, 60, "cuda", qbuf=src.qbuf, label=src.label, off=off, cap=cap)
        H.hkv_quant_pack(cfg, src.c, qc.c, 0, H.HKV_PACK_SKIP_COND if what == "cond" else 0)
        with pytest.raises(H.HkvError) as e:
            H.hkv_quant_check(qc.c)
        assert e.value.status == code
        want = [1, 0, 6] if what == "cond" else [10, 0, 15]
        assert qc.len.tolist() == want


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D,dtype", [(64, "fp32"), (128, "bf16")])
@pytest.mark.parametrize("r_s,distance", [(0.5, 0), (0.0, 0), (1.0, 0), (0.5, 1)])
def test_update_of_codes(bits, D, dtype, r_s, distance):
    """Evicted rows as the oracle's update chooses them from what the rows
    stand for; survivors keep their codes and scales; heads whose buffer is
    not full, and uncompressed heads, are left alone."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import QuantCacheBuffers
    C, P, w, B, N, rl = 7, 12, 16, 60, 400, 20
    cfg = H.make_config(n_layers=2, n_seqs=1, n_heads=6, head_dim=D, dtype=dtype, n_cond=C, n_image=N,
                        row_len=rl, recent_w=w, local_w=w, period=P, group_at=40, global_budget=B,
                        r_s=r_s, distance_mode=distance)
    hp = O.HeadParams(n_cond=C, n_image=N, recent_w=w, local_w=w, period=P, group_at=40,
                      global_budget=B, tau=0.9, r_s=r_s, row_len=rl,
                      distance=O.GRID2D if distance else O.RASTER)
    rng = np.random.default_rng(bits + D)
    label = np.array([1, 1, 0, 255, 1, 0, 1, 1, 1, 0, 1, 1])
    hist = np.array([B - w + P, B - w + 3, 20, 30, B - w + P, 0, B - w + P, 5, B - w + 1, 44, B - w + P,
                     B - w + P])
    nbuf = np.array([P, P, P, P, P - 1, P, P, P, P, P, P, P])
    n = 12
    ln = C + hist + w
    caps = C + np.where(label == 0, w, B) + P
    caps = np.maximum(caps, ln)              # the local and dense heads of this test hold more
    caps[label == 1] = C + B + P
    tokens = int(caps.sum())
    off = np.cumsum(caps) - caps
    ntok = rng.integers(N // 2, N, size=n)
    k = rng.normal(size=(tokens, D)).astype(np.float32)
    k[off[10]:off[10] + ln[10]] = k[off[10]]          # equal scores: the older goes first
    v = rng.normal(size=(tokens, D)).astype(np.float32)
    kc, ks = S.quantise(k, bits)
    vc, vs = S.quantise(v, bits)
    pos = np.zeros(tokens, np.int32)
    for h in range(n):
        img = np.sort(rng.choice(ntok[h] - w, size=hist[h], replace=False))
        p = np.r_[np.arange(C), C + img, C + np.arange(ntok[h] - w, ntok[h])]
        tail = p[C:].copy()
        rng.shuffle(tail)                              # storage order is not position order
        pos[off[h]:off[h] + ln[h]] = np.r_[p[:C], tail]
    ring = rounded(rng.normal(size=(n, P, D)), dtype)
    t = lambda x, d: torch.from_numpy(np.ascontiguousarray(x)).to(d).cuda()  # noqa: E731
    qc = QuantCacheBuffers(cfg, bits, tokens, "cuda", qbuf=to_torch(ring, dtype),
                           label=t(label, torch.uint8), off=t(off, torch.int64), cap=t(caps, torch.int32))
    qc.k.copy_(t(S.packed(kc, bits), torch.uint8))
    qc.v.copy_(t(S.packed(vc, bits), torch.uint8))
    qc.ks.copy_(to_torch(ks, "bf16"))
    qc.vs.copy_(to_torch(vs, "bf16"))
    qc.pos.copy_(t(pos, torch.int32))
    for a, b in ((qc.len, ln), (qc.nbuf, nbuf), (qc.ntok, ntok)):
        a.copy_(t(b, torch.int32))
    H.hkv_quant_evict(cfg, qc.c, 0)
    mid = qc.len.cpu().numpy()
    assert np.array_equal(mid[6:], ln[6:])             # one layer only
    H.hkv_quant_evict_all(cfg, qc.c)
    H.hkv_quant_check(qc.c)
    K, kS, V, vS, ps = (x.float().cpu().numpy() for x in (qc.k, qc.ks, qc.v, qc.vs, qc.pos))
    new_len, new_buf = qc.len.cpu().numpy(), qc.nbuf.cpu().numpy()
    pk, pv, kv = S.packed(kc, bits), S.packed(vc, bits), S.values(kc, ks)
    for h in range(n):
        a = slice(off[h], off[h] + ln[h])
        row_of = {int(p): off[h] + j for j, p in enumerate(pos[a])}
        if label[h] == 255 or nbuf[h] < P:
            want = np.sort(pos[a])
            assert new_buf[h] == nbuf[h]
        else:
            keys = np.zeros((C + N, D), np.float32)
            for p, r in row_of.items():
                keys[p] = kv[r]
            # the ring in the order of its tokens
            q = np.zeros((N, D), np.float32)
            for tt in range(ntok[h] - P, ntok[h]):
                q[tt] = ring[h, tt % P]
            want = np.sort(O.cache_update(np.sort(pos[a]).astype(np.int64), int(label[h]), hp, q, keys,
                                          int(ntok[h]) - 1).pos)
            assert new_buf[h] == 0
        b = slice(off[h], off[h] + new_len[h])
        assert np.array_equal(np.sort(ps[b]), want), h
        src = np.array([row_of[int(p)] for p in ps[b]])
        for got, ref in ((K, pk), (V, pv), (kS, ks), (vS, vs)):
            assert np.array_equal(got[b], ref[src]), h


def prefix_rows(rng, G, Hh, T, D, dtype, layout):
    """k, v [G][H][T][D] views over memory of the given layout."""
    import torch
    gain = np.exp(0.5 * rng.normal(size=D))
    k = to_torch(rounded(rng.normal(size=(G, Hh, T, D)) * gain, dtype), dtype)
    v = to_torch(rounded(rng.normal(size=(G, Hh, T, D)), dtype), dtype)
    if layout == "thd":              # [G][T][H][D]
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    elif layout == "padded":         # rows 16 bytes apart from packed, offset base
        pad = 16 // k.element_size()
        def spread(x):
            y = torch.full((G, Hh, T + 1, D + pad), float("nan"), dtype=x.dtype, device="cuda")
            z = y[:, :, 1:, :D]
            z.copy_(x)
            return z
        k, v = spread(k), spread(v)
    return k, v


def check_prefix(D, dtype, G, seqs, T, lens, layout, Hh):
    import torch
    from paper_2605_20600_gb300 import hkv as H
    rng = np.random.default_rng(D + T + seqs)
    cfg = H.make_config(n_layers=1, n_seqs=G * seqs, n_heads=Hh, head_dim=D, dtype=dtype, n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k, v = prefix_rows(rng, G, Hh, T, D, dtype, layout)
    for g, ln in enumerate(lens):       # rows past a prompt's length are not looked at
        k[g, :, ln:], v[g, :, ln:] = float("nan"), float("nan")
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    pre = H.make_prefix(k, v, ln, err)
    q = rounded(rng.normal(size=(G * seqs, Hh, D)) * 1.5, dtype)
    ws = torch.zeros(H.hkv_prefix_workspace_size(cfg, pre), dtype=torch.uint8, device="cuda")
    out = torch.full((G * seqs, Hh, D), 3.0, device="cuda")
    lse = torch.full((G * seqs, Hh), 3.0, device="cuda")
    for _ in range(2):
        H.hkv_prefix_attention(cfg, pre, to_torch(q, dtype), out, lse, ws, ws.numel())
    torch.cuda.synchronize()
    assert int(err) == 0
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    kf, vf = k.float().cpu().numpy(), v.float().cpu().numpy()
    for s in range(G * seqs):
        g = s // seqs
        for h in range(Hh):
            K, V = kf[g, h, :lens[g]], vf[g, h, :lens[g]]
            o, l = S.attention_lse(q[s, h], K, V)
            to, tl = tolerances(q[s, h], K, V)
            assert np.abs(got[s, h] - o).max() <= to, (s, h, np.abs(got[s, h] - o).max(), to)
            assert gl[s, h] == l or abs(gl[s, h] - l) <= tl, (s, h)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (64, "fp32"), (128, "fp32")])
@pytest.mark.parametrize("G,seqs,T,lens,layout", [
    (1, 1, 1, [1], "htd"), (1, 3, 17, [17], "thd"), (1, 16, 64, [64], "padded"),
    (2, 9, 130, [130, 0], "htd"), (3, 17, 333, [200, 333, 1], "thd"), (1, 40, 1025, [1025], "htd"),
    (2, 70, 257, [255, 256], "padded"), (1, 130, 500, [463], "thd")])
def test_prefix_attention(D, dtype, G, seqs, T, lens, layout):
    check_prefix(D, dtype, G, seqs, T, lens, layout, 3)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,seqs,T,lens,layout,heads", [
    (2, 40, 333, [200, 333], "thd", 20), (1, 64, 1025, [1025], "padded", 10),
    (1, 130, 500, [463], "thd", 10), (3, 70, 257, [255, 0, 256], "htd", 12),
    (1, 17, 2049, [2049], "htd", 10)])
def test_prefix_attention_of_large_batches(D, G, seqs, T, lens, layout, heads):
    check_prefix(D, "bf16", G, seqs, T, lens, layout, heads)


def test_prefix_length_out_of_range():
    import torch
    from paper_2605_20600_gb300 import hkv as H
    cfg = H.make_config(n_layers=1, n_seqs=4, n_heads=2, head_dim=64, dtype="bf16", n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k = torch.ones(2, 2, 50, 64, dtype=torch.bfloat16, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    pre = H.make_prefix(k, k, torch.tensor([50, 51], dtype=torch.int32, device="cuda"), err)
    ws = torch.zeros(H.hkv_prefix_workspace_size(cfg, pre), dtype=torch.uint8, device="cuda")
    q = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, 2, device="cuda")
    H.hkv_prefix_attention(cfg, pre, q, out, lse, ws, ws.numel())
    torch.cuda.synchronize()
    assert int(err) == H.HKV_ERR_BOUNDS
    assert torch.isnan(out[2:]).all() and torch.isnan(lse[2:]).all()
    assert torch.allclose(out[:2], torch.ones_like(out[:2]))


class SharedPrompt:
    """DeviceSynth whose conditioning tokens are sequence 0's for everyone."""

    def __init__(self, w):
        from synth.gpu import DeviceSynth
        self.base = DeviceSynth(w, "cuda")
        self.image = self.base.image

    def cond(self, kc, vc, layer, stream):
        self.base.cond(kc, vc, layer, stream)
        kc.copy_(kc[:1].expand_as(kc))
        vc.copy_(vc[:1].expand_as(vc))


@pytest.mark.parametrize("bits,shared,name", [(8, False, "tiny"), (8, True, "tiny"), (4, False, "tiny"),
                                              (4, True, "tiny"), (8, True, "janus_pro_7b"),
                                              (4, False, "llamagen_xl")])
def test_generation_with_a_quantised_cache(bits, shared, name):
    """A whole generation: plain until the grouping token, then on codes, the
    shared conditioning tokens in a prompt; outputs and retained positions as
    the oracle's, step by step."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import Engine
    from paper_2605_20600_gb300.runner import generate
    from synth.gpu import DeviceSynth
    w = configs.ALL[name].with_(n_seqs=2, n_layers=min(2, configs.ALL[name].n_layers), n_heads=8)
    if name != "tiny":
        w = w.with_(beta_fixed=(4.0, 4.0, 0.3, 4.0, 0.3, 0.3, 0.3, 4.0))
    eng = Engine(cfg_of(H, w), "cuda")
    E, N = w.group_at, w.n_image
    steps = sorted({0, E - 1, E, E + 1, E + w.period - 1, E + w.period, E + 3 * w.period + 1, N - 1})
    got = {}
    generate(eng, (SharedPrompt if shared else lambda x: DeviceSynth(x, "cuda"))(w),
             on_step=lambda t, out: got.__setitem__(t, out.cpu().numpy()) if t in steps else None,
             cache_format=bits, shared_prompt=shared)
    eng.check()
    labels = eng.labels.cpu().numpy()
    off, ln = eng.quant.off.cpu().numpy(), eng.quant.len.cpu().numpy()
    pos = eng.quant.pos.cpu().numpy()
    hp = O.HeadParams.of(w)
    C = w.n_cond
    heads = [(s, l, h) for s in range(2) for l in range(w.n_layers) for h in (0, 2, 5, 7)]
    for s, l, h in heads:
        hi = gen.HeadInputs(w, s, l, h)
        k, v = hi.k.copy(), hi.v.copy()
        if shared:
            first = gen.HeadInputs(w, 0, l, h)
            k[:C], v[:C] = first.k[:C], first.v[:C]
        i = flat(w, s, l, h)
        outs, want_pos = S.run_head_stored(hp, hi.q, k, v, bits, int(labels[i]), steps, plain_cond=shared)
        p = np.sort(pos[off[i]:off[i] + ln[i]]) + (C if shared else 0)
        assert np.array_equal(p, want_pos[want_pos >= C] if shared else want_pos), (s, l, h)
        for t in steps:
            to = 2e-3 if t < E and w.dtype == "bf16" else tolerances(hi.q[t], k[:C + t + 1], v[:C + t + 1])[0]
            assert np.abs(got[t][l, s, h] - outs[t]).max() <= 2 * to, (s, l, h, t)


def test_steps_in_a_graph_on_a_side_stream():
    """Prompt attention and steps of two layers captured once and replayed:
    the same cache and outputs as eager calls."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    D, n = 128, 8
    res = []
    for graph in (False, True):
        c = QCache([300, 1, 64, 900, 0, 17, 511, 40] * 2, D, 8, "bf16", seed=2, n_seqs=4, slack=6)
        c.cfg.n_layers, c.cfg.n_heads = 2, 2
        ws_bytes = H.hkv_quant_workspace_size(c.cfg)
        ws = torch.zeros(ws_bytes, dtype=torch.uint8, device="cuda")
        rng = np.random.default_rng(0)
        k, v = prefix_rows(rng, 2, 2, 90, D, "bf16", "htd")
        pre = H.make_prefix(k, v, torch.tensor([90, 13], dtype=torch.int32, device="cuda"), c.err)
        pws = torch.zeros(H.hkv_prefix_workspace_size(c.cfg, pre), dtype=torch.uint8, device="cuda")
        q, kn, vn = (to_torch(x, "bf16").view(2, n, D) for x in (c.q, c.k_new, c.v_new))
        out = torch.zeros(2, n, D, device="cuda")
        po, pl = torch.zeros(n, D, device="cuda"), torch.zeros(n, device="cuda")

        def token(st):
            for layer in range(2):
                H.hkv_prefix_attention(c.cfg, pre, q[layer], po, pl, pws, pws.numel(), st)
                H.hkv_quant_step(c.cfg, c.c, layer, q[layer], kn[layer], vn[layer], out[layer], ws,
                                 ws_bytes, prior=(po, pl), flags=H.HKV_STEP_PREFETCH, stream=st)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            token(side.cuda_stream)
            if graph:
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=side):
                    token(side.cuda_stream)
                g.replay()
                g.replay()
            else:
                token(side.cuda_stream)
                token(side.cuda_stream)
        side.synchronize()
        H.hkv_quant_check(c.c, side.cuda_stream)
        res.append([out.cpu(), c.len.cpu(), c.ntok.cpu(), c.ck.cpu(), c.cv.cpu()])
    for a, b in zip(*res):
        assert torch.equal(a, b)
    assert np.array_equal(res[0][1].numpy(), c.lens + 3)


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [
    [255], [223], [2000], [40] * 3, [9000, 1], [1, 9000, 1, 0, 33], [31, 32, 33] * 11, [65] * 700,
    [20000, 0, 0, 0, 20000], [0] * 40, [96 * 32 - 1], [12 * 32 - 1], [7 * 32 - 1, 32]])
def test_steps_of_any_split(bits, D, lens):
    """Heads whose tiles are dealt over warps and CTAs in every way: one tile a
    warp, warps without tiles, heads that span many CTAs, many heads a warp.
    Two steps in a row, then the attention alone over the same cache."""
    import torch
    c = QCache(lens, D, bits, "bf16", seed=len(lens) + D)
    H = c.H
    q, k, v = (to_torch(x, "bf16") for x in (c.q, c.k_new, c.v_new))
    out = torch.empty(c.n, D, device="cuda")
    lse = torch.empty(c.n, device="cuda")
    H.hkv_quant_step(c.cfg, c.c, 0, q, k, v, out, c.ws, c.ws_bytes)
    H.hkv_quant_step(c.cfg, c.c, 0, q, k, v, out, c.ws, c.ws_bytes, lse=lse)
    again = torch.empty_like(out)
    H.hkv_quant_attention(c.cfg, c.c, 0, q, again, c.ws, c.ws_bytes)
    H.hkv_quant_check(c.c)
    assert np.array_equal(c.len.cpu().numpy(), c.lens + 2)
    got, gl, ga = out.cpu().numpy(), lse.cpu().numpy(), again.cpu().numpy()
    for h in range(c.n) if c.n <= 50 else range(0, c.n, 37):
        K, V = c.rows(h, step=True)
        K, V = np.concatenate([K, K[-1:]]), np.concatenate([V, V[-1:]])
        o, l = S.attention_lse(c.q[h], K, V)
        to, tl = tolerances(c.q[h], K, V)
        assert np.abs(got[h] - o).max() <= to and abs(gl[h] - l) <= tl, h
        assert np.abs(ga[h] - o).max() <= to, h
    assert int(c.ws[:4 * (c.n + 2)].sum()) == 0


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n,most", [(330, 611), (700, 301), (200, 1100)])
def test_steps_of_many_uneven_heads(bits, D, n, most):
    test_steps_of_any_split(bits, D, [53 * i % most for i in range(n)])


def test_prompts_between_products_of_a_library():
    """Prompt attention on tcgen05 in a row with bf16 products that may hold
    tensor memory of their own, eager and in a graph: nothing waits for
    anything for good, and the results stay the same."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    D, Hh, seqs, T = 128, 12, 64, 700
    rng = np.random.default_rng(3)
    cfg = H.make_config(n_layers=1, n_seqs=seqs, n_heads=Hh, head_dim=D, dtype="bf16", n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k, v = prefix_rows(rng, 1, Hh, T, D, "bf16", "htd")
    pre = H.make_prefix(k, v, torch.tensor([T], dtype=torch.int32, device="cuda"))
    ws = torch.zeros(H.hkv_prefix_workspace_size(cfg, pre), dtype=torch.uint8, device="cuda")
    q = to_torch(rng.normal(size=(seqs, Hh, D)), "bf16")
    a = to_torch(rng.normal(size=(2048, 2048)), "bf16")
    outs = [torch.zeros(seqs, Hh, D, device="cuda") for _ in range(4)]
    lse = torch.zeros(seqs, Hh, device="cuda")

    def row(st):
        prods = []
        for o in outs:
            prods.append(a @ a)
            H.hkv_prefix_attention(cfg, pre, q, o, lse, ws, ws.numel(), st)
        return prods

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(5):
            prods = row(side.cuda_stream)
        side.synchronize()
        want, prod = outs[0].clone(), prods[0].clone()
        for x in outs:
            assert torch.equal(x, want)
            x.zero_()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            prods = row(side.cuda_stream)
        for _ in range(5):
            g.replay()
        side.synchronize()
    for x, y in zip(outs, prods):
        assert torch.equal(x, want) and torch.equal(y, prod)
    o, _ = S.attention_lse(q[5, 3].float().cpu().numpy(), k[0, 3].float().cpu().numpy(),
                           v[0, 3].float().cpu().numpy())
    to, _ = tolerances(q[5, 3].float().cpu().numpy(), k[0, 3].float().cpu().numpy(),
                       v[0, 3].float().cpu().numpy())
    assert np.abs(want[5, 3].cpu().numpy() - o).max() <= to


@pytest.mark.parametrize("what", ["head", "strides"])
def test_a_refused_quantisation_leaves_the_plain_cache(what):
    """A head that the pack refuses, or a prompt whose rows the attention does
    not take: the engine keeps its plain rows and goes on with them, and can
    be quantised when the cause is gone."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import Engine
    from paper_2605_20600_gb300.runner import generate
    from synth.gpu import DeviceSynth
    w = configs.TINY
    engines = []
    for refused in (False, True):
        eng = Engine(cfg_of(H, w), "cuda")
        generate(eng, DeviceSynth(w, "cuda"), last_step=w.group_at - 1)
        if refused:
            old, prompt = eng.ragged.len.clone(), None
            if what == "head":
                eng.ragged.len[3] = -1
            else:
                x = torch.zeros(1, 1, w.n_heads, w.n_cond, w.head_dim + 1, device="cuda")
                prompt = (x[..., :-1], x[..., :-1])
            with pytest.raises(H.HkvError):
                eng.quantise(8, prompt)
            eng.ragged.len.copy_(old)
            assert eng.quant is None and eng.prompt is None and eng.cache is eng.ragged
            assert eng.off is eng.ragged.off and eng.ragged.k is not None
        generate(eng, DeviceSynth(w, "cuda"), first_step=w.group_at, last_step=w.group_at + 20)
        eng.quantise(8)
        outs = []
        generate(eng, DeviceSynth(w, "cuda"), first_step=w.group_at + 21, last_step=w.group_at + 40,
                 on_step=lambda t, out: outs.append(out.clone()))
        eng.check()
        engines.append((outs, eng.quant.len.clone(), eng.quant.k.clone()))
    a, b = engines
    assert all(torch.equal(x, y) for x, y in zip(a[0], b[0])) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("bits", FMT)
def test_generation_of_a_guided_batch(bits):
    """Two prompts, two sequences each: conditional and unconditional."""
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import Engine
    from paper_2605_20600_gb300.runner import generate
    from synth.gpu import DeviceSynth

    class Guided(DeviceSynth):
        def cond(self, kc, vc, layer, stream=0):
            super().cond(kc, vc, layer, stream)
            for x in (kc, vc):
                x[1], x[3] = x[0].clone(), x[2].clone()

    w = configs.TINY.with_(n_seqs=4)
    E, N, C = w.group_at, w.n_image, w.n_cond
    steps = sorted({E, E + w.period, N - 1})
    with pytest.raises(ValueError):       # the two prompts differ
        generate(Engine(cfg_of(H, w), "cuda"), Guided(w), cache_format=bits, shared_prompt=True)
    eng = Engine(cfg_of(H, w), "cuda")
    got = {}
    generate(eng, Guided(w), cache_format=bits, shared_prompt=2,
             on_step=lambda t, out: got.__setitem__(t, out.cpu().numpy()) if t in steps else None)
    eng.check()
    labels, hp = eng.labels.cpu().numpy(), O.HeadParams.of(w)
    for s in range(4):
        for h in (1, 6):
            hi, first = gen.HeadInputs(w, s, 0, h), gen.HeadInputs(w, s // 2 * 2, 0, h)
            k, v = hi.k.copy(), hi.v.copy()
            k[:C], v[:C] = first.k[:C], first.v[:C]
            outs, _ = S.run_head_stored(hp, hi.q, k, v, bits, int(labels[flat(w, s, 0, h)]), steps,
                                        plain_cond=True)
            for t in steps:
                to = tolerances(hi.q[t], k[:C + t + 1], v[:C + t + 1])[0]
                assert np.abs(got[t][0, s, h] - outs[t]).max() <= 2 * to, (s, h, t)


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread", [20, 30, 60])
def test_queries_whose_groups_differ_in_size(bits, D, spread):
    """Queries small by 2^-spread in one group, whose keys are as much larger:
    the group counts as much as the others, and the scores keep the accuracy
    of any other query. Within a group the elements are of one size, so that
    two parts hold 22 bits of them (elements far below their group's largest
    keep fewer, down to 2^-36 of that)."""
    import torch
    c = QCache([1, 70, 300, 4000], D, bits, "fp32", seed=bits + D + spread)
    for h, g in ((1, 0), (2, 1), (3, D // 32 - 1)):
        a = slice(c.off[h], c.off[h] + c.lens[h])
        c.q[h, g * 32:g * 32 + 32] *= np.float32(2.0 ** -spread)
        c.k_scales[a, g] *= np.float32(2.0 ** spread)
        c.sk[a] = to_torch(c.k_scales[a], "bf16")
    out = torch.empty(c.n, D, device="cuda")
    lse = torch.empty(c.n, device="cuda")
    c.H.hkv_quant_attention(c.cfg, c.c, 0, to_torch(c.q, "fp32"), out, c.ws, c.ws_bytes, lse=lse)
    c.H.hkv_quant_check(c.c)
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    for h in range(c.n):
        K, V = c.rows(h)
        o, l = S.attention_lse(c.q[h], K, V)
        to, tl = tolerances(c.q[h], K, V)
        assert np.abs(got[h] - o).max() <= to, (h, np.abs(got[h] - o).max(), to)
        assert abs(gl[h] - l) <= tl, (h, gl[h], l, tl)


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread", [16, 22, 28])
def test_a_row_that_takes_the_weight_with_small_values(bits, D, spread):
    """One row has all the weight but 2^-spread of it, and V values 2^-spread of
    the others': both count alike. A channel is off by 2 eps + 2^-19 (the
    tolerance of any attention) of its own sum of |w v|, and for each row by
    2^-50 of the largest scale times a code of up to M; not by a part of the
    largest |v|."""
    import torch
    c = QCache([1, 31, 32, 300], D, bits, "fp32", seed=D + spread)
    M = 127 if bits == 8 else 7
    for h in range(c.n):
        a, top = slice(c.off[h], c.off[h] + c.lens[h]), int(c.off[h] + c.lens[h] // 2)
        # K: equal logits of 0 but the row's, which is spread * ln 2
        c.k_codes[a] = 0
        c.k_codes[top, 0], c.k_scales[top, 0] = 1, 1.0
        c.q[h, 0] = np.float32(spread * math.log(2) * math.sqrt(D))
        c.v_scales[a] *= np.float32(2.0 ** spread)
        c.v_scales[top] *= np.float32(2.0 ** -spread)
        c.ck[a] = torch.from_numpy(S.packed(c.k_codes[a], bits)).cuda()
        c.sk[a], c.sv[a] = to_torch(c.k_scales[a], "bf16"), to_torch(c.v_scales[a], "bf16")
    out = torch.empty(c.n, D, device="cuda")
    c.H.hkv_quant_attention(c.cfg, c.c, 0, to_torch(c.q, "fp32"), out, c.ws, c.ws_bytes)
    c.H.hkv_quant_check(c.c)
    got = out.cpu().numpy()
    for h in range(c.n):
        K, V = c.rows(h)
        want, _ = S.attention_lse(c.q[h], K, V)
        x = (K @ c.q[h].astype(np.float64)) / math.sqrt(D)
        w = np.exp(x - x.max())
        w /= w.sum()
        eps = 2.0 ** -19 * float((np.abs(K) @ np.abs(c.q[h])).max()) / math.sqrt(D)
        scales = c.v_scales[c.off[h]:c.off[h] + c.lens[h]].astype(np.float64)
        floor = np.repeat(scales.max(0), 32) * len(w) * M * 2.0 ** -50
        tol = (2 * eps + 2.0 ** -19) * (w @ np.abs(V)) + floor
        assert (np.abs(got[h] - want) <= tol).all(), (h, (np.abs(got[h] - want) / tol).max())


@pytest.mark.parametrize("bits", FMT)
@pytest.mark.parametrize("power", [-100, -60, 60, 110, 125])
def test_queries_of_any_size(bits, power):
    """fp32 queries near both ends of the range against keys near the other."""
    import torch
    D = 128
    c = QCache([1, 33, 200], D, bits, "fp32", seed=bits)
    c.q = np.clip(c.q, -3.9, 3.9) * np.float32(2.0 ** power)
    c.k_scales = S.round_bf16(c.k_scales * np.float32(2.0 ** -power)).reshape(c.k_scales.shape)
    for o, n in zip(c.off, c.lens):
        c.sk[o:o + n] = to_torch(c.k_scales[o:o + n], "bf16")
    out, lse = torch.empty(c.n, D, device="cuda"), torch.empty(c.n, device="cuda")
    c.H.hkv_quant_attention(c.cfg, c.c, 0, to_torch(c.q, "fp32"), out, c.ws, c.ws_bytes, lse=lse)
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    for h in range(c.n):
        K, V = c.rows(h)
        q = c.q[h].astype(np.float64)
        o, l = S.attention_lse(q, K, V)
        to, tl = tolerances(q, K, V)
        assert np.abs(got[h] - o).max() <= to and abs(gl[h] - l) <= tl, h


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("seqs", [1, 20, 40])
def test_prompt_elements_near_the_largest_fp32(D, seqs):
    """fp32 elements above the largest bf16 number (3.39e38): in V, in
    K against a query element of 2^-126, and in the query against such a key.
    One row has (nearly) all the weight, so that no sum leaves the range."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    rng = np.random.default_rng(seqs + D)
    T, Hh, big = 150, 3, np.float32(3.4e38)
    cfg = H.make_config(n_layers=1, n_seqs=seqs, n_heads=Hh, head_dim=D, dtype="fp32", n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k = rng.normal(size=(1, Hh, T, D)).astype(np.float32)
    v = rng.normal(size=(1, Hh, T, D)).astype(np.float32)
    q = rng.normal(size=(seqs, Hh, D)).astype(np.float32)
    # head 0: V; row 77 has the weight
    k[0, 0, :, 0], q[:, 0, 0] = 0.0, 8.0 * math.sqrt(D)
    k[0, 0, 77, 0] = 8.0
    v[0, 0, 77] = np.linspace(-1, 1, D).astype(np.float32) * big
    v[0, 0, 77, -1] = np.finfo(np.float32).max
    # heads 1 and 2: a key's element, a query's
    q[:, 1, 5], k[0, 1, :, 5] = np.float32(2.0 ** -126), 0.0
    k[0, 1, 33, 5], k[0, 1, 140, 5] = big, -big
    q[:, 2, 5], k[0, 2, :, 5] = big, 0.0
    k[0, 2, 33, 5], k[0, 2, 140, 5] = np.float32(2.0 ** -126), np.float32(-2.0 ** -126)
    kt, vt, qt = (to_torch(x, "fp32") for x in (k, v, q))
    pre = H.make_prefix(kt, vt, torch.tensor([T], dtype=torch.int32, device="cuda"))
    ws = torch.zeros(H.hkv_prefix_workspace_size(cfg, pre), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(seqs, Hh, D, device="cuda"), torch.zeros(seqs, Hh, device="cuda")
    H.hkv_prefix_attention(cfg, pre, qt, out, lse, ws, ws.numel())
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    for s in range(seqs):
        for h in range(Hh):
            K, V = (x[0, h].astype(np.float64) for x in (k, v))
            o, l = S.attention_lse(q[s, h], K, V)
            to, tl = tolerances(q[s, h], K, V)
            assert np.abs(got[s, h] - o).max() <= to and abs(gl[s, h] - l) <= tl, (s, h)


def test_scores_below_the_range_weigh_nothing():
    """Keys whose scores leave fp32 downwards, whole tiles of them before any
    other key: no weight, as in 64 bits, where theirs underflow. Tolerances
    from the keys that count."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    rng = np.random.default_rng(11)
    D, T, low, Hh = 64, 300, 130, 3
    for dtype, seqs, heads in (("bf16", 3, Hh), ("fp32", 3, Hh), ("fp32", 40, Hh), ("bf16", 64, 32)):
        cfg = H.make_config(n_layers=1, n_seqs=seqs, n_heads=heads, head_dim=D, dtype=dtype, n_cond=0,
                            n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                            global_budget=1)
        k = rounded(rng.normal(size=(1, heads, T, D)), dtype)
        v = rounded(rng.normal(size=(1, heads, T, D)), dtype)
        q = rounded(1 + np.abs(rng.normal(size=(seqs, heads, D))), dtype)
        k[0, :, :low] = rounded(np.float32(-3e38), dtype)
        pre = H.make_prefix(to_torch(k, dtype), to_torch(v, dtype),
                            torch.tensor([T], dtype=torch.int32, device="cuda"))
        ws = torch.zeros(H.hkv_prefix_workspace_size(cfg, pre), dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros(seqs, heads, D, device="cuda"), torch.zeros(seqs, heads, device="cuda")
        H.hkv_prefix_attention(cfg, pre, to_torch(q, dtype), out, lse, ws, ws.numel())
        got, gl = out.cpu().numpy(), lse.cpu().numpy()
        for s in range(seqs):
            for h in range(heads):
                o, l = S.attention_lse(q[s, h], k[0, h, low:], v[0, h, low:])
                to, tl = tolerances(q[s, h], k[0, h, low:], v[0, h, low:])
                assert np.abs(got[s, h] - o).max() <= to and abs(gl[s, h] - l) <= tl, (dtype, seqs, s, h)
    for bits in FMT:
        c = QCache([T, 2000], D, bits, "fp32", seed=bits)
        c.q = 1 + np.abs(c.q)
        for h in range(2):
            a = slice(c.off[h], c.off[h] + low)
            c.k_codes[a], c.k_scales[a] = -7, np.float32(2.0 ** 120)
            c.ck[a], c.sk[a] = torch.from_numpy(S.packed(c.k_codes[a], bits)).cuda(), to_torch(c.k_scales[a], "bf16")
        out, lse = torch.empty(2, D, device="cuda"), torch.empty(2, device="cuda")
        H.hkv_quant_attention(c.cfg, c.c, 0, to_torch(c.q, "fp32"), out, c.ws, c.ws_bytes, lse=lse)
        for h in range(2):
            K, V = (x[low:] for x in c.rows(h))
            o, l = S.attention_lse(c.q[h], K, V)
            to, tl = tolerances(c.q[h], K, V)
            assert np.abs(out[h].cpu().numpy() - o).max() <= to and abs(float(lse[h]) - l) <= tl, (bits, h)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,seqs,heads", [("bf16", 3, 5), ("fp32", 3, 5), ("fp32", 40, 5), ("bf16", 64, 20),
                                              ("bf16", 100, 20)])
def test_prompt_elements_that_are_not_finite(D, dtype, seqs, heads):
    """They show where their products enter, and nowhere else: a V element in
    its channel, a key's or a query's in the head or the query."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    rng = np.random.default_rng(D + seqs)
    T = 520
    cfg = H.make_config(n_layers=1, n_seqs=seqs, n_heads=heads, head_dim=D, dtype=dtype, n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k = rounded(rng.normal(size=(1, heads, T, D)), dtype)
    v = rounded(rng.normal(size=(1, heads, T, D)), dtype)
    q = rounded(rng.normal(size=(seqs, heads, D)), dtype)
    v[0, 0, 100, 3], v[0, 0, 300, 40], v[0, 0, 519, 62] = np.inf, -np.inf, np.nan
    k[0, 1, 77, 9] = np.nan
    q[seqs - 1, 2, 5] = np.nan
    finite = np.ones((seqs, heads, D), bool)
    finite[:, 0, [3, 40, 62]] = False
    finite[:, 1] = False
    finite[seqs - 1, 2] = False
    pre = H.make_prefix(to_torch(k, dtype), to_torch(v, dtype),
                        torch.tensor([T], dtype=torch.int32, device="cuda"))
    ws = torch.zeros(H.hkv_prefix_workspace_size(cfg, pre), dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros(seqs, heads, D, device="cuda"), torch.zeros(seqs, heads, device="cuda")
    H.hkv_prefix_attention(cfg, pre, to_torch(q, dtype), out, lse, ws, ws.numel())
    got, gl = out.cpu().numpy(), lse.cpu().numpy()
    assert np.array_equal(np.isfinite(got), finite)
    assert np.array_equal(np.isfinite(gl), finite[:, :, 0])
    for s in (0, seqs - 1):
        for h in (0, 2, 3):
            if not np.isfinite(gl[s, h]):
                continue
            vv = np.where(np.isfinite(v[0, h]), v[0, h], 0)
            o, l = S.attention_lse(q[s, h], k[0, h], vv)
            to, tl = tolerances(q[s, h], k[0, h], vv)
            assert np.abs(got[s, h] - o)[finite[s, h]].max() <= to and abs(gl[s, h] - l) <= tl, (s, h)


def test_updates_of_the_longest_segments_that_fit():
    """The longest segment the header's rule admits is launched, one token more
    is a capacity error, for plain and quantised caches (uncompressed heads:
    nothing is due)."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    from paper_2605_20600_gb300.engine import CacheBuffers, QuantCacheBuffers
    D, room = 64, 227 * 1024 - 4 * 64 - 2544
    for stage, quant in ((256 * (D * 2 + 16), False), (32 * D * 8, True)):
        for over in (0, 1, 20):
            cfg = H.make_config(n_layers=1, n_seqs=1, n_heads=2, head_dim=D, dtype="bf16", n_cond=0,
                                n_image=20000, row_len=100, recent_w=16, local_w=16, period=8,
                                group_at=(room - stage) // 16 + over, global_budget=24)
            c = CacheBuffers(cfg, 16, "cuda")
            if quant:
                c = QuantCacheBuffers(cfg, 8, 16, "cuda", qbuf=c.qbuf, label=c.label, off=c.off, cap=c.cap)
            for call in ((lambda: H.hkv_quant_evict_all(cfg, c.c), lambda: H.hkv_quant_evict(cfg, c.c, 0))
                         if quant else (lambda: H.hkv_evict_all(cfg, c.c), lambda: H.hkv_evict(cfg, c.c, 0))):
                if over == 0:
                    call()
                else:
                    with pytest.raises(H.HkvError) as e:
                        call()
                    assert e.value.status == H.HKV_ERR_CAPACITY
            (H.hkv_quant_check if quant else H.hkv_check)(c.c)
    assert torch.ones(3, device="cuda").sum().item() == 3     # no error left behind


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,seqs,T,lens,layout,heads", [
    (1, 40, 200, [187], "htd", 160), (2, 64, 333, [333, 0], "thd", 80), (1, 17, 640, [577], "padded", 160),
    (1, 100, 257, [257], "padded", 160), (2, 130, 130, [64, 129], "htd", 40), (2, 65, 200, [0, 1], "thd", 80)])
def test_prefix_attention_of_many_heads(D, G, seqs, T, lens, layout, heads):
    """Batches whose (group, head) pairs fill the device: one range of keys
    each, finished without a join."""
    from paper_2605_20600_gb300 import hkv as H
    import torch
    cfg = H.make_config(n_layers=1, n_seqs=G * seqs, n_heads=heads, head_dim=D, dtype="bf16", n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k = torch.zeros(G, heads, T, D, dtype=torch.bfloat16)
    assert H.hkv_prefix_workspace_size(cfg, H.make_prefix(k, k, torch.zeros(G, dtype=torch.int32))) == 256
    check_prefix(D, "bf16", G, seqs, T, lens, layout, heads)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,seqs,heads,T,joined", [
    ("bf16", 3, 2, 300, True), ("bf16", 3, 160, 70, False), ("fp32", 40, 2, 300, True),
    ("bf16", 40, 20, 600, True), ("bf16", 100, 20, 600, True), ("bf16", 40, 100, 300, False),
    ("bf16", 100, 100, 300, False)])
def test_prefix_length_out_of_range_on_every_kernel(D, dtype, seqs, heads, T, joined):
    """The group gets NaN, the other groups are as without it, and the error
    word says so, with one range of keys and with several."""
    import torch
    from paper_2605_20600_gb300 import hkv as H
    rng = np.random.default_rng(T)
    cfg = H.make_config(n_layers=1, n_seqs=3 * seqs, n_heads=heads, head_dim=D, dtype=dtype, n_cond=0,
                        n_image=8, row_len=1, recent_w=1, local_w=1, period=1, group_at=8,
                        global_budget=1)
    k, v = prefix_rows(rng, 3, heads, T, D, dtype, "htd")
    q = to_torch(rng.normal(size=(3 * seqs, heads, D)), dtype)
    res = []
    for bad in (None, T + 1, -1, 1 << 30):
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        lens = [T, T if bad is None else bad, T - 5]
        pre = H.make_prefix(k, v, torch.tensor(lens, dtype=torch.int32, device="cuda"), err)
        n = H.hkv_prefix_workspace_size(cfg, pre)
        assert (n > 256) == joined
        ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
        out, lse = torch.zeros(3, seqs, heads, D, device="cuda"), torch.zeros(3, seqs, heads, device="cuda")
        H.hkv_prefix_attention(cfg, pre, q, out, lse, ws, n)
        torch.cuda.synchronize()
        assert int(err) == (0 if bad is None else H.HKV_ERR_BOUNDS)
        res.append((out, lse))
    for out, lse in res[1:]:
        assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
        for g in (0, 2):
            assert torch.equal(out[g], res[0][0][g]) and torch.equal(lse[g], res[0][1][g])
    assert torch.isfinite(res[0][0]).all() and torch.isfinite(res[0][1]).all()
