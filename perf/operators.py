"""Cases of the serving-cache operators: a KV cache held in 8 or 4 bits (written, read back,
attended over, trimmed) and attention over a prompt that the sequences of a batch share.

Kinds of cases (the field "kind"):
  step    one decode step of `layers` layers: the new token's K and V are quantised into the
          cache and every head attends over what the cache then holds; with prompt > 0 the
          conditioning tokens live outside the cache, shared by the sequences of a group, and
          their attention is computed once for all and joined in the same pass
  attend  the attention alone over an uncompressed cache in 8 or 4 bits
  trip    a plain cache quantised head by head and read back into a plain one
  update  the periodic head-aware update (eviction) of a cache in 8 or 4 bits
  prompt  the attention of a batch over shared prompts alone

A cache row of D values is kept as D codes and D/32 bf16 scales: of 32 neighbours x with the
largest magnitude a, the scale is s = bf16(a / M), M = 127 (8 bits) or 7 (4 bits), the code
c = clamp(rint(x / s), -M, M), ties to even, and the row stands for s * c. The quotients are
taken in fp32 and the codes stored with 128 (8 bits) or 8 (4 bits) added, two 4-bit codes a
byte, the even channel in the low half.
"""
import math

import torch

own = False

GROUP = 32
LOCAL, GLOBAL, DENSE = 0, 1, 255


def _case(kind, name=None, **kw):
    c = {"kind": kind, "bits": 8, "dtype": "bf16", "dim": 128, "layers": 1, "seqs": 1, "heads": 32,
         "cond": 0, "budget": 0, "window": 0, "period": 0, "image": 0, "buffered": 0,
         "prompt": 0, "prompts": 1}
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the decode step of Lumina-mGPT 1024 at rho = 1/4 with 8 sequences, 8 of its layers
        _case("step", "step8 lumina1024", layers=8, seqs=8, cond=128, budget=1040, window=130,
              period=65, image=4160, buffered=32),
        # Janus-Pro-7B with 64 sequences of one prompt: its 64 conditioning tokens shared
        _case("step", "step4 janus prompt", bits=4, layers=6, seqs=64, budget=72, window=48,
              period=24, image=576, buffered=12, prompt=64),
        # LlamaGen-XL, 128 sequences of short segments, half of the layers' 36 heads x 128
        _case("step", "step8 llamagen", layers=6, seqs=128, heads=20, dim=64, cond=1, budget=96,
              window=48, period=24, image=576, buffered=12),
        # the smallest call: one sequence of the tiny workload's heads, latency counts
        _case("attend", "attend8 tiny", dtype="fp32", dim=64, heads=8, image=128),
        # one long uncompressed cache of an odd length in 4 bits
        _case("attend", "attend4 long", bits=4, image=65537),
        # a grouped Lumina-mGPT 1024 cache quantised after its compression, and read back
        _case("trip", "trip8 lumina1024", layers=2, seqs=8, cond=128, budget=1040, window=130,
              period=65, image=4160, buffered=0),
        # few heads, fp32 rows of 64, odd sizes
        _case("trip", "trip4 odd", bits=4, dtype="fp32", dim=64, layers=3, seqs=3, heads=11,
              cond=17, budget=333, window=41, period=19, image=1001, buffered=7),
        # the update of every layer when the buffers of 65 tokens are full
        _case("update", "update8 lumina1024", layers=4, seqs=8, cond=128, budget=1040, window=130,
              period=65, image=4160, buffered=65),
        _case("update", "update4 odd", bits=4, dtype="fp32", dim=64, layers=2, seqs=3, heads=13,
              cond=9, budget=301, window=40, period=21, image=900, buffered=21),
        # 64 sequences over one long prompt (an editing or interleaved prompt)
        _case("prompt", "prompt 64 seqs", seqs=64, prompt=4099),
        # conditional and unconditional prompts of a guided batch, heads of 64
        _case("prompt", "prompt guided", seqs=128, heads=20, dim=64, prompt=1000, prompts=2),
        # the fp32 parity type on a ragged size
        _case("prompt", "prompt fp32", dtype="fp32", seqs=5, heads=8, dim=64, prompt=777),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["step", "step", "attend", "trip", "update", "prompt"])
    c = _case(kind, bits=rng.choice([8, 4]), dtype=rng.choice(["bf16", "bf16", "bf16", "fp32"]),
              dim=rng.choice([64, 128]), heads=rng.randint(1, 40), seqs=_spread(rng, 1, 64))
    if kind == "prompt":
        c["prompts"] = rng.choice([1, 1, 2])
        c["seqs"] = c["prompts"] * max(1, c["seqs"] // c["prompts"])
        c["prompt"] = _spread(rng, 1, 8000)
        while c["prompt"] * c["heads"] * max(16, c["seqs"]) > 4100 * 32 * 64:
            c["prompt"] = c["prompt"] // 2 + 1
        return c
    if kind == "attend":
        c["image"] = _spread(rng, 2, 60000)
        while c["image"] * c["seqs"] * c["heads"] > 2000000:
            c["seqs"], c["image"] = c["seqs"] // 2 + 1, c["image"] * 3 // 4
        return c
    c["layers"] = rng.randint(1, 6)
    c["cond"] = rng.choice([0, 1, rng.randint(2, 160)])
    c["window"] = _spread(rng, 8, 140)
    c["period"] = _spread(rng, 4, 70)
    c["budget"] = c["window"] + _spread(rng, 1, 950)
    c["image"] = c["budget"] * rng.randint(2, 6) + 2 * c["period"] + c["window"]
    c["buffered"] = c["period"] if kind == "update" else rng.randrange(c["period"])
    per = c["cond"] + c["window"] + c["period"] + (c["budget"] - c["window"]) // 2
    most = 1600000 if kind == "step" else 400000
    while per * c["layers"] * c["seqs"] * c["heads"] > most:
        c["seqs"] = c["seqs"] // 2 + (c["seqs"] > 2)
        c["layers"] = max(1, c["layers"] - 1)
        if c["seqs"] == 1 and c["layers"] == 1:
            break
        c["seqs"] = max(1, c["seqs"])
    if kind == "step" and rng.random() < 0.5:
        c["prompt"], c["prompts"], c["cond"] = _spread(rng, 1, 600), rng.choice([1, 2]), 0
        c["seqs"] = c["prompts"] * max(1, c["seqs"] // c["prompts"])
    return c


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _shape(case, gen):
    """Per head of all layers, [L][S][H] flat: label, segment capacity, live tokens."""
    n = case["layers"] * case["seqs"] * case["heads"]
    if case["kind"] == "attend":
        label = torch.full((n,), DENSE, device="cuda")
        cap = torch.full((n,), case["image"], device="cuda")
        return label, cap, cap.clone()
    # half of the heads global, at places of their own in each batch
    label = (torch.randperm(n, generator=gen, device="cuda") < n // 2).long()
    keep = torch.where(label == GLOBAL, case["budget"], case["window"])
    return label, case["cond"] + keep + case["period"], case["cond"] + keep + case["buffered"]


def _quantise(x, bits):
    """x [..., D] -> codes as floats in [-M, M] and scales [..., D / 32] in bf16."""
    most = 127.0 if bits == 8 else 7.0
    g = x.float().reshape(*x.shape[:-1], -1, GROUP)
    # (a Python number as divisor would become a product with its reciprocal)
    scale = (g.abs().amax(-1) / torch.full((), most, device=x.device)).to(torch.bfloat16)
    s = scale.float().unsqueeze(-1)
    code = torch.where(s > 0, torch.round(g / s), torch.zeros_like(g)).clamp(-most, most)
    return code.reshape(x.shape), scale


def _packed(code, bits):
    if bits == 8:
        return (code + 128).to(torch.uint8)
    c = (code + 8).to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _codes(packed, bits):
    if bits == 8:
        return packed.float() - 128
    return torch.stack([packed & 15, packed >> 4], -1).flatten(-2).float() - 8


def _values(packed, scale, bits):
    code = _codes(packed, bits)
    return (code.unflatten(-1, (-1, GROUP)) * scale.float().unsqueeze(-1)).flatten(-2)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 13)
    L, S, H, D, dt = case["layers"], case["seqs"], case["heads"], case["dim"], _type(case)
    n = L * S * H
    st = {"case": dict(case)}
    # keys with channels of uneven size, as models have them; queries that make the attention
    # neither flat nor a single token
    gain = torch.exp(0.5 * _normal(gen, H, D))
    qgain = 1.0 / gain
    if case["prompt"]:
        G, T = case["prompts"], case["prompt"]
        shape = (L, G, H, T, D)
        st["pk"] = (_normal(gen, *shape) * gain[:, None]).to(dt)
        st["pv"] = _normal(gen, *shape).to(dt)
        # the prompts of a guided batch differ in length
        st["plen"] = torch.tensor([max(1, T - g * (T // 3)) for g in range(G)], dtype=torch.int32,
                                  device="cuda")
    st["q"] = (_normal(gen, L, S, H, D) * 1.5 * qgain).to(dt)
    st["out"] = torch.zeros(L, S, H, D, device="cuda")
    st["lse"] = torch.zeros(L, S, H, device="cuda")
    if case["prompt"]:
        st["pout"], st["plse"] = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"])
    if case["kind"] == "prompt":
        return st
    st["k"] = (_normal(gen, L, S, H, D) * gain).to(dt)
    st["v"] = _normal(gen, L, S, H, D).to(dt)
    label, cap, live = _shape(case, gen)
    off = torch.cumsum(cap, 0) - cap
    tokens = int(cap.sum())
    head = torch.repeat_interleave(torch.arange(n, device="cuda"), cap) % H
    row = torch.arange(tokens, device="cuda") - torch.repeat_interleave(off, cap)
    # positions: the conditioning tokens, a thinned history, the recent window and the buffer
    last = case["image"] - case["period"] + case["buffered"] if case["kind"] != "attend" else case["image"]
    i = row - case["cond"]
    tail = case["window"] + case["buffered"] if case["kind"] != "attend" else 0
    hist = torch.repeat_interleave(live, cap) - case["cond"] - tail
    thin = i * (last - tail) // hist.clamp(min=1)
    pos = torch.where(i < 0, row, case["cond"] + torch.where(i < hist, thin, last - tail + i - hist))
    k = _normal(gen, tokens, D)
    for a in range(0, tokens, 1 << 20):
        k[a:a + (1 << 20)] *= gain[head[a:a + (1 << 20)]]
    v = _normal(gen, tokens, D)
    st["off"], st["cap"] = off, cap.to(torch.int32)
    st["label"] = label.to(torch.uint8)
    st["qbuf"] = (_normal(gen, n, max(1, case["period"]), D) * 1.5).to(dt)
    counters = torch.stack([live, torch.full_like(live, case["buffered"]), torch.full_like(live, last)])
    if case["kind"] == "trip":
        st["plain"] = {"k": k.to(dt), "v": v.to(dt), "pos": pos.to(torch.int32),
                       "counters": counters.to(torch.int32)}
        st["back"] = {"k": torch.zeros_like(st["plain"]["k"]), "v": torch.zeros_like(st["plain"]["v"]),
                      "pos": torch.zeros_like(st["plain"]["pos"]),
                      "counters": torch.zeros_like(st["plain"]["counters"])}
        del k, v
        k = v = None
    # the quantised cache in one piece of memory, so that a pass that changes it can begin by
    # putting the old one back: counters, positions, codes, scales
    rowb = D * case["bits"] // 8
    sizes = [3 * n * 4, tokens * 4, tokens * rowb, tokens * rowb, tokens * D // GROUP * 2,
             tokens * D // GROUP * 2]
    at = [0]
    for b in sizes:
        at.append(at[-1] + (b + 255) // 256 * 256)
    blob = torch.zeros(at[-1], dtype=torch.uint8, device="cuda")
    part = [blob[a:a + b] for a, b in zip(at, sizes)]
    st["blob"] = blob
    st["counters"] = part[0].view(torch.int32).view(3, n)
    st["pos"] = part[1].view(torch.int32)
    st["ck"], st["cv"] = part[2].view(tokens, rowb), part[3].view(tokens, rowb)
    st["sk"], st["sv"] = (p.view(torch.bfloat16).view(tokens, D // GROUP) for p in part[4:])
    if k is not None:
        st["counters"].copy_(counters)
        st["pos"].copy_(pos)
        for x, codes, scales in ((k, st["ck"], st["sk"]), (v, st["cv"], st["sv"])):
            for a in range(0, tokens, 1 << 20):
                c, s = _quantise(x[a:a + (1 << 20)], case["bits"])
                codes[a:a + (1 << 20)] = _packed(c, case["bits"])
                scales[a:a + (1 << 20)] = s
        if case["kind"] == "step":
            st["first"] = st["counters"].clone()
        elif case["kind"] == "update":
            st["first"] = blob.clone()
    return st


# ---------------------------------------------------------------------------------------------
# plain forms, 32 bits
# ---------------------------------------------------------------------------------------------
def _rows(off, live):
    """Arena rows of every head, padded: indexes [n, longest] and which of them are live."""
    i = torch.arange(int(live.max()), device=off.device)
    return off[:, None] + torch.minimum(i, (live[:, None] - 1).clamp(min=0)), i < live[:, None]


def _softmax_parts(x, mask):
    """x [..., m] logits -> weights, natural log of the sum of exp; rows of no key: 0 and -inf."""
    x = torch.where(mask, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, 1.0), (m + torch.log(total)).squeeze(-1)


def _joined(out, lse, other, other_lse):
    both = torch.logaddexp(lse, other_lse)
    return (torch.exp(lse - both)[..., None] * out + torch.exp(other_lse - both)[..., None] * other), both


def _prompt_plain(st):
    case = st["case"]
    L, S, H, D, G = case["layers"], case["seqs"], case["heads"], case["dim"], case["prompts"]
    q = st["q"].float().view(L, G, S // G, H, D).transpose(2, 3)
    x = torch.matmul(q, st["pk"].float().transpose(-1, -2)) / math.sqrt(D)
    mask = torch.arange(case["prompt"], device="cuda") < st["plen"][:, None]
    w, lse = _softmax_parts(x, mask[None, :, None, None, :])
    out = torch.matmul(w, st["pv"].float())
    return out.transpose(2, 3).reshape(L, S, H, D), lse.transpose(2, 3).reshape(L, S, H)


def _attend_plain(st):
    case = st["case"]
    L, S, H, D = case["layers"], case["seqs"], case["heads"], case["dim"]
    rows, mask = _rows(st["off"], st["counters"][0].long())
    k = _values(st["ck"][rows], st["sk"][rows], case["bits"])
    q = st["q"].float().view(L * S * H, D, 1)
    w, lse = _softmax_parts(torch.matmul(k, q).squeeze(-1) / math.sqrt(D), mask)
    del k
    v = _values(st["cv"][rows], st["sv"][rows], case["bits"])
    return torch.matmul(w[:, None, :], v).view(L, S, H, D), lse.view(L, S, H)


def _append_plain(st):
    case = st["case"]
    n, D = st["off"].numel(), case["dim"]
    live, buffered, count = st["counters"]
    row = st["off"] + live
    for x, codes, scales in ((st["k"], st["ck"], st["sk"]), (st["v"], st["cv"], st["sv"])):
        c, s = _quantise(x.view(n, D), case["bits"])
        codes[row], scales[row] = _packed(c, case["bits"]), s
    st["pos"][row] = case["cond"] + count
    st["qbuf"][torch.arange(n, device="cuda"), (count % case["period"]).long()] = st["q"].view(n, D)
    buffered += (st["label"] != DENSE).to(torch.int32)
    live += 1
    count += 1


def _rank(x, among):
    """Rank of each entry of a row by (x, storage order), entries not `among` last."""
    order = torch.sort(torch.where(among, x, math.inf), dim=-1, stable=True).indices
    return torch.empty_like(order).scatter_(-1, order, torch.arange(x.shape[-1], device=x.device).expand_as(order))


def _update_plain(st):
    case = st["case"]
    C, P, w, n = case["cond"], case["period"], case["window"], st["off"].numel()
    live, buffered, count = (x.long() for x in st["counters"])
    due = (st["label"] != DENSE) & (buffered >= P)
    rows, mask = _rows(st["off"], live)
    pos = torch.where(mask, st["pos"][rows].long(), -1)
    hist = mask & (pos >= C) & (pos < (C + (count - w).clamp(min=0))[:, None])
    NH = hist.sum(-1)
    budget = (st["cap"].long() - C - P - w).clamp(min=0)
    M = torch.where(st["label"] == LOCAL, NH, (NH - budget).clamp(min=0))
    M = torch.where(due, M, torch.zeros_like(M))
    # the oldest half of the history is the long-range subset; half of the evictions from each
    n_long = torch.floor(NH.double() * 0.5).long()
    is_long = hist & (_rank(pos.double(), hist) < n_long[:, None])
    near = hist & ~is_long
    m_long = torch.minimum(M // 2, n_long)
    m_near = M - m_long
    over = (m_near - (NH - n_long)).clamp(min=0)
    m_long, m_near = m_long + over, m_near - over
    # scores of the summed queries, both sums in a fixed order: which rows go depends on them
    slots = (count[:, None] - P + torch.arange(P, device="cuda")) % P
    ring = st["qbuf"].float()[torch.arange(n, device="cuda")[:, None], slots]
    qsum = torch.zeros(n, case["dim"], device="cuda")
    for p in range(P):
        qsum = qsum + ring[:, p]
    k = _values(st["ck"][rows], st["sk"][rows], case["bits"])
    score = torch.zeros(rows.shape, device="cuda")
    for d in range(case["dim"]):
        score = score + qsum[:, d:d + 1] * k[:, :, d]
    # equal scores: the older token first
    by_age = torch.sort(pos, dim=-1).indices
    rank = torch.zeros_like(rows)
    for subset in (is_long, near):
        r = _rank(score.double().gather(-1, by_age), subset.gather(-1, by_age))
        rank = torch.where(subset, torch.zeros_like(rank).scatter_(-1, by_age, r), rank)
    gone = (is_long & (rank < m_long[:, None])) | (near & (rank < m_near[:, None]))
    gone = torch.where((st["label"] == LOCAL)[:, None], hist, gone) & (M > 0)[:, None]
    # the i-th evicted row below the new length takes the i-th surviving row above it
    left = live - M
    i = torch.arange(rows.shape[1], device="cuda")
    hole, fill = gone & (i < left[:, None]), mask & ~gone & (i >= left[:, None])
    to, src = rows[hole], rows[fill]
    for x in (st["pos"], st["ck"], st["cv"], st["sk"], st["sv"]):
        x[to] = x[src]
    st["counters"][0].copy_(left)
    st["counters"][1].copy_(torch.where(due, torch.zeros_like(buffered), buffered))


def _trip_plain(st):
    case, a, b = st["case"], st["plain"], st["back"]
    n = st["off"].numel()
    live = a["counters"][0].long()
    tokens = a["pos"].numel()
    seg = torch.repeat_interleave(torch.arange(n, device="cuda"), st["cap"].long())
    on = torch.arange(tokens, device="cuda") - st["off"][seg] < live[seg]
    for name, codes, scales in (("k", st["ck"], st["sk"]), ("v", st["cv"], st["sv"])):
        c, s = _quantise(a[name], case["bits"])
        codes.copy_(torch.where(on[:, None], _packed(c, case["bits"]), codes))
        scales.copy_(torch.where(on[:, None], s, scales))
        b[name].copy_(torch.where(on[:, None], _values(codes, scales, case["bits"]).to(b[name].dtype), b[name]))
    for to in (st["pos"], b["pos"]):
        to.copy_(torch.where(on, a["pos"], to))
    for to in (st["counters"], b["counters"]):
        to.copy_(a["counters"])


# ---------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------
def _handle(st):
    """The plan a program keeps beside its buffers: config, cache structs, workspaces."""
    if "handle" in st:
        return st["handle"]
    from paper_2605_20600_gb300 import hkv as H
    case = st["case"]
    dense = case["kind"] in ("attend", "prompt")
    cfg = H.make_config(
        n_layers=case["layers"], n_seqs=case["seqs"], n_heads=case["heads"], head_dim=case["dim"],
        dtype=case["dtype"], n_cond=case["cond"], n_image=max(1, case["image"]), row_len=1,
        recent_w=1 if dense else case["window"], local_w=1 if dense else case["window"],
        period=1 if dense else case["period"],
        group_at=max(1, case["image"]) if dense else case["period"],
        global_budget=1 if dense else case["budget"])
    h = {"H": H, "cfg": cfg, "stream": torch.cuda.current_stream().cuda_stream}
    err = h["err"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if case["prompt"]:
        h["prefix"] = [H.make_prefix(st["pk"][layer], st["pv"][layer], st["plen"])
                       for layer in range(case["layers"])]
        h["pws_bytes"] = H.hkv_prefix_workspace_size(cfg, h["prefix"][0])
        h["pws"] = torch.zeros(h["pws_bytes"], dtype=torch.uint8, device="cuda")
    if case["kind"] != "prompt":
        live, buffered, count = st["counters"]
        h["cache"] = H.make_qcache(case["bits"], st["ck"], st["cv"], st["sk"], st["sv"], st["pos"],
                                   st["off"], st["cap"], live, buffered, count, st["label"],
                                   st["qbuf"], err, st["pos"].numel())
        h["ws_bytes"] = H.hkv_quant_workspace_size(cfg)
        h["ws"] = torch.zeros(h["ws_bytes"], dtype=torch.uint8, device="cuda")
    if case["kind"] == "trip":
        def plain(x):
            live, buffered, count = x["counters"]
            return H.hkv_cache(x["k"].data_ptr(), x["v"].data_ptr(), x["pos"].data_ptr(),
                               st["off"].data_ptr(), st["cap"].data_ptr(), live.data_ptr(),
                               buffered.data_ptr(), count.data_ptr(), st["label"].data_ptr(),
                               st["qbuf"].data_ptr(), err.data_ptr(), x["pos"].numel())
        h["plain"], h["back"] = plain(st["plain"]), plain(st["back"])
    st["handle"] = h
    return h


def _run_own(st):
    h, kind = _handle(st), st["case"]["kind"]
    H, cfg, stream = h["H"], h["cfg"], h["stream"]
    if kind == "trip":
        H.hkv_quant_pack(cfg, h["plain"], h["cache"], H.HKV_ALL_LAYERS, 0, stream)
        H.hkv_quant_unpack(cfg, h["cache"], h["back"], H.HKV_ALL_LAYERS, stream)
        return
    if kind == "update":
        H.hkv_quant_evict_all(cfg, h["cache"], stream)
        return
    for layer in range(cfg.n_layers):
        q, out, lse, prior = st["q"][layer], st["out"][layer], st["lse"][layer], None
        if st["case"]["prompt"]:
            prior = (st["pout"][layer], st["plse"][layer]) if kind == "step" else (out, lse)
            H.hkv_prefix_attention(cfg, h["prefix"][layer], q, prior[0], prior[1], h["pws"],
                                   h["pws_bytes"], stream)
        if kind == "step":
            # the kernel before this one works on another layer, or on the prompt
            H.hkv_quant_step(cfg, h["cache"], layer, q, st["k"][layer], st["v"][layer], out,
                             h["ws"], h["ws_bytes"], prior=prior, lse=lse,
                             flags=H.HKV_STEP_PREFETCH if layer or prior else 0, stream=stream)
        elif kind == "attend":
            H.hkv_quant_attention(cfg, h["cache"], layer, q, out, h["ws"], h["ws_bytes"], lse=lse,
                                  stream=stream)


def _run_plain(st):
    kind = st["case"]["kind"]
    if kind == "trip":
        _trip_plain(st)
    elif kind == "update":
        _update_plain(st)
    elif kind == "prompt":
        st["out"], st["lse"] = _prompt_plain(st)
    else:
        if kind == "step":
            _append_plain(st)
        st["out"], st["lse"] = _attend_plain(st)
        if st["case"]["prompt"]:
            st["out"], st["lse"] = _joined(st["out"], st["lse"], *_prompt_plain(st))


def run(st):
    kind = st["case"]["kind"]
    # a pass that changes its cache starts from the same one each time
    if kind == "step":
        st["counters"].copy_(st["first"])
    elif kind == "update":
        st["blob"].copy_(st["first"])
    (_run_own if own else _run_plain)(st)
    if kind in ("prompt", "attend"):
        return {"out": st["out"], "lse": st["lse"]}
    # codes go out as they are stored: both sides have to write the same bits
    state = {"counters": st["counters"], "pos": st["pos"], "k_codes": st["ck"], "v_codes": st["cv"],
             "k_scales": st["sk"], "v_scales": st["sv"]}
    if kind == "step":
        return {"out": st["out"], "lse": st["lse"], "qbuf": st["qbuf"], **state}
    if kind == "trip":
        return {"k": st["back"]["k"], "v": st["back"]["v"], "back_pos": st["back"]["pos"],
                "back_counters": st["back"]["counters"], **state}
    return state


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------
def _unit64(x, bits):
    """What rows x stand for after they were stored."""
    top = 127 if bits == 8 else 7
    x = x.double()
    a = x.unflatten(-1, (-1, 32)).abs().max(-1, keepdim=True).values.float()
    s = (a / torch.tensor(float(top), device=x.device)).bfloat16().double()
    c = torch.round(x.unflatten(-1, (-1, 32)) / torch.where(s == 0, torch.ones_like(s), s))
    return (c.clip(-top, top) * s).flatten(-2)


def _stored64(codes, scales, bits):
    c = codes.long()
    if bits == 4:
        c = torch.stack((c % 16, c // 16), -1).flatten(-2)
    c = c - (128 if bits == 8 else 8)
    return (c.unflatten(-1, (-1, 32)) * scales.double().unsqueeze(-1)).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    kind, bits, D = case["kind"], case["bits"], case["dim"]
    if kind == "update":
        return None     # rows are chosen and moved, nothing is computed
    if kind == "trip":
        def back(x):
            y = _unit64(x, bits)
            seg = torch.repeat_interleave(torch.arange(st["cap"].numel(), device=x.device), st["cap"].long())
            row = torch.arange(x.shape[0], device=x.device) - st["off"][seg]
            return torch.where((row < st["plain"]["counters"][0].long()[seg])[:, None], y, 0.0)
        return {"k": back(st["plain"]["k"]), "v": back(st["plain"]["v"]), "back_pos": None,
                "back_counters": None, "counters": None, "pos": None, "k_codes": None,
                "v_codes": None, "k_scales": None, "v_scales": None}
    L, S, H, G = case["layers"], case["seqs"], case["heads"], case["prompts"]
    out = torch.zeros(L, S, H, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(L, S, H, dtype=torch.float64, device="cuda")
    q = st["q"].double() / D ** 0.5
    if kind != "prompt":
        live = st["counters"][0].tolist()
        off = st["off"].tolist()
    for layer in range(L):
        for s in range(S):
            g = s // (S // G)
            for h in range(H):
                ks, vs = [], []
                if case["prompt"]:
                    t = int(st["plen"][g])
                    ks.append(st["pk"][layer, g, h, :t].double())
                    vs.append(st["pv"][layer, g, h, :t].double())
                if kind != "prompt":
                    i = (layer * S + s) * H + h
                    a = slice(off[i], off[i] + live[i])
                    ks.append(_stored64(st["ck"][a], st["sk"][a], bits))
                    vs.append(_stored64(st["cv"][a], st["sv"][a], bits))
                if kind == "step":
                    ks.append(_unit64(st["k"][layer, s, h][None], bits))
                    vs.append(_unit64(st["v"][layer, s, h][None], bits))
                x = torch.cat(ks) @ q[layer, s, h]
                m = x.max()
                e = torch.exp(x - m)
                out[layer, s, h] = (e / e.sum()) @ torch.cat(vs)
                lse[layer, s, h] = m + torch.log(e.sum())
    got = {"out": out, "lse": lse}
    if kind == "step":
        got.update({x: None for x in ("qbuf", "counters", "pos", "k_codes", "v_codes", "k_scales", "v_scales")})
    return got


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    L, S, H, D, P = case["layers"], case["seqs"], case["heads"], case["dim"], case["period"]
    n, es = L * S * H, 2 if case["dtype"] == "bf16" else 4
    row = D * case["bits"] // 8 + D // GROUP * 2        # codes and scales of one K or V row
    nbytes, flops = 0.0, 0.0
    if case["prompt"]:
        T = sum(max(1, case["prompt"] - g * (case["prompt"] // 3)) for g in range(case["prompts"]))
        nbytes += L * H * T * D * 2 * es
        flops += 4.0 * L * H * D * T * (S // case["prompts"])
        if case["kind"] == "prompt":
            return {"bytes": nbytes + n * (D * es + D * 4 + 4), "flops": flops}
    if case["kind"] == "attend":
        live = n * case["image"]
        return {"bytes": live * 2 * row + n * (D * es + D * 4 + 4), "flops": 4.0 * live * D}
    keep = (case["budget"] + case["window"]) / 2        # half of the heads are global
    live = n * (case["cond"] + keep + case["buffered"])
    if case["kind"] == "step":
        nbytes += live * 2 * row + n * (2 * row + 4 * D * es + D * 4 + 4)
        return {"bytes": nbytes, "flops": flops + 4.0 * (live + n) * D}
    if case["kind"] == "trip":
        # plain rows in, codes out and in again, plain rows out; positions with them
        return {"bytes": live * (4 * D * es + 4 * row + 16), "flops": 8.0 * live * D}
    # update: the history's keys of the global heads (half of them) and the queries for their
    # scores, the positions, and the rows that move; at least P rows of each head leave, and
    # about half of those have to be replaced
    scored = n / 2 * (case["budget"] - case["window"] + P)
    moved = n * P / 2
    return {"bytes": scored * row + n / 2 * P * D * es + live * 4 + moved * (4 * row + 8),
            "flops": 2.0 * scored * D}
