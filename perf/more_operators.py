"""Cases of what a model does to queries, keys and values around the cache: rotary positions, the
norms of queries and keys with the rotation in the same pass, and attention of many queries (or one)
over states of another length.

Kinds of cases (the field "kind"):
  rotate   rotary positions of [sequences][tokens][heads][dim] rows; with back, the rotation undone
           (its gradient, and how cached keys move to other positions)
  prepare  queries and keys of a fused projection normed for each head and rotated, values carried
           along: queries stay by tokens, keys and values go by heads, as a cache takes them
  cross    attention over the states of an encoder, or (causal) of a prompt's own tokens

Pair i of the rot / 2 pairs of a head turns by the angle position * f_i. In the "half" layout channel
i pairs with i + rot / 2, in the "pairs" layout 2i with 2i + 1. f_i = base^(-2i / d) with d = rot; on
two axes the first half of the pairs turns by the row and the other by the column, each with
frequencies of its own (d = rot / 2, i from 0). For contexts longer than the original one by a factor
s: "linear" f / s; "base" takes base * s^(d / (d - 2)); "parts" f * (g + (1 - g) / s), g the turns in
the original length from 1 to 32 as a ramp, and cos and sin times an amplitude.
"""
import math

import torch

own = False

BASE = 10000.0
EPS = 1e-5
LOW, HIGH = 1.0, 32.0


def _case(kind, name=None, **kw):
    c = {"kind": kind, "dtype": "bf16", "dim": 128, "seqs": 1, "heads": 32, "kv": 32, "tokens": 1,
         "ragged": False}
    if kind == "cross":
        c.update(keys=1, causal=False, single=False)
    else:
        c.update(rot=128, layout="half", grid=0, start=0, scaling="none", factor=1.0, original=4096)
        c.update({"back": False} if kind == "rotate" else {"norm": "rms"})
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: the new token's keys of the tiny workload, latency counts
        _case("rotate", "rotate tiny step", dtype="fp32", dim=64, rot=64, heads=8, start=77),
        # the image tokens of LlamaGen-XL, 128 sequences on a grid of 24 x 24
        _case("rotate", "rotate llamagen grid", dim=64, rot=64, layout="pairs", grid=24, seqs=128,
              heads=20, tokens=576),
        # a long context, part of the head, odd sizes, padded sequences, rotated back
        _case("rotate", "rotate part of long", dtype="fp32", rot=32, seqs=3, heads=11, tokens=3001,
              start=900000, scaling="parts", factor=8.0, ragged=True, back=True),
        # one decode step of Lumina-mGPT 1024: layer norms and rotation of 8 sequences
        _case("prepare", "prepare lumina1024 step", seqs=8, norm="layer", start=2000),
        # one decode step of Janus-Pro-7B's batch, RMS norms
        _case("prepare", "prepare janus step", seqs=64, start=500),
        # all tokens of Lumina-mGPT 1024's 8 sequences: conditioning and image
        _case("prepare", "prepare lumina1024 prompt", seqs=8, tokens=4288, norm="layer"),
        # grouped heads, odd sizes, padded, heads of 64, a larger base
        _case("prepare", "prepare grouped odd", dim=64, rot=64, layout="pairs", seqs=5, heads=14, kv=2,
              tokens=1001, scaling="base", factor=4.0, ragged=True),
        # one query per sequence over a text encoder's states of unequal length
        _case("cross", "cross text step", seqs=64, keys=300, ragged=True, single=True),
        # a prompt's own tokens: Lumina-mGPT 1024's whole sequence, for two sequences
        _case("cross", "cross causal lumina1024", seqs=2, tokens=4288, keys=4288, causal=True),
        # an image's queries over text states, grouped heads of 64, padded
        _case("cross", "cross image grouped", dim=64, seqs=16, heads=20, kv=4, tokens=577, keys=1025,
              ragged=True),
        # few queries of few heads over one long context
        _case("cross", "cross long few", heads=8, kv=2, tokens=5, keys=65537),
        # the fp32 parity type on ragged sizes
        _case("cross", "cross fp32", dtype="fp32", dim=64, seqs=5, heads=8, kv=8, tokens=257, keys=777,
              ragged=True),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "prepare", "cross", "cross"])
    dim = rng.choice([64, 128])
    c = _case(kind, dtype=rng.choice(["bf16", "bf16", "fp32"]), dim=dim, seqs=_spread(rng, 1, 64),
              ragged=rng.random() < 0.5)
    c["kv"] = rng.randint(1, 12)
    c["heads"] = c["kv"] * rng.choice([1, 1, 2, 4, 7])
    if kind == "cross":
        c["keys"] = _spread(rng, 1, 8000)
        c["tokens"] = _spread(rng, 1, 4000)
        if rng.random() < 0.3:
            c["tokens"], c["single"] = 1, c["dtype"] == "bf16"
        c["causal"] = c["tokens"] > 1 and rng.random() < 0.4
        most = 5.0e8 if c["dtype"] == "bf16" else 1.0e8
        while c["seqs"] * c["heads"] * c["tokens"] * c["keys"] > most:
            if c["seqs"] > 1:
                c["seqs"] //= 2
            else:
                c["tokens"] = c["tokens"] // 2 + 1
                c["keys"] = c["keys"] * 3 // 4 + 1
        return c
    c["rot"] = rng.choice([dim, dim, dim // 2, dim // 4, dim // 8 * 3])
    c["layout"] = rng.choice(["half", "pairs"])
    c["tokens"] = rng.choice([1, _spread(rng, 2, 4000)])
    c["start"] = rng.choice([0, _spread(rng, 1, 1000000)])
    c["scaling"] = rng.choice(["none", "linear", "base", "parts"])
    c["factor"] = 1.0 if c["scaling"] == "none" else rng.choice([2.0, 4.0, 8.0, 40.0])
    c["original"] = rng.choice([2048, 4096, 8192])
    if c["rot"] % 4 == 0 and rng.random() < 0.3:
        c["grid"] = _spread(rng, 8, 65)
    if kind == "rotate":
        c["back"] = rng.random() < 0.3
    else:
        c["norm"] = rng.choice(["rms", "layer"])
    most = 4.0e8 if c["dtype"] == "bf16" else 2.0e8
    while c["seqs"] * c["tokens"] * (c["heads"] + 2 * c["kv"]) * dim > most:
        c["seqs"] = c["seqs"] // 2 + (c["seqs"] == 1)
        c["tokens"] = c["tokens"] * 3 // 4 + 1
    return c


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _lengths(case, most):
    """Tokens of each sequence: all, or from all of them down, the last of three or more empty."""
    n = case["seqs"]
    if not case["ragged"]:
        return [most] * n
    got = [most - i * most // n for i in range(n)]
    if n > 2:
        got[-1] = 0
    return got


def _frequencies(case):
    R = case["rot"]
    d = R // 2 if case["grid"] else R
    i = torch.arange(d // 2, dtype=torch.float64)
    s, base = case["factor"], BASE
    if case["scaling"] == "base" and d > 2:
        base *= s ** (d / (d - 2))
    f = base ** (-2 * i / d)
    if case["scaling"] == "linear":
        f = f / s
    if case["scaling"] == "parts":
        g = ((case["original"] * f / (2 * math.pi) - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * (g + (1 - g) / s)
    return torch.cat((f, f)) if case["grid"] else f


def _amplitude(case):
    return 0.1 * math.log(case["factor"]) + 1 if case["scaling"] == "parts" else 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    S, H, KV, T, D = (case[x] for x in ("seqs", "heads", "kv", "tokens", "dim"))
    dt = _type(case)
    st = {"case": dict(case)}
    # channels of uneven size in keys, as models have them, and values with a mean
    gain = torch.exp(0.5 * normal(KV, D))
    st["lens"] = torch.tensor(_lengths(case, T), dtype=torch.int32, device="cuda")
    if case["kind"] == "cross":
        qgain = (1.5 / gain).repeat_interleave(H // KV, 0)
        st["q"] = (normal(S, T, H, D) * qgain).to(dt)
        st["k"] = (normal(S, KV, case["keys"], D) * gain[:, None]).to(dt)
        st["v"] = (normal(S, KV, case["keys"], D) + 0.5 * normal(KV, 1, D)).to(dt)
        # queries and keys do not end together: the longest prompt need not have the most keys
        st["klens"] = torch.tensor(_lengths(case, case["keys"])[::-1] if not case["causal"] else
                                   _lengths(case, case["keys"]), dtype=torch.int32, device="cuda")
        st["out"] = torch.zeros(S, T, H, D, dtype=torch.float32 if case["single"] else dt,
                                device="cuda")
        st["lse"] = torch.zeros(S, H, T, device="cuda")
        if case["single"]:
            st["lens"].fill_(1)
        return st
    # each sequence at a place of its own; on a grid rows and columns
    t = torch.arange(T, device="cuda") + torch.arange(S, device="cuda")[:, None] * 3
    if case["grid"]:
        t = t + case["start"] % 4000
        pos = torch.stack((t // case["grid"], t % case["grid"]))
    else:
        pos = (t + case["start"])[None]
    st["pos"] = pos.to(torch.int32).contiguous()
    st["freq"] = _frequencies(case).cuda()
    if case["kind"] == "rotate":
        st["x"] = normal(S, T, H, D).to(dt)
        st["out"] = torch.zeros_like(st["x"])
        return st
    x = normal(S, T, H + 2 * KV, D)
    x[:, :, H:H + KV] *= gain
    st["x"] = x.to(dt)
    for name in ("qw", "kw"):
        st[name] = (1 + 0.2 * normal(D)).to(dt)
    if case["norm"] == "layer":
        st["qb"], st["kb"] = (0.1 * normal(D)).to(dt), (0.1 * normal(D)).to(dt)
    st["q"] = torch.zeros(S, T, H, D, dtype=dt, device="cuda")
    st["k"] = torch.zeros(S, KV, T, D, dtype=dt, device="cuda")
    st["v"] = torch.zeros_like(st["k"])
    return st


# ---------------------------------------------------------------------------------------------
# plain forms, 32 bits (angles 64)
# ---------------------------------------------------------------------------------------------
def _turned(st, x):
    """x [S, T, heads, D] fp32 -> rotated."""
    case = st["case"]
    R = case["rot"]
    pos = st["pos"].double()
    if case["grid"]:
        half = st["freq"].numel() // 2
        angle = torch.cat((pos[0, :, :, None] * st["freq"][:half], pos[1, :, :, None] * st["freq"][half:]), -1)
    else:
        angle = pos[0, :, :, None] * st["freq"]
    amp = _amplitude(case)
    cos, sin = ((amp * f(angle)).float()[:, :, None] for f in (torch.cos, torch.sin))
    if case.get("back"):
        sin = -sin
    y, rest = x[..., :R], x[..., R:]
    if case["layout"] == "half":
        a, b = y[..., :R // 2], y[..., R // 2:]
        return torch.cat((a * cos - b * sin, a * sin + b * cos, rest), -1)
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.cat((torch.stack((a * cos - b * sin, a * sin + b * cos), -1).flatten(-2), rest), -1)


def _normed(st, x, which):
    w = st[which + "w"].float()
    if st["case"]["norm"] == "rms":
        return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w + st[which + "b"].float()


def _live(st):
    T = st["case"]["tokens"]
    return torch.arange(T, device="cuda") < st["lens"][:, None]      # [S, T]


def _put(to, new, live):
    """Rows that count are written, the others stay as they were."""
    to.copy_(torch.where(live, new.to(to.dtype), to))


def _rotate_plain(st):
    _put(st["out"], _turned(st, st["x"].float()), _live(st)[:, :, None, None])


def _prepare_plain(st):
    H, KV = st["case"]["heads"], st["case"]["kv"]
    x, live = st["x"].float(), _live(st)
    _put(st["q"], _turned(st, _normed(st, x[:, :, :H], "q")), live[:, :, None, None])
    _put(st["k"], _turned(st, _normed(st, x[:, :, H:H + KV], "k")).transpose(1, 2), live[:, None, :, None])
    _put(st["v"], x[:, :, H + KV:].transpose(1, 2), live[:, None, :, None])


def _cross_plain(st):
    case = st["case"]
    S, H, KV, T, N, D = (case[x] for x in ("seqs", "heads", "kv", "tokens", "keys", "dim"))
    q = st["q"].float().view(S, T, KV, H // KV, D).permute(0, 2, 3, 1, 4)       # [S, KV, g, T, D]
    x = torch.matmul(q.reshape(S, KV, -1, D), st["k"].float().transpose(-1, -2)) / math.sqrt(D)
    x = x.view(S, KV, H // KV, T, N)
    j = torch.arange(N, device="cuda")
    mask = (j < st["klens"][:, None])[:, None]                                  # [S, 1, N]
    if case["causal"]:
        i = torch.arange(T, device="cuda")[None, :, None] + (st["klens"] - st["lens"])[:, None, None]
        mask = mask & (j <= i)
    x.masked_fill_(~mask[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = x.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    lse = (m + torch.log(total)).view(S, H, T)
    o = torch.matmul(e.view(S, KV, -1, N), st["v"].float()).view(S, KV, H // KV, T, D)
    o = (o / torch.where(total > 0, total, 1.0)).permute(0, 3, 1, 2, 4).reshape(S, T, H, D)
    live = _live(st)
    _put(st["out"], o, live[:, :, None, None])
    _put(st["lse"], lse, live[:, None])


# ---------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------
def _handle(st):
    """What a user's program keeps between calls: config, rotation, views, workspace."""
    if "handle" in st:
        return st["handle"]
    from paper_2605_20600_gb300 import hkv as H
    case = st["case"]
    cfg = H.make_config(n_layers=1, n_seqs=case["seqs"], n_heads=case["heads"], head_dim=case["dim"],
                        dtype=case["dtype"], n_cond=0, n_image=1, row_len=1, recent_w=1, local_w=1,
                        period=1, group_at=1, global_budget=1)
    h = {"H": H, "cfg": cfg, "stream": torch.cuda.current_stream().cuda_stream}
    lens = st["lens"] if case["ragged"] else None
    if case["kind"] == "cross":
        h["tokens"] = H.make_tokens(case["tokens"], None if case["single"] else lens)
        h["states"] = H.make_states(st["k"], st["v"], st["klens"])
        h["q"], h["out"] = H.make_rows(st["q"]), H.make_rows(st["out"])
        h["flags"] = H.HKV_ATTN_CAUSAL if case["causal"] else 0
        h["ws_bytes"] = H.hkv_cross_workspace_size(cfg, h["states"], h["tokens"])
        h["ws"] = torch.zeros(h["ws_bytes"], dtype=torch.uint8, device="cuda")
    else:
        h["tokens"] = H.make_tokens(case["tokens"], lens, st["pos"])
        rot = case["rot"]
        h["rope"] = H.hkv_make_rope(
            head_dim=case["dim"], rot_dim=rot,
            layout=H.HKV_ROPE_HALF if case["layout"] == "half" else H.HKV_ROPE_PAIRS,
            sections=(rot // 4, rot // 4) if case["grid"] else (rot // 2,), base=BASE,
            scaling={"none": H.HKV_ROPE_PLAIN, "linear": H.HKV_ROPE_LINEAR, "base": H.HKV_ROPE_BASE,
                     "parts": H.HKV_ROPE_PARTS}[case["scaling"]],
            factor=case["factor"], original=case["original"], low=LOW, high=HIGH,
            amplitude=_amplitude(case))
        if case["kind"] == "rotate":
            h["x"], h["out"] = H.make_rows(st["x"]), H.make_rows(st["out"])
            h["flags"] = H.HKV_ROPE_BACK if case["back"] else 0
        else:
            n, kv = case["heads"], case["kv"]
            h["norm"] = H.make_norm(H.HKV_NORM_RMS if case["norm"] == "rms" else H.HKV_NORM_LAYER, EPS,
                                    st["qw"], st["kw"], st.get("qb"), st.get("kb"))
            x = st["x"]
            h["qkv"] = [H.make_rows(y) for y in (x[:, :, :n], x[:, :, n:n + kv], x[:, :, n + kv:])]
            h["outs"] = [H.make_rows(st["q"])] + [H.make_rows(st[y].transpose(1, 2)) for y in "kv"]
    st["handle"] = h
    return h


def _run_own(st):
    h, kind = _handle(st), st["case"]["kind"]
    H, cfg, stream = h["H"], h["cfg"], h["stream"]
    if kind == "rotate":
        H.hkv_rope_rotate(cfg, h["rope"], h["tokens"], h["x"], h["out"], flags=h["flags"], stream=stream)
    elif kind == "prepare":
        H.hkv_qk_norm_rope(cfg, h["norm"], h["rope"], h["tokens"], *h["qkv"], *h["outs"], stream=stream)
    else:
        H.hkv_cross_attention(cfg, h["states"], h["tokens"], h["q"], h["out"], st["lse"], h["ws"],
                              h["ws_bytes"], flags=h["flags"], stream=stream)


def run(st):
    kind = st["case"]["kind"]
    if own:
        _run_own(st)
    else:
        {"rotate": _rotate_plain, "prepare": _prepare_plain, "cross": _cross_plain}[kind](st)
    if kind == "rotate":
        return st["out"]
    if kind == "prepare":
        return {"q": st["q"], "k": st["k"], "v": st["v"]}
    return {"out": st["out"], "lse": st["lse"]}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------
def _rotated64(case, row, positions):
    """One sequence's rows [T, heads, D] in 64 bits, pair by pair, as complex numbers turned."""
    R, n = case["rot"], case["rot"] // 2
    out = row.clone()
    for i in range(n):
        axis, j, d = (i // (n // 2), i % (n // 2), R / 2) if case["grid"] else (0, i, R)
        s, theta = case["factor"], 1.0
        if case["scaling"] == "base" and d > 2:
            theta = (BASE * s ** (d / (d - 2))) ** (-2.0 * j / d)
        else:
            theta = BASE ** (-2.0 * j / d)
        if case["scaling"] == "linear":
            theta = theta / s
        elif case["scaling"] == "parts":
            turns = case["original"] * theta / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - LOW) / (HIGH - LOW)))
            theta = (1 - keep) * theta / s + keep * theta
        a, b = (i, i + n) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.polar(torch.full_like(positions[axis], _amplitude(case)),
                        positions[axis] * (-theta if case.get("back") else theta))[:, None]
        turned = torch.complex(row[..., a], row[..., b]) * z
        out[..., a], out[..., b] = turned.real, turned.imag
    return out


def exact(case, seed):
    st = prepare(case, seed)
    S, H, KV = case["seqs"], case["heads"], case["kv"]
    lens = st["lens"].tolist()
    if case["kind"] == "cross":
        out, lse = st["out"].double(), st["lse"].double()
        klens = st["klens"].tolist()
        for s in range(S):
            n, m = lens[s], klens[s]
            if n == 0:
                continue
            for h in range(H):
                q = st["q"][s, :n, h].double()
                k, v = (st[x][s, h * KV // H, :m].double() for x in "kv")
                if m == 0:
                    out[s, :n, h], lse[s, h, :n] = 0.0, -math.inf
                    continue
                x = (q @ k.T) * case["dim"] ** -0.5
                if case["causal"]:
                    x += torch.full_like(x, -math.inf).triu(1 + m - n)
                lse[s, h, :n] = torch.logsumexp(x, -1)
                w = torch.exp(x - lse[s, h, :n, None])
                out[s, :n, h] = torch.where(torch.isneginf(lse[s, h, :n, None]), 0.0, w) @ v
        return {"out": out, "lse": lse}
    pos = st["pos"].double()

    def head_norm(x, which):
        scale = st[which + "w"].double()
        if case["norm"] == "layer":
            var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
            return (x - mean) / torch.sqrt(var + EPS) * scale + st[which + "b"].double()
        return x / torch.sqrt(x.square().sum(-1, keepdim=True) / case["dim"] + EPS) * scale

    if case["kind"] == "rotate":
        out = st["out"].double()
        for s in range(S):
            out[s, :lens[s]] = _rotated64(case, st["x"][s, :lens[s]].double(), pos[:, s, :lens[s]])
        return out
    got = {x: st[x].double() for x in "qkv"}
    for s in range(S):
        n = lens[s]
        x = st["x"][s, :n].double()
        got["q"][s, :n] = _rotated64(case, head_norm(x[:, :H], "q"), pos[:, s, :n])
        got["k"][s, :, :n] = _rotated64(case, head_norm(x[:, H:H + KV], "k"), pos[:, s, :n]).transpose(0, 1)
        got["v"][s, :, :n] = x[:, H + KV:].transpose(0, 1)
    return got


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
def work(case):
    S, H, KV, D = case["seqs"], case["heads"], case["kv"], case["dim"]
    es = 2 if case["dtype"] == "bf16" else 4
    lens = [1] * S if case.get("single") else _lengths(case, case["tokens"])
    rows = sum(lens)
    if case["kind"] != "cross":
        axes = 2 if case["grid"] else 1
        pairs = case["rot"] // 2
        if case["kind"] == "rotate":
            return {"bytes": rows * (2.0 * H * D * es + 4 * axes), "flops": 6.0 * rows * H * pairs}
        return {"bytes": rows * (2.0 * (H + 2 * KV) * D * es + 4 * axes),
                "flops": rows * (H + KV) * (6.0 * pairs + 5.0 * D)}
    klens = _lengths(case, case["keys"])
    if not case["causal"]:
        klens = klens[::-1]
    seen, read = 0, 0
    for n, m in zip(lens, klens):
        if case["causal"]:
            # query i sees i + 1 + m - n keys, none where that is not positive
            first, last = max(1, m - n + 1), m
            seen += (first + last) * (last - first + 1) // 2 if n else 0
        else:
            seen += n * m
        read += m if n else 0
    out = D * (4 if case["single"] else es) + 4
    return {"bytes": float(rows * H * (D * es + out) + read * KV * 2 * D * es),
            "flops": 4.0 * D * H * seen}
