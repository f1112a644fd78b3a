"""Drives one full image generation through the Engine (Sec. 4 Steps 1-3 and
the decode loop), taking per-step inputs from a provider object with

    provider.cond(kc, vc, layer, stream)                 # kc/vc [S][H][C][D]
    provider.image(q, k, v, l0, nl, t0, nt, stream)     # [nt][nl][S][H][D]

and handing each step's attention outputs to an optional callback.
"""
from __future__ import annotations

import torch

from .engine import Engine, Heads, torch_dtype


def generate(engine: Engine, provider, *, last_step: int | None = None, on_step=None,
             before_compress=None, fused: bool = True, first_step: int = 0,
             identify: str | None = None, cache_format: int | None = None,
             shared_prompt: int = False, heads: Heads | None = None) -> None:
    """Runs image tokens first_step..last_step (default N-1) for every layer.

    fused: hkv_evict_all (every layer in one launch) when the update is due,
    then hkv_decode_step per layer; otherwise hkv_append_evict then
    hkv_decode_attention per layer.
    on_step(t, out) receives out [L][S][H][D] (fp32, device) after step t.
    before_compress(engine) runs after grouping, before budgets and repack.
    first_step > 0 continues a generation (the prefill is skipped).
    identify: "fused" decides the head types inside the grouping token's
    decode step (fused path only; no n_h), "separate" runs
    hkv_identify_heads after it (labels and n_h), "multi" runs
    hkv_identify_heads_multi after it (the recent queries' averaged
    attention; labels and n_h). Default: fused when the path is fused and
    the distances are the raster ones.
    cache_format: None keeps the compressed cache in the config dtype;
    HKV_Q8 or HKV_Q4 quantises it after compression, at the start where the
    engine continues with a compressed cache (fused path only). An engine that
    is quantised already goes on with its format.
    shared_prompt: with a cache_format, the number of prompts (True: one) of
    which each belongs to an equal run of sequences, whose conditioning tokens
    are then kept once for the run. Tokens that differ within a run raise
    ValueError: with guidance, the conditional and the unconditional sequences
    are two runs.
    heads: what the model does to queries and keys between its projections and
    the cache (norms and rotary positions); the provider's q, k and kc are then
    the projections' outputs. None: they are ready for the cache.
    """
    if cache_format is not None and not fused:
        raise ValueError("a quantised cache needs the fused path")
    if shared_prompt and (cache_format is None or first_step > 0 or engine.cfg.n_cond < 1):
        raise ValueError("a shared prompt needs a cache_format, conditioning tokens and a whole run")
    if shared_prompt and (shared_prompt < 0 or engine.cfg.n_seqs % shared_prompt != 0):
        raise ValueError(f"{engine.cfg.n_seqs} sequences are not {shared_prompt} equal runs")
    if identify is None:   # the fused count is the raster one
        identify = "fused" if fused and engine.cfg.distance_mode == 0 else "separate"
    if identify not in ("fused", "separate", "multi") or (identify == "fused" and not fused):
        raise ValueError(f"identify={identify!r} with fused={fused}")
    if identify == "fused" and engine.cfg.distance_mode != 0:
        raise ValueError("the fused identification counts in raster order only")
    cfg = engine.cfg
    L, S, H, D, C = cfg.n_layers, cfg.n_seqs, cfg.n_heads, cfg.head_dim, cfg.n_cond
    E = cfg.group_at
    dev, dt = engine.device, torch_dtype(cfg)
    st = engine.stream()
    quant = engine.quant
    if quant is not None and (not fused or cache_format not in (None, quant.c.format)):
        raise ValueError(f"the engine's cache is quantised (format {quant.c.format}): "
                         f"fused={fused}, cache_format={cache_format}")
    if cache_format is not None and quant is None and first_step >= E:
        engine.quantise(cache_format)
    if C > 0 and first_step == 0:
        kc = torch.empty(S, H, C, D, dtype=dt, device=dev)
        vc = torch.empty_like(kc)
        for layer in range(L):
            provider.cond(kc, vc, layer, st)
            if heads is not None:
                engine.prepare(heads, layer, None, kc.transpose(1, 2), 0)
            if shared_prompt:
                G = int(shared_prompt)
                if layer == 0:
                    prompt = (torch.empty(L, G, H, C, D, dtype=dt, device=dev),
                              torch.empty(L, G, H, C, D, dtype=dt, device=dev))
                for x, rows in zip((kc, vc), prompt):
                    runs = x.view(G, S // G, H, C, D)
                    bits = runs.view(torch.int16 if dt == torch.bfloat16 else torch.int32)
                    if not torch.equal(bits, bits[:, :1].expand_as(bits)):
                        raise ValueError(f"the conditioning tokens of layer {layer} differ between "
                                         f"sequences that share a prompt ({G} of {S} sequences)")
                    rows[layer].copy_(runs[:, 0])
            engine.prefill(layer, kc, vc)
    q = torch.empty(L, S, H, D, dtype=dt, device=dev)
    k, v = torch.empty_like(q), torch.empty_like(q)
    out = torch.empty(L, S, H, D, dtype=torch.float32, device=dev)
    last = cfg.n_image - 1 if last_step is None else last_step
    for t in range(first_step, last + 1):
        provider.image(q, k, v, 0, L, t, 1, st)
        due = engine.update_due(t)
        if fused and due:
            engine.evict_all()       # every layer's buffer fills at the same token
        for layer in range(L):
            if heads is not None:
                engine.prepare(heads, layer, q[layer], k[layer], C + t)
            if fused:
                if t == E - 1 and identify == "fused":
                    engine.step_identify(layer, q[layer], k[layer], v[layer], out[layer])
                else:
                    engine.step(layer, q[layer], k[layer], v[layer], out[layer])
            else:
                engine.append(layer, q[layer], k[layer], v[layer])
                engine.attend(layer, q[layer], out[layer])
            if t == E - 1 and identify == "separate":
                engine.identify(layer, q[layer])
            elif t == E - 1 and identify == "multi":
                engine.identify_multi(layer)
        if on_step is not None:
            on_step(t, out)
        if t == E - 1:
            if before_compress is not None:
                before_compress(engine)
            engine.compress()
            if cache_format is not None:
                engine.quantise(cache_format, prompt if shared_prompt else None)
