"""Schedule driver over the HeadKV C-ABI.

Owns the device buffers (allocated with torch, which serves only as the
memory and stream provider) and sequences the calls of one image generation
(Sec. 4): Step 1 cache prefilling into an uncompressed cache, Step 2 head
grouping at image token E-1, Step 3 head-aware compression (budgets, arena
allocation, repack), then decode steps of append/evict + attention. After
compression the cache may be quantised (Engine.quantise): the decode steps
and updates then run on codes, and conditioning tokens that all sequences
share may be kept once, outside the cache. All compute runs in libheadkv.so
kernels.
"""
from __future__ import annotations

import copy

import torch

from . import hkv as H

_TORCH_DTYPE = {H.HKV_FP32: torch.float32, H.HKV_BF16: torch.bfloat16}


def torch_dtype(cfg: H.hkv_config) -> torch.dtype:
    return _TORCH_DTYPE[cfg.dtype]


class CacheBuffers:
    """Device buffers behind one hkv_cache (layout documented in hkv.h)."""

    def __init__(self, cfg: H.hkv_config, capacity_tokens: int, device, *, qbuf=None, label=None,
                 off=None, cap=None):
        n = cfg.n_layers * cfg.n_seqs * cfg.n_heads
        D, dt = cfg.head_dim, torch_dtype(cfg)
        self.k = torch.empty(max(capacity_tokens, 1), D, dtype=dt, device=device)
        self.v = torch.empty(max(capacity_tokens, 1), D, dtype=dt, device=device)
        self.pos = torch.full((max(capacity_tokens, 1),), -1, dtype=torch.int32, device=device)
        self.off = off if off is not None else torch.zeros(n, dtype=torch.int64, device=device)
        self.cap = cap if cap is not None else torch.zeros(n, dtype=torch.int32, device=device)
        self.len = torch.zeros(n, dtype=torch.int32, device=device)
        self.nbuf = torch.zeros(n, dtype=torch.int32, device=device)
        self.ntok = torch.zeros(n, dtype=torch.int32, device=device)
        self.label = label if label is not None else torch.full((n,), H.HKV_DENSE, dtype=torch.uint8,
                                                                 device=device)
        self.qbuf = qbuf if qbuf is not None else torch.zeros(n, cfg.period, D, dtype=dt, device=device)
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.capacity_tokens = capacity_tokens
        self.c = H.hkv_cache(self.k.data_ptr(), self.v.data_ptr(), self.pos.data_ptr(),
                             self.off.data_ptr(), self.cap.data_ptr(), self.len.data_ptr(),
                             self.nbuf.data_ptr(), self.ntok.data_ptr(), self.label.data_ptr(),
                             self.qbuf.data_ptr(), self.err.data_ptr(), capacity_tokens)


class QuantCacheBuffers:
    """Device buffers behind one hkv_qcache (layout documented in hkv_serve.h)."""

    def __init__(self, cfg: H.hkv_config, fmt: int, capacity_tokens: int, device, *, qbuf, label,
                 off, cap):
        n = cfg.n_layers * cfg.n_seqs * cfg.n_heads
        D, rows = cfg.head_dim, max(capacity_tokens, 1)

        def arena(width, dt):
            return torch.empty(rows, width, dtype=dt, device=device)

        self.k, self.v = arena(D * fmt // 8, torch.uint8), arena(D * fmt // 8, torch.uint8)
        self.ks, self.vs = arena(D // 32, torch.bfloat16), arena(D // 32, torch.bfloat16)
        self.pos = torch.full((rows,), -1, dtype=torch.int32, device=device)
        self.off, self.cap, self.label, self.qbuf = off, cap, label, qbuf
        self.len, self.nbuf, self.ntok = (torch.zeros(n, dtype=torch.int32, device=device)
                                          for _ in range(3))
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.capacity_tokens = capacity_tokens
        self.c = H.make_qcache(fmt, self.k, self.v, self.ks, self.vs, self.pos, self.off, self.cap,
                               self.len, self.nbuf, self.ntok, self.label, self.qbuf, self.err,
                               capacity_tokens)


class Engine:
    """One batch of sequences through the HeadKV decode path."""

    def __init__(self, cfg: H.hkv_config, device="cuda"):
        H.hkv_validate_config(cfg)
        self.cfg = cfg
        self.device = torch.device(device)
        self.n = cfg.n_layers * cfg.n_seqs * cfg.n_heads
        seg = cfg.n_cond + cfg.group_at
        self.dense = CacheBuffers(cfg, self.n * seg, self.device)
        self.labels = torch.full((self.n,), H.HKV_DENSE, dtype=torch.uint8, device=self.device)
        self.n_h = torch.zeros(self.n, dtype=torch.int32, device=self.device)
        self.ws_bytes = H.hkv_workspace_size(cfg)
        self.ws = torch.zeros(self.ws_bytes, dtype=torch.uint8, device=self.device)
        self.ragged: CacheBuffers | None = None
        self.budget = self.cap = self.off = None
        self.total_tokens = 0
        self.quant: QuantCacheBuffers | None = None
        self.prompt = None            # shared prompts: one hkv_prefix per layer
        H.hkv_init_dense(cfg, self.dense.c, self.stream())
        self.cache = self.dense

    @staticmethod
    def stream() -> int:
        return torch.cuda.current_stream().cuda_stream

    # Step 1
    def prefill(self, layer: int, kc, vc) -> None:
        H.hkv_prefill(self.cfg, self.dense.c, layer, kc, vc, self.stream())

    def _plain(self, name: str) -> None:
        if self.quant is not None:     # calls that have no form for codes
            raise H.HkvError(name, H.HKV_ERR_STATE)

    # per decode step and layer
    def append(self, layer: int, q, k, v) -> None:
        self._plain("append_evict")
        H.hkv_append_evict(self.cfg, self.cache.c, layer, q, k, v, self.stream())

    def attend(self, layer: int, q, out) -> None:
        self._plain("decode_attention")
        H.hkv_decode_attention(self.cfg, self.cache.c, layer, q, out, self.ws, self.ws_bytes,
                               self.stream())

    # fused path: the update when due, then append + attention in one launch
    def evict(self, layer: int) -> None:
        if self.quant is not None:
            H.hkv_quant_evict(self.quant_cfg, self.quant.c, layer, self.stream())
            return
        H.hkv_evict(self.cfg, self.cache.c, layer, self.stream())

    def evict_all(self) -> None:
        """The periodic update of every layer in one launch."""
        if self.quant is not None:
            H.hkv_quant_evict_all(self.quant_cfg, self.quant.c, self.stream())
            return
        H.hkv_evict_all(self.cfg, self.cache.c, self.stream())

    def step(self, layer: int, q, k, v, out) -> None:
        # layers run in order, so with two or more layers the kernel before a
        # decode step belongs to another layer (or is hkv_evict, which never
        # lets its successor start early): the step may prefetch
        flags = H.HKV_STEP_PREFETCH if self.cfg.n_layers >= 2 else 0
        if self.quant is not None:
            self._quant_step(layer, q, k, v, out, flags)
            return
        H.hkv_decode_step(self.cfg, self.cache.c, layer, q, k, v, out, self.ws, self.ws_bytes,
                          flags, self.stream())

    def update_due(self, t: int) -> bool:
        """Whether image token t's step starts with the periodic update
        (decided by the library, hkv_update_due)."""
        return H.hkv_update_due(self.cfg, t)

    # Step 2
    def step_identify(self, layer: int, q, k, v, out) -> None:
        """The decode step of the grouping token with the head types (Sec. 4,
        Step 2) decided in the same pass, into self.labels (no n_h)."""
        self._plain("decode_step_identify")
        flags = H.HKV_STEP_PREFETCH if self.cfg.n_layers >= 2 else 0
        H.hkv_decode_step_identify(self.cfg, self.cache.c, layer, q, k, v, out, self.labels, self.ws,
                                   self.ws_bytes, flags, self.stream())

    def identify(self, layer: int, q) -> None:
        H.hkv_identify_heads(self.cfg, self.dense.c, layer, q, self.labels, self.n_h, self.stream())

    def identify_multi(self, layer: int) -> None:
        """Step 2 from the ring's recent queries (a variant the paper does not
        have): labels and n_h."""
        H.hkv_identify_heads_multi(self.cfg, self.dense.c, layer, self.labels, self.n_h, self.stream())

    # Step 3: budgets, arena, repack of every layer
    def compress(self, labels=None) -> None:
        if labels is not None:
            self.labels.copy_(labels)
        dev = self.device
        self.budget = torch.empty(self.n, dtype=torch.int32, device=dev)
        self.cap = torch.empty(self.n, dtype=torch.int32, device=dev)
        self.off = torch.empty(self.n, dtype=torch.int64, device=dev)
        self.total_tokens = H.hkv_allocate_budgets(self.cfg, self.labels, self.budget, self.cap,
                                                   self.off, self.stream())
        self.ragged = CacheBuffers(self.cfg, self.total_tokens, dev, qbuf=self.dense.qbuf,
                                   label=self.labels, off=self.off, cap=self.cap)
        for layer in range(self.cfg.n_layers):
            H.hkv_repack(self.cfg, self.dense.c, self.ragged.c, layer, self.stream())
        self.cache = self.ragged

    # the serving cache
    def quantise(self, fmt: int, prompt=None) -> None:
        """Puts the compressed cache into 8 or 4 bits (HKV_Q8 or HKV_Q4) and
        frees its plain rows; decode steps and updates run on the codes from
        here on. prompt: None, or (k, v), [L][groups][H][C][head_dim] tensors
        in the config dtype of the conditioning tokens that each of `groups`
        equal runs of sequences shares; they then stay plain and are kept once
        instead of in every sequence's segments. Synchronises the stream: an
        error leaves the engine as it was, on its plain rows."""
        if self.ragged is None or self.quant is not None:
            raise H.HkvError("quantise", H.HKV_ERR_STATE)
        cfg, dev = self.cfg, self.device
        off, cap, total = self.off, self.cap, self.total_tokens
        flags = 0
        quant_cfg = copy.copy(cfg)
        if prompt is not None:
            k, v = prompt
            shape = (cfg.n_layers, k.shape[1] if k.dim() == 5 else 0, cfg.n_heads, cfg.n_cond,
                     cfg.head_dim)
            if k.shape != shape or v.shape != shape or cfg.n_cond < 1 or shape[1] < 1 \
                    or cfg.n_seqs % shape[1] != 0 or not k.dtype == v.dtype == torch_dtype(cfg):
                raise H.HkvError("quantise", H.HKV_ERR_SHAPE)
            if not k.device == v.device == self.labels.device:
                raise H.HkvError("quantise", H.HKV_ERR_INVALID_ARG)
            quant_cfg.n_cond = 0
            off, cap = torch.empty_like(off), torch.empty_like(cap)
            total = H.hkv_allocate_budgets(quant_cfg, self.labels, torch.empty_like(self.budget),
                                           cap, off, self.stream())
            flags = H.HKV_PACK_SKIP_COND
        quant = QuantCacheBuffers(cfg, fmt, total, dev, qbuf=self.ragged.qbuf, label=self.labels,
                                  off=off, cap=cap)
        ws_bytes = H.hkv_quant_workspace_size(quant_cfg)
        ws = torch.zeros(ws_bytes, dtype=torch.uint8, device=dev)
        if prompt is not None:
            prompt_len = torch.full((shape[1],), cfg.n_cond, dtype=torch.int32, device=dev)
            prefixes = [H.make_prefix(k[layer], v[layer], prompt_len, quant.err)
                        for layer in range(cfg.n_layers)]
            prompt_ws_bytes = min(H.hkv_prefix_workspace_size(cfg, p) for p in prefixes)
            if prompt_ws_bytes == 0:       # strides or alignment the attention does not take
                raise H.HkvError("quantise", H.HKV_ERR_SHAPE)
            prompt_ws = torch.zeros(prompt_ws_bytes, dtype=torch.uint8, device=dev)
            prior = (torch.empty(cfg.n_seqs, cfg.n_heads, cfg.head_dim, dtype=torch.float32, device=dev),
                     torch.empty(cfg.n_seqs, cfg.n_heads, dtype=torch.float32, device=dev))
        H.hkv_quant_pack(cfg, self.ragged.c, quant.c, H.HKV_ALL_LAYERS, flags, self.stream())
        H.hkv_quant_check(quant.c, self.stream())     # every head is in, or nothing changes
        if prompt is not None:
            self.prompt, self.prompt_ws_bytes, self.prompt_ws = prefixes, prompt_ws_bytes, prompt_ws
            self.prior = prior
        self.quant_cfg, self.quant_ws_bytes, self.quant_ws = quant_cfg, ws_bytes, ws
        self.off, self.cap, self.total_tokens = off, cap, total
        self.cache = self.quant = quant
        self.ragged.k = self.ragged.v = self.ragged.pos = None

    def _quant_step(self, layer: int, q, k, v, out, flags: int) -> None:
        prior = None
        if self.prompt is not None:
            prior = self.prior
            H.hkv_prefix_attention(self.cfg, self.prompt[layer], q, prior[0], prior[1],
                                   self.prompt_ws, self.prompt_ws_bytes, self.stream())
        H.hkv_quant_step(self.quant_cfg, self.quant.c, layer, q, k, v, out, self.quant_ws,
                         self.quant_ws_bytes, prior=prior, flags=flags, stream=self.stream())

    def release_dense(self) -> None:
        """Frees the uncompressed arena once the ragged cache holds everything."""
        self.dense.k = self.dense.v = self.dense.pos = None

    def check(self) -> None:
        if self.quant is not None:
            H.hkv_quant_check(self.quant.c, self.stream())
        if self.ragged is not None:
            H.hkv_check(self.ragged.c, self.stream())
        H.hkv_check(self.dense.c, self.stream())
