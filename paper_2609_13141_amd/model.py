"""A decoder stack served with SAS (Sec. 5.1, Alg. 2), over the C ABI.

The prompt is prefilled densely through every layer, which fills each
layer's paged KV cache and block summaries; every generated token is then
embedded, runs the SAS decode step in each layer (Top-K blocks per KV group
by the selector, attention to them plus the current block without gate bias)
and the greedy LM head (final RMSNorm, logits in fp32, lowest id on ties).
Sequences may also take several new tokens at once over what is cached (a piece
of a long prompt, drafted tokens): ``extend``, a dense chunk in every layer.
Every step runs in the library's kernels; this module only sequences them.
"""
from __future__ import annotations

import torch

from . import sas
from .configs import Workload


class Stack:
    def __init__(self, w: Workload, layers: list, ends: dict, *, max_len: int, page_size: int | None = None,
                 device="cuda", packed: bool = True):
        """layers: per-layer device weight dicts; ends: device tensors
        'embed' [V, d], 'w_lm' [V, d], 'rms_final' [d].  packed: the decode
        steps stream a packed copy of each layer's linear weights (made here
        when the configuration has a packed layout; results are identical)."""
        self.w = w
        self.ends = ends
        self.device = device
        self.cfg_prefill = sas.make_config(w, "dense")
        self.cfg_decode = sas.make_config(w, "sparse")
        if packed and sas.lib().sas_decode_packed_bytes(sas.C.byref(self.cfg_decode)) > 0:
            layers = [sas.pack_decode_weights(self.cfg_decode, W) for W in layers]
        self.layers = layers
        ps = page_size or w.page_size
        self.caches = [sas.alloc_cache(self.cfg_decode, w.batch, max_len, page_size=ps, device=device, seed=l)
                       for l in range(len(layers))]
        self.ws = sas.Workspace(device)
        self.max_len = max_len
        self.pos = None     # cached tokens of every sequence: a number, after extend a device tensor [b]

    def prefill(self, ids, img=None, *, logits: bool = False, on_layer=None):
        """ids [b, n] int32 on the device (-1 = next image embedding row);
        returns the first generated token of every sequence [b] int32 (and
        its fp32 logits when asked).  on_layer(l, x), when given, sees the
        input x [b, n, d] of every layer l and the last layer's output (l = L)."""
        x = sas.embed(self.cfg_prefill, ids, self.ends["embed"], img)
        for l, (W, cache) in enumerate(zip(self.layers, self.caches)):
            if on_layer is not None:
                on_layer(l, x)
            x = sas.layer_forward(self.cfg_prefill, x, W, stats=False, cache=cache, ws=self.ws)["y"]
        if on_layer is not None:
            on_layer(len(self.layers), x)
        self.pos = ids.shape[1]
        tok, lg = sas.lm_head_argmax(self.cfg_decode, x[:, -1].contiguous(), self.ends["rms_final"],
                                     self.ends["w_lm"], logits=logits, ws=self.ws)
        return (tok, lg) if logits else tok

    def positions(self, steps: int):
        """Device position vectors for the next `steps` decode steps, behind the prompt,
        the last `extend` and the steps since.  (A replayed graph moves nothing here, and
        after drafts that were not accepted the lengths are the caller's to know.)"""
        b = self.w.batch
        if isinstance(self.pos, torch.Tensor):
            return [self.pos + s for s in range(steps)]
        return [torch.full((b,), self.pos + s, dtype=torch.int32, device=self.device) for s in range(steps)]

    def step(self, tok, pos, *, logits: bool = False, sel_idx: bool = False, taps: bool = False):
        """One generated token per sequence: tok [b] at positions pos [b]
        (device int32).  Returns the next tokens, the logits and per-layer
        selections when asked, and with taps a per-layer list of
        {"x": layer input, "q", "k", "v", "h1", "y": layer output}."""
        x = sas.embed(self.cfg_decode, tok.view(-1, 1), self.ends["embed"])[:, 0].contiguous()
        sels, tps = [], []
        for W, cache in zip(self.layers, self.caches):
            r = sas.decode_step(self.cfg_decode, x, pos, W, cache, sel_idx=sel_idx, taps=taps, ws=self.ws)
            if taps:
                r[2]["x"] = x
                r[2]["y"] = r[0]
                tps.append(r[2])
            x, sel = r[0], r[1]
            sels.append(sel)
        nxt, lg = sas.lm_head_argmax(self.cfg_decode, x, self.ends["rms_final"], self.ends["w_lm"], logits=logits,
                                     ws=self.ws)
        self.pos = self.pos + 1
        out = (nxt, lg, (sels if sel_idx else None))
        return out + (tps,) if taps else out

    def extend(self, ids, ctx_len, new_len):
        """New tokens of every sequence, any number each, over the caches: ids
        [rows] int32, sequence i's new_len[i] after each other at positions
        ctx_len[i] .. (ctx_len, new_len [b] int32, all on the device; rows past
        their sum are padding; tokens past the rows wait for another call, those at
        positions from max_len on have no page and leave no key).  Returns the last
        layer's output [rows, d] and the rows' plan (see sas.plan_chunk): kv_len, the
        lengths after the call, are where the next tokens go."""
        x = sas.embed(self.cfg_prefill, ids.view(1, -1), self.ends["embed"])[0]
        none = torch.zeros(1, dtype=torch.int32, device=ids.device)
        plan = None
        # (every position's page is there already, in another order in each layer)
        held = torch.full_like(ctx_len, self.caches[0].block_table.shape[1])
        for W, cache in zip(self.layers, self.caches):
            plan = sas.plan_chunk(cache, ctx_len, new_len, held, none, none, ids.numel())
            x = sas.layer_chunk(self.cfg_prefill, x, W, cache, ctx_len, plan, ws=self.ws)
        self.pos = plan["kv_len"].clone()
        return x, plan

    def logits(self, x):
        """fp32 logits [rows, V] of hidden rows x [rows, d], 16 at a time (the LM head's rows)."""
        return torch.cat([sas.lm_head_argmax(self.cfg_decode, r.contiguous(), self.ends["rms_final"], self.ends["w_lm"],
                                             logits=True, ws=self.ws)[1] for r in x.split(16)])

    def generate(self, ids, img, steps: int):
        """Greedy generation: [b, steps + 1] tokens (the prefill's and `steps` more)."""
        tok = self.prefill(ids, img)
        out = [tok]
        for pos in self.positions(steps):
            tok, _, _ = self.step(tok, pos)
            out.append(tok)
        return torch.stack(out, 1)
