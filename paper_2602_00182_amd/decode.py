"""Greedy decode loop over libdetinfer (host orchestration only: every step runs in the library's
kernels, on one stream, with no host round trip inside the loop).

One step, for B sequences at step t (the paper's section 6.6: greedy decoding in a fixed order):
    token select -> embedding gather -> L x decoder layer -> final RMSNorm -> lm_head GEMM (fp32
    logits) -> argmax.
greedy_decode feeds prompts through the same step one token at a time; prefill_decode pushes all
prompt tokens of all sequences through each layer in one call (rows that name their cache slot) and
then decodes.  Either way a sequence's bytes are those of the single-sequence, token-by-token run,
whatever batch it sits in.

With an 8-bit paged cache (DecodeModel(..., cache8=True)) the prompts of several continuations are run once, their pages shared (`samples`) and read once
a step, long sequences may give up the pages that get little weight (`evict`), and speculative_decode lets a second model draft tokens that the first one
verifies several at a time.  `rules` come between the output head and the choice of a token: penalties, biases, a grammar's masks."""
from __future__ import annotations

import contextlib
import copy
import os
from dataclasses import dataclass

import torch

from . import api
from .pages import KVPages


@dataclass
class ModelCfg:
    H: int
    Hq: int
    Hkv: int
    D: int
    F: int
    V: int
    n_layers: int
    eps: float = 1e-5
    scale: float = 0.08838834764831845  # 1/sqrt(128)


class DecodeModel:
    """Weights of a Llama-style decoder, packed for det_gemm_bf16, or with quantized=True block-quantized
    to 4 bits and packed for det_qgemm_w4a8 (every projection, the lm_head included; embedding and norm
    weights stay bf16).  With cache8=True the keys and values are kept in 8 bits, in pages (KVPages).

    `weights` holds logical row-major bf16 tensors on the GPU:
        embed [V,H], lm_head [H,V], final_norm [H], and per layer i:
        layers[i] = dict(norm1 [H], wqkv [H,(Hq+2Hkv)D], wo [Hq*D,H], norm2 [H], wgu [H,2F], wdown [F,H])
    """

    def __init__(self, cfg: ModelCfg, weights: dict, quantized: bool = False, cache8: bool = False):
        self.cfg = cfg
        self.quantized = quantized
        self.cache8 = cache8
        pack = api.quant_pack_weight if quantized else api.pack_weight
        pack_gu = api.quant_pack_gate_up if quantized else api.pack_gate_up
        self.embed = weights["embed"].contiguous()
        self.final_norm = weights["final_norm"].contiguous()
        self.lm_head = pack(weights["lm_head"])
        self.layers = []
        for lw in weights["layers"]:
            wqkv = pack(lw["wqkv"]) if cache8 else (api.quant_pack_qkv if quantized else api.pack_qkv)(lw["wqkv"], cfg.Hq, cfg.Hkv, cfg.D)
            packed = dict(norm1=lw["norm1"].contiguous(), wqkv=wqkv,
                          wo=pack(lw["wo"]), norm2=lw["norm2"].contiguous(),
                          wgu=pack_gu(lw["wgu"]), wdown=pack(lw["wdown"]))
            struct = api.layer_weights(packed["norm1"], packed["wqkv"], packed["wo"], packed["norm2"],
                                       packed["wgu"], packed["wdown"])
            self.layers.append((packed, struct))

    def layer_workspace_bytes(self, lcfg, rows: int, named: bool = False, step=None) -> int:
        """For steps of `rows` rows; named: rows that name their slots, which takes less of an 8-bit cache; step: as layer takes it."""
        if self.cache8:
            kind = "det_qdecoder_layer_kv8" if self.quantized else "det_decoder_layer_kv8"
            if step is not None:
                return getattr(api, kind + "_step_workspace_bytes")(lcfg, rows, -(-lcfg.Lmax // api.KV8_PAGE), bool(step.weights))
            size = getattr(api, kind + ("_rows_workspace_bytes" if named else "_workspace_bytes"))
            return size(lcfg, rows, -(-lcfg.Lmax // api.KV8_PAGE))
        if self.quantized:
            return api.det_qdecoder_layer_workspace_bytes(lcfg, rows)
        return api.det_decoder_layer_workspace_bytes(lcfg, rows)

    def layer(self, struct, lcfg, x, kcache, vcache, positions, slots, rope_cos, rope_sin, ws, stream=None, step=None):
        """One decoder layer on rows x; slots None: row r is the sequence in cache slot r.  With an 8-bit cache kcache is the layer's pool,
        vcache the page table, and step (api.kv8_step) may say which rows share what and where the pages' weights go."""
        if self.cache8 and step is not None:
            run = api.det_qdecoder_layer_kv8_step if self.quantized else api.det_decoder_layer_kv8_step
            run(struct, lcfg, x, kcache, vcache, positions, slots, rope_cos, rope_sin, step, ws, stream)
        elif self.cache8:
            run = api.det_qdecoder_layer_kv8 if self.quantized else api.det_decoder_layer_kv8
            run(struct, lcfg, x, kcache, vcache, positions, slots, rope_cos, rope_sin, ws, stream)
        elif self.quantized:
            api.det_qdecoder_layer(struct, lcfg, x, kcache, vcache, positions, slots, rope_cos, rope_sin, ws, stream)
        elif slots is None:
            api.det_decoder_layer(struct, lcfg, x, kcache, vcache, positions, rope_cos, rope_sin, ws, stream)
        else:
            api.det_decoder_layer_rows(struct, lcfg, x, kcache, vcache, positions, slots, rope_cos, rope_sin, ws,
                                       stream)

    def new_state(self, B: int, Lmax: int, rope_cos: torch.Tensor, rope_sin: torch.Tensor, reserve: bool = True, n_pages: int | None = None):
        return DecodeState(self, B, Lmax, rope_cos, rope_sin, reserve, n_pages)


class DecodeState:
    """KV caches, workspace and step buffers for B sequences of up to Lmax tokens.  With an 8-bit cache `pages` holds n_pages
    pages (None: room for all of them), reserved at once unless reserve is False; `groups` (the first sequence of each group, and B; None) says which
    sequences share pages that a step is to read once, and to `weights` ([B, pages of a sequence] fp32 or None) it adds what weight each page gets, over all
    layers.  What a group shares is what the pages' tables say when the step is launched, or, of a captured step, when `tell` is called."""

    def __init__(self, model: DecodeModel, B: int, Lmax: int, rope_cos, rope_sin, reserve: bool = True, n_pages: int | None = None):
        c = model.cfg
        dev = model.embed.device
        self.model, self.B, self.Lmax = model, B, Lmax
        self.lcfg = api.layer_cfg(c.H, c.Hq, c.Hkv, c.D, c.F, Lmax, c.eps, c.scale)
        if rope_cos.shape != (Lmax, c.D // 2):
            raise ValueError("rope tables must be [Lmax, D/2]")
        self.rope_cos, self.rope_sin = rope_cos, rope_sin
        if model.cache8:
            each = -(-Lmax // api.KV8_PAGE)
            self.pages = KVPages(c.n_layers, B * each if n_pages is None else n_pages, c.Hkv, B, each, c.D, dev)
            if reserve:
                self.pages.reserve(range(B), [Lmax] * B)
            self.kcache, self.vcache = list(self.pages.pool), [self.pages.table] * c.n_layers
        else:
            self.kcache = [torch.zeros((B, c.Hkv, Lmax, c.D), dtype=torch.bfloat16, device=dev)
                           for _ in range(c.n_layers)]
            self.vcache = [torch.zeros_like(k) for k in self.kcache]
        self.ws = torch.empty(model.layer_workspace_bytes(self.lcfg, B), dtype=torch.uint8, device=dev)
        self.groups = self.weights = None
        self._told, self._spaces = {}, {}  # group_rows, shared and the table's version of groups; workspaces without and with weights
        self._buffers(B)

    def _buffers(self, rows: int):
        c, dev = self.model.cfg, self.model.embed.device
        self.x = torch.empty((rows, c.H), dtype=torch.bfloat16, device=dev)
        self.xn = torch.empty((rows, c.H), dtype=torch.bfloat16, device=dev)
        if self.model.quantized:  # the final norm's output as activation codes for the quantized lm_head
            self.xn_codes = torch.empty((rows, c.H), dtype=torch.int8, device=dev)
            self.xn_scales = torch.empty(api.det_quant_act_scales_bytes(rows, c.H) // 4, dtype=torch.float32, device=dev)
        self.logits = torch.empty((rows, c.V), dtype=torch.float32, device=dev)
        self.tokens = torch.empty(rows, dtype=torch.int32, device=dev)
        self.positions = torch.empty(rows, dtype=torch.int32, device=dev)
        self.slots = None

    def tell(self, stream=None):
        """What the layers are told of groups and weights, and their workspace: brought in line with the pages' tables.  A step does so by itself; a captured one
        keeps the groups and the weights of its capture, needs a step or a call of this with them in front of it, and another call, outside the graph, when
        the tables have changed."""
        if self.groups is None and self.weights is None:
            return None, self.ws
        if not self.model.cache8 or (self.groups is not None and self.slots is not None):
            raise ValueError("groups and weights are those of an 8-bit cache's sequences, a row each")
        rows, dev, g = self.tokens.shape[0], self.tokens.device, tuple(self.groups or ())
        if self.groups is not None and (len(g) < 2 or g[0] != 0 or g[-1] != rows or any(a >= b for a, b in zip(g, g[1:]))):
            raise ValueError("groups of sequences, one behind the other")
        weighs, told = self.weights is not None, self._told.get(g)
        if weighs not in self._spaces or (g and (told is None or told[2] != self.pages.version)):
            if dev.type == "cuda" and torch.cuda.is_current_stream_capturing():
                raise RuntimeError("groups, weights and tables of a captured step are those of one before it")
            with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
                if g:  # their addresses stay, for graphs
                    shared = torch.tensor([self.pages.shared_tokens(range(a, b)) for a, b in zip(g, g[1:])], dtype=torch.int32)
                    told = told or [torch.tensor(g, dtype=torch.int32).to(dev), torch.empty(len(g) - 1, dtype=torch.int32, device=dev), None]
                    told[1].copy_(shared)
                    told[2] = self.pages.version
                    self._told[g] = told
                if weighs not in self._spaces:
                    size = self.model.layer_workspace_bytes(self.lcfg, rows, step=api.kv8_step(weights=self.weights))
                    self._spaces[weighs] = self.ws if size <= self.ws.nbytes else torch.empty(size, dtype=torch.uint8, device=dev)
        step = api.kv8_step(*(told[:2] if g else (None, None)), self.weights)
        return step, self._spaces[weighs]

    def of_rows(self, slots: torch.Tensor) -> "DecodeState":
        """A state over the same caches whose steps take one row for each entry of slots (several rows may name one sequence)."""
        st = copy.copy(self)
        st.groups = st.weights = None
        st._told, st._spaces = {}, {}
        st.ws = torch.empty(self.model.layer_workspace_bytes(self.lcfg, slots.shape[0], named=True), dtype=torch.uint8, device=slots.device)
        st._buffers(slots.shape[0])
        st.slots = slots
        return st

    def forward(self, stream=None):
        """One decode step on self.tokens / self.positions; leaves fp32 logits in self.logits."""
        m, c = self.model, self.model.cfg
        step, ws = self.tell(stream)
        api.det_embed_gather(m.embed, self.tokens, self.x, stream)
        for i, (_, struct) in enumerate(m.layers):
            m.layer(struct, self.lcfg, self.x, self.kcache[i], self.vcache[i], self.positions, self.slots, self.rope_cos,
                    self.rope_sin, ws, stream, step)
        self.head(stream)

    def head(self, stream=None):
        """Final RMSNorm and lm_head on self.x; fp32 logits in self.logits."""
        m, c = self.model, self.model.cfg
        if m.quantized:
            api.det_rmsnorm_quant_q8(self.x, m.final_norm, self.xn_codes, self.xn_scales, c.eps, stream)
            api.det_qgemm_w4a8(self.xn_codes, self.xn_scales, m.lm_head, self.logits, c.V, stream)
        else:
            api.det_rmsnorm_gemm_bf16(self.x, m.final_norm, c.eps, m.lm_head, self.xn, self.logits, c.V, stream)


@dataclass
class SamplingPolicy:
    """Seeded decode policy: det_sample with these parameters instead of det_argmax.  `seq_ids`
    [B] int32 on the device names each sequence, so that its random stream does not depend on the
    batch it runs in."""
    temperature: float
    top_k: int
    top_p: float
    seed: int
    seq_ids: torch.Tensor


@dataclass
class Grammar:
    """Which tokens may come where, as an automaton over classes of tokens: in state s the tokens whose bit in masks[s] ([n_states, ceil(V / 32)] int32) is
    set; a token leads to transitions[s, class] ([n_states, n_classes] int32; -1: nothing is barred from there on).  token_class [V] int32 or None (every
    token is its own class); start: the state in which every sequence begins.  Tensors on the device.  A state that start leads to has to allow a token:
    in one without, every logit would be -inf, the choice a barred token all the same, and nothing barred behind it.  That is looked at once, when it is made."""
    masks: torch.Tensor
    transitions: torch.Tensor
    token_class: torch.Tensor | None = None
    start: int = 0

    def __post_init__(self):
        if self.masks.dim() != 2 or self.transitions.dim() != 2 or (self.token_class is not None and self.token_class.dim() != 1):
            raise ValueError("masks [n_states, words], transitions [n_states, n_classes] and the class of each token")
        if self.masks.shape[0] != self.transitions.shape[0] or 32 * self.masks.shape[1] < self.tokens or not 0 <= self.start < self.masks.shape[0]:
            raise ValueError("a mask over all tokens for each state, and one of them to begin in")
        self.check(self.tokens)

    @property
    def tokens(self) -> int:
        return self.transitions.shape[1] if self.token_class is None else self.token_class.shape[0]

    def check(self, V: int, barred=()) -> None:
        """Refuses states that start leads to without a token below V beside the barred ones."""
        n, n_classes = self.transitions.shape
        V, dev = min(V, self.tokens), self.masks.device
        bit = torch.arange(32, dtype=torch.int32, device=dev)
        there = torch.ones(V, dtype=torch.bool, device=dev)
        there[[t for t in barred if 0 <= t < V]] = False
        of = None
        if self.token_class is not None:  # tokens without a class, in a column behind the others
            of = self.token_class[:V].long()
            of = torch.where((of >= 0) & (of < n_classes), of, n_classes)
        seen, todo = {self.start}, [self.start]
        while todo:
            states, todo = todo[:64], todo[64:]  # some at a time: a state's tokens take 128 bytes a word of its mask
            at = torch.tensor(states, device=dev)
            allowed = ((self.masks[at][..., None] >> bit) & 1).flatten(1)[:, :V].bool() & there
            some = allowed.any(1).tolist()
            if not all(some):
                raise ValueError(f"state {states[some.index(False)]} of the grammar allows no token")
            classes = allowed
            if of is not None:
                row, token = allowed.nonzero(as_tuple=True)
                classes = torch.zeros((len(states), n_classes + 1), dtype=torch.bool, device=dev)
                classes[row, of[token]] = True
            to = self.transitions[at][:, :classes.shape[1]][classes[:, :n_classes]].unique().tolist()
            new = [s for s in to if 0 <= s < n and s not in seen]
            seen.update(new)
            todo += new


@dataclass
class LogitsPolicy:
    """Rules on the logits of every step (det_logits_process): tokens of the prompt or generated so far are made less likely by `repetition` (their
    logits divided, where positive, or multiplied by it), generated ones also by `frequency` for each time and by `presence` once; `biases`
    {token: added}; `grammar`, of which the biases may not bar (-inf) all that a state allows.  The same for every sequence of a call."""
    repetition: float = 1.0
    frequency: float = 0.0
    presence: float = 0.0
    biases: dict | None = None
    grammar: Grammar | None = None


@dataclass
class EvictPolicy:
    """A sequence of an 8-bit cache comes back to `keep` pages every `every` steps: of those but its first and last ones it gives up the pages that its
    generated tokens, over all layers and heads, have given the least weight (KVPages.evict).  A step then reads less; the call's pool has room for all tokens
    all the same, and what is given up serves no other sequence of it."""
    keep: int
    every: int = 64
    first: int = 1
    recent: int = 4


class _Rules:
    """A LogitsPolicy while B sequences are decoded: their history and grammar states, on the device."""

    def __init__(self, policy: LogitsPolicy, prompts, lens_host, n_new: int, V: int, out):
        B, dev = len(lens_host), prompts.device
        i32 = dict(dtype=torch.int32, device=dev)
        self.out = out
        self.history = self.lens = self.grammar = self.states = None
        given = {}
        if (policy.repetition, policy.frequency, policy.presence) != (1.0, 0.0, 0.0):
            if not policy.repetition > 0:
                raise ValueError("repetition is a factor above 0")
            self.history = torch.zeros((B, int(lens_host.max()) + n_new), **i32)
            self.history[:, :prompts.shape[1]] = prompts[:, :self.history.shape[1]]
            begin = lens_host.to(torch.int32).to(dev)
            self.lens = begin.clone()
            values = torch.tensor([policy.repetition, policy.frequency, policy.presence], dtype=torch.float32)
            given |= dict(penalties=values.repeat(B, 1).to(dev), history=self.history, history_lens=self.lens, generated_from=begin)
        barred = []
        if policy.biases:
            n = len(policy.biases)
            tokens, added = torch.tensor(list(policy.biases), dtype=torch.int32), torch.tensor(list(policy.biases.values()), dtype=torch.float32)
            barred = tokens[torch.isneginf(added)].tolist()
            given |= dict(bias_begin=(torch.arange(B + 1, dtype=torch.int32) * n).to(dev), bias_tokens=tokens.repeat(B).to(dev),
                          bias_values=added.repeat(B).to(dev))
        if policy.grammar is not None:
            self.grammar = policy.grammar
            if barred or V < self.grammar.tokens:
                self.grammar.check(V, barred)
            self.states = torch.full((B,), policy.grammar.start, **i32)
            given |= dict(masks=policy.grammar.masks, mask_rows=self.states)
        self.rules = api.logits_rules(**given)

    def process(self, logits, stream):
        """The logits with the rules applied, in `out` (None: in their own place)."""
        out = logits if self.out is None else self.out
        api.det_logits_process(logits, out, self.rules, stream)
        return out

    def advance(self, tokens, stream):
        g = self.grammar
        if self.history is not None or g is not None:
            api.det_logits_advance(tokens, self.history, self.lens, self.lens, None if g is None else g.transitions,
                                   None if g is None else g.token_class, self.states, self.states, stream)


def greedy_decode(model: DecodeModel, prompts: torch.Tensor, prompt_lens: torch.Tensor, n_new: int,
                  rope_cos: torch.Tensor, rope_sin: torch.Tensor, keep_logits_at=(), stream=None,
                  policy: SamplingPolicy | None = None):
    """Runs B sequences together.  prompts [B, Tp] int32 (padded), prompt_lens [B] int32.
    With `policy`, tokens are drawn by det_sample (step = position) instead of det_argmax.

    Returns (generated [B, n_new] int32 on the device, {step: logits [B, V] fp32 clone}).
    Step t feeds prompt token t while t < len, else the token sampled at step t-1; sequence b's
    generated tokens are the samples of steps len_b-1 .. len_b+n_new-2."""
    # allocations, clones and the final gather are torch operations: they follow torch's current stream,
    # which is made the library's stream for the whole run
    with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
        return _greedy_decode(model, prompts, prompt_lens, n_new, rope_cos, rope_sin, keep_logits_at, stream, policy)


def _greedy_decode(model, prompts, prompt_lens, n_new, rope_cos, rope_sin, keep_logits_at, stream, policy):
    B, Tp = prompts.shape
    lens_host = prompt_lens.cpu()
    T = int(lens_host.max()) + n_new - 1
    if rope_cos.shape[0] < T:
        raise ValueError("rope tables shorter than the run")
    st = model.new_state(B, T, rope_cos[:T].contiguous(), rope_sin[:T].contiguous())
    dev = prompts.device
    sampled = torch.zeros((T, B), dtype=torch.int32, device=dev)
    history = torch.zeros((B, T), dtype=torch.int32, device=dev)
    kept = {}
    for t in range(T):
        last = sampled[t - 1] if t > 0 else sampled[0]
        api.det_next_token(prompts, prompt_lens, last, st.tokens, st.positions, history, t, stream)
        st.forward(stream)
        if policy is None:
            api.det_argmax(st.logits, sampled[t], stream)
        else:
            api.det_sample(st.logits, policy.temperature, policy.top_k, policy.top_p, policy.seed, policy.seq_ids,
                           st.positions, sampled[t], stream)
        if t in keep_logits_at:
            kept[t] = st.logits.clone()
    idx = (lens_host.to(torch.int64) - 1)[:, None] + torch.arange(n_new)[None, :]
    gen = sampled.t().contiguous().gather(1, idx.to(dev))
    return gen, kept


def _select(policy, logits, positions, out, stream, rules=None):
    if rules is not None:
        logits = rules.process(logits, stream)
        _select(policy, logits, positions, out, stream)
        rules.advance(out, stream)
    elif policy is None:
        api.det_argmax(logits, out, stream)
    else:
        api.det_sample(logits, policy.temperature, policy.top_k, policy.top_p, policy.seed, policy.seq_ids,
                       positions, out, stream)


# Where groups pay: `saved` tokens that a step need not read, `behind` tokens that its rows read for themselves, of n_groups of `samples` rows.  Beside the
# fixed cost of groups each of them costs some, what rows read behind them is read slower, and two rows a group hardly gain: plain calls find in cache what
# another row has read.  Over 5468 calls of 1 to 32 KV heads, 1 to 16 heads each, 1 to 48 prompts of 260 to 16400 tokens, 2 to 64 rows each and up to
# 4000 tokens of their own the rule takes groups for 2283: together 90 ms without and 62 with them, 8 lose more than 3 % (7 % at most).  Of 700 others, drawn, it
# took 423, of which 2 lost more than 3 % (10 %).  (saved * Hkv >= 80000 and 2 * saved >= behind alone let 317 of 3459 lose that much: 48 prompts of 300 tokens with 3
# rows each, 32/32 heads 59 -> 79 us, 16 of 4100 with 2 rows and 4000 tokens of their own, 32/8 heads 95 -> 120.)  Groups gain most with many rows: 64
# of 4 prompts of 4000 tokens, 16/4 heads, 43 -> 21 us.
GROUPS_FROM = 80_000


def _groups_pay(n_groups: int, samples: int, Hkv: int, saved: int, behind: int) -> bool:
    return (saved - 0.8 * behind) * Hkv >= GROUPS_FROM * ((3 if samples == 2 else 1) + n_groups * Hkv / 80)


def prefill_decode(model: DecodeModel, prompts: torch.Tensor, prompt_lens: torch.Tensor, n_new: int,
                   rope_cos: torch.Tensor, rope_sin: torch.Tensor, stream=None,
                   policy: SamplingPolicy | None = None, keep_logits: bool = False, samples: int = 1, rules: LogitsPolicy | None = None,
                   evict: EvictPolicy | None = None):
    """Same results as greedy_decode, with the prompts processed in one pass.

    samples > 1 (8-bit cache): that many continuations of each prompt, sequence b * samples + i the i-th of prompt b, as if every prompt
    stood samples times in `prompts`; each prompt is run once and its pages are shared, but for the last one where it is not full, and read once a step.

    rules: what the logits go through before a token is chosen (kept logits are those of the head).  evict (8-bit cache): sequences give up pages as they
    go on, which changes what they attend to, but not with the batch they are in.

    Prefill: row r is token prompts[b, p] with position p and cache slot b, for every b and p < len_b
    (R = sum of the lengths).  Each layer writes all keys and values first and then lets row r attend
    to positions 0..p of its slot, which is exactly what the token-by-token run computes for that
    token.  The last row of each sequence goes on to the final norm, lm_head and token selection.
    Decode: sequence b then advances from its own position len_b, one token per step.

    Returns (generated [B, n_new] int32 on the device, list of n_new logits clones [B, V] if
    keep_logits else [])."""
    with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
        return _prefill_decode(model, prompts, prompt_lens, n_new, rope_cos, rope_sin, stream, policy, keep_logits, samples, rules, evict)


def _prefill_decode(model, prompts, prompt_lens, n_new, rope_cos, rope_sin, stream, policy, keep_logits, samples, rules, evict):
    c = model.cfg
    B, _ = prompts.shape
    dev = prompts.device
    lens_host = prompt_lens.cpu().to(torch.int64)
    if samples < 1 or (samples > 1 and not model.cache8):
        raise ValueError("several continuations of a prompt need the 8-bit paged cache")
    if evict is not None and (not model.cache8 or evict.keep < 1 or evict.every < 1 or evict.first < 0 or evict.recent < 1):
        raise ValueError("pages that are given up need the 8-bit paged cache, and a page that stays")
    T = int(lens_host.max()) + n_new - 1
    if rope_cos.shape[0] < T:
        raise ValueError("rope tables shorter than the run")
    n_pages = None
    if samples > 1:  # a prompt's full pages once, what is behind them for each continuation
        full, each = lens_host // api.KV8_PAGE, -(-T // api.KV8_PAGE)
        n_pages = int((full + samples * (each - full)).sum())
    st = model.new_state(B * samples, T, rope_cos[:T].contiguous(), rope_sin[:T].contiguous(), reserve=samples == 1, n_pages=n_pages)
    if samples > 1:
        st.pages.reserve(range(0, B * samples, samples), lens_host.tolist(), stream=stream)

    # row tables, built on the host once (integer bookkeeping only)
    slots_h = torch.repeat_interleave(torch.arange(B), lens_host)
    starts = torch.cumsum(lens_host, 0) - lens_host
    pos_h = torch.arange(int(lens_host.sum())) - torch.repeat_interleave(starts, lens_host)
    R = int(lens_host.sum())
    row_tokens = prompts.cpu()[slots_h, pos_h].to(torch.int32).to(dev)
    row_slots = (slots_h * samples).to(torch.int32).to(dev)
    row_pos = pos_h.to(torch.int32).to(dev)
    last_rows = torch.repeat_interleave(starts + lens_host - 1, samples).to(torch.int32).to(dev)

    xr = torch.empty((R, c.H), dtype=torch.bfloat16, device=dev)
    ws = torch.empty(model.layer_workspace_bytes(st.lcfg, R, named=True), dtype=torch.uint8, device=dev)
    api.det_embed_gather(model.embed, row_tokens, xr, stream)
    for i, (_, struct) in enumerate(model.layers):
        model.layer(struct, st.lcfg, xr, st.kcache[i], st.vcache[i], row_pos, row_slots, st.rope_cos, st.rope_sin, ws,
                    stream)
    api.det_embed_gather(xr, last_rows, st.x, stream)  # row gather: the last token of each sequence
    st.head(stream)
    if samples > 1:
        for b, n in enumerate(lens_host.tolist()):
            st.pages.fork(b * samples, range(b * samples + 1, (b + 1) * samples), n, stream)
        st.pages.reserve(range(B * samples), [T] * (B * samples), torch.repeat_interleave(lens_host, samples).tolist(), stream)
    shared = int((lens_host // api.KV8_SHARED_CHUNK).sum()) * api.KV8_SHARED_CHUNK
    weights = torch.zeros(st.pages.table.shape, dtype=torch.float32, device=dev) if evict is not None else None
    st.groups, st.weights = list(range(0, B * samples + 1, samples)) if samples > 1 else None, weights
    of_rules = None
    if rules is not None:
        out = torch.empty_like(st.logits) if keep_logits else None
        of_rules = _Rules(rules, torch.repeat_interleave(prompts.to(torch.int32), samples, 0), torch.repeat_interleave(lens_host, samples), n_new, c.V, out)
    kept_pages = torch.full((B * samples,), evict.keep, dtype=torch.int32, device=dev) if evict is not None else None

    gen = torch.zeros((n_new, B * samples), dtype=torch.int32, device=dev)
    kept = []
    base_pos = torch.repeat_interleave(lens_host - 1, samples).to(torch.int32).to(dev)   # position of each sequence's last prompt token
    st.positions.copy_(base_pos)
    _select(policy, st.logits, st.positions, gen[0], stream, of_rules)
    if keep_logits:
        kept.append(st.logits.clone())
    for j in range(1, n_new):
        api.det_decode_advance(gen[j - 1], base_pos, j, st.tokens, st.positions, stream)
        if evict is not None and j % evict.every == 0:
            gone = st.pages.evict(weights, st.positions, kept_pages, evict.first, evict.recent, stream)
            if st.groups is not None and any(gone):  # continuations give up pages of their own choice, and share those in front of the first that differs
                shared = sum(st.pages.shared_tokens(range(a, b)) // api.KV8_SHARED_CHUNK for a, b in zip(st.groups, st.groups[1:])) * api.KV8_SHARED_CHUNK
        if st.groups is not None:
            saved, behind = (samples - 1) * shared, samples * (R - shared + j * B)  # tokens that groups need not read, and that rows read for themselves
            if not _groups_pay(B, samples, c.Hkv, saved, behind):
                st.groups = None
        st.forward(stream)
        _select(policy, st.logits, st.positions, gen[j], stream, of_rules)
        if keep_logits:
            kept.append(st.logits.clone())
    return gen.t().contiguous(), kept


def speculative_decode(model: DecodeModel, draft: DecodeModel, prompts: torch.Tensor, prompt_lens: torch.Tensor, n_new: int, n_draft: int,
                       uniforms, rope_cos: torch.Tensor, rope_sin: torch.Tensor, stream=None):
    """Draws n_new tokens for each sequence from the model's own distribution (temperature 1), n_draft at a time proposed by `draft` (a model of the
    same vocabulary) and verified in one pass of `model` over n_draft + 1 rows of each sequence (det_verify_drafts).

    uniforms: a function (round, shape) -> independent fp32 numbers in [0, 1) on the device, called once a round for (B, 2 n_draft + 1): n_draft
    draws of the draft model, then n_draft + 1 of the verification.  Round -1 gives the (B, 2) numbers of the first token, of which the second is used.
    The tokens are a function of the models, the prompts and these numbers; what a sequence gets does not depend on the batch.

    Rejected drafts need no undoing: a sequence's length ends in front of them and their places in the caches are written again.

    Returns (tokens [B, n_new] int32 on the host, accepted drafts of each round, a list of [B] int32 host tensors; a sequence that has its
    tokens goes on until the last one has)."""
    if n_draft < 1 or n_draft > 62 or n_new < 1 or model.cfg.V != draft.cfg.V:
        raise ValueError("1 to 62 drafts of a model with the same vocabulary")
    with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
        return _speculative_decode(model, draft, prompts, prompt_lens, n_new, n_draft, uniforms, rope_cos, rope_sin, stream)


def _fill_prompts(model, st, prompts, lens_host, stream):
    """The prompts' rows through the model's layers; the last row of each into st.x, logits into st.logits."""
    B = prompts.shape[0]
    dev = prompts.device
    slots_h = torch.repeat_interleave(torch.arange(B), lens_host)
    starts = torch.cumsum(lens_host, 0) - lens_host
    pos_h = torch.arange(int(lens_host.sum())) - torch.repeat_interleave(starts, lens_host)
    rows = st.of_rows(slots_h.to(torch.int32).to(dev))
    rows.positions.copy_(pos_h)
    api.det_embed_gather(model.embed, prompts.cpu()[slots_h, pos_h].to(torch.int32).to(dev), rows.x, stream)
    for i, (_, struct) in enumerate(model.layers):
        model.layer(struct, st.lcfg, rows.x, st.kcache[i], st.vcache[i], rows.positions, rows.slots, st.rope_cos, st.rope_sin, rows.ws, stream)
    api.det_embed_gather(rows.x, (starts + lens_host - 1).to(torch.int32).to(dev), st.x, stream)
    st.head(stream)


def _speculative_decode(model, draft, prompts, prompt_lens, n_new, n_draft, uniforms, rope_cos, rope_sin, stream):
    B, dev, V, N = prompts.shape[0], prompts.device, model.cfg.V, n_draft
    lens_host = prompt_lens.cpu().to(torch.int64)
    if int(lens_host.min()) < 1 or int(lens_host.max()) > prompts.shape[1]:
        raise ValueError("a prompt's length outside 1..its row")
    T = int(lens_host.max()) + n_new + N  # the last token is drawn at position length + n_new - 1 at most, drafts behind it
    if rope_cos.shape[0] < T:
        raise ValueError("rope tables shorter than the run")
    cos, sin = rope_cos[:T].contiguous(), rope_sin[:T].contiguous()
    target, small = model.new_state(B, T, cos, sin), draft.new_state(B, T, cos, sin)
    rows = target.of_rows(torch.repeat_interleave(torch.arange(B, dtype=torch.int32), N + 1).to(dev))
    i32, f32 = dict(dtype=torch.int32, device=dev), dict(dtype=torch.float32, device=dev)
    width = torch.full((B * (N + 1),), V, **i32)
    p, q, sums = torch.empty((B, N + 1, V), **f32), torch.empty((N, B, V), **f32), torch.empty((2, B * (N + 1)), **f32)
    drafts, drawn, none = torch.empty((B, N), **i32), torch.empty((B, 2), **i32), torch.zeros(B, **i32)
    accepted, tokens = torch.empty(B, **i32), torch.empty((B, N + 1), **i32)
    first = torch.empty((B, 2, V), **f32)
    ws = torch.empty(api.det_verify_drafts_workspace_bytes(B, V), dtype=torch.uint8, device=dev)

    def draw(st, probabilities, u, out):
        """One token of each sequence from st.logits: a verification without drafts.  u [B, 2], the second is used."""
        api.det_softmax_f32(st.logits, width[:B], probabilities, sums[0, :B], sums[1, :B], stream)
        first[:, 0].copy_(probabilities)
        api.det_verify_drafts(first, None, none[:, None], none, u, accepted, drawn, ws, stream)
        out.copy_(drawn[:, 0])

    _fill_prompts(model, target, prompts, lens_host, stream)
    _fill_prompts(draft, small, prompts, lens_host, stream)
    current, at = torch.empty(B, **i32), lens_host.to(torch.int32).to(dev)
    draw(target, q[0], uniforms(-1, (B, 2)), current)
    made = [[int(t)] for t in current.cpu()]
    counts, turn = [], 0
    step_numbers = torch.arange(N + 1, **i32)
    two = torch.zeros((B, 2), **f32)
    while min(map(len, made)) < n_new:
        # the draft model's own tokens; one step more, so that its cache has the last of them too.  A sequence that has its tokens stays where it is.
        u = uniforms(turn, (B, 2 * N + 1))
        for i in range(N + 1):
            small.tokens.copy_(current if i == 0 else drafts[:, i - 1])
            small.positions.copy_(at + i)
            small.forward(stream)
            if i < N:
                two[:, 1].copy_(u[:, i])
                draw(small, q[i], two, drafts[:, i])
        rows.tokens.copy_(torch.cat([current[:, None], drafts], 1).flatten())
        rows.positions.copy_((at[:, None] + step_numbers).flatten())
        rows.forward(stream)
        api.det_softmax_f32(rows.logits, width, p.view(B * (N + 1), V), sums[0], sums[1], stream)
        api.det_verify_drafts(p, q.transpose(0, 1).contiguous(), drafts, None, u[:, N:].contiguous(), accepted, tokens, ws, stream)
        host, took = tokens.cpu(), accepted.cpu()
        counts.append(took)
        on = [len(m) < n_new for m in made]
        for b in range(B):
            if on[b]:
                made[b] += host[b, :int(took[b]) + 1].tolist()
        # a sequence that has its tokens stays where it is, so that no row passes the end of the caches
        go = torch.tensor([len(m) < n_new for m in made], device=dev)
        current = torch.where(go, tokens.gather(1, accepted.long()[:, None])[:, 0], current)
        at = torch.where(go, at + accepted + 1, at)
        turn += 1
    return torch.tensor([m[:n_new] for m in made], dtype=torch.int32), counts


def commit_outputs(prompts: torch.Tensor, prompt_lens: torch.Tensor, logits_steps, generated: torch.Tensor):
    """Per-sequence output commitment, the hash the paper records for every execution (section 6.7):
    SHA256(prompt || logits || tokens) with prompt = the sequence's own prompt ids (int32,
    little-endian), logits = the fp32 logits rows of its generated steps in step order, tokens = its
    generated ids (int32).  `logits_steps` is the list prefill_decode(keep_logits=True) returns.
    Downloads to host memory and hashes there (det_commit_sha256).  Returns a list of 32-byte digests;
    together with api.det_fingerprint() they are what a receipt would carry for the run."""
    B = prompts.shape[0]
    lens = prompt_lens.cpu().tolist()
    p_host = prompts.to(torch.int32).cpu().contiguous()
    g_host = generated.to(torch.int32).cpu().contiguous()
    l_host = torch.stack(list(logits_steps)).permute(1, 0, 2).contiguous().cpu()  # [B, steps, V]
    # one SHA-256 chain per sequence, the chains on separate host threads (the call releases the GIL)
    from concurrent.futures import ThreadPoolExecutor

    def one(b):
        return api.det_commit_sha256(p_host[b, :lens[b]].contiguous(), l_host[b], g_host[b])

    with ThreadPoolExecutor(max_workers=min(B, os.cpu_count() or 1, 16)) as pool:
        return list(pool.map(one, range(B)))
