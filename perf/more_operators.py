"""The calls of serving several continuations of a prompt, as cases that can be measured: attention that reads a shared prefix once, attention that
also adds up what weight every page of the cache gets, the choice of the pages that go, and the rules on logits before a token is chosen.

A case is a dict of plain values; `kind` names the call.  The cache is the 8-bit paged one: a pool is [pages, KV heads, RECORD] bytes, a record holds the
64 tokens of a page for one KV head, K codes [64, 128], V codes [4, 128, 16] (sixteen tokens of a column side by side), 64 K scales and 64 V scales
(fp32); a code times its token's scale is the value.  `run` computes the plain form in elementary torch operations, or, where `own` is true, through the
package's public entry points.  Heads, widths and vocabularies are those of the models the benchmark runs, or odd neighbours of them."""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
D = 128
PAGE = 64
RECORD = 2 * PAGE * D + 2 * 4 * PAGE
SCALE = 0.08838834764831845  # 1/sqrt(128)


def listed():
    return [
        # A few continuations of one question: all latency.
        dict(name="shared-few", kind="shared", P=1, least=4, most=4, shortest=1000, longest=1000, tail=60, gone=0, Hq=16, Hkv=4),
        # Sixteen continuations of a prompt a few thousand tokens long.
        dict(name="shared-samples-16", kind="shared", P=1, least=16, most=16, shortest=2900, longest=2900, tail=500, gone=0, Hq=32, Hkv=8),
        # A batch of prompts, each with as many continuations as were asked for.
        dict(name="shared-prompts-6", kind="shared", P=6, least=3, most=17, shortest=300, longest=4000, tail=300, gone=0, Hq=32, Hkv=8),
        # A long document that every request of the batch begins with.
        dict(name="shared-long-64", kind="shared", P=1, least=64, most=64, shortest=32000, longest=32000, tail=1000, gone=0, Hq=32, Hkv=8),
        # A serving batch whose pages are weighed while it decodes.
        dict(name="weights-batch-24", kind="weights", P=24, least=1, most=1, shortest=500, longest=6000, tail=64, gone=0, Hq=32, Hkv=8),
        # Long sequences that have given up three of four pages already.
        dict(name="weights-holes-8", kind="weights", P=8, least=1, most=1, shortest=4000, longest=20000, tail=64, gone=75, Hq=16, Hkv=4),
        # Continuations of three prompts, weighed.
        dict(name="weights-shared-12", kind="weights", P=3, least=4, most=4, shortest=2000, longest=7000, tail=200, gone=0, Hq=32, Hkv=8),
        # The pages that one sequence gives up.
        dict(name="pick-one", kind="pick", S=1, shortest=4001, longest=4001, keep=40, ties=0),
        # A batch of long sequences comes back into its budgets.
        dict(name="pick-batch-64", kind="pick", S=64, shortest=3000, longest=32768, keep=128, ties=1),
        # One chat: penalties over its history, a few biases.
        dict(name="logits-one", kind="logits", B=1, V=32000, shortest=200, longest=200, penalties=1, biases=10, states=0, bf16=0),
        # A serving batch with everything set: penalties, biases, and a grammar's masks.
        dict(name="logits-batch-64", kind="logits", B=64, V=128000, shortest=100, longest=4000, penalties=1, biases=30, states=40, bf16=0),
        # Structured answers of a batch, from bf16 logits of an odd width.
        dict(name="logits-grammar-24", kind="logits", B=24, V=32001, shortest=1, longest=300, penalties=0, biases=0, states=100, bf16=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["shared", "shared", "shared", "weights", "weights", "pick", "logits", "logits"])
    if kind in ("shared", "weights"):
        Hkv = rng.choice([1, 2, 4, 8])
        Hq = Hkv * rng.choice([1, 2, 4, 8])
        longest = _log(rng, 1, 32000)
        shortest = max(1, int(longest * rng.uniform(0.1, 1.0)))
        tail = _log(rng, 1, 1000)
        if kind == "shared" or rng.random() < 0.4:
            P = _log(rng, 1, max(1, min(16, 40000 // longest)))
            most = _log(rng, 1, max(1, min(64, 200 // P, 2000000 // (P * longest))))
            least = rng.randint(1, most)
        else:
            P, least, most = _log(rng, 1, max(1, min(48, 200000 // longest))), 1, 1
        gone = rng.choice([0, 0, rng.randint(1, 90)]) if kind == "weights" else 0
        return dict(kind=kind, P=P, least=least, most=most, shortest=shortest, longest=longest, tail=tail, gone=gone, Hq=Hq, Hkv=Hkv)
    if kind == "pick":
        longest = _log(rng, 1, 32768)
        return dict(kind=kind, S=_log(rng, 1, 64), shortest=rng.randint(1, longest), longest=longest, keep=_log(rng, 1, 300), ties=rng.randint(0, 1))
    V = _log(rng, 1000, 128000)
    longest = _log(rng, 1, 8000)
    return dict(kind=kind, B=_log(rng, 1, 64), V=V, shortest=rng.randint(1, longest), longest=longest, penalties=rng.randint(0, 1),
                biases=rng.choice([0, _log(rng, 1, 300)]), states=rng.choice([0, _log(rng, 2, 100)]), bf16=rng.randint(0, 1))


def _spread(n, a, b):
    """n whole numbers spread evenly from a to b."""
    return [a + (b - a) * i // max(1, n - 1) for i in range(n)]


def _rows(case):
    """The groups' first rows (and the number of rows behind them), the tokens that each group shares (whole pages of its prompt) and each row's length."""
    begin, shared, lengths = [0], [], []
    for n, prompt in zip(_spread(case["P"], case["least"], case["most"]), _spread(case["P"], case["shortest"], case["longest"])):
        shared.append(prompt // PAGE * PAGE if n > 1 else 0)
        lengths += [prompt + t for t in _spread(n, 1, case["tail"])]
        begin.append(len(lengths))
    return begin, shared, lengths


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pool(g, pages, Hkv):
    """Records of rows of different sizes and channels of different weight."""
    pool = torch.zeros((pages, Hkv, RECORD), dtype=torch.uint8, device=DEV)
    scales = pool.view(torch.float32)
    for part, shape in ((0, (PAGE, D)), (1, (4, D, 16))):
        x = _normal(g, pages, Hkv, *shape)
        if part == 0:
            x *= torch.exp(0.5 * _normal(g, Hkv, 1, D))
            amax = x.abs().amax(-1)
            codes = torch.round(x * (127 / amax)[..., None])
        else:
            x *= torch.exp(0.5 * _normal(g, pages, Hkv, 4, 1, 16))
            amax = x.abs().amax(-2)
            codes = torch.round(x * (127 / amax)[..., None, :])
        pool[..., part * PAGE * D:(part + 1) * PAGE * D] = codes.to(torch.int8).view(torch.uint8).flatten(2)
        scales[..., 2 * PAGE * D // 4 + part * PAGE:2 * PAGE * D // 4 + (part + 1) * PAGE] = (amax / 127).flatten(2)
    return pool


def _prepare_attention(case, seed, st):
    g = _generator(seed)
    rng = random.Random(seed)
    begin, shared, lengths = _rows(case)
    Hq, Hkv, R = case["Hq"], case["Hkv"], len(lengths)
    counts = [-(-n // PAGE) for n in lengths]
    pages = sum(s // PAGE for s in shared) + sum(counts) + 2
    order = iter(rng.sample(range(pages), pages))  # pages in no order
    table = torch.full((R, max(counts) + 1), -1, dtype=torch.int32)
    for b, e, s in zip(begin, begin[1:], shared):
        common = [next(order) for _ in range(s // PAGE)]
        for r in range(b, e):
            row = common + [next(order) for _ in range(counts[r] - len(common))]
            table[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
        if case["gone"]:  # pages given up: not the first, not the last few; of a group's common ones the same in every row
            lost = [i for i in range(1, max(counts[b:e]) - 4) if rng.random() * 100 < case["gone"]]
            table[b:e, lost] = -1
    st["pool"], st["table"] = _pool(g, pages, Hkv), table.to(DEV)
    st["q"] = (1.5 * _normal(g, R, Hq, D)).to(torch.bfloat16)
    st["lengths"], st["group_rows"], st["shared"] = _int32(lengths), _int32(begin), _int32(shared)
    st["out"] = torch.empty_like(st["q"])
    st["grouped"] = any(shared)
    st["group"] = torch.tensor([i for i in range(case["P"]) for _ in range(begin[i], begin[i + 1])], device=DEV)
    st["index"] = torch.tensor([r - begin[i] for i in range(case["P"]) for r in range(begin[i], begin[i + 1])], device=DEV)
    st["many"] = max(e - b for b, e in zip(begin, begin[1:]))
    st["common_pages"] = max(shared) // PAGE
    st["tail_pages"] = max(counts[r] - shared[i] // PAGE for i in range(case["P"]) for r in range(begin[i], begin[i + 1]))
    if case["kind"] == "weights":
        st["before"] = 2 * torch.rand(table.shape, generator=g, device=DEV)
        st["weights"] = torch.empty_like(st["before"])


def _prepare_logits(case, seed, st):
    g = _generator(seed)
    rng = np.random.default_rng(seed)
    B, V = case["B"], case["V"]
    logits = 3.0 * _normal(g, B, V)
    st["logits"] = logits.to(torch.bfloat16) if case["bf16"] else logits
    st["out"] = torch.empty_like(st["logits"])
    lens = _spread(B, case["shortest"], case["longest"])
    # a history takes some tokens again and again; the last token waits to join it
    history = np.minimum((rng.random((B, case["longest"] + 1)) ** 3 * V).astype(np.int64), V - 1)
    st["history"], st["lens"] = _int32(history), _int32(lens)
    st["tokens"] = _int32(history[np.arange(B), lens])
    st["from"] = _int32([n // 3 for n in lens])
    st["new_lens"] = torch.empty(B, dtype=torch.int32, device=DEV)
    if case["penalties"]:
        st["penalties"] = torch.stack([1.0 + 0.5 * torch.rand(B, generator=g, device=DEV), 0.3 * torch.rand(B, generator=g, device=DEV),
                                       0.5 * torch.rand(B, generator=g, device=DEV)], 1).contiguous()
    if case["biases"]:
        each = [rng.choice(V, min(V, 1 + (case["biases"] + b) % case["biases"] if b % 2 else case["biases"]), replace=False) for b in range(B)]
        st["bias_begin"] = _int32(np.cumsum([0] + [len(e) for e in each]))
        st["bias_tokens"] = _int32(np.concatenate(each))
        st["bias_values"] = torch.from_numpy(rng.normal(0, 4, sum(len(e) for e in each)).astype(np.float32)).to(DEV)
        st["bias_rows"] = torch.tensor(np.repeat(np.arange(B), [len(e) for e in each]), device=DEV)
    if case["states"]:
        n, words, classes = case["states"], -(-V // 32), 64
        # a state allows most tokens or few of them
        bits = rng.integers(0, 2 ** 32, (n, words), dtype=np.uint32)
        strict = np.arange(n) % 3 != 0
        for _ in range(4):
            bits[strict] &= rng.integers(0, 2 ** 32, (int(strict.sum()), words), dtype=np.uint32)
        st["masks"] = torch.from_numpy(bits.view(np.int32)).to(DEV)
        st["classes"] = _int32(rng.integers(0, classes, V))
        st["transitions"] = _int32(rng.integers(-1, n, (n, classes)))
        st["states"] = _int32(rng.integers(-1, n, B))
        st["new_states"] = torch.empty(B, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    st = dict(kind=case["kind"])
    if case["kind"] in ("shared", "weights"):
        _prepare_attention(case, seed, st)
    elif case["kind"] == "logits":
        _prepare_logits(case, seed, st)
    else:
        g = _generator(seed)
        S = case["S"]
        lengths = _spread(S, case["shortest"], case["longest"])
        width = -(-case["longest"] // PAGE) + 1
        weights = torch.rand((S, width), generator=g, device=DEV) ** 4 * 100
        st["weights"] = weights.floor() if case["ties"] else weights
        present = torch.rand((S, width), generator=g, device=DEV) < 0.95
        inside = torch.arange(width, device=DEV) < _int32([-(-n // PAGE) for n in lengths])[:, None]
        st["table"] = torch.where(present & inside, torch.arange(S * width, device=DEV).view(S, width), -1).to(torch.int32)
        st["lengths"] = _int32(lengths)
        st["keep"] = _int32([case["keep"] + s % 7 for s in range(S)])
        st["dropped"] = torch.empty((S, width), dtype=torch.uint8, device=DEV)
        st["n_pages"] = S * width
    return st


FIRST, RECENT = 1, 4  # pages of a sequence that always stay: the first, and the last ones


def _parts(pool):
    """K codes [P, Hkv, 64, 128], V codes [P, Hkv, 4, 128, 16] and the scales [P, Hkv, 64] of a pool, as views."""
    codes, scales = pool.view(torch.int8), pool.view(torch.float32)[..., 2 * PAGE * D // 4:]
    return (codes[..., :PAGE * D].unflatten(-1, (PAGE, D)), codes[..., PAGE * D:2 * PAGE * D].unflatten(-1, (4, D, 16)),
            scales[..., :PAGE], scales[..., PAGE:])


def _values(pool, table):
    """K and V [N, Hkv, tokens, 128] of the pages in a table [N, pages]."""
    N, pages = table.shape
    Hkv = pool.shape[1]
    kc, vc, ks, vs = (x[table.clamp(min=0)] for x in _parts(pool))
    k = (kc.float() * ks[..., None]).transpose(1, 2).reshape(N, Hkv, pages * PAGE, D)
    v = (vc.transpose(-1, -2).reshape(N, pages, Hkv, PAGE, D).float() * vs[..., None]).transpose(1, 2).reshape(N, Hkv, pages * PAGE, D)
    return k, v


def _attention_plain(st):
    """The prompts' pages once for each group, the rows' own pages row by row, one softmax over both."""
    pool, table, q = st["pool"], st["table"].long(), st["q"].float()
    R, Hq, _ = q.shape
    Hkv, P, many = pool.shape[1], st["shared"].shape[0], st["many"]
    G, n_common, n_tail, max_pages = Hq // Hkv, st["common_pages"], st["tail_pages"], table.shape[1]
    group, index = st["group"], st["index"]
    first = st["group_rows"][:-1].long()
    common = st["shared"].long() // PAGE                                                   # [P]
    at = torch.arange(n_common, device=DEV)
    pages = torch.where(at < common[:, None], table[first][:, :n_common], -1)              # [P, n_common]
    own_at = common[group][:, None] + torch.arange(n_tail, device=DEV)                     # [R, n_tail]
    own_pages = torch.where(own_at < max_pages, table.gather(1, own_at.clamp(max=max_pages - 1)), -1)

    ko, vo = _values(pool, own_pages)
    so = torch.matmul(q.view(R, Hkv, G, D), ko.transpose(-1, -2).contiguous()) * SCALE       # [R, Hkv, G, tokens]
    token = (own_at * PAGE)[..., None] + torch.arange(PAGE, device=DEV)
    seen = ((token < st["lengths"][:, None, None]) & (own_pages >= 0)[..., None]).flatten(1)
    so = so.masked_fill_(~seen[:, None, None], float("-inf"))
    top = so.amax(-1)
    if n_common:
        kp, vp = _values(pool, pages)
        rows = torch.zeros((P, many, Hq, D), device=DEV)
        rows[group, index] = q
        rows = rows.view(P, many, Hkv, G, D).transpose(1, 2).reshape(P, Hkv, many * G, D)
        sp = torch.matmul(rows, kp.transpose(-1, -2).contiguous()) * SCALE
        there = (pages >= 0).repeat_interleave(PAGE, 1)
        sp = sp.masked_fill_(~there[:, None, None], float("-inf")).view(P, Hkv, many, G, -1)
        tops = torch.full((P, many, Hkv, G), float("-inf"), device=DEV)
        tops[group, index] = torch.maximum(top, sp.amax(-1).transpose(1, 2)[group, index])
        top = tops[group, index]
        safe = torch.where(tops == float("-inf"), 0.0, tops).transpose(1, 2)
        ep = torch.exp(sp - safe[..., None])                                                # [P, Hkv, many, G, tokens]
    eo = torch.exp(so - torch.where(top == float("-inf"), 0.0, top)[..., None])
    total, o = eo.sum(-1), torch.matmul(eo, vo)
    if n_common:
        total = total + ep.sum(-1).transpose(1, 2)[group, index]
        o = o + torch.matmul(ep.view(P, Hkv, many * G, -1), vp).view(P, Hkv, many, G, D).transpose(1, 2)[group, index]
    by = torch.where(total > 0, 1 / total, 0.0)
    out = (o * by[..., None]).view(R, Hq, D).to(torch.bfloat16)
    if st["kind"] == "shared":
        return out
    weights = torch.zeros((R, max_pages + 1), device=DEV)
    pw = (eo * by[..., None]).view(R, Hq, n_tail, PAGE).sum((1, 3))
    weights.scatter_add_(1, own_at.clamp(max=max_pages), pw)
    if n_common:
        pw = ep.view(P, Hkv, many, G, n_common, PAGE).sum(-1).transpose(1, 2)[group, index]      # [R, Hkv, G, n_common]
        weights[:, :n_common] += (pw * by[..., None]).sum((1, 2))
    return [out, st["before"] + weights[:, :max_pages]]


def _pick_plain(st):
    weights, table = st["weights"], st["table"]
    S, width = weights.shape
    at = torch.arange(width, device=DEV)
    pages = ((st["lengths"] + PAGE - 1) // PAGE)[:, None]
    there = (table >= 0) & (table < st["n_pages"]) & (at < pages)
    candidate = there & (at >= FIRST) & (at < pages - RECENT)
    drop = (there.sum(1) - st["keep"]).clamp(min=0)
    order = torch.where(candidate, weights, float("inf")).argsort(dim=1, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, at.expand(S, width))
    return (candidate & (rank < drop[:, None])).to(torch.uint8)


def _logits_plain(st):
    logits, lens, tokens = st["logits"], st["lens"].long(), st["tokens"]
    B, V = logits.shape
    row = torch.arange(B, device=DEV)
    history = st["history"].clone()
    history[row, lens] = tokens
    lens = lens + 1
    z = logits.float()
    if "penalties" in st:
        at = torch.arange(history.shape[1], device=DEV)
        ids = history.long()
        zero = torch.zeros((B, V), device=DEV)
        seen = zero.scatter_add(1, ids, (at < lens[:, None]).float()) > 0
        count = zero.scatter_add(1, ids, ((at >= st["from"][:, None]) & (at < lens[:, None])).float())
        repetition, frequency, presence = (st["penalties"][:, i:i + 1] for i in range(3))
        z = torch.where(seen, torch.where(z > 0, z / repetition, z * repetition), z)
        z = z - frequency * count
        z = torch.where(count > 0, z - presence, z)
    if "bias_tokens" in st:
        z = z.index_put((st["bias_rows"], st["bias_tokens"].long()), st["bias_values"], accumulate=True)
    more = []
    if "masks" in st:
        state = torch.where(st["states"] >= 0, st["transitions"][st["states"].long().clamp(min=0), st["classes"][tokens.long()].long()], -1)
        bits = (st["masks"][state.long().clamp(min=0)][..., None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        allowed = (bits.flatten(1)[:, :V] != 0) | (state < 0)[:, None]
        z = torch.where(allowed, z, float("-inf"))
        more = [state]
    return [z.to(logits.dtype), lens.int()] + more


def run(st):
    if own:
        return _calls(st)
    if st["kind"] == "pick":
        return _pick_plain(st)
    return _logits_plain(st) if st["kind"] == "logits" else _attention_plain(st)


def _calls(st):
    import paper_2602_00182_amd as det

    if st["kind"] in ("shared", "weights"):
        R, Hq, _ = st["q"].shape
        if "ws" not in st:  # kept by a program for all its calls of these sizes
            size = getattr(det, "det_attn_decode_kv8_%s_workspace_bytes" % st["kind"])(R, Hq, st["pool"].shape[1], D, st["table"].shape[1])
            st["ws"] = torch.empty(size, dtype=torch.uint8, device=DEV)
        if st["kind"] == "shared":
            det.det_attn_decode_kv8_shared(st["q"], st["pool"], st["table"], st["lengths"], None, st["group_rows"], st["shared"], st["out"], st["ws"],
                                           SCALE)
            return st["out"]
        groups = (st["group_rows"], st["shared"]) if st["grouped"] else (None, None)
        det.det_attn_decode_kv8_weights(st["q"], st["pool"], st["table"], st["lengths"], None, *groups, st["before"], st["weights"], st["out"],
                                        st["ws"], SCALE)
        return [st["out"], st["weights"]]
    if st["kind"] == "pick":
        det.det_kv8_pick_pages(st["weights"], st["table"], st["n_pages"], st["lengths"], st["keep"], FIRST, RECENT, st["dropped"])
        return st["dropped"]
    more = []
    if "rules" not in st:  # pointers of the tensors above, kept by a program while it decodes
        st["rules"] = det.logits_rules(history=st["history"], history_lens=st["new_lens"], generated_from=st["from"], penalties=st.get("penalties"),
                                       bias_begin=st.get("bias_begin"), bias_tokens=st.get("bias_tokens"), bias_values=st.get("bias_values"),
                                       masks=st.get("masks"), mask_rows=st.get("new_states"))
    if "masks" in st:
        det.det_logits_advance(st["tokens"], st["history"], st["lens"], st["new_lens"], st["transitions"], st["classes"], st["states"],
                               st["new_states"])
        more = [st["new_states"]]
    else:
        det.det_logits_advance(st["tokens"], st["history"], st["lens"], st["new_lens"])
    det.det_logits_process(st["logits"], st["out"], st["rules"])
    return [st["out"], st["new_lens"]] + more


def work(case):
    if case["kind"] in ("shared", "weights"):
        begin, shared, lengths = _rows(case)
        R, Hq, Hkv = len(lengths), case["Hq"], case["Hkv"]
        rows = [e - b for b, e in zip(begin, begin[1:])]
        there = 1 - case["gone"] / 100
        tokens = sum(lengths) - sum((n - 1) * s for n, s in zip(rows, shared))   # each shared token once
        each = 2 * D + 8                                                         # bytes of a token of a KV head: codes and two scales
        weights = 8 * R * (max(lengths) // PAGE + 1) if case["kind"] == "weights" else 0
        return dict(bytes=int(there * tokens) * Hkv * each + 4 * R * Hq * D + weights, flops=int(there * 4 * D * Hq * sum(lengths)))
    if case["kind"] == "pick":
        pages = sum(-(-n // PAGE) for n in _spread(case["S"], case["shortest"], case["longest"]))
        return dict(bytes=9 * pages, flops=2 * pages)
    B, V = case["B"], case["V"]
    size = 2 if case["bf16"] else 4
    history = 4 * sum(_spread(B, case["shortest"], case["longest"])) if case["penalties"] else 0
    return dict(bytes=2 * size * B * V + history + 8 * B * case["biases"] + (B * V // 8 if case["states"] else 0), flops=4 * B * V)


def _exact_tokens(st, row):
    """Which of a row's tokens have a page, and K and V [Hkv, those, 128] in 64 bits, by the byte each value stands at."""
    pool, Hkv = st["pool"], st["pool"].shape[1]
    t = torch.arange(int(st["lengths"][row]), device=DEV)
    t = t[st["table"][row, t // PAGE] >= 0]
    page, at = st["table"][row, t // PAGE].long(), t % PAGE
    base = (page[None, :] * Hkv + torch.arange(Hkv, device=DEV)[:, None]) * RECORD        # [Hkv, tokens]
    d = torch.arange(D, device=DEV)
    codes, scales = pool.flatten().view(torch.int8), pool.flatten().view(torch.float32)
    k = codes[base[..., None] + (at * D)[None, :, None] + d].double()
    v = codes[base[..., None] + (PAGE * D + at // 16 * (16 * D) + at % 16)[None, :, None] + 16 * d].double()
    dk = scales[base // 4 + 2 * PAGE * D // 4 + at].double()
    dv = scales[base // 4 + 2 * PAGE * D // 4 + PAGE + at].double()
    return t, k * dk[..., None], v * dv[..., None]


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("shared", "weights"):
        R, Hq, _ = st["q"].shape
        G = Hq // case["Hkv"]
        out = torch.zeros((R, Hq, D), dtype=torch.float64, device=DEV)
        weights = st["before"].double() if case["kind"] == "weights" else None
        for r in range(R):
            t, k, v = _exact_tokens(st, r)
            for h in range(Hq):
                if not len(t):
                    continue
                p = torch.softmax(k[h // G] @ st["q"][r, h].double() / math.sqrt(D), 0)
                out[r, h] = p @ v[h // G]
                if weights is not None:
                    weights[r].index_add_(0, t // PAGE, p)
        return out if weights is None else [out, weights]
    if case["kind"] == "pick":
        dropped = np.zeros(st["dropped"].shape, dtype=np.uint8)
        for s, (n, keep) in enumerate(zip(st["lengths"].tolist(), st["keep"].tolist())):
            pages = -(-n // PAGE)
            there = [i for i, p in enumerate(st["table"][s, :pages].tolist()) if 0 <= p < st["n_pages"]]
            weights = st["weights"][s].tolist()
            order = sorted((weights[i], i) for i in there if FIRST <= i < pages - RECENT)
            for _, i in order[:max(0, len(there) - keep)]:
                dropped[s, i] = 1
        return dropped
    B, V = case["B"], case["V"]
    z = st["logits"].double().cpu().numpy()
    history, lens, tokens = (st[w].cpu().numpy() for w in ("history", "lens", "tokens"))
    states = np.full(B, -1, dtype=np.int32)
    for b in range(B):
        ids = np.append(history[b, :lens[b]], tokens[b])
        if case["penalties"]:
            repetition, frequency, presence = st["penalties"][b].double().tolist()
            seen = np.unique(ids)
            z[b, seen] = np.where(z[b, seen] > 0, z[b, seen] / repetition, z[b, seen] * repetition)
            made, counts = np.unique(ids[int(st["from"][b]):], return_counts=True)
            z[b, made] -= frequency * counts + presence
        if case["biases"]:
            at = slice(int(st["bias_begin"][b]), int(st["bias_begin"][b + 1]))
            z[b, st["bias_tokens"][at].cpu().numpy()] += st["bias_values"][at].double().cpu().numpy()
        if case["states"] and int(st["states"][b]) >= 0:
            states[b] = int(st["transitions"][int(st["states"][b]), int(st["classes"][tokens[b]])])
            if states[b] >= 0:
                words = st["masks"][states[b]].cpu().numpy().view(np.uint32)
                z[b, (words[np.arange(V) // 32] >> (np.arange(V, dtype=np.uint32) % 32)) & 1 == 0] = -np.inf
    return [z, lens + 1] + ([states] if case["states"] else [])
