"""What surrounds the decoding calls on the paged cache, as timed cases: cached keys carried to other positions, and tokens drawn
from logits under rules.

A case is a dict of plain sizes and options.  `prepare` builds what a program holds before the call, `run` makes one pass
through one operator.  Three kinds:

  reposition   cached keys turned from their positions to others, or to other rotary frequencies, in place (`Decoder.reposition`)
  penalize     biases, penalties for tokens that the history holds, and grammar masks on logits (`Sampler.penalize`)
  sample       a token per row of logits: temperature, top-k, top-p, min-p, one uniform number a row (`Sampler.sample`)

With `own` false, `run` computes the same in elementary torch operations.  `exact` is the definition in float64.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
VOCAB = 151936

REPOSITION = dict(kind="reposition", layers=1, kv_heads=8, head_dim=128, page=16, requests=1, len_lo=1000, len_hi=1000, prefix=0,
                  rotary=128, axes=1, interleaved=False, per_unit=True, rescale=False, shape=1)
PENALIZE = dict(kind="penalize", requests=16, win_lo=1, win_hi=1, vocab=VOCAB, hist_lo=2000, hist_hi=34000, biases=0, grammar=0.0,
                in_place=True, bf16=False, shape=1)
SAMPLE = dict(kind="sample", rows=16, vocab=VOCAB, top_k=0, top_p=1.0, min_p=0.0, temperature=1.0, mixed=False, masked=False, bf16=False)


def listed():
    return [
        # One agent's cache cut to about 1000 tokens, one layer, every head with survivors of its own: positions without gaps again.
        dict(REPOSITION, name="reposition_1k_x1", len_lo=1021, len_hi=1021, prefix=64),
        # The benchmark's cache after its compression (8 requests, 26 % of 35000 tokens, 4 KV heads), 6 layers of it.
        dict(REPOSITION, name="reposition_9k_x8", layers=6, kv_heads=4, requests=8, len_lo=9100, len_hi=9100, prefix=300),
        # Contexts have outgrown what the model was trained on: all cached keys go over to scaled frequencies, positions stay.
        dict(REPOSITION, name="reposition_rescale_x8", layers=2, kv_heads=4, requests=8, len_lo=20000, len_hi=35000, per_unit=False,
             rescale=True, shape=3),
        # Images in the trace (time, height, width), pairs side by side, half of a head turned; ragged requests behind a compression.
        dict(REPOSITION, name="reposition_axes_x16", layers=2, head_dim=64, page=32, requests=16, len_lo=500, len_hi=6000, prefix=100,
             rotary=32, axes=3, interleaved=True, shape=4),
        # One decode step of 16 agents with long histories: repetition, frequency and presence penalties, a few biases.
        dict(PENALIZE, name="penalize_decode_x16", biases=8),
        # 64 agents, most of them inside a tool call: a grammar leaves them a part of the vocabulary.
        dict(PENALIZE, name="penalize_grammar_x64", requests=64, hist_lo=8192, hist_hi=32768, grammar=0.75, shape=5),
        # Drafted tokens are verified, 4 to 8 of 16 agents: bf16 logits, the raw ones are kept for their log probabilities.
        dict(PENALIZE, name="penalize_draft_x16", win_lo=4, win_hi=8, hist_lo=500, hist_hi=9000, grammar=0.5, biases=3, in_place=False,
             bf16=True, shape=6),
        # Sampled actions are scored under the rules they were drawn with: 6 actions of 200 to 300 tokens.
        dict(PENALIZE, name="penalize_score_x6", requests=6, win_lo=200, win_hi=300, hist_lo=3000, hist_hi=20000, grammar=0.3, in_place=False,
             shape=7),
        # One decode step of 16 agents with a model's usual settings.
        dict(SAMPLE, name="sample_decode_x16", top_k=20, top_p=0.8, temperature=0.7),
        # Free text of 64 agents: top-p alone, at a temperature at which thousands of tokens stay.
        dict(SAMPLE, name="sample_open_x64", rows=64, top_p=0.95),
        # Rollouts for training: 1024 rows of bf16 logits, the whole distribution mostly, other settings and greedy rows among them.
        dict(SAMPLE, name="sample_rollout_x1024", rows=1024, mixed=True, bf16=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["reposition", "penalize", "sample"])
    shape = rng.randrange(1, 1 << 20)
    if kind == "reposition":
        rows = _log_uniform(rng, 300, 400000)                    # (token, layer) pairs
        mean = min(rows, _log_uniform(rng, 100, 30000))
        layers = max(1, min(rng.choice([1, 2, 6]), rows // mean))
        dim = rng.choice([64, 128, 128, 80])
        return dict(REPOSITION, layers=layers, kv_heads=rng.choice([1, 2, 4]), head_dim=dim, page=rng.choice([16, 16, 32, 64, 5]),
                    requests=max(1, min(64, rows // layers // mean)), len_lo=max(1, int(mean * 0.6)), len_hi=max(1, int(mean * 1.4)),
                    prefix=rng.choice([0, 0, 50, 300]), rotary=rng.choice([dim, dim, dim // 2, 2 * rng.randrange(1, dim // 2)]),
                    axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.3, per_unit=rng.random() < 0.7, rescale=rng.random() < 0.3,
                    shape=shape)
    if kind == "penalize":
        rows = _log_uniform(rng, 1, 800)
        win = rng.choice([1, 1, rng.randrange(2, 9), _log_uniform(rng, 10, 300)])
        requests = max(1, min(96, rows // win))
        lo = _log_uniform(rng, 20, 15000)
        return dict(PENALIZE, requests=requests, win_lo=max(1, int(win * 0.7)), win_hi=win, vocab=rng.choice([VOCAB, VOCAB, 32003, 1009]),
                    hist_lo=max(lo, win), hist_hi=max(lo, win) * 2, biases=rng.choice([0, 0, 1, 40, 300]), grammar=rng.choice([0.0, 0.0, 0.5, 1.0]),
                    in_place=rng.random() < 0.5, bf16=rng.random() < 0.4, shape=shape)
    return dict(SAMPLE, rows=_log_uniform(rng, 1, 600), vocab=rng.choice([VOCAB, VOCAB, 32003, 1009]), top_k=rng.choice([0, 0, 1, 20, 50, 1000]),
                top_p=rng.choice([1.0, 1.0, 0.5, 0.9, 0.99]), min_p=rng.choice([0.0, 0.0, 0.05]),
                temperature=rng.choice([1.0, 1.0, 0.6, round(rng.uniform(0.3, 2.0), 3)]), mixed=rng.random() < 0.3,
                masked=rng.random() < 0.3, bf16=rng.random() < 0.4)


# ---------------------------------------------------------------------------------------------------------------
# what the sizes of a case come to, from the case alone


def _lengths(case):
    rng = random.Random(case["shape"])
    R = case["requests"]
    if case["kind"] == "reposition":
        return [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(R)]
    win = [rng.randint(case["win_lo"], case["win_hi"]) for _ in range(R)]
    hist = [max(w, rng.randint(case["hist_lo"], case["hist_hi"])) for w in win]
    masked = [rng.random() < case["grammar"] for _ in range(R)]
    return win, hist, masked


def _share(at):
    """The part of the vocabulary that the `at`-th masked row's grammar allows: a few tokens behind a bracket, nearly all of them in a string."""
    return (0.0005, 0.02, 0.1, 0.9)[at % 4]


def _distinct(tokens, vocab):
    """How many different tokens that many drawn ones are, about: the cube of a uniform number times the vocabulary."""
    edge = (torch.arange(vocab + 1, dtype=torch.float64) / vocab) ** (1.0 / 3.0)
    return float((1.0 - (1.0 - (edge[1:] - edge[:-1])) ** tokens).sum())


def work(case):
    if case["kind"] == "reposition":
        units = case["layers"] * case["kv_heads"]
        L = _lengths(case)
        moved = sum(L) if case["rescale"] else sum(max(0, n - case["prefix"]) for n in L)
        positions = 0 if case["rescale"] and not case["per_unit"] else 4 * case["axes"] * sum(L) * (units if case["per_unit"] else 1)
        return {"bytes": moved * units * case["rotary"] * 4 + positions, "flops": moved * units * case["rotary"] * 3}
    item = 2 if case["bf16"] else 4
    if case["kind"] == "penalize":
        win, hist, masked = _lengths(case)
        V, words = case["vocab"], (case["vocab"] + 31) // 32
        at, written = 0, 0.0
        for w, m in zip(win, masked):
            for _ in range(w if m else 0):
                written += (1 - _share(at)) * V * item
                at += 1
        if not case["in_place"]:
            moved = 2.0 * sum(win) * V * item
        else:
            touched = sum(w * _distinct(n, V) for w, n in zip(win, hist)) + sum(win) * case["biases"]
            moved = min(2.0 * touched * item, 2.0 * sum(win) * V * item) + written
        return {"bytes": moved + 4 * sum(hist) + 4 * words * at + 8 * case["biases"] * len(win), "flops": sum(win) * V}
    return {"bytes": case["rows"] * (case["vocab"] * item + 28), "flops": case["rows"] * case["vocab"] * 4}


# ---------------------------------------------------------------------------------------------------------------
# inputs


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _indptr(x):
    return _i32([0] + torch.tensor(x).cumsum(0).tolist())


def _sections(pairs, axes):
    if axes == 1 or pairs < axes:
        return [pairs] + [0] * (axes - 1)
    first = max(1, pairs // (axes + 1))
    rest = [(pairs - first) // (axes - 1)] * (axes - 1)
    rest[-1] += pairs - first - sum(rest)
    return [first] + rest


def _logits(rows, vocab, gen, bf16):
    x = torch.randn((rows, vocab), generator=gen, device=DEV)
    x.mul_(2.5)
    n = min(24, vocab)
    hot = torch.randint(vocab, (rows, n), generator=gen, device=DEV)                          # a few tokens stand out
    x.scatter_add_(1, hot, 9.0 * torch.rand((rows, n), generator=gen, device=DEV))
    return x.to(torch.bfloat16) if bf16 else x


def _prepare_reposition(case, gen):
    L, page = _lengths(case), case["page"]
    nl, hk, d, R, n = case["layers"], case["kv_heads"], case["head_dim"], case["requests"], sum(_lengths(case))
    need = [-(-x // page) for x in L]
    perm = torch.randperm(sum(need) + 5, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((R, max(need)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for r, x in enumerate(need):
        table[r, :x] = perm[at:at + x]
        at += x
    free = torch.full((sum(need) + 5,), -1, dtype=torch.int32, device=DEV)
    free[:5] = perm[at:]
    s = {"case": case, "table": table, "seq_len": _i32(L), "tok_indptr": _indptr(L), "max_tok": max(L), "free": free, "free_count": _i32([5]),
         "pool": torch.randn((nl, 2, sum(need) + 5, page, hk, d), generator=gen, device=DEV, dtype=torch.bfloat16)}
    s["req"] = torch.repeat_interleave(torch.arange(R, device=DEV), torch.tensor(L, device=DEV))
    s["token"] = torch.cat([torch.arange(x, device=DEV) for x in L])
    pairs, axes, units = case["rotary"] // 2, case["axes"], nl * hk if case["per_unit"] else 1
    s["inv_freq"] = (1e6 ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / pairs)).float()
    s["sections"] = _sections(pairs, axes)
    s["axis"] = torch.repeat_interleave(torch.arange(axes, device=DEV), torch.tensor(s["sections"], device=DEV))
    s["to_inv_freq"] = None
    if case["rescale"]:                                          # slow pairs four times slower, fast ones as they were
        ramp = torch.linspace(0, 1, pairs, device=DEV, dtype=torch.float64)
        s["to_inv_freq"] = (s["inv_freq"].double() * (1 - ramp * 0.75)).float()
    if case["rescale"] and not case["per_unit"]:
        s["from_pos"] = s["to_pos"] = None                       # a token's position is its index, before and after
        return s
    # the survivors of a compaction: a kept prefix, then tokens with gaps between them; they move up to their index
    gap = 1 + (torch.rand((axes, units, n), generator=gen, device=DEV) ** 4 * 16).to(torch.int32)
    head = (s["token"] < case["prefix"])[None, None]
    gap = torch.where(head, 1, gap + (s["token"] == case["prefix"]).to(torch.int32)[None, None])
    run = gap.cumsum(-1, dtype=torch.int32)
    start = s["tok_indptr"][:-1].long()[s["req"]]
    s["from_pos"] = (run - run[..., start] + gap[..., start] - 1).contiguous()
    s["to_pos"] = None
    return s


def _prepare_penalize(case, gen):
    win, hist, masked = _lengths(case)
    R, V, rows = case["requests"], case["vocab"], sum(win)
    f = lambda lo, hi: lo + (hi - lo) * torch.rand(R, generator=gen, device=DEV)
    off = torch.rand(R, generator=gen, device=DEV) < 0.1         # some requests ask for no penalty
    s = {"case": case, "rows": rows, "max_win": max(win), "max_hist": max(hist), "win_indptr": _indptr(win), "hist_len": _i32(hist)}
    s["logits"] = _logits(rows, V, gen, case["bf16"])
    s["tokens"] = (torch.rand((R, max(hist)), generator=gen, device=DEV, dtype=torch.float64) ** 3 * V).to(torch.int32).clamp_(max=V - 1)
    s["prompt_len"] = (s["hist_len"] * f(0.2, 0.9)).to(torch.int32)
    s["repetition"] = torch.where(off, 1.0, f(1.0, 1.3))
    s["frequency"], s["presence"] = torch.where(off, 0.0, f(0.0, 0.6)), torch.where(off, 0.0, f(0.0, 0.8))
    s["bias_indptr"] = s["bias_token"] = s["bias_value"] = None
    if case["biases"]:
        n = min(case["biases"], V)
        s["bias_indptr"] = _indptr([n] * R)
        s["bias_token"] = torch.rand((R, V), generator=gen, device=DEV).topk(n, dim=1).indices.sort(1).values.to(torch.int32).flatten()
        s["bias_value"] = torch.randn(R * n, generator=gen, device=DEV).mul_(3.0)
        s["bias_value"][::7] = -math.inf                         # tokens that must not be drawn
    s["allow"] = s["allow_row"] = None
    n = sum(w for w, m in zip(win, masked) if m)
    if n:
        share = torch.tensor([_share(i) for i in range(n)], device=DEV)[:, None]
        words = (V + 31) // 32
        s["allow"] = torch.zeros((n, words), dtype=torch.int32, device=DEV)
        for bit in range(32):
            s["allow"] |= (torch.rand((n, words), generator=gen, device=DEV) < share).to(torch.int32) << bit
        rows_of, at = [], 0
        for w, m in zip(win, masked):
            rows_of += list(range(at, at + w)) if m else [-1] * w
            at += w if m else 0
        s["allow_row"] = _i32(rows_of)
    s["out"] = s["logits"] if case["in_place"] else torch.empty_like(s["logits"])
    # what the plain form looks up: each row's request and how much of the history it stands behind
    w = torch.tensor(win, device=DEV)
    s["row_req"] = torch.repeat_interleave(torch.arange(R, device=DEV), w)
    behind = torch.cat([torch.arange(x, device=DEV) for x in win]) - w[s["row_req"]] + 1
    s["row_len"] = s["hist_len"].long()[s["row_req"]] + behind
    return s


def _prepare_sample(case, gen):
    n = case["rows"]
    x = _logits(n, case["vocab"], gen, False)
    if case["masked"]:                                           # a grammar allows a tenth of the vocabulary
        x.masked_fill_(torch.rand(x.shape, generator=gen, device=DEV) > 0.1, -math.inf)
    full = lambda v, t: torch.full((n,), v, dtype=t, device=DEV)
    s = {"case": case, "logits": x.to(torch.bfloat16) if case["bf16"] else x, "u": torch.rand(n, generator=gen, device=DEV),
         "temperature": full(case["temperature"], torch.float32), "top_k": full(case["top_k"], torch.int32),
         "top_p": full(case["top_p"], torch.float32), "min_p": full(case["min_p"], torch.float32)}
    if case["mixed"]:                                            # every fourth row has settings of its own, some of them greedy
        odd = torch.rand(n, generator=gen, device=DEV) < 0.25
        pick = lambda *v: torch.tensor(v, device=DEV)[torch.randint(len(v), (n,), generator=gen, device=DEV)]
        s["temperature"] = torch.where(odd, pick(0.0, 0.5, 0.7, 1.3), s["temperature"])
        s["top_k"] = torch.where(odd, pick(0, 0, 20, 40), s["top_k"]).to(torch.int32)
        s["top_p"] = torch.where(odd, pick(1.0, 0.95, 0.8, 0.9), s["top_p"])
        s["min_p"] = torch.where(odd, pick(0.0, 0.0, 0.0, 0.1), s["min_p"])
    return s


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return {"reposition": _prepare_reposition, "penalize": _prepare_penalize, "sample": _prepare_sample}[case["kind"]](case, gen)


# ---------------------------------------------------------------------------------------------------------------
# one pass


def _handle(s):
    """What a program keeps beside its cache and its logits: the decoder, the rotary description, rules, result buffers."""
    from paper_2609_31395_b200 import harness as H
    case = s["case"]
    if case["kind"] == "reposition":
        s["rope"] = H.Rope(s["inv_freq"], s["sections"], case["interleaved"])
        s["handle"] = H.Decoder(s["pool"], s["table"], s["seq_len"], s["free"], s["free_count"], case["kv_heads"], max_tok=s["max_tok"],
                                layers_per_call=case["layers"])
    elif case["kind"] == "penalize":
        s["rules"] = H.LogitRules(s["tokens"], s["hist_len"], s["prompt_len"], s["repetition"], s["frequency"], s["presence"],
                                  s["bias_indptr"], s["bias_token"], s["bias_value"], s["allow"], s["allow_row"])
        s["handle"] = H.Sampler(s["rows"], DEV)
    else:
        s["handle"] = H.Sampler(case["rows"], DEV)
    return s["handle"]


def run(s):
    case = s["case"]
    if own:
        h = s["handle"] if "handle" in s else _handle(s)
        if case["kind"] == "reposition":
            h.reposition(s["rope"], s["tok_indptr"], s["max_tok"], s["from_pos"], s["to_pos"], s["to_inv_freq"])
            return {"pool": s["pool"]}
        if case["kind"] == "penalize":
            h.penalize(s["logits"], s["win_indptr"], s["rules"], s["max_win"], s["max_hist"], out=s["out"])
            return {"logits": s["out"]}
        h.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
        return {"token": h.token, "logprob": h.logprob, "kept": h.kept}
    return {"reposition": _reposition, "penalize": _penalize, "sample": _sample}[case["kind"]](s)


def _reposition(s):
    case, pool, P = s["case"], s["pool"], s["case"]["page"]
    nl, hk, pairs = case["layers"], case["kv_heads"], case["rotary"] // 2
    f0 = s["inv_freq"].double()
    f1 = f0 if s["to_inv_freq"] is None else s["to_inv_freq"].double()
    index = s["token"][None, None]
    p0, p1 = (index if p is None else p for p in (s["from_pos"], s["to_pos"]))
    axis = s["axis"] if p0.shape[0] > 1 else torch.zeros_like(s["axis"])
    a = p0.double()[axis] * f0[:, None, None]                    # [pair, unit or 1, token]; angles of far positions: in 64 bits
    b = p1.double()[axis if p1.shape[0] > 1 else torch.zeros_like(axis)] * f1[:, None, None]
    turn = (b - a).permute(2, 1, 0)
    turn = turn.expand(turn.shape[0], nl * hk, pairs) if turn.shape[1] == 1 else turn
    turn = turn.reshape(-1, nl, hk, pairs).transpose(0, 1)       # [layer, token, head, pair]
    cos, sin = turn.cos().float(), turn.sin().float()
    page, slot = s["table"].long()[s["req"], s["token"] // P], s["token"] % P
    x = pool[:, 0, page, slot]                                   # [layer, token, head, dim]
    lo, hi = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if case["interleaved"] else (slice(0, pairs), slice(pairs, 2 * pairs))
    y = x.clone()
    u, v = x[..., lo].float(), x[..., hi].float()
    y[..., lo] = (u * cos - v * sin).to(torch.bfloat16)
    y[..., hi] = (v * cos + u * sin).to(torch.bfloat16)
    pool[:, 0, page, slot] = y
    return {"pool": pool}


def _penalize(s):
    V, rr = s["case"]["vocab"], s["row_req"]
    z = s["logits"].float()
    rows = z.shape[0]
    if s["bias_indptr"] is not None:
        per = s["bias_token"].view(s["hist_len"].shape[0], -1)
        z = z.scatter_add(1, per.long()[rr], s["bias_value"].view_as(per)[rr])
    at = torch.arange(s["tokens"].shape[1], device=DEV)
    held = at < s["row_len"][:, None]
    made = held & (at >= s["prompt_len"].long()[rr][:, None])
    place = s["tokens"].long()[rr]
    count = torch.zeros((rows, V + 1), dtype=torch.int32, device=DEV)
    count.scatter_add_(1, torch.where(made, place, V), torch.ones_like(place, dtype=torch.int32))
    seen = torch.zeros((rows, V + 1), dtype=torch.bool, device=DEV)
    seen.scatter_(1, torch.where(held, place, V), True)
    n = count[:, :V].float()
    theta = s["repetition"][rr][:, None]
    z = torch.where(seen[:, :V], torch.where(z > 0, z / theta, z * theta), z)
    z = z - (s["frequency"][rr][:, None] * n + s["presence"][rr][:, None] * (n > 0))
    if s["allow"] is not None:
        t = torch.arange(V, device=DEV)
        free = (s["allow"][:, t // 32] >> (t % 32).to(torch.int32)) & 1
        row = s["allow_row"].long()
        z = torch.where((row < 0)[:, None] | (free[row.clamp_min(0)] != 0), z, -math.inf)
    s["out"].copy_(z)
    return {"logits": s["out"]}


def _sample(s):
    x = s["logits"].float()
    T = s["temperature"].double()[:, None]
    n, V = x.shape
    z, order = x.sort(dim=1, descending=True, stable=True)       # equal logits: the lowest token first
    y = z.double() - z[:, :1].double()
    w = torch.where(T > 0, (y / torch.where(T > 0, T, 1.0)).exp(), 0.0)    # sums next to a border: in 64 bits
    place = torch.arange(V, device=DEV)
    k = s["top_k"].long()[:, None]
    w = torch.where((k <= 0) | (place < k), w, 0.0)
    p = s["top_p"].double()[:, None]
    before = w.cumsum(1) - w
    inside = (p >= 1.0) | (before < p * w.sum(1, keepdim=True))
    keep = (inside & ((k <= 0) | (place < k)) & (w >= s["min_p"].double()[:, None]) & (z > -math.inf) & (T > 0)) | (place == 0)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    wv = torch.where(kept, torch.where(T > 0, ((x.double() - z[:, :1].double()) / torch.where(T > 0, T, 1.0)).exp(), 1.0), 0.0)
    run_ = wv.cumsum(1)
    total = run_[:, -1:]
    token = (run_ <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp_max(V - 1)
    logprob = (wv.gather(1, token) / total).log()
    return {"token": token[:, 0].to(torch.int32), "logprob": logprob[:, 0].float(), "kept": kept.sum(1).to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in float64


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "reposition":
        P, nl, hk, half = case["page"], case["layers"], case["kv_heads"], case["rotary"] // 2
        pool, table, L = s["pool"].double(), s["table"].long(), s["seq_len"].tolist()
        to_freq = s["inv_freq"] if s["to_inv_freq"] is None else s["to_inv_freq"]
        for r, n in enumerate(L):
            j = torch.arange(n, device=DEV)
            first = int(s["tok_indptr"][r])
            for layer in range(nl):
                for h in range(hk):
                    old = pool[layer, 0, table[r, j // P], j % P, h]
                    k = torch.complex(torch.zeros_like(old[:, :half]), torch.zeros_like(old[:, :half]))
                    a, b = (old[:, 0:2 * half:2], old[:, 1:2 * half:2]) if case["interleaved"] else (old[:, :half], old[:, half:2 * half])
                    was = j[:, None].double().expand(n, half)
                    if s["from_pos"] is not None:
                        unit = layer * hk + h if case["per_unit"] else 0
                        was = s["from_pos"][:, unit, first:first + n][s["axis"]].T.double()
                    angle = j[:, None].double() * to_freq.double() - was * s["inv_freq"].double()
                    k = torch.complex(a, b) * torch.polar(torch.ones_like(angle), angle)
                    new = old.clone()
                    if case["interleaved"]:
                        new[:, 0:2 * half:2], new[:, 1:2 * half:2] = k.real, k.imag
                    else:
                        new[:, :half], new[:, half:2 * half] = k.real, k.imag
                    pool[layer, 0, table[r, j // P], j % P, h] = new
        return {"pool": pool}
    if case["kind"] == "penalize":
        V = case["vocab"]
        out = torch.empty((s["rows"], V), dtype=torch.float64, device=DEV)
        for i in range(s["rows"]):
            r, n = int(s["row_req"][i]), int(s["row_len"][i])
            z = s["logits"][i].double()
            if case["biases"]:
                lo, hi = s["bias_indptr"][r:r + 2].tolist()
                z[s["bias_token"][lo:hi].long()] += s["bias_value"][lo:hi].double()
            past = s["tokens"][r, :n].long()
            made = torch.bincount(past[int(s["prompt_len"][r]):], minlength=V)
            any_ = torch.bincount(past, minlength=V) > 0
            theta = float(s["repetition"][r])
            z = torch.where(any_ & (z > 0), z / theta, torch.where(any_, z * theta, z))
            z = z - float(s["frequency"][r]) * made - float(s["presence"][r]) * made.clamp_max(1)
            if s["allow"] is not None and int(s["allow_row"][i]) >= 0:
                words = s["allow"][int(s["allow_row"][i])]
                bits = (words[:, None] >> torch.arange(32, dtype=torch.int32, device=DEV)) & 1
                z[bits.flatten()[:V] == 0] = -math.inf
            out[i] = z
        return {"logits": out}
    logprob = torch.zeros(case["rows"], dtype=torch.float64, device=DEV)
    for i in range(case["rows"]):
        t, k, p, m = (float(s[name][i]) for name in ("temperature", "top_k", "top_p", "min_p"))
        if t == 0:
            continue
        z = s["logits"][i].double()
        by = torch.argsort(-z, stable=True)
        by = by[:int(k)] if k > 0 else by
        by = by[z[by] > -math.inf]
        prob = torch.softmax(z[by] / t, 0)
        if p < 1:
            by = by[:int(torch.searchsorted(prob.cumsum(0), torch.tensor(p, dtype=torch.float64, device=DEV))) + 1]
        lead = torch.exp((z[by] - z[by[0]]) / t)
        by = by[: max(1, int((lead >= m).sum()))].sort().values
        prob = torch.softmax(z[by] / t, 0)
        at = int(torch.searchsorted(prob.cumsum(0), s["u"][i].double(), right=True))
        logprob[i] = prob[min(at, len(by) - 1)].log()
    return {"token": None, "logprob": logprob, "kept": None}
