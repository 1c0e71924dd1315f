"""Decoding on the paged cache between two compression steps, as timed cases.

A case is a dict of plain sizes and options.  `prepare` builds what a program holds before the call, `run` makes one pass
through one operator.  Five kinds:

  attend   attention of the newest tokens of every request over its pages; output and LSE (`Decoder.attend`)
  append   rotary positions of new queries and keys, keys and values written into their pages (`Decoder.append`)
  resize   requests grow by new tokens, are cut back or freed: pages from and to the free list (`Decoder.resize`)
  copy     the cache of requests copied into branches of them (`Decoder.copy`)
  logprob  log probabilities of given tokens, entropy and the most probable alternatives (`actkv_logprob`)

With `own` false, `run` computes the same in elementary torch operations.  `exact` is the definition in float64.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
VOCAB = 151936

ATTEND = dict(kind="attend", layers=1, kv_heads=8, group=4, head_dim=128, page=16, requests=1, len_lo=1000, len_hi=1000,
              win_lo=1, win_hi=1, causal=True, sliding=0, shape=1)
APPEND = dict(kind="append", layers=1, kv_heads=8, group=4, head_dim=128, page=16, requests=1, win_lo=1, win_hi=1,
              context=200, rotary=128, axes=1, interleaved=False, shape=1)
RESIZE = dict(kind="resize", page=16, requests=16, len_lo=4000, len_hi=16000, grow=1, freed=0, cut=0, shape=1)
COPY = dict(kind="copy", layers=1, kv_heads=8, head_dim=128, page=16, requests=1, branches=1, len_lo=1000, len_hi=1000,
            shape=1)
LOGPROB = dict(kind="logprob", rows=16, vocab=VOCAB, given=1, top=20, bf16=False, masked=False)


def listed():
    return [
        # One decode step of one agent with a 4096-token cache cut to about 1000: called once per layer, latency counts.
        dict(ATTEND, name="attend_1k_x1", len_lo=1021, len_hi=1021),
        # The benchmark's cache, 8 requests x 35000 tokens, 4 KV heads of 8 query heads: one decode step of one layer.
        dict(ATTEND, name="attend_35k_x8", kv_heads=4, group=8, requests=8, len_lo=35000, len_hi=35000),
        # The serving mix: 64 requests of 8K to 32K tokens in a fragmented pool, one decode step of one layer.
        dict(ATTEND, name="attend_mix_x64", kv_heads=4, group=8, requests=64, len_lo=8192, len_hi=32768, shape=4),
        # Drafted tokens are verified: 4 to 8 of them per request, causal among themselves; head_dim 64, pages of 32.
        dict(ATTEND, name="attend_draft_x16", group=8, head_dim=64, page=32, requests=16, len_lo=12000, len_hi=20000,
             win_lo=4, win_hi=8, shape=5),
        # The new tokens of one decode step of 8 requests, one layer: the smallest call, behind the QKV product.
        dict(APPEND, name="append_decode_x8", kv_heads=4, group=8, requests=8),
        # Observations of tools (with images: positions of time, height, width) come in: 16 requests, 300 to 700 tokens.
        dict(APPEND, name="append_chunk_x16", requests=16, win_lo=300, win_hi=700, axes=3, shape=6),
        # Pages for one more token of 16 requests.
        dict(RESIZE, name="resize_decode_x16"),
        # A scheduler's turn over 64 requests: observations of up to 700 tokens come in, some requests end, some drafts
        # are taken back.
        dict(RESIZE, name="resize_round_x64", requests=64, len_lo=8192, len_hi=32768, grow=700, freed=8, cut=8, shape=7),
        # One agent tries a second action: its compressed cache of 1000 tokens, 8 layers of it.
        dict(COPY, name="copy_1k_x1", layers=8, len_lo=1021, len_hi=1021),
        # A 35000-token trace goes on in three branches; 6 layers of 4 KV heads.
        dict(COPY, name="copy_35k_x3", layers=6, kv_heads=4, branches=3, len_lo=35000, len_hi=35000),
        # One decode step of 16 requests: log probability of the sampled token, entropy, 20 alternatives (the monitor's k).
        dict(LOGPROB, name="logprob_decode_x16"),
        # Sampled actions are scored: the logits of 1500 action tokens at once.
        dict(LOGPROB, name="logprob_score_x1500", rows=1500, top=8),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend", "append", "append", "resize", "copy", "logprob", "logprob"])
    shape = rng.randrange(1, 1 << 20)
    if kind == "attend":
        tokens = _log_uniform(rng, 100, 400000)                  # of all requests together
        mean = min(tokens, _log_uniform(rng, 64, 40000))
        requests = max(1, min(96, tokens // mean))
        win = rng.choice([1, 1, 1, rng.randrange(2, 9)])
        return dict(ATTEND, layers=1 if tokens > 100000 else rng.choice([1, 1, 2]), kv_heads=rng.choice([1, 2, 4, 8]),
                    group=rng.choice([1, 4, 7, 8]), head_dim=rng.choice([64, 128, 128, 80]), page=rng.choice([16, 16, 32, 64]),
                    requests=requests, len_lo=max(win, int(mean * 0.6)), len_hi=max(win, int(mean * 1.4)), win_lo=(win + 1) // 2,
                    win_hi=win, causal=rng.random() < 0.8, sliding=rng.choice([0, 0, 0, 128, 1000]), shape=shape)
    if kind == "append":
        tokens = _log_uniform(rng, 1, 9000)
        requests = max(1, min(tokens, _log_uniform(rng, 1, 64)))
        win = max(1, tokens // requests)
        dim = rng.choice([64, 128, 128, 80])
        return dict(APPEND, layers=rng.choice([1, 1, 2]) if tokens < 2000 else 1, kv_heads=rng.choice([1, 4, 8]),
                    group=rng.choice([1, 4, 7, 8]), head_dim=dim, page=rng.choice([16, 16, 32]), requests=requests,
                    win_lo=max(1, win // 2), win_hi=win, context=rng.randrange(0, 300),
                    rotary=rng.choice([dim, dim, dim // 2, 0]), axes=rng.choice([1, 1, 2, 3]),
                    interleaved=rng.random() < 0.3, shape=shape)
    if kind == "resize":
        requests = _log_uniform(rng, 1, 96)
        lo = _log_uniform(rng, 100, 20000)
        return dict(RESIZE, page=rng.choice([16, 16, 32, 5]), requests=requests, len_lo=lo, len_hi=lo * 2,
                    grow=_log_uniform(rng, 1, 1500), freed=rng.randrange(0, requests // 4 + 1),
                    cut=rng.randrange(0, requests // 4 + 1), shape=shape)
    if kind == "copy":
        rows = _log_uniform(rng, 500, 120000)                    # (token, layer) pairs written
        mean = min(rows, _log_uniform(rng, 100, 30000))
        branches = rng.choice([1, 2, 3, 5])
        requests = max(1, min(8, rows // mean // branches))
        return dict(COPY, layers=max(1, min(12, rows // (mean * requests * branches))), kv_heads=rng.choice([2, 4, 8]),
                    head_dim=rng.choice([64, 128, 80]), page=rng.choice([16, 32]), requests=requests, branches=branches,
                    len_lo=max(1, int(mean * 0.6)), len_hi=max(1, int(mean * 1.4)), shape=shape)
    top = rng.choice([0, 1, 5, 20, 64])
    return dict(LOGPROB, rows=_log_uniform(rng, 1, 1200), vocab=rng.choice([VOCAB, VOCAB, 32003, 1009]),
                given=rng.choice([1, 1, 0, 4]), top=top, bf16=rng.random() < 0.4, masked=rng.random() < 0.3)


# ---------------------------------------------------------------------------------------------------------------
# what the sizes of a case come to, from the case alone


def _lengths(case):
    rng = random.Random(case["shape"])
    R = case["requests"]
    L = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(R)] if "len_lo" in case else None
    W = [rng.randint(case["win_lo"], case["win_hi"]) for _ in range(R)] if "win_lo" in case else None
    return L, W, rng


def _new_lengths(case):
    L, _, rng = _lengths(case)
    order = rng.sample(range(len(L)), len(L))
    freed, cut = set(order[:case["freed"]]), set(order[case["freed"]:case["freed"] + case["cut"]])
    new = [0 if r in freed else max(0, n - rng.randint(1, 40)) if r in cut else n + rng.randint(1, case["grow"])
           for r, n in enumerate(L)]
    return L, new


def _visible(case):
    """Per request the keys that at least one of its rows sees."""
    L, W, _ = _lengths(case)
    S = case["sliding"]
    return [min(n, S + (w - 1 if case["causal"] else 0)) if S else n for n, w in zip(L, W)]


def work(case):
    if case["kind"] == "attend":
        L, W, _ = _lengths(case)
        hq, d, nl = case["kv_heads"] * case["group"], case["head_dim"], case["layers"]
        keys = _visible(case)
        rows = sum(W)
        return {"bytes": nl * (sum(keys) * case["kv_heads"] * d * 4 + rows * hq * (d * 4 + 4)),
                "flops": nl * sum(4 * d * hq * w * n for w, n in zip(W, keys))}
    if case["kind"] == "append":
        _, W, _ = _lengths(case)
        hq, hk, d, nl = case["kv_heads"] * case["group"], case["kv_heads"], case["head_dim"], case["layers"]
        n = sum(W)
        return {"bytes": nl * n * (hq + 2 * hk) * d * 4 + 4 * case["axes"] * n,
                "flops": nl * n * (hq + hk) * case["rotary"] * 3}
    if case["kind"] == "resize":
        L, new = _new_lengths(case)
        p = case["page"]
        moved = sum(abs(-(-a // p) - -(-b // p)) for a, b in zip(L, new))
        return {"bytes": moved * 8 + 12 * len(L), "flops": 0}
    if case["kind"] == "copy":
        L, _, _ = _lengths(case)
        return {"bytes": sum(L) * (1 + case["branches"]) * case["layers"] * case["kv_heads"] * case["head_dim"] * 4, "flops": 0}
    item = 2 if case["bf16"] else 4
    return {"bytes": case["rows"] * (case["vocab"] * item + 8 * case["given"] + 8 * case["top"] + 8),
            "flops": case["rows"] * case["vocab"] * 6}


# ---------------------------------------------------------------------------------------------------------------
# inputs


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _indptr(x):
    return _i32([0] + torch.tensor(x).cumsum(0).tolist())


def _tables(lens, page, max_pages, spare, gen):
    """Pages of all requests drawn from one shuffled pool; the others are on the free list."""
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + spare
    perm = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(lens), max_pages), -1, dtype=torch.int32, device=DEV)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = perm[at:at + n]
        at += n
    free = torch.full((n_pages,), -1, dtype=torch.int32, device=DEV)
    free[:spare] = perm[at:]
    return table, free, n_pages


def _normal(shape, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16).mul_(scale)


def _sections(pairs, axes):
    """The rotary pairs of each axis: the first one a little shorter, as time has it beside height and width."""
    if axes == 1 or pairs < axes:
        return [pairs] + [0] * (axes - 1)
    first = max(1, pairs // (axes + 1))
    rest = [(pairs - first) // (axes - 1)] * (axes - 1)
    rest[-1] += pairs - first - sum(rest)
    return [first] + rest


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = {"case": case}
    kind = case["kind"]
    if kind == "logprob":
        x = torch.randn((case["rows"], case["vocab"]), generator=gen, device=DEV)
        x.mul_(2.5)
        hot = torch.randint(case["vocab"], (case["rows"], 24), generator=gen, device=DEV)     # a few tokens stand out
        x.scatter_add_(1, hot, 9.0 * torch.rand((case["rows"], 24), generator=gen, device=DEV))
        if case["masked"]:                                       # a grammar allows a tenth of the vocabulary
            x.masked_fill_(torch.rand(x.shape, generator=gen, device=DEV) > 0.1, -math.inf)
        given = torch.randint(case["vocab"], (case["rows"], case["given"]), generator=gen, device=DEV).to(torch.int32)
        if case["given"]:                                        # a sampled token is mostly a probable one
            given[:, 0] = torch.where(torch.rand(case["rows"], generator=gen, device=DEV) < 0.8, hot[:, 0].to(torch.int32), given[:, 0])
        s["logits"] = x.to(torch.bfloat16) if case["bf16"] else x
        s["given"] = given
        return s
    page = case["page"]
    L, W, rng = _lengths(case)
    if kind == "resize":
        L, new = _new_lengths(case)
        width = max(-(-max(a, b) // page) for a, b in zip(L, new))
        grown = sum(max(0, -(-b // page) - -(-a // page)) for a, b in zip(L, new))
        table, free, n_pages = _tables(L, page, width, grown + 7, gen)
        # the tables in one buffer, as a serving program uploads them before the call
        now = torch.cat([table.flatten(), _i32(L), free, _i32([grown + 7])])
        work_buf = now.clone()
        R = len(L)
        cut = [R * width, R * width + R, R * width + R + n_pages]
        s["pool"] = torch.empty((1, 2, n_pages, page, 1, 8), dtype=torch.bfloat16, device=DEV)
        s.update(now=now, buf=work_buf, table=work_buf[:cut[0]].view(R, width), seq_len=work_buf[cut[0]:cut[1]],
                 free=work_buf[cut[1]:cut[2]], free_count=work_buf[cut[2]:], new_len=_i32(new), n_pages=n_pages)
        return s
    nl, hk, d = case["layers"], case["kv_heads"], case["head_dim"]
    if kind == "append":
        ctx = [rng.randint(0, case["context"]) for _ in W]
        L = [a + b for a, b in zip(ctx, W)]
    if kind == "copy":
        src, dst = list(range(len(L))), []
        pairs = [(r, b) for r in src for b in range(case["branches"])]
        s["src"] = _i32([r for r, _ in pairs])
        s["dst"] = _i32([len(L) + i for i in range(len(pairs))])
        s["len"] = _i32([L[r] for r, _ in pairs])
        s["max_len"] = max(L)
        L = L + [L[r] for r, _ in pairs]
    table, free, n_pages = _tables(L, page, max(-(-n // page) for n in L), 5, gen)
    s.update(pool=_normal((nl, 2, n_pages, page, hk, d), gen), table=table, seq_len=_i32(L), free=free, free_count=_i32([5]),
             max_tok=max(L))
    if kind == "copy":
        return s
    hq, rows = hk * case["group"], sum(W)
    s.update(win_indptr=_indptr(W), rows=rows, max_win=max(W),
             row_req=torch.repeat_interleave(torch.arange(len(W), device=DEV), torch.tensor(W, device=DEV)),
             row_win=torch.cat([torch.arange(w, device=DEV) for w in W]))
    if kind == "attend":
        # logits of standard deviation 2: some keys matter, most hardly do
        s["q"] = _normal((nl, rows, hq, d), gen, 2.0)
        s["scale"] = 1.0 / math.sqrt(d)
        return s
    # q, k and v lie side by side in the rows of one product
    s["qkv"] = _normal((nl, rows, hq + 2 * hk, d), gen)
    pairs = case["rotary"] // 2
    base = torch.tensor([rng.randint(0, 120000) for _ in W], device=DEV)
    s["positions"] = (base[s["row_req"]] + s["row_win"] + torch.arange(case["axes"], device=DEV)[:, None] * 17).to(torch.int32)
    s["inv_freq"] = (1e6 ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / max(1, pairs))).float()
    s["sections"] = _sections(pairs, case["axes"])
    s["axis"] = torch.repeat_interleave(torch.arange(case["axes"], device=DEV), torch.tensor(s["sections"], device=DEV))
    return s


# ---------------------------------------------------------------------------------------------------------------
# one pass


def _handle(s):
    """What a program keeps beside its cache: the decoder with its workspace, and output buffers."""
    if "handle" not in s:
        from paper_2609_31395_b200 import harness as H
        case = s["case"]
        if case["kind"] == "logprob":
            s["out"] = H.LogprobBuffers(case["rows"], case["given"], case["top"], DEV)
            s["handle"] = None
            return None
        hq = case.get("kv_heads", 1) * case.get("group", 1)
        s["handle"] = H.Decoder(s["pool"], s["table"], s["seq_len"], s["free"], s["free_count"], hq, max_rows=s.get("rows", 0),
                                max_win=s.get("max_win", 1), max_tok=s.get("max_tok", 1), layers_per_call=case.get("layers", 1))
        if case["kind"] == "append" and case["rotary"]:
            s["rope"] = H.Rope(s["inv_freq"], s["sections"], case["interleaved"])
        if case["kind"] in ("attend", "append"):
            q = s["q"] if case["kind"] == "attend" else s["qkv"][:, :, :hq]
            s["out"] = torch.empty(q.shape, dtype=torch.bfloat16, device=DEV)
            s["lse"] = torch.empty(q.shape[:3], dtype=torch.float32, device=DEV)
    return s["handle"]


def run(s):
    case = s["case"]
    if own:
        h = s["handle"] if "handle" in s else _handle(s)
        if case["kind"] == "attend":
            h.attend(s["q"], s["win_indptr"], s["scale"], case["causal"], s["out"], s["lse"], window_left=case["sliding"])
            return {"out": s["out"], "lse": s["lse"]}
        if case["kind"] == "append":
            hk = case["kv_heads"]
            hq = hk * case["group"]
            q, k, v = s["qkv"][:, :, :hq], s["qkv"][:, :, hq:hq + hk], s["qkv"][:, :, hq + hk:]
            h.append(k, v, s["win_indptr"], q=q, q_out=s["out"], rope=s.get("rope"), positions=s["positions"])
            return {"q": s["out"], "pool": s["pool"]}
        if case["kind"] == "resize":
            s["buf"].copy_(s["now"])
            h.resize(s["new_len"])
            return {"table": s["table"], "seq_len": s["seq_len"], "free": s["free"], "free_count": s["free_count"]}
        if case["kind"] == "copy":
            h.copy(s["src"], s["dst"], s["len"], s["max_len"])
            return {"pool": s["pool"]}
        from paper_2609_31395_b200 import binding as B
        o = s["out"]
        B.actkv_logprob(s["logits"], s["given"] if case["given"] else None, o.logprob, o.entropy, o.lse, o.top_logprob, o.top_index, o.status)
        return {"logprob": o.logprob, "entropy": o.entropy, "lse": o.lse, "top_logprob": o.top_logprob, "top_index": o.top_index}
    return {"attend": _attend, "append": _append, "resize": _resize, "copy": _copy, "logprob": _logprob}[case["kind"]](s)


def _attend(s):
    case, pool, q = s["case"], s["pool"], s["q"]
    nl, rows, hq, d = q.shape
    hk, G, R, W = case["kv_heads"], case["group"], case["requests"], s["max_win"]
    pages = s["table"].long().clamp_min(0)
    kv = pool[:, :, pages].float().flatten(3, 4)                               # [layer, 2, request, key, head, dim]
    N = kv.shape[3]
    key = torch.arange(N, device=DEV)
    L = s["seq_len"].long()
    held = (key < L[:, None])[:, :, None, None]
    k = torch.where(held, kv[:, 0], 0.0).permute(0, 1, 3, 4, 2)                # [layer, request, head, dim, key]
    v = torch.where(held, kv[:, 1], 0.0).transpose(2, 3)                       # [layer, request, head, key, dim]
    qp = torch.zeros((nl, R, W, hk, G, d), device=DEV)
    qp[:, s["row_req"], s["row_win"]] = q.float().view(nl, rows, hk, G, d)
    qp = qp.permute(0, 1, 3, 2, 4, 5).reshape(nl, R, hk, W * G, d)
    x = (qp @ k * s["scale"]).view(nl, R, hk, W, G, N)
    n_win = (s["win_indptr"][1:] - s["win_indptr"][:-1]).long()
    w = torch.arange(W, device=DEV)
    at = (L - n_win)[:, None] + w if case["causal"] else (L - 1)[:, None] + 0 * w    # the cache position a row stands at
    seen = (key < L[:, None, None]) & (key <= at[:, :, None])
    if case["sliding"]:
        seen = seen & (key > at[:, :, None] - case["sliding"])
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = (x - torch.where(top == -math.inf, 0.0, top)).exp()
    total = p.sum(-1)
    o = (p.view(nl, R, hk, W * G, N) @ v).view(nl, R, hk, W, G, d) / total.clamp_min(1e-38)[..., None]
    lse = top[..., 0] + total.log()
    pick = lambda t: t.transpose(2, 3)[:, s["row_req"], s["row_win"]]          # [layer, row, head, group, ...]
    return {"out": pick(o).reshape(nl, rows, hq, d).to(torch.bfloat16), "lse": pick(lse).reshape(nl, rows, hq)}


def _rotated(x, cos, sin, rotary, interleaved):
    """x [layer, row, head, dim] in the type of cos; cos, sin [row, 1, pair]."""
    y = x.clone()
    if not rotary:
        return y
    a, b = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, rotary // 2), slice(rotary // 2, rotary))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _append(s):
    case, qkv, pool = s["case"], s["qkv"], s["pool"]
    hk = case["kv_heads"]
    hq = hk * case["group"]
    # angles of far positions: in 64 bits
    turn = s["positions"][s["axis"]].double() * s["inv_freq"].double()[:, None]
    cos, sin = turn.cos().T[:, None, :].float(), turn.sin().T[:, None, :].float()
    qk = _rotated(qkv[:, :, :hq + hk].float(), cos, sin, case["rotary"], case["interleaved"]).to(torch.bfloat16)
    r = s["row_req"]
    at = s["seq_len"].long()[r] - (s["win_indptr"][1:] - s["win_indptr"][:-1]).long()[r] + s["row_win"]
    page, slot = s["table"].long()[r, at // case["page"]], at % case["page"]
    pool[:, 0, page, slot] = qk[:, :, hq:]
    pool[:, 1, page, slot] = qkv[:, :, hq + hk:]
    return {"q": qk[:, :, :hq], "pool": pool}


def _resize(s):
    s["buf"].copy_(s["now"])
    P, table, L, new = s["case"]["page"], s["table"], s["seq_len"].long(), s["new_len"].long()
    n_pages = s["n_pages"]
    Y, X = (L + P - 1) // P, (new + P - 1) // P
    grow, shrink = (X - Y).clamp_min(0), (Y - X).clamp_min(0)
    first, put = grow.cumsum(0) - grow, shrink.cumsum(0) - shrink
    count = s["free_count"].long()
    col = torch.arange(table.shape[1], device=DEV)
    rel = col - Y[:, None]
    popped = s["free"][(count - 1 - (first[:, None] + rel)).clamp(0, n_pages - 1)]
    mid = torch.where((rel >= 0) & (col < X[:, None]), popped, table)
    gone = (col >= X[:, None]) & (col < Y[:, None])
    to = torch.where(gone, count - grow.sum() + put[:, None] + col - X[:, None], n_pages)      # the others: a place behind the list
    longer = torch.cat([s["free"], s["free"][:1]])
    longer[to.flatten()] = mid.flatten()
    s["free"].copy_(longer[:n_pages])
    table.copy_(torch.where(gone, -1, mid))
    s["seq_len"].copy_(new)
    s["free_count"].copy_(count - grow.sum() + shrink.sum())
    return {"table": table, "seq_len": s["seq_len"], "free": s["free"], "free_count": s["free_count"]}


def _copy(s):
    pool, P = s["pool"], s["case"]["page"]
    tok = torch.minimum(torch.arange(s["max_len"], device=DEV), s["len"].long()[:, None] - 1)  # behind the end: the last token again
    src, dst = s["src"].long()[:, None], s["dst"].long()[:, None]
    a, b, slot = s["table"].long()[src, tok // P], s["table"].long()[dst, tok // P], tok % P
    pool[:, :, b, slot] = pool[:, :, a, slot]
    return {"pool": pool}


def _logprob(s):
    case = s["case"]
    x = s["logits"].float()
    top = x.amax(-1, keepdim=True)
    y = x - top
    e = y.exp()
    total = e.sum(-1)
    lse = top[:, 0] + total.log()
    entropy = total.log() - torch.where(e > 0, e * y, 0.0).sum(-1) / total
    logprob = x.gather(1, s["given"].long()) - lse[:, None]
    # equal logits: the lowest token first.  The bits of a float as an integer in the same order, the token below them
    bits = (x + 0.0).view(torch.int32).long()
    order = torch.where(bits < 0, bits ^ 0x7fffffff, bits)
    token = torch.arange(case["vocab"], device=DEV)
    index = (case["vocab"] - 1) - ((order << 20) | ((case["vocab"] - 1) - token)).topk(case["top"], dim=1).values % (1 << 20)
    return {"logprob": logprob, "entropy": entropy, "lse": lse, "top_logprob": x.gather(1, index) - lse[:, None],
            "top_index": index.to(torch.int32)}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in float64


def exact(case, seed):
    kind = case["kind"]
    if kind in ("resize", "copy"):
        return None                                              # nothing computed: whole numbers, and bytes moved
    s = prepare(case, seed)
    if kind == "logprob":
        out = {k: [] for k in ("logprob", "entropy", "lse", "top_logprob")}
        for r0 in range(0, case["rows"], 64):
            z = s["logits"][r0:r0 + 64].double()
            lse = torch.logsumexp(z, 1, keepdim=True)
            lp = z - lse
            out["lse"].append(lse[:, 0])
            out["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum(1))
            out["logprob"].append(lp.gather(1, s["given"][r0:r0 + 64].long()))
            out["top_logprob"].append(lp.sort(1, descending=True).values[:, :case["top"]])
        return {**{k: torch.cat(v) for k, v in out.items()}, "top_index": None}
    hk, G, P = case["kv_heads"], case["group"], case["page"]
    hq = hk * G
    L, n_win, table = s["seq_len"].tolist(), s["win_indptr"].diff().tolist(), s["table"].long()
    if kind == "append":
        x = s["qkv"].double()
        pool = s["pool"].double()
        half = case["rotary"] // 2
        places = [(2 * i, 2 * i + 1) if case["interleaved"] else (i, i + half) for i in range(half)]
        y = x.clone()
        for i, (a, b) in enumerate(places):
            t = (s["positions"][int(s["axis"][i])].double() * s["inv_freq"][i].double())[:, None]
            y[:, :, :hq + hk, a] = x[:, :, :hq + hk, a] * t.cos() - x[:, :, :hq + hk, b] * t.sin()
            y[:, :, :hq + hk, b] = x[:, :, :hq + hk, a] * t.sin() + x[:, :, :hq + hk, b] * t.cos()
        row = 0
        for r, w in enumerate(n_win):
            j = torch.arange(L[r] - w, L[r], device=DEV)
            pool[:, 0, table[r, j // P], j % P] = y[:, row:row + w, hq:hq + hk]
            pool[:, 1, table[r, j // P], j % P] = y[:, row:row + w, hq + hk:]
            row += w
        return {"q": y[:, :, :hq], "pool": pool}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:3], -math.inf, dtype=torch.float64, device=DEV)
    for layer in range(case["layers"]):
        row = 0
        for r, w in enumerate(n_win):
            j = torch.arange(L[r], device=DEV)
            k, v = (s["pool"][layer, c, table[r, j // P], j % P].double() for c in (0, 1))
            for i in range(w):
                at = L[r] - w + i if case["causal"] else L[r] - 1
                lo = max(0, at - case["sliding"] + 1) if case["sliding"] else 0
                q = s["q"][layer, row + i].double().view(hk, G, -1)
                z = torch.einsum("hgd,nhd->hgn", q, k[lo:at + 1]) * s["scale"]
                lse[layer, row + i] = torch.logsumexp(z, -1).reshape(-1)
                out[layer, row + i] = torch.einsum("hgn,nhd->hgd", torch.softmax(z, -1), v[lo:at + 1]).reshape(hq, -1)
            row += w
    return {"out": out, "lse": lse}
