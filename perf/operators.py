"""The operators of a speech-token language model's step in front of the decoder, as they are measured:

append   queries and keys normalised per head and rotated by their positions, keys and values written into
         the session's cache rows, in one pass (TokenCache.append)
attend   attention over that cache: a sliding window and a few first tokens that stay visible
         (TokenCache.attend)
sample   the next token of every row of logits: temperature, top-k, top-p, min-p, from given random
         numbers (sample_tokens)

The cache of a session is the decoder's own retention rule: the first `sinks` positions keep their rows,
the positions behind them share a ring of `ring` rows. A case's sequences are sessions of one pool, in an
order of their own; "ragged" ones have histories and chunks of different lengths. Where `own` is false,
`run` computes the operators' plain forms in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6
THETA = 10000.0


# ---- the cases ---------------------------------------------------------------------------------------------------------


def cached(name, op, sessions, tokens, start, heads, kv_heads, head_dim, sinks, window, ring, type="bf16", ragged=False, rot=None, interleaved=False):
    c = {"name": name, "op": op, "sessions": sessions, "tokens": tokens, "start": start, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
         "sinks": sinks, "window": window, "ring": ring, "type": type, "ragged": ragged}
    if op == "append":
        c.update(rot=head_dim if rot is None else rot, interleaved=interleaved)
    return c


def sampled(name, rows, vocab, type, how):
    return {"name": name, "op": "sample", "rows": rows, "vocab": vocab, "type": type, "how": how}


def listed():
    return [
        # one listener's next token: the heads of the flow decoder
        cached("append_one_token", "append", 1, 1, 700, 8, 8, 64, 4, 256, 320),
        # a serving round: 64 sessions of different ages, half of each head rotated
        cached("append_64_sessions", "append", 64, 1, 9000, 16, 2, 128, 4, 2048, 2304, ragged=True, rot=64),
        # prompts of up to 2000 tokens for five sessions, pairs side by side
        cached("append_prompts", "append", 5, 2000, 0, 32, 8, 128, 4, 4096, 8192, ragged=True, interleaved=True),
        # one listener's next token over a short window, ring wrapped
        cached("attend_one_token", "attend", 1, 1, 700, 8, 8, 64, 4, 256, 320),
        # one session, long window: a single query row per head reads all of it
        cached("attend_one_long", "attend", 1, 1, 60000, 28, 4, 128, 16, 32768, 33000, type="fp16"),
        # a full server: sessions of different ages
        cached("attend_48_sessions", "attend", 48, 1, 9000, 32, 8, 128, 4, 4096, 4608, ragged=True),
        # a round of chunks: 50 new rows at most for each of eight sessions, behind a prompt of 302 rows
        cached("attend_chunks", "attend", 8, 50, 1100, 16, 2, 128, 302, 512, 640, ragged=True),
        # a long prompt in one call: the window slides through it
        cached("attend_prompt", "attend", 1, 8192, 0, 16, 4, 128, 4, 2048, 12288),
        # one listener's next speech token
        sampled("sample_one", 1, 4097, "fp32", "nucleus"),
        # a serving round, half precision
        sampled("sample_48_rows", 48, 32001, "bf16", "mixed"),
        # many rows of a large vocabulary, every rule among them
        sampled("sample_256_rows", 256, 131072, "fp32", "mixed"),
    ]


def spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "sample"])
    type = rng.choice(["bf16", "bf16", "fp16"])
    if op == "sample":
        vocab = spread(rng, 64, 131072)
        rows = spread(rng, 1, min(256, 24_000_000 // vocab))
        return {"op": op, "rows": rows, "vocab": vocab, "type": rng.choice(["fp32", "bf16", "fp16"]), "how": rng.choice(["nucleus", "mixed", "plain"])}
    head_dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 4, 5, 7, 8])
    sinks = rng.choice([0, 1, 4, 16, 302])
    window = spread(rng, 1, 8192)
    kind = rng.choice(["step", "chunk", "prompt"])
    if kind == "step":
        tokens, sessions = 1, spread(rng, 1, 64)
    elif kind == "chunk":
        tokens, sessions = rng.randint(2, 80), spread(rng, 1, 16)
    else:
        tokens, sessions = spread(rng, 100, 3000), rng.randint(1, 3)
    # no dearer than the largest listed ones: rows read, pairs of query and key, and the plain form's table of scores
    while sessions > 1 and sessions * kv_heads * head_dim * window > 48 * 8 * 128 * 4096:
        sessions = (sessions + 1) // 2
    while tokens > 1 and (sessions * tokens * heads * (window + sinks) > 16 * 8192 * 2048 or sessions * tokens * heads * (window + tokens) > 16 * 8192 * 10000):
        tokens = (tokens + 1) // 2
    ring = window + tokens - 1 + rng.choice([0, 1, 37, 512])
    start = rng.choice([0, spread(rng, 1, 100), spread(rng, 100, 100000)])
    c = {"op": op, "sessions": sessions, "tokens": tokens, "start": start, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "sinks": sinks,
         "window": window, "ring": ring, "type": type, "ragged": sessions > 1 and rng.random() < 0.6}
    if op == "append":
        c.update(rot=rng.choice([head_dim, head_dim, head_dim // 2, 32, 0]), interleaved=rng.random() < 0.3)
    return c


def counts(case):
    """Tokens and histories of the case's sequences."""
    n, part = case["sessions"], lambda i, by: (0.98 + by * i) % 1.0
    if not case["ragged"]:
        return [case["tokens"]] * n, [case["start"]] * n
    return [1 + int(part(i, 0.618034) * (case["tokens"] - 1) + 0.5) for i in range(n)], [int(part(i, 0.754878) * case["start"]) for i in range(n)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, type=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda").to(type)

    if case["op"] == "sample":
        n, vocab, type = case["rows"], case["vocab"], TYPES[case["type"]]
        # a model's logits: most of the vocabulary far behind a few candidates
        logits = 2.0 * normal(n, vocab)
        row, some = torch.arange(n, device="cuda"), torch.arange(24, device="cuda") * (vocab // 24)
        logits[row[:, None], (torch.randint(vocab, (n, 1), generator=gen, device="cuda") + some) % vocab] += 6.0 + 2.0 * normal(n, 24)
        every = {"temperature": 0.6 + 0.2 * (row % 4).float(), "top_k": None, "top_p": torch.full((n,), 0.9, device="cuda"), "min_p": None}
        if case["how"] == "plain":
            every["top_p"] = None
        if case["how"] == "mixed":  # neighbours ask for different rules: one of eight is greedy
            every["temperature"] = torch.where(row % 8 == 7, 0.0, every["temperature"])
            every["top_k"] = torch.tensor([0, 50, 0, 1, 1000, 20, 0, 0], device="cuda", dtype=torch.int32)[row % 8]
            every["top_p"] = torch.tensor([1.0, 0.95, 0.9, 1.0, 0.8, 1.0, 0.99, 1.0], device="cuda")[row % 8]
            every["min_p"] = torch.tensor([0.0, 0.0, 0.0, 0.0, 0.02, 0.1, 0.0, 0.0], device="cuda")[row % 8]
        return {"case": case, "logits": logits.to(type), "u": torch.rand(n, generator=gen, device="cuda"),
                "tokens": torch.zeros(n, dtype=torch.int32, device="cuda"), "probs": torch.zeros(n, device="cuda"), **every}
    type, d, H, Hkv = TYPES[case["type"]], case["head_dim"], case["heads"], case["kv_heads"]
    new, before = counts(case)
    n, rows = len(new), case["sinks"] + case["ring"]
    pool = n + 2
    used = sum(new)
    total = used if max(new) == 1 else -(-used // 16) * 16  # a padded batch: rows behind the last sequence
    k, v = normal(pool, Hkv, rows, d, type=type), normal(pool, Hkv, rows, d, type=type)
    ends = np.concatenate([[0], np.cumsum(new)])
    s = {"case": case, "used": used, "max_tokens": max(new), "k": k, "v": v,
         "sessions": torch.randperm(pool, generator=gen, device="cuda")[:n].to(torch.int32),
         "cu_tokens": None if max(new) == 1 else torch.tensor(ends, dtype=torch.int32, device="cuda"),
         "start": torch.tensor(before, dtype=torch.int32, device="cuda"),
         "seq": torch.tensor(np.repeat(np.arange(n), new), device="cuda"),  # each token's sequence and place in it
         "place": torch.tensor(np.concatenate([np.arange(t) for t in new]), device="cuda")}
    if case["op"] == "append":
        half = max(case["rot"] // 2, 1)
        s.update(qkv=1.5 * normal(total, (H + 2 * Hkv) * d), q_gain=1.0 + 0.2 * normal(d), k_gain=1.0 + 0.2 * normal(d),
                 inv_freq=torch.tensor([THETA ** (-j / half) for j in range(case["rot"] // 2)], dtype=torch.float32, device="cuda"),
                 q=torch.zeros(total, H, d, dtype=type, device="cuda"))
        s["qkv"] = s["qkv"].to(type)
    else:
        s.update(q=normal(total, H, d, type=type), out=torch.zeros(total, H, d, dtype=type, device="cuda"))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------


def handles(s):
    """What a program makes once and keeps: the cache's handle and the description of the round's batch."""
    if "cache" not in s:
        import paper_2609_35115_b200 as dc
        c = s["case"]
        s["cache"] = dc.TokenCache(s["k"], s["v"], n_heads=c["heads"], n_sink=c["sinks"], window=c["window"])
        rows = s["qkv"].shape[0] if c["op"] == "append" else s["q"].shape[0]
        s["batch"] = dc.TokenBatch(s["sessions"], s["start"], cu_tokens=s["cu_tokens"], n_tokens=rows, max_tokens=s["max_tokens"])
        if c["op"] == "append":
            s["norm"] = dc.QKNorm(s["q_gain"], s["k_gain"], s["inv_freq"], eps=EPS, interleaved=c["interleaved"])
    return s["cache"], s["batch"]


def run(s):
    op = s["case"]["op"]
    if own:
        if op == "sample":
            import paper_2609_35115_b200 as dc
            dc.sample_tokens(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], tokens=s["tokens"], probs=s["probs"])
            return {"tokens": s["tokens"], "probs": s["probs"]}
        cache, batch = handles(s)
        if op == "append":
            cache.append(s["qkv"], batch, s["norm"], q=s["q"])
            return {"q": s["q"], "k": s["k"], "v": s["v"]}
        return {"out": cache.attend(s["q"], batch, out=s["out"])}
    return {"append": plain_append, "attend": plain_attend, "sample": plain_sample}[op](s)


def ring_row(case, at):
    return torch.where(at < case["sinks"], at, case["sinks"] + (at - case["sinks"]) % case["ring"])


def plain_append(s):
    case, used = s["case"], s["used"]
    d, H, Hkv, half = case["head_dim"], case["heads"], case["kv_heads"], case["rot"] // 2
    x = s["qkv"][:used].float().view(used, H + 2 * Hkv, d)
    at = s["start"][s["seq"]].long() + s["place"]
    y = x[:, : H + Hkv]
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
    y = torch.cat([y[:, :H] * s["q_gain"], y[:, H:] * s["k_gain"]], 1)
    angle = at.double()[:, None] * s["inv_freq"].double()  # far positions: 32 bits lose the angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if case["interleaved"]:
        a, b = y[..., 0:2 * half:2], y[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    y = torch.cat([turned, y[..., 2 * half:]], -1)
    s["q"][:used] = y[:, :H].to(s["q"].dtype)
    session, row = s["sessions"][s["seq"]].long(), ring_row(case, at)
    s["k"][session, :, row] = y[:, H:].to(s["k"].dtype)
    s["v"][session, :, row] = s["qkv"][:used].view(used, H + 2 * Hkv, d)[:, H + Hkv:]
    return {"q": s["q"], "k": s["k"], "v": s["v"]}


def plain_attend(s):
    case, used, most = s["case"], s["used"], s["max_tokens"]
    d, H, Hkv = case["head_dim"], case["heads"], case["kv_heads"]
    n, rows, sinks = len(s["sessions"]), case["sinks"] + case["ring"], case["sinks"]
    q = torch.zeros(n, most, H, d, device="cuda")
    q[s["seq"], s["place"]] = s["q"][:used].float()
    q = q.view(n, most, Hkv, H // Hkv, d)
    k, v = s["k"][s["sessions"].long()].float(), s["v"][s["sessions"].long()].float()
    # the position that each row holds once the sequence's last token is in: the newest of those that share the row
    start = s["start"].long()
    last = torch.zeros(n, dtype=torch.long, device="cuda").scatter_reduce_(0, s["seq"], start[s["seq"]] + s["place"], "amax")
    row = torch.arange(rows, device="cuda")
    held = torch.where(row < sinks, row, last[:, None] - (last[:, None] - row) % case["ring"])
    written = torch.where(row < sinks, row <= last[:, None], held >= sinks)
    at = start[:, None, None] + torch.arange(most, device="cuda")[:, None]
    seen = written[:, None] & (held[:, None] <= at) & ((held[:, None] < sinks) | (held[:, None] > at - case["window"]))
    score = torch.einsum("nthgd,nhrd->nhgtr", q, k) / math.sqrt(d)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    score = torch.exp(score - score.amax(-1, keepdim=True))
    out = torch.einsum("nhgtr,nhrd->nthgd", score / score.sum(-1, keepdim=True), v)
    s["out"][:used] = out.reshape(n, most, H, d)[s["seq"], s["place"]].to(s["out"].dtype)
    return {"out": s["out"]}


def plain_sample(s):
    logits = s["logits"].double()  # sums over a vocabulary are compared with borders: 64 bits
    n, vocab = logits.shape
    cold = s["temperature"] <= 0
    value, index = logits.sort(dim=1, descending=True, stable=True)
    w = torch.exp((value - value[:, :1]) / torch.where(cold, 1.0, s["temperature"]).double()[:, None])
    rank = torch.arange(vocab, device="cuda")
    keep = torch.ones_like(w, dtype=torch.bool)
    if s["top_k"] is not None:
        keep &= rank < torch.where(s["top_k"] > 0, s["top_k"], vocab)[:, None]
    if s["top_p"] is not None:
        mass = (w * keep).cumsum(1)
        before = mass - w * keep
        keep &= (before < s["top_p"].double()[:, None] * mass[:, -1:]) | (s["top_p"] >= 1)[:, None]
    if s["min_p"] is not None:
        keep &= w >= s["min_p"].double()[:, None]
    keep &= (rank == 0) | ~cold[:, None]
    kept = torch.zeros_like(w).scatter_(1, index, w * keep)  # back in the vocabulary's order
    mass = kept.cumsum(1)
    token = (mass <= s["u"].double()[:, None] * mass[:, -1:]).sum(1)
    s["tokens"].copy_(token)
    s["probs"].copy_(kept.gather(1, token[:, None])[:, 0] / mass[:, -1])
    return {"tokens": s["tokens"], "probs": s["probs"]}


# ---- the same in 64 bits, from the definitions --------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": exact_append, "attend": exact_attend, "sample": exact_sample}[case["op"]](case, s)


def row_of(case, p):
    return p if p < case["sinks"] else case["sinks"] + (p - case["sinks"]) % case["ring"]


def exact_append(case, s):
    d, H, Hkv, half = case["head_dim"], case["heads"], case["kv_heads"], case["rot"] // 2
    new, before = counts(case)
    x = s["qkv"].double().cpu().numpy().reshape(-1, H + 2 * Hkv, d)
    q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
    gains, freq = [s[g].double().cpu().numpy() for g in ("q_gain", "k_gain")], s["inv_freq"].double().cpu().numpy()
    first, second = (np.arange(half) * 2, np.arange(half) * 2 + 1) if case["interleaved"] else (np.arange(half), np.arange(half) + half)
    sessions, at = s["sessions"].tolist(), 0
    for session, t, p0 in zip(sessions, new, before):
        part = x[at:at + t]
        heads = part[:, : H + Hkv] / np.sqrt(np.mean(part[:, : H + Hkv] ** 2, axis=-1, keepdims=True) + EPS)
        heads[:, :H] *= gains[0]
        heads[:, H:] *= gains[1]
        turn = np.exp(1j * np.outer(np.arange(p0, p0 + t, dtype=np.float64), freq))[:, None]
        z = (heads[..., first] + 1j * heads[..., second]) * turn
        heads[..., first], heads[..., second] = z.real, z.imag
        rows = torch.tensor([row_of(case, p) for p in range(p0, p0 + t)], device="cuda")
        q[at:at + t] = torch.tensor(heads[:, :H], device="cuda")
        k[session, :, rows] = torch.tensor(heads[:, H:], device="cuda").transpose(0, 1)
        v[session, :, rows] = torch.tensor(part[:, H + Hkv:], device="cuda").transpose(0, 1)
        at += t
    return {"q": q, "k": k, "v": v}


def exact_attend(case, s):
    d, H, Hkv, sinks, window = case["head_dim"], case["heads"], case["kv_heads"], case["sinks"], case["window"]
    new, before = counts(case)
    out, at, G = s["out"].double(), 0, H // Hkv
    for session, t, p0 in zip(s["sessions"].tolist(), new, before):
        for lo in range(0, t, 512):  # a block of queries and the positions that any of them sees
            hi = min(t, lo + 512)
            far = max(0, p0 + lo - window + 1)
            keys = list(range(min(sinks, far))) + list(range(far, p0 + hi))
            rows = torch.tensor([row_of(case, p) for p in keys], device="cuda")
            key, query = torch.tensor(keys, device="cuda"), torch.arange(p0 + lo, p0 + hi, device="cuda")[:, None]
            hidden = (key > query) | ((key <= query - window) & (key >= sinks))
            for h in range(Hkv):
                kk, vv = s["k"][session, h, rows].double(), s["v"][session, h, rows].double()
                qq = s["q"][at + lo:at + hi, h * G:(h + 1) * G].double().transpose(0, 1)
                p = torch.softmax((qq @ kk.T / math.sqrt(d)).masked_fill(hidden, -math.inf), -1)
                out[at + lo:at + hi, h * G:(h + 1) * G] = (p @ vv).transpose(0, 1)
        at += t
    return {"out": out}


def exact_sample(case, s):
    def rule(name, off):
        return np.full(case["rows"], off) if s[name] is None else s[name].double().cpu().numpy()

    logits, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    temperature, top_k, top_p, min_p = rule("temperature", 1.0), rule("top_k", 0), rule("top_p", 1.0), rule("min_p", 0.0)
    tokens, probs = np.zeros(case["rows"], np.int64), np.zeros(case["rows"])
    for r, l in enumerate(logits):
        if temperature[r] <= 0:
            tokens[r], probs[r] = np.argmax(l), 1.0
            continue
        order = np.argsort(-l, kind="stable")
        if top_k[r] > 0:
            order = order[:int(top_k[r])]
        w = np.exp((l[order] - l[order[0]]) / temperature[r])
        many = len(order)
        if top_p[r] < 1:
            many = 1 + int(np.searchsorted(np.cumsum(w), top_p[r] * w.sum()))
        many = min(many, int(np.sum(w >= min_p[r])))
        kept = np.sort(order[:many])
        w = np.exp((l[kept] - l[order[0]]) / temperature[r])
        mass = np.cumsum(w)
        i = int(np.searchsorted(mass, u[r] * mass[-1], side="right"))
        tokens[r], probs[r] = kept[i], w[i] / mass[-1]
    return {"tokens": tokens.astype(np.int32), "probs": probs}


# ---- what a pass cannot do without -----------------------------------------------------------------------------------------


def work(case):
    if case["op"] == "sample":
        values = case["rows"] * case["vocab"]
        return {"bytes": values * TYPES[case["type"]].itemsize + case["rows"] * 8, "flops": 4 * values}
    d, H, Hkv, sinks, window = case["head_dim"], case["heads"], case["kv_heads"], case["sinks"], case["window"]
    new, before = counts(case)
    if case["op"] == "append":
        values = sum(new) * (H + 2 * Hkv) * d
        return {"bytes": 4 * values, "flops": 10 * values}
    pairs = read = 0
    for t, p0 in zip(new, before):
        at = np.arange(p0, p0 + t)
        pairs += int(np.sum(np.minimum(at + 1, window) + np.minimum(sinks, np.maximum(0, at + 1 - window))))
        first = max(0, p0 - window + 1)
        read += p0 + t - first + min(sinks, first)
    return {"bytes": 2 * (2 * sum(new) * H * d + 2 * read * Hkv * d), "flops": 4 * d * H * pairs}
