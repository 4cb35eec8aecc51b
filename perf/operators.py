"""The serving operators of ``paper_2509_22622_amd.binding`` as cases that can be prepared, run and counted one by one.

``append``   new tokens' keys and values into a paged cache, turned by the rotary embedding on the way, with the queries
             turned and scaled beside them.  Each sequence brings ``new`` tokens; its pages lie anywhere in the pool.
``attend``   attention of each sequence's last token (or last few) over the paged cache: everything before it, or a sink
             of first tokens and a window of last ones.
``linear``   y = act(x w^T + bias) + residual: the products around them.

With ``own`` the calls are the library's; without it the same operators are computed by elementary torch operations in 32 bits.
Inputs are normal numbers in bfloat16; sequences differ in length, the last one of a batch may be idle (length 0).
"""
import math

import torch

own = False

LOG2E = 1.4426950408889634


# ---- cases -------------------------------------------------------------------------------------------------------

def _append(name, **kw):
    case = {"name": name, "op": "append", "cache": "bf16", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "seqs": 16,
            "new": 1, "longest": 4096, "rope": "halves", "theta": 500000.0, "idle": False}
    return {**case, **kw}


def _attend(name, **kw):
    case = {"name": name, "op": "attend", "cache": "bf16", "q_heads": 32, "kv_heads": 8, "head_dim": 128, "page": 64, "seqs": 16,
            "new": 1, "longest": 4096, "sink": 0, "window": 0, "q_std": 1.0, "idle": False}
    return {**case, **kw}


def _linear(name, **kw):
    case = {"name": name, "op": "linear", "rows": 1, "n_in": 1536, "n_out": 1536, "bias": True, "act": "none", "residual": False}
    return {**case, **kw}


def listed():
    return [
        # the first steps of two small sequences (4 heads x 64): launches and latency
        _append("append_first_tokens", q_heads=4, kv_heads=4, head_dim=64, page=16, seqs=2, longest=77, rope="pairs", theta=10000.0),
        # one step of a full batch with an 8-bit cache; one place of the batch is idle
        _append("append_batch_8bit", cache="fp8_e4m3", seqs=96, longest=30000, idle=True),
        # prompts of different lengths, all at once
        _append("append_prompts", seqs=7, new=2500, longest=2500),
        # a three-frame chunk of 30 x 52 video tokens, turned by frame, row and column, into an 8-bit cache
        _append("append_chunk_8bit", cache="fp8_e4m3", q_heads=12, kv_heads=12, page=128, seqs=1, new=4680, longest=23400, rope="grid",
                theta=10000.0),
        # the attention of those first steps
        _attend("attend_first_tokens", q_heads=4, kv_heads=4, head_dim=64, page=16, seqs=2, longest=77),
        # one step of a batch of long sequences
        _attend("attend_batch", seqs=64, longest=16384),
        # one user with a very long context, 8-bit cache
        _attend("attend_long_8bit", cache="fp8_e4m3", page=128, seqs=1, longest=131072),
        # sink and window (three frames and nine of 1560 tokens) of streams that have run for long, every head its own keys
        _attend("attend_sink_window", q_heads=12, kv_heads=12, page=16, seqs=24, longest=60000, sink=4680, window=14040, q_std=2.0),
        # up to four drafted tokens a sequence are checked at once; five query heads a key head, head_dim 64, 8-bit cache
        _attend("attend_draft_8bit", cache="fp8_e4m3", q_heads=40, kv_heads=8, head_dim=64, page=32, seqs=16, new=4, longest=6000),
        # the output projection of one token, added to the stream
        _linear("linear_token", residual=True),
        # the widening product of a batch of tokens
        _linear("linear_batch", rows=37, n_out=6144, act="gelu_tanh"),
        # the narrowing product of a chunk's tokens, added to the stream
        _linear("linear_chunk", rows=4680, n_in=6144, residual=True),
    ]


DRAW_KEYS = 1 << 28       # a drawn attention has at most so many numbers in its keys
DRAW_FLOPS = 4e10


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["append", "attend", "attend", "linear"])
    if op == "linear":
        while True:
            case = _linear("", rows=_log_int(rng, 1, 8192), n_in=8 * _log_int(rng, 8, 1024), n_out=_log_int(rng, 33, 8192),
                           bias=rng.random() < 0.7, act=rng.choice(["none", "none", "gelu_tanh", "gelu", "silu"]), residual=rng.random() < 0.5)
            if work(case)["flops"] <= DRAW_FLOPS:
                break
    else:
        kv_heads = rng.choice([1, 2, 4, 5, 8, 12])
        dims = {"cache": rng.choice(["bf16", "bf16", "fp8_e4m3"]), "kv_heads": kv_heads, "q_heads": kv_heads * rng.choice([1, 2, 3, 4, 8]),
                "head_dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 48, 64, 128]), "idle": rng.random() < 0.3}
        while True:
            if op == "append":
                new = 1 if rng.random() < 0.4 else _log_int(rng, 2, 2000)
                case = _append("", seqs=_log_int(rng, 1, 128), new=new, longest=new + _log_int(rng, 1, 30000),
                               rope=rng.choice(["halves", "halves", "pairs", "grid", "none"]), theta=rng.choice([10000.0, 500000.0]), **dims)
                if case["seqs"] * new <= 8192 and case["seqs"] * case["longest"] <= 1 << 18:
                    break
            else:
                new = 1 if rng.random() < 0.7 else rng.randint(2, 8)
                far = rng.random() < 0.25
                case = _attend("", seqs=_log_int(rng, 1, 96), new=new, longest=new + _log_int(rng, 1, 120000),
                               sink=_log_int(rng, 1, 5000) if far else 0, window=_log_int(rng, 1, 16000) if far else 0,
                               q_std=rng.choice([1.0, 1.0, 2.0]), **dims)
                if case["seqs"] * case["longest"] * kv_heads * dims["head_dim"] <= DRAW_KEYS:
                    break
    del case["name"]
    return case


def _spread(case):
    """Per sequence (length with the new tokens, new tokens), by a rule on the case alone: the first sequence is the longest and
    brings ``new`` tokens, the others are spread over an octave and a half below it; where ``idle``, the last of several has nothing."""
    lens, news = [], []
    for i in range(case["seqs"]):
        part = (i * 0.6180339887498949) % 1.0
        new = case["new"] if i == 0 or case["new"] == 1 else max(1, int(case["new"] * (1 - 0.7 * part)))
        lens.append(max(new, int(case["longest"] * 2.0 ** (-1.5 * part))))
        news.append(new)
    if case["idle"] and case["seqs"] > 1:
        lens[-1], news[-1] = 0, (1 if case["new"] == 1 else 0)     # one token a sequence: the idle one's row is padding
    return lens, news


# ---- inputs ------------------------------------------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _normal(g, *shape, std=1.0):
    return (torch.randn(*shape, generator=g, device=g.device, dtype=torch.float32) * std).to(torch.bfloat16)


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 17)
    s = {"case": case}
    if case["op"] == "linear":
        m, k, n = case["rows"], case["n_in"], case["n_out"]
        s["x"] = _normal(g, m, k)
        s["w"] = _normal(g, n, k, std=k ** -0.5)
        s["bias"] = _normal(g, n, std=0.5) if case["bias"] else None
        s["residual"] = _normal(g, m, n) if case["residual"] else None
        if own:
            from paper_2509_22622_amd import binding as B
            s["linear"] = B.Linear(s["w"])            # laid out once, when the model is loaded
        s["y"] = torch.empty(m, n, dtype=torch.bfloat16, device=dev)
        return s

    hq, hkv, d, t = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    lens, news = _spread(case)
    tokens, wide = sum(news), max(1, -(-max(lens) // t))
    need = [-(-x // t) for x in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device=dev)
    table = torch.full((case["seqs"], wide), -1, dtype=torch.int64, device=dev)   # no page yet
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    s["table"] = table.to(torch.int32)
    s["spare"] = order[-1]                                                        # no sequence has it
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    ends = [0]
    for n in news:
        ends.append(ends[-1] + n)
    s["cu"] = None if case["new"] == 1 else torch.tensor(ends, dtype=torch.int32, device=dev)
    cache = None
    if own:
        from paper_2509_22622_amd import binding as B
        rope = {"rope": case["rope"], "rope_theta": case["theta"]} if case["op"] == "append" else {}
        cache = s["cache"] = B.PagedCache(1, hq, hkv, d, t, n_pages, kv_format=case["cache"], device=dev, **rope)
    if case["op"] == "append":
        qkv = _normal(g, tokens, (hq + 2 * hkv) * d)              # the product that makes all three leaves them side by side
        s["q"] = qkv[:, :hq * d].view(tokens, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].view(tokens, hkv, d)
        s["v"] = qkv[:, (hq + hkv) * d:].view(tokens, hkv, d)
        s["q_out"] = torch.empty(tokens, hq, d, dtype=torch.bfloat16, device=dev)
        s["positions"] = None
        if case["rope"] == "grid":                                # frame, row, column of 30 x 52 tokens a frame
            flat = torch.cat([torch.arange(x - n, x, device=dev) for x, n in zip(lens, news)] or [torch.zeros(0, device=dev)])
            flat = flat.to(torch.int64).clamp(min=0)
            s["positions"] = torch.stack([flat // 1560, flat % 1560 // 52, flat % 52], 1).to(torch.int32).contiguous()
        if cache is None:
            kind = torch.bfloat16 if case["cache"] == "bf16" else torch.float8_e4m3fn
            s["pool"] = [torch.zeros(n_pages, t, hkv, d, dtype=torch.bfloat16, device=dev).to(kind) for _ in "kv"]
        return s

    s["q"] = _normal(g, tokens, hq, d, std=case["q_std"] * LOG2E / math.sqrt(d))   # turned and scaled, as append hands them on
    s["out"] = torch.zeros(tokens, hq, d, dtype=torch.bfloat16, device=dev)
    pool = [_normal(g, n_pages, t, hkv, d) for _ in "kv"]
    if case["cache"] == "fp8_e4m3":
        pool = [x.to(torch.float8_e4m3fn) for x in pool]
    if cache is None:
        s["pool"] = pool
    else:
        cache.keys(0).copy_(pool[0].view(cache.keys(0).shape))
        cache.values(0).copy_(pool[1].view(cache.values(0).shape))
        s["longest"] = max(lens)
        s["workspace"] = cache.attn_workspace(case["seqs"], max_new=case["new"], max_len=s["longest"], sink_tokens=case["sink"],
                                              window_tokens=case["window"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    return {"append": _run_append, "attend": _run_attend, "linear": _run_linear}[s["case"]["op"]](s)


def _natural(pool, case, values):
    """A pool [pages, page, heads, head_dim] with its dimensions cut as the library's views of its own layout have them."""
    n, t, h, d = pool.shape
    if case["cache"] == "bf16":
        return pool.view(n, t // 16, 4, 4, h, d // 32, 2, 16) if values else pool.view(n, t // 16, 16, h, d // 32, 4, 8)
    return pool.view(n, t // 16, 4, 4, h, d // 64, 4, 16) if values else pool.view(n, t // 16, 16, h, d // 64, 2, 4, 8)


def _run_append(s):
    if own:
        c = s["cache"]
        c.append(0, s["lens"], s["table"], s["k"], s["v"], q=s["q"], q_out=s["q_out"], cu_tokens=s["cu"], positions=s["positions"])
        return {"q": s["q_out"], "k": c.keys(0), "v": c.values(0)}
    case = s["case"]
    d, t = case["head_dim"], case["page"]
    tokens = s["q"].shape[0]
    row = torch.arange(tokens, device=s["q"].device)
    if s["cu"] is None:
        seq, place = row, s["lens"].long() - 1
    else:
        seq = torch.searchsorted(s["cu"][1:].long(), row, right=True)
        place = s["lens"].long()[seq] - s["cu"].long()[seq + 1] + row
    # the angles of far positions in 64 bits
    rope = case["rope"]
    if rope == "grid":
        by_axis = (d // 2 - 2 * (d // 6), d // 6, d // 6)
        freq = torch.cat([case["theta"] ** (-torch.arange(n, dtype=torch.float64, device=row.device) / n) for n in by_axis])
        axis = torch.repeat_interleave(torch.arange(3, device=row.device), torch.tensor(by_axis, device=row.device), output_size=d // 2)
        angle = s["positions"].double()[:, axis] * freq
    else:
        angle = place.double()[:, None] * case["theta"] ** (-torch.arange(d // 2, dtype=torch.float64, device=row.device) / (d // 2))
    if rope == "none":
        angle = torch.zeros_like(angle)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x):
        x = x.float()
        if rope == "halves":
            a, b = x[..., :d // 2], x[..., d // 2:]
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)

    s["q_out"].copy_((turned(s["q"]) * (LOG2E / math.sqrt(d))).to(torch.bfloat16))
    there = (place >= 0) & (place < s["lens"].long()[seq])
    page = s["table"].long()[seq, (place.clamp(min=0) // t)]
    page = torch.where(there & (page >= 0), page, s["spare"])                      # an idle row: to where nothing changes
    off = torch.where(there, place % t, 0)
    for pool, x in zip(s["pool"], (turned(s["k"]), s["v"].float())):
        if case["cache"] == "bf16":
            codes, x = pool, x.to(torch.bfloat16)
        else:
            codes, x = pool.view(torch.uint8), x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        codes[page, off] = torch.where(there[:, None, None], x, codes[page, off])
    return {"q": s["q_out"], "k": _natural(s["pool"][0], case, False), "v": _natural(s["pool"][1], case, True)}


def _run_attend(s):
    case = s["case"]
    if own:
        s["cache"].attn(0, s["lens"], s["table"], s["q"], s["out"], s["workspace"], cu_tokens=s["cu"], max_new=case["new"],
                        max_len=s["longest"], sink_tokens=case["sink"], window_tokens=case["window"])
        return s["out"]
    hq, hkv, d, t, new = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], case["new"]
    dev, seqs, tokens = s["q"].device, case["seqs"], s["q"].shape[0]
    lens, table = s["lens"].long(), s["table"].long().clamp(min=0)
    first = torch.arange(seqs, device=dev) if s["cu"] is None else s["cu"].long()[:-1]
    brings = torch.ones_like(lens) if s["cu"] is None else s["cu"].long()[1:] - first
    j = torch.arange(new, device=dev)
    row = torch.where(j < brings[:, None], first[:, None] + j, tokens)                        # [seqs, new]; `tokens`: no such row
    place = lens[:, None] - brings[:, None] + j
    long = table.shape[1] * t
    key = torch.arange(long, device=dev)
    seen = (key <= place[..., None]) & (key < lens[:, None, None])                            # [seqs, new, long]
    if case["window"]:
        seen &= (key < case["sink"]) | (key > place[..., None] - case["window"])
    q = torch.cat([s["q"], torch.zeros_like(s["q"][:1])])[row].float()                        # [seqs, new, hq, d]
    q = q.view(seqs, new, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(seqs, hkv, new * (hq // hkv), d)
    k, v = ((p[table] if case["cache"] == "bf16" else p.view(torch.uint8)[table].view(torch.float8_e4m3fn)) for p in s["pool"])
    k, v = (x.view(seqs, long, hkv, d).float().transpose(1, 2).contiguous() for x in (k, v))
    score = torch.matmul(q, k.transpose(-1, -2)).view(seqs, hkv, new, hq // hkv, long)
    score = score.masked_fill(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp2(score - torch.where(top == -math.inf, 0.0, top))
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight.view(seqs, hkv, -1, long), v).view(seqs, hkv, new, hq // hkv, d) / torch.where(total == 0, 1.0, total)
    out = out.permute(0, 2, 1, 3, 4).reshape(seqs * new, hq, d).to(torch.bfloat16)
    all_rows = torch.cat([s["out"], s["out"][:1]]).index_copy(0, row.flatten().clamp(max=tokens), out)
    s["out"].copy_(all_rows[:tokens])
    return s["out"]


def _run_linear(s):
    case = s["case"]
    if own:
        s["linear"].forward(s["x"], s["y"], bias=s["bias"], activation=case["act"], residual=s["residual"])
        return s["y"]
    y = torch.matmul(s["x"].float(), s["w"].float().t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["act"] == "gelu_tanh":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    elif case["act"] == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    elif case["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    if s["residual"] is not None:
        y = y + s["residual"].float()
    s["y"].copy_(y.to(torch.bfloat16))
    return s["y"]


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    if case["op"] == "linear":
        m, k, n = case["rows"], case["n_in"], case["n_out"]
        return {"bytes": 2 * (m * k + n * k + m * n * (2 if case["residual"] else 1) + (n if case["bias"] else 0)), "flops": 2.0 * m * n * k}
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    size = 2 if case["cache"] == "bf16" else 1
    lens, news = _spread(case)
    tokens = sum(news)
    if case["op"] == "append":
        kept = sum(min(x, n) for x, n in zip(lens, news))
        return {"bytes": tokens * hq * d * 2 * 2 + kept * hkv * d * 2 * (2 + size), "flops": tokens * (hq + hkv) * d * 3.0}
    keys = pairs = 0
    for x, n in zip(lens, news):
        if x == 0:
            continue
        low = x - n - case["window"] + 1 if case["window"] else 0        # first key of the first new token's window
        keys += x if low <= case["sink"] else case["sink"] + x - low
        for j in range(n):
            seen = x - n + j + 1
            pairs += seen if not case["window"] else min(seen, case["sink"] + case["window"])
    return {"bytes": keys * hkv * d * 2 * size + tokens * hq * d * 2 * 2, "flops": 4.0 * pairs * hq * d}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _inputs(case, seed):
    """The inputs in plain tensors, whatever ``own`` says."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "linear":
        y = s["x"].double() @ s["w"].double().t()
        if s["bias"] is not None:
            y += s["bias"].double()
        if case["act"] == "gelu_tanh":
            y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
        elif case["act"] == "gelu":
            y = y * torch.special.ndtr(y)
        elif case["act"] == "silu":
            y = y * torch.sigmoid(y)
        return y if s["residual"] is None else y + s["residual"].double()
    return _exact_append(case, s) if case["op"] == "append" else _exact_attend(case, s)


def _exact_append(case, s):
    d, t = case["head_dim"], case["page"]
    lens, news = _spread(case)
    half = d // 2
    q, k, v = (s[x].double() for x in "qkv")
    owner = [(i, x - n + j) for i, (x, n) in enumerate(zip(lens, news)) for j in range(n)]
    place = torch.tensor([p for _, p in owner], dtype=torch.float64, device=q.device)
    angle = torch.zeros(len(owner), half, dtype=torch.float64, device=q.device)
    if case["rope"] == "grid":
        n_x = d // 6
        n_t = half - 2 * n_x
        for p in range(half):
            axis, i, n = (0, p, n_t) if p < n_t else (1, p - n_t, n_x) if p < n_t + n_x else (2, p - n_t - n_x, n_x)
            angle[:, p] = s["positions"][:, axis].double() * case["theta"] ** (-i / n)
    elif case["rope"] != "none":
        for p in range(half):
            angle[:, p] = place * case["theta"] ** (-2.0 * p / d)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def turned(x):                                     # each pair as a complex number
        if case["rope"] == "halves":
            z = torch.complex(x[..., :half].contiguous(), x[..., half:].contiguous()) * turn
            return torch.cat([z.real, z.imag], -1)
        z = torch.view_as_complex(x.reshape(*x.shape[:-1], half, 2).contiguous()) * turn
        return torch.view_as_real(z).reshape(x.shape)

    n_pages = s["pool"][0].shape[0]
    pools = [torch.zeros(n_pages * t, case["kv_heads"], d, dtype=torch.float64, device=q.device) for _ in "kv"]
    table = s["table"].cpu()
    rows = [r for r, (i, p) in enumerate(owner) if 0 <= p < lens[i]]
    slots = [int(table[owner[r][0], owner[r][1] // t]) * t + owner[r][1] % t for r in rows]
    rows, slots = (torch.tensor(x, dtype=torch.int64, device=q.device) for x in (rows, slots))
    for pool, x in zip(pools, (turned(k), v)):
        pool[slots] = x[rows] if case["cache"] == "bf16" else x[rows].clamp(-448, 448)
    k, v = (_natural(p.view(n_pages, t, case["kv_heads"], d), case, i == 1) for i, p in enumerate(pools))
    return {"q": turned(q) * (LOG2E / math.sqrt(d)), "k": k, "v": v}


def _exact_attend(case, s):
    hq, hkv, d, t = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    lens, news = _spread(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    row = 0
    for i, (x, n) in enumerate(zip(lens, news)):
        if x == 0:
            row += n
            continue
        pages = s["table"][i, :-(-x // t)].long()
        k, v = ((p.view(torch.uint8) if p.dtype == torch.float8_e4m3fn else p)[pages].view(p.dtype).double().flatten(0, 1)[:x] for p in s["pool"])
        for j in range(n):
            at = x - n + j
            seen = torch.arange(at + 1, device=k.device)
            if case["window"] and at + 1 > case["sink"] + case["window"]:
                seen = torch.cat([seen[:case["sink"]], seen[at + 1 - case["window"]:]])
            for h in range(hkv):
                mine = slice(h * (hq // hkv), (h + 1) * (hq // hkv))
                z = s["q"][row, mine].double() @ k[seen, h].t() / LOG2E        # natural logits
                out[row, mine] = torch.softmax(z, -1) @ v[seen, h]
            row += 1
    return out
