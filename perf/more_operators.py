"""The operators around the attention of ``paper_2509_22622_amd.binding`` that training and serving share, as cases that can be
prepared, run and counted one by one.

``norm``         layer norm of rows of features, with a weight and a bias that all rows share, or one of each for every ``group`` rows
                 (a frame's tokens, modulated by that frame's scale and shift).
``norm_step``    its forward and its backward pass: the inputs' gradients, with the gradient that went past the norm added, and those of
                 weight and bias.
``attend``       attention of each sequence's queries over the states of an encoder, of other lengths and without a mask.
``attend_step``  its forward and its backward pass: the gradients of queries, keys and values.

With ``own`` the calls are the library's; without it the same operators are computed by elementary torch operations in 32 bits.
Inputs are normal numbers; sequences differ in length, the last one of a batch may have no keys at all.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------------------------------

def _norm(name, **kw):
    case = {"name": name, "op": "norm", "rows": 1, "features": 1536, "x": "bf16", "y": "bf16", "w": "bf16", "weight": True, "bias": True,
            "group": 0, "residual": False}
    return {**case, **kw}


def _attend(name, **kw):
    case = {"name": name, "op": "attend", "q_heads": 12, "kv_heads": 12, "head_dim": 128, "seqs": 1, "queries": 1, "keys": 512,
            "padded": False, "idle": False, "q_std": 1.0}
    return {**case, **kw}


def listed():
    return [
        # one token's features before a product
        _norm("norm_token"),
        # a three-frame chunk of 30 x 52 video tokens on a 32-bit stream, each frame with its own scale and shift
        _norm("norm_chunk", rows=4680, x="f32", w="f32", group=1560),
        # rows of an odd width, which no wide load fits
        _norm("norm_odd", rows=1111, features=1531),
        # a training step of few rows
        _norm("norm_step_few", op="norm_step", rows=77, features=512),
        # a training step of a 21-frame clip, each frame with its own scale and shift, the stream's gradient added
        _norm("norm_step_clip", op="norm_step", rows=32760, w="f32", group=1560, residual=True),
        # wide rows on a 32-bit stream, a weight and no bias
        _norm("norm_step_wide", op="norm_step", rows=2100, features=8192, x="f32", bias=False, residual=True),
        # one new token each of a batch, over what the encoder made of inputs of different lengths
        _attend("attend_tokens", q_heads=32, kv_heads=8, seqs=24, keys=1500),
        # one token over a long document
        _attend("attend_long", q_heads=32, kv_heads=8, keys=32000),
        # chunks of several videos over their prompts, padded to the longest; one has none
        _attend("attend_chunks", seqs=4, queries=4680, padded=True, idle=True),
        # a training step of two small sequences
        _attend("attend_step_few", op="attend_step", q_heads=4, kv_heads=4, head_dim=64, seqs=2, queries=77, keys=33),
        # a training step of a 21-frame clip over its prompt
        _attend("attend_step_clip", op="attend_step", queries=32760),
        # a training step of sequences of different lengths over longer ones, five query heads a key head
        _attend("attend_step_ragged", op="attend_step", q_heads=40, kv_heads=8, head_dim=64, seqs=6, queries=1200, keys=2500),
    ]


DRAW_NUMBERS = 50e6       # of a drawn norm's rows, or of a drawn attention's queries or keys
DRAW_SCORES = 2e8         # of a drawn attention


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """One more case of the same ranges."""
    step = rng.random() < 0.5
    if rng.random() < 0.45:
        types = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        while True:
            rows, features = _log_int(rng, 1, 32760), _log_int(rng, 33, 16384)
            if rng.random() < 0.7:
                features = (features + 7) // 8 * 8
            if rows * features <= DRAW_NUMBERS:
                break
        weight = rng.random() < 0.9
        case = _norm("", op="norm_step" if step else "norm", rows=rows, features=features, x=types[0], y=types[1], w=rng.choice(["bf16", "f32"]),
                     weight=weight, bias=weight and rng.random() < 0.7, group=_log_int(rng, 1, rows) if rows > 100 and rng.random() < 0.3 else 0,
                     residual=step and rng.random() < 0.5)
        if case["group"] and case["group"] < 20:
            case["group"] += 20
    else:
        kv_heads = rng.choice([1, 2, 4, 5, 8, 12])
        while True:
            case = _attend("", op="attend_step" if step else "attend", kv_heads=kv_heads, q_heads=kv_heads * rng.choice([1, 1, 2, 3, 4, 5, 8]),
                           head_dim=rng.choice([64, 128, 128]), seqs=_log_int(rng, 1, 64),
                           queries=1 if rng.random() < 0.3 else _log_int(rng, 2, 32760), keys=_log_int(rng, 1, 32000),
                           padded=rng.random() < 0.3, idle=rng.random() < 0.3, q_std=rng.choice([1.0, 1.0, 2.0]))
            tokens, states = case["seqs"] * case["queries"], case["seqs"] * case["keys"]
            if (tokens * case["keys"] * case["q_heads"] <= DRAW_SCORES and tokens * case["q_heads"] * case["head_dim"] <= DRAW_NUMBERS
                    and states * kv_heads * case["head_dim"] <= DRAW_NUMBERS):
                break
    del case["name"]
    return case


def _spread(case):
    """Per sequence (queries, keys), by a rule on the case alone: the first one has the most, the others are spread over an octave and a
    half below it, queries of a padded batch excepted; where ``idle``, the last of several has no keys."""
    queries, keys = [], []
    for i in range(case["seqs"]):
        part, other = (i * 0.6180339887498949) % 1.0, (i * 0.7548776662466927) % 1.0
        queries.append(case["queries"] if case["padded"] else max(1, int(case["queries"] * 2.0 ** (-1.5 * part))))
        keys.append(max(1, int(case["keys"] * 2.0 ** (-1.5 * other))))
    if case["idle"] and case["seqs"] > 1:
        keys[-1] = 0
    return queries, keys


# ---- inputs ------------------------------------------------------------------------------------------------------

def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _normal(g, *shape, std=1.0, mean=0.0, dtype=torch.bfloat16):
    return (torch.randn(*shape, generator=g, device=g.device, dtype=torch.float32) * std + mean).to(dtype)


def prepare(case, seed):
    dev = _device()
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 29)
    s = {"case": case}
    if case["op"].startswith("norm"):
        m, n = case["rows"], case["features"]
        xt, yt, wt = TYPES[case["x"]], TYPES[case["y"]], TYPES[case["w"]]
        groups = -(-m // case["group"]) if case["group"] else 1
        level = _normal(g, n, dtype=torch.float32)                                 # features have levels of their own
        s["x"] = (_normal(g, m, n, std=2.0, dtype=torch.float32) + level).to(xt)
        s["weight"] = _normal(g, groups, n, std=0.2, mean=1.0, dtype=wt) if case["weight"] else None
        s["bias"] = _normal(g, groups, n, std=0.2, dtype=wt) if case["bias"] else None
        s["dy"] = _normal(g, m, n, dtype=yt) if case["op"] == "norm_step" else None
        s["residual"] = _normal(g, m, n, dtype=xt) if case["residual"] else None
        if own:
            from paper_2509_22622_amd import binding as B
            norm = s["norm"] = B.LayerNorm(n, eps=EPS, device=dev)
            s["y"] = torch.empty(m, n, dtype=yt, device=dev)
            if case["op"] == "norm_step":
                s["stats"] = torch.empty(m, 2, dtype=torch.float32, device=dev)
                s["dx"] = torch.empty_like(s["x"])
                s["dweight"] = torch.empty(groups, n, dtype=torch.float32, device=dev) if case["weight"] else None
                s["dbias"] = torch.empty(groups, n, dtype=torch.float32, device=dev) if case["bias"] else None
                s["workspace"] = norm.backward_workspace(m, group_rows=case["group"])
        return s

    hq, hkv, d, step = case["q_heads"], case["kv_heads"], case["head_dim"], case["op"] == "attend_step"
    queries, keys = _spread(case)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    ends = lambda x: [sum(x[:i]) for i in range(len(x) + 1)]  # noqa: E731
    if case["padded"]:                                             # every sequence has as many rows as the longest
        tokens, states = case["seqs"] * max(queries), case["seqs"] * max(max(keys), 1)
        s["cu_q"], s["cu_k"], s["k_lens"] = None, None, ints(keys)
    else:
        tokens, states = sum(queries), sum(keys)
        s["cu_q"], s["cu_k"], s["k_lens"] = ints(ends(queries)), ints(ends(keys)), None
        if case["queries"] == 1:
            s["cu_q"] = None                                       # a row each
    s["n"], s["max_q"], s["max_k"] = case["seqs"], max(queries), max(keys)
    s["q"] = _normal(g, tokens, hq, d, std=case["q_std"])
    kv = _normal(g, states, 2 * hkv * d)                           # one product makes both
    s["k"], s["v"] = kv[:, :hkv * d].view(states, hkv, d), kv[:, hkv * d:].view(states, hkv, d)
    s["dout"] = _normal(g, tokens, hq, d) if step else None
    if own:
        from paper_2509_22622_amd import binding as B
        attn = s["attn"] = B.EncoderAttention(hq, hkv, d, device=dev)
        s["out"] = torch.empty_like(s["q"])
        s["workspace"] = attn.workspace(s["n"], s["max_q"], s["max_k"])
        if step:
            s["lse"] = torch.empty(hq, tokens, dtype=torch.float32, device=dev)
            s["dq"] = torch.empty_like(s["q"])
            s["dk"], s["dv"] = (torch.empty(states, hkv, d, dtype=torch.bfloat16, device=dev) for _ in "kv")
            s["back"] = attn.backward_workspace(s["n"], tokens, s["max_q"], s["max_k"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    if s["case"]["op"].startswith("norm"):
        return _own_norm(s) if own else _plain_norm(s)
    return _own_attend(s) if own else _plain_attend(s)


def _own_norm(s):
    case, norm = s["case"], s["norm"]
    if case["op"] == "norm":
        norm.forward(s["x"], s["y"], weight=s["weight"], bias=s["bias"], group_rows=case["group"])
        return {"y": s["y"]}
    norm.forward(s["x"], s["y"], weight=s["weight"], bias=s["bias"], group_rows=case["group"], stats=s["stats"])
    norm.backward(s["dy"], s["x"], s["stats"], s["dx"], weight=s["weight"], dweight=s["dweight"], dbias=s["dbias"], group_rows=case["group"],
                  residual=s["residual"], workspace=s["workspace"])
    return {k: s[k] for k in ("y", "dx", "dweight", "dbias") if s[k] is not None}


def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    m, group = case["rows"], case["group"] or case["rows"]
    of = torch.arange(m, device=x.device) // group                 # the group of each row
    mean = x.mean(1, keepdim=True)
    x = x - mean
    rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    x = x * rstd
    w = None if s["weight"] is None else s["weight"].float()
    y = x if w is None else x * (w[of] if len(w) > 1 else w)
    if s["bias"] is not None:
        y = y + (s["bias"].float()[of] if len(s["bias"]) > 1 else s["bias"].float())
    out = {"y": y.to(TYPES[case["y"]])}
    if case["op"] == "norm":
        return out
    dy = s["dy"].float()
    g = dy if w is None else dy * (w[of] if len(w) > 1 else w)
    dx = rstd * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    out["dx"] = dx.to(TYPES[case["x"]])

    def by_group(t):
        if len(s["weight"]) == 1:
            return t.sum(0, keepdim=True)
        pad = len(s["weight"]) * group - m
        if pad:
            t = torch.cat([t, t.new_zeros(pad, t.shape[1])])
        return t.view(-1, group, t.shape[1]).sum(1)

    if w is not None:
        out["dweight"] = by_group(dy * x)
    if s["bias"] is not None:
        out["dbias"] = by_group(dy)
    return out


def _own_attend(s):
    step = s["case"]["op"] == "attend_step"
    batch = {"n_seqs": s["n"], "cu_q": s["cu_q"], "cu_k": s["cu_k"], "k_lens": s["k_lens"], "max_q": s["max_q"], "max_k": s["max_k"]}
    s["attn"].forward(s["q"], s["k"], s["v"], s["out"], lse=s["lse"] if step else None, workspace=s["workspace"], **batch)
    if not step:
        return {"out": s["out"]}
    s["attn"].backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dq"], s["dk"], s["dv"], workspace=s["back"], **batch)
    return {k: s[k] for k in ("out", "lse", "dq", "dk", "dv")}


def _rows(cu, lens, n_seqs, total, longest):
    """[n_seqs, longest] rows of each sequence; ``total`` where there is none."""
    dev = _device()
    each = total // n_seqs
    first = torch.arange(n_seqs, device=dev) * each if cu is None else cu.long()[:-1]
    n = torch.full_like(first, each) if cu is None else cu.long()[1:] - first
    if lens is not None:
        n = torch.minimum(n, lens.long())
    j = torch.arange(longest, device=dev)
    return torch.where(j < n[:, None], first[:, None] + j, total)


def _plain_attend(s):
    case = s["case"]
    hq, hkv, d, n = case["q_heads"], case["kv_heads"], case["head_dim"], s["n"]
    tokens, states, per = s["q"].shape[0], s["k"].shape[0], hq // hkv
    qr, kr = _rows(s["cu_q"], None, n, tokens, s["max_q"]), _rows(s["cu_k"], s["k_lens"], n, states, s["max_k"])

    def queries(t):                                                # [n, hkv, max_q * per, d]
        t = torch.cat([t, torch.zeros_like(t[:1])])[qr].float()
        return t.view(n, -1, hkv, per, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d)

    def keys(t):                                                   # [n, hkv, max_k, d]
        return torch.cat([t, torch.zeros_like(t[:1])])[kr].float().transpose(1, 2).contiguous()

    def tokens_of(t):                                              # back from queries()
        t = t.view(n, hkv, -1, per, d).permute(0, 2, 1, 3, 4).reshape(-1, hq, d)
        return t.new_zeros(tokens + 1, hq, d).index_copy(0, qr.flatten(), t)[:tokens].to(torch.bfloat16)

    def states_of(t):                                              # back from keys()
        t = t.transpose(1, 2).reshape(-1, hkv, d)
        return t.new_zeros(states + 1, hkv, d).index_copy(0, kr.flatten(), t)[:states].to(torch.bfloat16)

    q, k, v = queries(s["q"]), keys(s["k"]), keys(s["v"])
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()) * (d ** -0.5)
    score = score.masked_fill((kr == states)[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)                  # no keys
    p = torch.exp(score - top)
    del score
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    out = {"out": tokens_of(torch.matmul(p, v))}
    if case["op"] == "attend":
        return out
    lse = (top + torch.log(total)).view(n, hkv, -1, per).permute(0, 2, 1, 3).reshape(-1, hq)
    out["lse"] = lse.new_zeros(tokens + 1, hq).index_copy(0, qr.flatten(), lse)[:tokens].t().contiguous()
    do = queries(s["dout"])
    out["dv"] = states_of(torch.matmul(p.transpose(-1, -2).contiguous(), do))
    ds = torch.matmul(do, v.transpose(-1, -2).contiguous())
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * (d ** -0.5)
    out["dq"] = tokens_of(torch.matmul(ds, k))
    out["dk"] = states_of(torch.matmul(ds.transpose(-1, -2).contiguous(), q))
    return {k: out[k] for k in ("out", "lse", "dq", "dk", "dv")}


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    if case["op"].startswith("norm"):
        size = {"bf16": 2, "f32": 4}
        numbers, groups = case["rows"] * case["features"], -(-case["rows"] // case["group"]) if case["group"] else 1
        shared = groups * case["features"] * (case["weight"] + case["bias"])
        if case["op"] == "norm":
            return {"bytes": numbers * (size[case["x"]] + size[case["y"]]) + shared * size[case["w"]], "flops": 8.0 * numbers}
        return {"bytes": numbers * (size[case["x"]] * (3 if case["residual"] else 2) + 2 * size[case["y"]]) + shared * (size[case["w"]] + 4), "flops": 22.0 * numbers}
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    queries, keys = _spread(case)
    q_numbers, k_numbers = sum(queries) * hq * d, sum(keys) * hkv * d
    products = 2.0 * sum(a * b for a, b in zip(queries, keys)) * hq * d
    if case["op"] == "attend":
        return {"bytes": 2 * (2 * q_numbers + 2 * k_numbers), "flops": 2 * products}
    return {"bytes": 2 * (4 * q_numbers + 4 * k_numbers) + 4 * sum(queries) * hq, "flops": 7 * products}


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
    return _exact_norm(case, s) if case["op"].startswith("norm") else _exact_attend(case, s)


def _exact_norm(case, s):
    step, leaves = case["op"] == "norm_step", {}
    for k in ("x", "weight", "bias"):
        if s[k] is not None:
            leaves[k] = s[k].double().requires_grad_(step)
    x, group = leaves["x"], case["group"] or case["rows"]
    parts = []
    for i, at in enumerate(range(0, case["rows"], group)):
        t = x[at:at + group]
        y = (t - t.mean(1, keepdim=True)) / torch.sqrt(t.var(1, unbiased=False, keepdim=True) + EPS)
        y = y * leaves["weight"][i] if "weight" in leaves else y
        parts.append(y + leaves["bias"][i] if "bias" in leaves else y)
    y = torch.cat(parts)
    out = {"y": y.detach()}
    if step:
        grads = dict(zip(leaves, torch.autograd.grad(y, list(leaves.values()), s["dy"].double())))
        out["dx"] = grads["x"] if s["residual"] is None else grads["x"] + s["residual"].double()
        for k in ("weight", "bias"):
            if k in grads:
                out["d" + k] = grads[k]
    return out


def _exact_attend(case, s):
    hq, hkv, d, step = case["q_heads"], case["kv_heads"], case["head_dim"], case["op"] == "attend_step"
    queries, keys = _spread(case)
    if case["padded"]:
        q_at, k_at = ([i * max(x) for i in range(len(x))] for x in (queries, keys))
    else:
        q_at, k_at = ([sum(x[:i]) for i in range(len(x))] for x in (queries, keys))
    kind = {"dtype": torch.float64, "device": s["q"].device}
    out = {"out": torch.zeros(s["q"].shape, **kind)}
    if step:
        out |= {"lse": torch.full((hq, s["q"].shape[0]), -math.inf, **kind), "dq": torch.zeros(s["q"].shape, **kind),
                "dk": torch.zeros(s["k"].shape, **kind), "dv": torch.zeros(s["k"].shape, **kind)}
    for i, (a, b) in enumerate(zip(queries, keys)):
        if b == 0:
            continue
        at, to = slice(q_at[i], q_at[i] + a), slice(k_at[i], k_at[i] + b)
        for h in range(hq):
            g = h // (hq // hkv)
            q, k, v = (x.double().requires_grad_(step) for x in (s["q"][at, h], s["k"][to, g], s["v"][to, g]))
            z = q @ k.t() / math.sqrt(d)
            o = torch.softmax(z, -1) @ v
            out["out"][at, h] = o.detach()
            if step:
                out["lse"][h, at] = torch.logsumexp(z.detach(), -1)
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), s["dout"][at, h].double())
                out["dq"][at, h] = dq
                out["dk"][to, g] += dk
                out["dv"][to, g] += dv
    return out
