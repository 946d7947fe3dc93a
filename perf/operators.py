"""Masked attention with its gradients, and one-token attention over a paged cache: the calls whose speed counts.

`listed()` holds the cases, `draw()` further ones of the same ranges.  A case is one of

    forward    masked_attention: scores capped by a tanh and biased by distance where asked for, keys limited to the
               row's document and, if causal, to what lies before the row or in its document's prefix
    train      masked_attention and masked_attention_backward on the same inputs, as a training step runs them
    decode     paged_append of one new token per sequence, then paged_attention over the cache

With `own` false `run` computes the same from elementary torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _dense(name, kind, batch, heads, kv_heads, q_len, kv_len, d, dtype="bf16", causal=False, docs="", prefix=0, cap=0.0,
           bias=False, tokens_first=False):
    """docs: lengths of the documents laid one behind the other ("" = one document of kv_len tokens; what they leave of
    kv_len is padding); batch element b has them rotated by b.  prefix: tokens at each document's start that all of its rows
    see.  cap: of the tanh, 0 for none.  tokens_first: memory order [batch, tokens, heads, d] in place of [batch, heads,
    tokens, d].  The q_len query rows are the last of the kv_len positions."""
    return {"name": name, "kind": kind, "batch": batch, "heads": heads, "kv_heads": kv_heads, "q_len": q_len, "kv_len": kv_len,
            "d": d, "dtype": dtype, "causal": causal, "docs": docs, "prefix": prefix, "cap": cap, "bias": bias,
            "tokens_first": tokens_first}


def _paged(name, seqs, heads, kv_heads, longest, spread, page, d, dtype="bf16", cap=0.0, bias=False, heads_first=False):
    """longest: tokens of the longest sequence, the new one included; the others are up to `spread` shorter.
    heads_first: pages of [kv_heads, page, d] in place of [page, kv_heads, d]."""
    return {"name": name, "kind": "decode", "seqs": seqs, "heads": heads, "kv_heads": kv_heads, "longest": longest,
            "spread": spread, "page": page, "d": d, "dtype": dtype, "cap": cap, "bias": bias, "heads_first": heads_first}


def listed():
    return [
        # a prompt of an image model's text side: two short rows of tokens, the first 40 seen by all; latency is all there is
        _dense("forward-text", "forward", 2, 8, 8, 200, 200, 64, causal=True, prefix=40),
        # image layers of several resolutions packed into one sequence of the repository's image length, full attention inside
        _dense("forward-packed", "forward", 1, 24, 24, 4608, 4608, 128, docs="1024,2304,577,703", tokens_first=True),
        # the next piece of a long sequence against what the cache holds already (odd lengths, distance bias, shared heads)
        _dense("forward-piece", "forward", 1, 24, 8, 500, 9001, 128, causal=True, bias=True, tokens_first=True),
        # the longest: capped scores, four query heads on one key head
        _dense("forward-long", "forward", 1, 16, 4, 16384, 16384, 128, causal=True, cap=50.0),
        # a reference run in fp32 at an odd length
        _dense("forward-fp32", "forward", 1, 8, 8, 4500, 4500, 128, dtype="fp32", causal=True, prefix=512, bias=True),
        # one training step of the packed image layer, two of its documents padded away behind the last
        _dense("train-packed", "train", 1, 24, 24, 4608, 4608, 128, docs="1024,2304,577,300"),
        # shared heads with capped and biased scores, 64 channels, an odd length
        _dense("train-shared", "train", 2, 12, 4, 2777, 2777, 64, causal=True, cap=30.0, bias=True, tokens_first=True),
        # a small fp32 step, as gradients are checked with
        _dense("train-fp32", "train", 1, 4, 2, 1000, 1000, 128, dtype="fp32", causal=True, prefix=77),
        # a long causal step
        _dense("train-long", "train", 1, 12, 12, 8192, 8192, 128, causal=True),
        # one user, a short cache in small pages: latency
        _paged("decode-one", 1, 8, 2, 1000, 0.0, 16, 128),
        # a batch of users of very different lengths, capped scores
        _paged("decode-batch", 48, 32, 8, 8000, 0.95, 64, 128, cap=50.0),
        # two users with very long sequences: all of the card has to read for each of them
        _paged("decode-long", 2, 40, 8, 200001, 0.2, 128, 128, heads_first=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["forward", "train", "decode"])
    d = rng.choice([128, 128, 64])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 5, 8])
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    bias = rng.random() < 0.3
    if kind == "decode":
        case = _paged("", _log_int(rng, 1, 64), heads, kv_heads, _log_int(rng, 1, 200000), rng.choice([0.0, 0.5, 0.95]),
                      rng.choice([16, 16, 24, 64, 128, 256]), d, dtype, cap, bias, rng.random() < 0.5)
        limit = work(listed()[-1])["bytes"]
        while work(case)["bytes"] > limit:
            if case["seqs"] > 1:
                case["seqs"] = max(1, case["seqs"] // 2)
            else:
                case["longest"] = max(1, case["longest"] // 2)
        return case
    most = 16384 if kind == "forward" else 8192
    kv_len = _log_int(rng, 1, most)
    q_len = kv_len if kind == "train" or rng.random() < 0.6 else _log_int(rng, 1, kv_len)
    docs = ""
    if rng.random() < 0.5 and kv_len >= 8:
        left, lengths = kv_len, []
        for _ in range(rng.randint(2, 6)):
            n = rng.randint(1, max(1, 2 * kv_len // 5))
            if n <= left:
                lengths.append(n)
                left -= n
        if rng.random() < 0.5 and left:
            lengths.append(left)
        docs = ",".join(map(str, lengths))
    causal = rng.random() < 0.6
    case = _dense("", kind, rng.choice([1, 1, 2]), heads, kv_heads, q_len, kv_len, d, dtype, causal, docs,
                  rng.choice([0, 0, max(1, kv_len // 9)]) if causal else 0, cap, bias, rng.random() < 0.5)
    cells = 16 * 16384 ** 2 if kind == "forward" else 12 * 8192 ** 2
    cells //= 8 if dtype == "fp32" else 1      # the 32-bit matrix rate is a sixteenth of the 16-bit one
    while case["batch"] * case["heads"] * case["q_len"] * case["kv_len"] > cells:
        if case["batch"] > 1:
            case["batch"] = 1
        elif case["kv_heads"] > 1:
            case["heads"] = case["heads"] // case["kv_heads"]
            case["kv_heads"] = 1
        elif case["heads"] > 1:
            case["heads"] = 1
        else:
            case["q_len"] = min(case["q_len"], max(1, cells // case["kv_len"]))
    return case


# ---- what a case's numbers stand for --------------------------------------------------------------------------


def _offsets(case):
    """[batch][documents + 1] positions of the document borders."""
    lengths = [int(x) for x in case["docs"].split(",")] if case["docs"] else [case["kv_len"]]
    return np.stack([np.concatenate([[0], np.cumsum(lengths[b % len(lengths):] + lengths[:b % len(lengths)])])
                     for b in range(case["batch"])])


def _intervals(case):
    """lo, hi [batch, q_len]: the keys lo <= j < hi that each query row sees (empty where lo == hi)."""
    pos = np.arange(case["q_len"]) + case["kv_len"] - case["q_len"]
    lows, highs = [], []
    for offs in _offsets(case):
        lo, hi = np.zeros_like(pos), np.zeros_like(pos)
        for a, e in zip(offs[:-1], offs[1:]):
            inside = (pos >= a) & (pos < e)
            lo[inside] = a
            hi[inside] = np.minimum(np.maximum(pos[inside] + 1, a + case["prefix"]), e) if case["causal"] else e
        lows.append(lo)
        highs.append(hi)
    return np.stack(lows), np.stack(highs)


def _lengths(case):
    """Cached tokens of each sequence, the new one included."""
    s = np.arange(case["seqs"])
    return np.maximum(1, np.round(case["longest"] * (1 - case["spread"] * ((s * 0.6180339887) % 1.0)))).astype(np.int64)


def _slopes(heads, device):
    return torch.exp2(-8.0 * (torch.arange(heads, device=device, dtype=torch.float32) + 1) / heads)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    h, kvh, d = case["heads"], case["kv_heads"], case["d"]
    if case["kind"] == "decode":
        total, n = int(_lengths(case).sum()), case["seqs"]
        cache = 2 * total * kvh * d * size                      # the new token's part is written, the rest read
        pages = int(np.sum(-(-_lengths(case) // case["page"])))
        return {"bytes": cache + 2 * n * kvh * d * size + n * h * (2 * d * size + 4) + 4 * (pages + n),
                "flops": 4 * d * h * total}
    lo, hi = _intervals(case)
    pairs = int((hi - lo).sum()) * h
    b = case["batch"]
    q, kv, lse = b * h * case["q_len"] * d * size, b * kvh * case["kv_len"] * d * size, 4 * b * h * case["q_len"]
    if case["kind"] == "forward":
        return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * d * pairs}
    return {"bytes": 4 * q + 4 * kv + lse, "flops": 14 * d * pairs}   # q, out, dout, dq; k, v, dk, dv; two products, then five


# ---- inputs ---------------------------------------------------------------------------------------------------


def _random(gen, batch, heads, length, case, scale=1.0):
    """[batch, heads, length, d] in the case's memory order."""
    shape = (batch, length, heads, case["d"]) if case["tokens_first"] else (batch, heads, length, case["d"])
    x = torch.randn(shape, generator=gen, device=gen.device).mul_(scale).to(_DTYPES[case["dtype"]])
    return x.transpose(1, 2) if case["tokens_first"] else x


def prepare(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device).manual_seed(seed)
    state = {"case": case, "slopes": _slopes(case["heads"], device) if case["bias"] else None}
    if case["kind"] == "decode":
        return _prepare_decode(case, gen, state)
    b, h, kvh, nq, nk = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "kv_len"))
    state["q"] = _random(gen, b, h, nq, case, 1.5)              # scores of spread 1.5, as trained layers reach and pass
    state["k"] = _random(gen, b, kvh, nk, case)
    state["v"] = _random(gen, b, kvh, nk, case)
    if case["kind"] == "train":
        state["dout"] = _random(gen, b, h, nq, case)
    offsets = torch.from_numpy(_offsets(case)).to(torch.int32)
    state["doc_offsets"] = offsets.to(device) if case["docs"] else None
    n = offsets.shape[1] - 1
    state["prefix"] = torch.full((b, n), case["prefix"], dtype=torch.int32, device=device) if case["prefix"] else None
    return state


def _prepare_decode(case, gen, state):
    device, dtype = gen.device, _DTYPES[case["dtype"]]
    n, h, kvh, d, page = (case[x] for x in ("seqs", "heads", "kv_heads", "d", "page"))
    lengths = torch.from_numpy(_lengths(case)).to(device)
    used = -(-lengths // page)
    width, total = -(-case["longest"] // page), int(used.sum())
    pool = total + 3                                            # pages of other users
    order = torch.randperm(pool, generator=gen, device=device)[:total]
    table = torch.full((n, width), -1, dtype=torch.int32, device=device)
    table[torch.arange(width, device=device)[None, :] < used[:, None]] = order.to(torch.int32)
    shape = (pool, kvh, page, d) if case["heads_first"] else (pool, page, kvh, d)
    for name in ("k_pages", "v_pages"):
        x = torch.empty(shape, dtype=dtype, device=device).normal_(generator=gen)
        state[name] = x.transpose(1, 2) if case["heads_first"] else x
    state["q"] = (1.5 * torch.randn(n, h, d, generator=gen, device=device)).to(dtype)
    state["k_new"], state["v_new"] = (torch.randn(n, kvh, d, generator=gen, device=device).to(dtype) for _ in range(2))
    state["offsets"] = torch.arange(n + 1, dtype=torch.int32, device=device)   # one new token each
    state["page_table"], state["lengths"] = table, lengths.to(torch.int32)
    state["out"] = torch.empty_like(state["q"])                 # a serving loop keeps its outputs' memory
    state["lse"] = torch.empty(n, h, dtype=torch.float32, device=device)
    return state


# ---- the plain forms ------------------------------------------------------------------------------------------


def _visible(case, offsets, prefix, device):
    """Truth values [batch, 1, q_len, kv_len]: does the row see the key."""
    key = torch.arange(case["kv_len"], device=device)
    row = key[case["kv_len"] - case["q_len"]:]
    if offsets is None:
        offsets = torch.tensor([[0, case["kv_len"]]], device=device)
    n = offsets.shape[1] - 1
    doc = (key[None, :, None] >= offsets[:, None, :]).sum(-1) - 1                  # [batch, kv_len]
    doc_row = doc[:, case["kv_len"] - case["q_len"]:]
    see = (doc_row[:, :, None] == doc[:, None, :]) & (doc_row < n)[:, :, None]
    if case["causal"]:
        before = key[None, None, :] <= row[None, :, None]
        if prefix is not None:
            end = (offsets[:, :-1] + prefix).gather(1, doc_row.clamp(max=n - 1))   # of the row's document's prefix
            before = before | (key[None, None, :] < end[:, :, None])
        see &= before
    return see[:, None]


def _plain_weights(state):
    """Softmax weights [batch, heads, q_len, kv_len] in 32 bits, log-sum-exp, and 1 - tanh^2 of capped scores."""
    case, q, k = state["case"], state["q"].float(), state["k"].float()
    group = case["heads"] // case["kv_heads"]
    s = torch.matmul(q * (1.0 / math.sqrt(case["d"])), k.repeat_interleave(group, 1).transpose(2, 3))
    slope = None
    if case["cap"]:
        s = torch.tanh(s.div_(case["cap"]))
        slope = 1 - s * s if case["kind"] == "train" else None
        s.mul_(case["cap"])
    if case["bias"]:
        key = torch.arange(case["kv_len"], device=s.device)
        far = (key[case["kv_len"] - case["q_len"]:, None] - key[None, :]).abs().float()
        s.sub_(state["slopes"][:, None, None] * far)
    s.masked_fill_(~_visible(case, state["doc_offsets"], state["prefix"], s.device), -math.inf)
    top = s.amax(-1, keepdim=True)
    s = s.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = s.sum(-1, keepdim=True)
    lse = (top + total.log())[..., 0]                           # -inf for a row that sees nothing
    return s.div_(total.masked_fill(total == 0, 1.0)), lse, slope


def _plain_forward(state):
    p, lse, _ = _plain_weights(state)
    group = state["case"]["heads"] // state["case"]["kv_heads"]
    out = torch.matmul(p, state["v"].float().repeat_interleave(group, 1))
    return {"out": out.to(state["q"].dtype), "lse": lse}


def _plain_train(state):
    case = state["case"]
    p, lse, slope = _plain_weights(state)
    b, kvh, nk, d = state["k"].shape
    group, dtype = case["heads"] // kvh, state["q"].dtype
    q, k, v, dout = (state[x].float() for x in ("q", "k", "v", "dout"))
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    out = torch.matmul(p, v)
    dv = torch.matmul(p.transpose(2, 3), dout)
    ds = torch.matmul(dout, v.transpose(2, 3))
    ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p)
    if slope is not None:
        ds.mul_(slope)
    ds.mul_(1.0 / math.sqrt(d))
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(2, 3), q)
    dk, dv = (x.view(b, kvh, group, nk, d).sum(2) for x in (dk, dv))
    return {"out": out.to(dtype), "lse": lse, "dq": dq.to(dtype), "dk": dk.to(dtype), "dv": dv.to(dtype)}


def _plain_decode(state):
    case, table, lengths = state["case"], state["page_table"].long(), state["lengths"].long()
    n, h, kvh, d, page = (case[x] for x in ("seqs", "heads", "kv_heads", "d", "page"))
    last = lengths - 1
    at = table.gather(1, (last // page)[:, None])[:, 0]
    state["k_pages"][at, last % page] = state["k_new"]
    state["v_pages"][at, last % page] = state["v_new"]
    k, v = (state[x][table.clamp(min=0)].reshape(n, -1, kvh, d).float() for x in ("k_pages", "v_pages"))
    q = state["q"].float().view(n, kvh, h // kvh, d) * (1.0 / math.sqrt(d))
    s = torch.matmul(q, k.permute(0, 2, 3, 1))                  # [seqs, kv_heads, group, keys]
    if case["cap"]:
        s = torch.tanh(s / case["cap"]) * case["cap"]
    key = torch.arange(s.shape[-1], device=s.device)
    if case["bias"]:
        far = (last[:, None] - key[None, :]).abs().float()
        s = s - state["slopes"].view(1, kvh, -1, 1) * far[:, None, None, :]
    s = s.masked_fill((key[None, :] >= lengths[:, None])[:, None, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    s = (s - top).exp()
    total = s.sum(-1, keepdim=True)
    out = torch.matmul(s, v.transpose(1, 2)) / total
    return {"out": out.view(n, h, d).to(state["q"].dtype), "lse": (top + total.log()).view(n, h),
            "k_pages": state["k_pages"], "v_pages": state["v_pages"]}


# ---- one pass -------------------------------------------------------------------------------------------------


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"forward": _plain_forward, "train": _plain_train, "decode": _plain_decode}[kind](state)
    import paper_2602_01077_amd as pisa
    cap, slopes = state["case"]["cap"], state["slopes"]
    if kind == "decode":
        k_pages, v_pages, table, lengths = (state[x] for x in ("k_pages", "v_pages", "page_table", "lengths"))
        pisa.paged_append(state["k_new"], state["v_new"], state["offsets"], k_pages, v_pages, table, lengths)
        out, lse = pisa.paged_attention(state["q"], k_pages, v_pages, table, lengths, softcap=cap, slopes=slopes,
                                        out=state["out"], lse=state["lse"])
        return {"out": out, "lse": lse, "k_pages": k_pages, "v_pages": v_pages}
    q, k, v = state["q"], state["k"], state["v"]
    mask = {"causal": state["case"]["causal"], "doc_offsets": state["doc_offsets"], "prefix": state["prefix"]}
    out, lse = pisa.masked_attention(q, k, v, softcap=cap, slopes=slopes, want_lse=True, **mask)
    if kind == "forward":
        return {"out": out, "lse": lse}
    dq, dk, dv = pisa.masked_attention_backward(q, k, v, out, lse, state["dout"], softcap=cap, slopes=slopes, **mask)
    return {"out": out, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


# ---- the definition in 64 bits --------------------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_decode(state) if case["kind"] == "decode" else _exact_dense(state)


def _exact_dense(state):
    case, f64 = state["case"], torch.float64
    b, h, kvh, nq, nk, d = (case[x] for x in ("batch", "heads", "kv_heads", "q_len", "kv_len", "d"))
    train, group, scale = case["kind"] == "train", h // kvh, 1.0 / math.sqrt(d)
    device = state["q"].device
    lo, hi = (torch.from_numpy(x).to(device) for x in _intervals(case))
    res = {"out": torch.zeros(b, h, nq, d, dtype=f64, device=device),
           "lse": torch.full((b, h, nq), -math.inf, dtype=f64, device=device)}
    if train:
        res["dq"] = torch.zeros(b, h, nq, d, dtype=f64, device=device)
        res["dk"] = torch.zeros(b, kvh, nk, d, dtype=f64, device=device)
        res["dv"] = torch.zeros(b, kvh, nk, d, dtype=f64, device=device)
    key = torch.arange(nk, device=device)
    for i in range(b):
        for j in range(h):
            k, v = state["k"][i, j // group].to(f64), state["v"][i, j // group].to(f64)
            for a in range(0, nq, 4096):
                rows = slice(a, min(a + 4096, nq))
                some = (hi[i, rows] > lo[i, rows]).nonzero()[:, 0] + a       # the rows that see a key
                if not len(some):
                    continue
                q = state["q"][i, j, some].to(f64)
                raw = q @ k.T * scale
                cut = torch.tanh(raw / case["cap"]) if case["cap"] else None
                z = cut * case["cap"] if case["cap"] else raw
                if case["bias"]:
                    z = z - state["slopes"][j].to(f64) * (some[:, None] + (nk - nq) - key[None, :]).abs()
                z = torch.where((key >= lo[i, some, None]) & (key < hi[i, some, None]), z, -math.inf)
                lse = torch.logsumexp(z, 1)
                p = torch.exp(z - lse[:, None])
                res["out"][i, j, some] = p @ v
                res["lse"][i, j, some] = lse
                if train:
                    dout = state["dout"][i, j, some].to(f64)
                    res["dv"][i, j // group] += p.T @ dout
                    dz = p * (dout @ v.T - (dout * (p @ v)).sum(1, keepdim=True))
                    if case["cap"]:
                        dz = dz * (1 - cut * cut)
                    res["dq"][i, j, some] = dz @ k * scale
                    res["dk"][i, j // group] += dz.T @ q * scale
    return res


def _exact_decode(state):
    case, f64 = state["case"], torch.float64
    h, kvh, d, page = (case[x] for x in ("heads", "kv_heads", "d", "page"))
    group = h // kvh
    out = torch.zeros(case["seqs"], h, d, dtype=f64, device=state["q"].device)
    lse = torch.zeros(case["seqs"], h, dtype=f64, device=state["q"].device)
    for i, length in enumerate(_lengths(case).tolist()):
        pages = state["page_table"][i, :-(-length // page)].tolist()
        for name in ("k", "v"):
            state[name + "_pages"][pages[-1], (length - 1) % page] = state[name + "_new"][i]
        at = torch.arange(length, device=out.device)
        ids = torch.tensor(pages, device=out.device)[at // page]
        for g in range(kvh):
            k, v = (state[x][ids, at % page, g].to(f64) for x in ("k_pages", "v_pages"))
            z = state["q"][i, g * group:(g + 1) * group].to(f64) @ k.T / math.sqrt(d)
            if case["cap"]:
                z = case["cap"] * torch.tanh(z / case["cap"])
            if case["bias"]:
                z = z - state["slopes"][g * group:(g + 1) * group, None].to(f64) * (length - 1 - at)
            top = torch.logsumexp(z, 1)
            lse[i, g * group:(g + 1) * group] = top
            out[i, g * group:(g + 1) * group] = torch.exp(z - top[:, None]) @ v
    return {"out": out, "lse": lse, "k_pages": None, "v_pages": None}
