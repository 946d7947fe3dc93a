"""pisa_paged_append and pisa_paged_attention against the fp64 oracle, and the way from a prompt to the next token."""
import numpy as np
import pytest
import torch

from oracle import masked_oracle as mo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def cache(seed, lengths, kvh, page, d, dtype, heads_first=False, spare=2, width=None):
    """Filled pages in random order; slots that belong to nobody hold NaN.  Returns pages, table, and the rows in order."""
    g = torch.Generator().manual_seed(seed)
    used = [-(-n // page) for n in lengths]
    width = width or max(1, max(used))
    pool = sum(used) + spare
    shape = (pool, kvh, page, d) if heads_first else (pool, page, kvh, d)
    pages = [torch.full(shape, float("nan"), dtype=DT[dtype]) for _ in range(2)]
    views = [x.transpose(1, 2) if heads_first else x for x in pages]
    order = torch.randperm(pool, generator=g)[:sum(used)].tolist()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    rows, at = [], 0
    for s, n in enumerate(lengths):
        mine = order[at:at + used[s]]
        at += used[s]
        table[s, :used[s]] = torch.tensor(mine, dtype=torch.int32)
        kv = [torch.randn(n, kvh, d, generator=g).to(DT[dtype]) for _ in range(2)]
        for x, view in zip(kv, views):
            for i, pg in enumerate(mine):
                part = x[i * page:(i + 1) * page]
                view[pg, :len(part)] = part
        rows.append(kv)
    dev = [x.to(DEV) for x in pages]
    dev = [x.transpose(1, 2) if heads_first else x for x in dev]
    return dev[0], dev[1], table.to(DEV), rows


def oracle(q, rows, lengths, scale, softcap=0.0, slopes=None, drop=None):
    """out, lse, mass, zmax; drop[s]: positions that do not count."""
    n, h, d = q.shape
    out, mass = np.zeros((n, h, d)), np.zeros((n, h, d))
    lse, zmax = np.full((n, h), -np.inf), 0.0
    for s, length in enumerate(lengths):
        if length == 0:
            continue
        see = np.ones((1, 1, length), bool)
        if drop is not None:
            see[0, 0, drop[s]] = False
        k, v = (x[:length].double().numpy().transpose(1, 0, 2)[None] for x in rows[s])
        r = mo.attention(q[s].double().cpu().numpy()[None, :, None], k, v, see, scale, softcap, slopes)
        out[s], mass[s], lse[s] = r["out"][0, :, 0], r["mass"][0, :, 0], r["lse"][0, :, 0]
        zmax = max(zmax, r["zmax"])
    return {"out": out, "mass": mass, "lse": lse, "zmax": zmax}


def close(got, lse, ref, dtype, longest, d):
    eps = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    terms = longest + 4 * d + 64
    bound = mo.forward_bounds(ref, eps, terms)
    diff = np.abs(got.double().cpu().numpy() - ref["out"])
    assert np.all(diff <= bound), f"{np.nanmax(diff / bound):.2f} of the bound"
    x = lse.double().cpu().numpy()
    empty = np.isneginf(ref["lse"])
    assert np.array_equal(np.isneginf(x), empty)
    assert np.abs(x[~empty] - ref["lse"][~empty]).max(initial=0) <= 2.0 ** -24 * terms * (1 + ref["zmax"])


LENGTHS = [[1], [0, 5, 0, 128, 129], [1000, 37, 1], [3, 0, 2047, 300, 1, 640, 0]]


@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
@pytest.mark.parametrize("heads,kvh,page", [(1, 1, 16), (6, 2, 24), (20, 1, 1), (8, 8, 100), (32, 2, 256)])
def test_against_oracle(lib, lengths, dtype, d, heads, kvh, page):
    kp, vp, table, rows = cache(1, lengths, kvh, page, d, dtype, heads_first=page == 24)
    q = (1.5 * torch.randn(len(lengths), heads, d, generator=torch.Generator().manual_seed(2))).to(DT[dtype]).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), want_lse=True)
    torch.cuda.synchronize()
    close(out, lse, oracle(q, rows, lengths, lib.resolved_scale(d)), dtype, max(lengths), d)


@pytest.mark.parametrize("softcap,bias", [(10.0, False), (0.0, True), (3.0, True)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_scores_capped_and_biased(lib, softcap, bias, dtype, d):
    lengths = [500, 1, 90]
    kp, vp, table, rows = cache(3, lengths, 2, 16, d, dtype)
    slopes = torch.tensor([0.3, 0.01, 0.0, 0.1], device=DEV) if bias else None
    q = (1.5 * torch.randn(3, 4, d, generator=torch.Generator().manual_seed(4))).to(DT[dtype]).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), softcap=softcap,
                                   slopes=slopes, want_lse=True)
    torch.cuda.synchronize()
    ref = oracle(q, rows, lengths, lib.resolved_scale(d), softcap, None if slopes is None else slopes.double().cpu().numpy())
    close(out, lse, ref, dtype, 500, d)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_sequences(lib, dtype):
    """More sequences than a workgroup has threads, most of them empty or short."""
    rng = np.random.default_rng(5)
    lengths = [int(x) for x in np.where(rng.random(700) < 0.4, 0, rng.integers(0, 200, 700))]
    lengths[699] = 150
    kp, vp, table, rows = cache(6, lengths, 1, 32, 64, dtype)
    q = torch.randn(700, 2, 64, generator=torch.Generator().manual_seed(7)).to(DT[dtype]).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), want_lse=True)
    torch.cuda.synchronize()
    close(out, lse, oracle(q, rows, lengths, lib.resolved_scale(64)), dtype, 200, 64)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_pages_outside_the_cache_do_not_count(lib, dtype):
    lengths, page = [300, 64, 40], 16
    kp, vp, table, rows = cache(8, lengths, 2, page, 64, dtype)
    table[0, 3], table[0, 7], table[0, 18] = -1, kp.shape[0], 2 ** 31 - 1
    table[1, :] = -5                                               # nothing of it is left
    drop = [np.r_[48:64, 112:128, 288:300], np.arange(64), np.arange(0)]
    q = torch.randn(3, 4, 64, generator=torch.Generator().manual_seed(9)).to(DT[dtype]).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), want_lse=True)
    torch.cuda.synchronize()
    close(out, lse, oracle(q, rows, lengths, lib.resolved_scale(64), drop=drop), dtype, 300, 64)
    assert torch.count_nonzero(out[1]) == 0


def test_lengths_are_clamped_to_the_table(lib):
    lengths = [64, 32]
    kp, vp, table, rows = cache(10, lengths, 1, 32, 64, "bf16")
    q = torch.randn(2, 2, 64, generator=torch.Generator().manual_seed(11)).to(torch.bfloat16).to(DEV)
    told = torch.tensor([2 ** 31 - 1, -7], dtype=torch.int32, device=DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, told, want_lse=True)
    torch.cuda.synchronize()
    close(out, lse, oracle(q, rows, [64, 0], lib.resolved_scale(64)), "bf16", 64, 64)


def test_a_cache_past_4_gib(lib):
    """Pages whose byte offsets pass 32 bits."""
    page, kvh, d = 256, 8, 128
    pool = (5 << 30) // (page * kvh * d * 2)
    kp, vp = (torch.empty(pool, page, kvh, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.tensor([[pool - 1, 3, pool - 2]], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(12)
    n = 700
    rows = [[torch.randn(n, kvh, d, generator=g).to(torch.bfloat16) for _ in range(2)]]
    lengths = torch.tensor([n], dtype=torch.int32, device=DEV)
    offsets = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    lib.paged_append(rows[0][0].to(DEV), rows[0][1].to(DEV), offsets, kp, vp, table, lengths)
    q = torch.randn(1, 16, d, generator=g).to(torch.bfloat16).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, lengths, want_lse=True)
    torch.cuda.synchronize()
    assert torch.equal(kp[pool - 2, :n - 512].cpu(), rows[0][0][512:]) and torch.equal(vp[3].cpu(), rows[0][1][256:512])
    close(out, lse, oracle(q, rows, [n], lib.resolved_scale(d)), "bf16", n, d)


@pytest.mark.parametrize("dtype,heads_first", [("bf16", False), ("bf16", True), ("fp32", False)])
def test_append_writes_its_rows_and_nothing_else(lib, dtype, heads_first):
    kvh, page, d = 3, 24, 64
    before, new = [40, 0, 23, 7], [1, 50, 0, 18]
    after = [a + b for a, b in zip(before, new)]
    kp, vp, table, _ = cache(13, after, kvh, page, d, dtype, heads_first)
    tokens = sum(new) + 4                                          # rows ahead of the first sequence and behind the last
    offsets = np.concatenate([[2], 2 + np.cumsum(new)])
    g = torch.Generator().manual_seed(14)
    k, v = (torch.randn(tokens, kvh, d, generator=g).to(DT[dtype]).to(DEV) for _ in range(2))
    lengths = torch.tensor(after, dtype=torch.int32, device=DEV)
    table[3, 0] = kp.shape[0]                                      # a page that does not exist: its tokens go nowhere
    want = [kp.clone(), vp.clone()]
    for s in range(4):
        for i in range(new[s]):
            pos = before[s] + i
            pg = int(table[s, pos // page])
            if 0 <= pg < kp.shape[0]:
                for w, x in zip(want, (k, v)):
                    w[pg, pos % page] = x[offsets[s] + i]
    lib.paged_append(k, v, torch.tensor(offsets, dtype=torch.int32, device=DEV), kp, vp, table, lengths)
    torch.cuda.synchronize()
    bits = torch.int16 if dtype == "bf16" else torch.int32
    for w, x in zip(want, (kp, vp)):
        assert torch.equal(w.contiguous().view(bits), x.contiguous().view(bits))


def test_append_of_more_than_a_sequence_holds(lib):
    """Positions below 0 and past the table are left out, and no token is no work."""
    kp, vp, table, _ = cache(15, [32], 1, 16, 64, "bf16", spare=0)
    k = torch.randn(40, 1, 64).to(torch.bfloat16).to(DEV)
    offsets = torch.tensor([0, 40], dtype=torch.int32, device=DEV)
    lib.paged_append(k, k, offsets, kp, vp, table, torch.tensor([36], dtype=torch.int32, device=DEV))     # positions -4 .. 35
    lib.paged_append(k[:0], k[:0], torch.tensor([0, 0], dtype=torch.int32, device=DEV), kp, vp, table,
                     torch.tensor([36], dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for half in range(2):
        assert torch.equal(kp[int(table[0, half])], k[4 + 16 * half:20 + 16 * half])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_from_a_prompt_to_the_next_tokens(lib, dtype):
    """Prompt through masked_attention, its keys and values into the cache, then token by token: every step's row is the last
    row of masked attention over the whole sequence."""
    d, h, kvh, page, prompt, steps = 128, 8, 2, 16, [75, 130], 4
    g = torch.Generator().manual_seed(16)
    total = [p + steps for p in prompt]
    q, k, v = ([(torch.randn(n, x, d, generator=g)).to(DT[dtype]).to(DEV) for n in total] for x in (h, kvh, kvh))
    pool = sum(-(-n // page) for n in total)
    kp, vp = (torch.full((pool, page, kvh, d), float("nan"), dtype=DT[dtype], device=DEV) for _ in range(2))
    width = max(-(-n // page) for n in total)
    table = torch.full((2, width), -1, dtype=torch.int32, device=DEV)
    first = -(-total[0] // page)
    table[0, :first] = torch.arange(first, dtype=torch.int32, device=DEV)
    table[1, :pool - first] = torch.arange(first, pool, dtype=torch.int32, device=DEV)
    # both prompts as documents of one packed sequence
    pack = lambda xs: torch.cat([x[:p] for x, p in zip(xs, prompt)])
    borders = torch.tensor([[0, prompt[0], sum(prompt)]], dtype=torch.int32, device=DEV)
    view = lambda x: x[None].transpose(1, 2)
    out, _ = lib.masked_attention(view(pack(q)), view(pack(k)), view(pack(v)), causal=True, doc_offsets=borders)
    lengths = torch.tensor(prompt, dtype=torch.int32, device=DEV)
    lib.paged_append(pack(k), pack(v), borders[0].contiguous(), kp, vp, table, lengths)
    one = torch.arange(3, dtype=torch.int32, device=DEV)
    bits = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    whole = []
    for s in range(2):
        ref = mo.attention(*(x[s].double().cpu().numpy().transpose(1, 0, 2)[None] for x in (q, k, v)),
                           mo.visible(1, total[s], total[s], True), lib.resolved_scale(d))
        whole.append((ref, mo.forward_bounds(ref, bits, total[s] + 4 * d + 64)))
    at = 0
    for s in range(2):
        ref, bound = whole[s]
        got = out[0, :, at:at + prompt[s]].double().cpu().numpy()
        assert np.all(np.abs(got - ref["out"][0, :, :prompt[s]]) <= bound[0, :, :prompt[s]])
        at += prompt[s]
    for i in range(steps):
        lengths += 1
        lib.paged_append(torch.stack([k[s][prompt[s] + i] for s in range(2)]), torch.stack([v[s][prompt[s] + i] for s in range(2)]),
                         one, kp, vp, table, lengths)
        got, _ = lib.paged_attention(torch.stack([q[s][prompt[s] + i] for s in range(2)]), kp, vp, table, lengths)
        got = got.double().cpu().numpy()
        for s in range(2):
            ref, bound = whole[s]
            assert np.all(np.abs(got[s] - ref["out"][0, :, prompt[s] + i]) <= bound[0, :, prompt[s] + i])


def test_graph_replays_follow_the_lengths(lib):
    """A captured step reads lengths and table from the device: replays serve the sequences as they grow."""
    kvh, h, d, page = 2, 8, 128, 16
    lengths0 = [100, 700]
    kp, vp, table, _ = cache(17, [n + 40 for n in lengths0], kvh, page, d, "bf16")
    lengths = torch.tensor(lengths0, dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(18)
    q = torch.randn(2, h, d, generator=g).to(torch.bfloat16).to(DEV)
    kn, vn = (torch.randn(2, kvh, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    one = torch.arange(3, dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(2, h, device=DEV)
    ws = torch.empty(lib.paged_attention_workspace_bytes(q, kp, vp, table), dtype=torch.uint8, device=DEV)

    def step():
        lib.paged_append(kn, vn, one, kp, vp, table, lengths)
        lib.paged_attention(q, kp, vp, table, lengths, out=out, lse=lse, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        lengths += 9
        q.copy_(torch.randn(2, h, d, generator=g).to(torch.bfloat16))
        step()
        torch.cuda.synchronize()
        eager = out.clone(), lse.clone()
        out.fill_(float("nan"))
        lse.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("softcap", [1e-3, 0.5, 1e6])
def test_caps_of_any_size(lib, dtype, softcap):
    lengths = [400, 3]
    kp, vp, table, rows = cache(20, lengths, 2, 16, 64, dtype)
    q = (1.5 * torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(21))).to(DT[dtype]).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), softcap=softcap, want_lse=True)
    torch.cuda.synchronize()
    close(out, lse, oracle(q, rows, lengths, lib.resolved_scale(64), softcap), dtype, 400, 64)


def test_sequences_that_share_pages(lib):
    """Three sequences go on from the same pages."""
    page, shared = 16, 48
    kp, vp, table, rows = cache(22, [100], 2, page, 128, "bf16", spare=8)
    free = sorted(set(range(kp.shape[0])) - set(table[0].tolist()))
    tables = table.expand(3, -1).contiguous()
    tables[1, 3], tables[2, 3] = free[0], free[1]
    lengths, mine = [100, 60, 49], [rows[0]]
    for s in (1, 2):
        new = [torch.randn(lengths[s] - shared, 2, 128, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for _ in range(2)]
        mine.append([torch.cat([old[:shared], x]) for old, x in zip(rows[0], new)])
        offsets = torch.tensor([0, 0, lengths[1] - shared if s == 1 else 0, lengths[s] - shared], dtype=torch.int32, device=DEV)
        lib.paged_append(new[0].to(DEV), new[1].to(DEV), offsets, kp, vp, tables, torch.tensor(lengths, dtype=torch.int32, device=DEV))
    q = torch.randn(3, 4, 128, generator=torch.Generator().manual_seed(23)).to(torch.bfloat16).to(DEV)
    out, lse = lib.paged_attention(q, kp, vp, tables, torch.tensor(lengths, dtype=torch.int32, device=DEV), want_lse=True)
    torch.cuda.synchronize()
    close(out, lse, oracle(q, mine, lengths, lib.resolved_scale(128)), "bf16", 100, 128)


def test_two_calls_at_once(lib):
    calls = []
    for seed, lengths in ((24, [3000, 5]), (25, [700] * 9)):
        kp, vp, table, _ = cache(seed, lengths, 2, 32, 128, "bf16")
        q = torch.randn(len(lengths), 8, 128, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).to(DEV)
        calls.append((q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV)))
    want = [lib.paged_attention(*c, want_lse=True) for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = []
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                got.append(lib.paged_attention(*c, want_lse=True))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_scores_of_minus_infinity_alone(lib, dtype):
    """A cached sequence whose keys all score -inf has out 0 and lse -inf, in one workgroup as over many."""
    for lengths in ([40, 100], [3000, 700]):
        kp, vp, table, rows = cache(26, lengths, 2, 16, 64, dtype)
        q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(27)).to(DT[dtype]).to(DEV)
        q[..., 7] = 2.0
        kp[table[0, :-(-lengths[0] // 16)].long(), :, :, 7] = torch.finfo(kp.dtype).min
        out, lse = lib.paged_attention(q, kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), want_lse=True)
        torch.cuda.synchronize()
        assert torch.count_nonzero(out[0]) == 0 and torch.isneginf(lse[0]).all()
        ref = oracle(q, rows, [0, lengths[1]], lib.resolved_scale(64))
        close(out, lse, ref, dtype, lengths[1], 64)
