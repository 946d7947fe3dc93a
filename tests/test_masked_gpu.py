"""pisa_masked_attention and pisa_masked_attention_backward against the fp64 oracle: types, masks that leave rows empty,
odd sizes, strides, shared heads, non-finite values in masked places, capture into a graph."""
import numpy as np
import pytest
import torch

from oracle import masked_oracle as mo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def make(seed, b, h, kvh, n, m, d, dtype, tokens_first=False, spread=1.5):
    g = torch.Generator().manual_seed(seed)

    def one(heads, length, s=1.0):
        shape = (b, length, heads, d) if tokens_first else (b, heads, length, d)
        x = (s * torch.randn(shape, generator=g)).to(DT[dtype])
        return (x.transpose(1, 2) if tokens_first else x)
    q, k, v, dout = one(h, n, spread), one(kvh, m), one(kvh, m), one(h, n)
    up = lambda x: x.to(DEV) if not tokens_first else x.transpose(1, 2).contiguous().to(DEV).transpose(1, 2)
    return up(q), up(k), up(v), up(dout)


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def n_terms(m, d):
    return m + 4 * d + 64        # products of a score, weights of a row, and what the exponential adds


def check(lib, q, k, v, dout, causal, docs, prefix, softcap=0.0, slopes=None, backward=True, **kw):
    b, h, n, d = q.shape
    m = k.shape[2]
    see = mo.visible(b, n, m, causal, docs, prefix)
    scale = lib.resolved_scale(d)
    slo = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device=DEV)
    args = dict(causal=causal, doc_offsets=ints(docs), prefix=ints(prefix), softcap=softcap, slopes=slo)
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args, **kw)
    grads = lib.masked_attention_backward(q, k, v, out, lse, dout, **args) if backward else None
    torch.cuda.synchronize()
    slo64 = None if slopes is None else slo.double().cpu().numpy()
    ref = mo.attention(f64(q), f64(k), f64(v), see, scale, softcap, slo64, f64(dout) if backward else None)
    eps = 2.0 ** -7 if q.dtype == torch.bfloat16 else 2.0 ** -23
    terms = n_terms(m, d)
    bound = mo.forward_bounds(ref, eps, terms)
    diff = np.abs(f64(out) - ref["out"])
    assert np.all(diff <= bound), f"out: {np.max(diff / bound):.2f} of the bound"
    lse_ref, lse_got = ref["lse"], f64(lse)
    empty = np.isneginf(lse_ref)
    assert np.array_equal(np.isneginf(lse_got), empty)
    assert np.all(f64(out)[empty] == 0)
    lse_tol = 2.0 ** -24 * terms * (1 + ref["zmax"])
    assert np.abs(lse_got[~empty] - lse_ref[~empty]).max(initial=0) <= lse_tol
    if backward:
        bounds = mo.gradient_bounds(ref, eps, n_terms(max(m, n * h // k.shape[1]), d), scale)
        for name, got in zip(("dq", "dk", "dv"), grads):
            diff = np.abs(f64(got) - ref[name])
            assert np.all(diff <= bounds[name]), f"{name}: {np.max(diff / bounds[name]):.2f} of the bound"
    return out, lse, grads


# (batch, heads, kv_heads, q_len, kv_len, causal, documents, prefix)
SHAPES = [
    (1, 1, 1, 1, 1, False, None, None),
    (2, 2, 1, 1, 77, True, None, None),
    (1, 3, 3, 64, 64, True, None, None),
    (2, 4, 2, 129, 129, True, None, [[40], [0]]),
    (1, 2, 2, 200, 200, False, [[0, 63, 64, 64, 150]], None),                     # a document of one token, an empty one, padding
    (2, 2, 1, 191, 191, True, [[0, 100, 191, 191], [5, 70, 70, 160]], [[10, 200, 3], [0, 4, 33]]),
    (1, 4, 1, 65, 333, True, [[0, 130, 290, 333]], None),                         # rows are the last of the positions
    (1, 2, 2, 90, 40, True, None, None),                                          # rows before position 0 see nothing
    (1, 2, 1, 300, 50, False, None, None),                                        # more rows than keys
    (1, 2, 2, 257, 511, True, None, [[300]]),
    (1, 1, 1, 130, 130, False, [[130, 130]], None),                               # nobody sees anything
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s[:6]))
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_against_oracle(lib, shape, dtype, d):
    b, h, kvh, n, m, causal, docs, prefix = shape
    q, k, v, dout = make(1, b, h, kvh, n, m, d, dtype, tokens_first=n % 2 == 1)
    check(lib, q, k, v, dout, causal, docs, prefix)


@pytest.mark.parametrize("softcap,bias", [(20.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_scores_capped_and_biased(lib, softcap, bias, dtype, d):
    q, k, v, dout = make(2, 1, 4, 2, 150, 211, d, dtype)
    slopes = [0.5, 0.25, 0.03, 0.0] if bias else None
    check(lib, q, k, v, dout, True, None, [[60]], softcap, slopes)
    check(lib, q, k, v, dout, False, [[0, 90, 211]], None, softcap, slopes)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_zero_keys(lib, dtype):
    q, k, v, dout = make(3, 2, 2, 1, 70, 0, 64, dtype)
    out, lse = lib.masked_attention(q, k, v, want_lse=True)
    dq, dk, dv = lib.masked_attention_backward(q, k, v, out, lse, dout)
    torch.cuda.synchronize()
    assert torch.count_nonzero(out) == 0 and torch.count_nonzero(dq) == 0
    assert torch.isneginf(lse).all()
    assert dk.shape == k.shape and dv.shape == v.shape


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("fp32", 64)])
def test_few_rows_and_many_keys_are_shared_out(lib, dtype, d):
    q, k, v, dout = make(4, 1, 2, 1, 3, 2500, d, dtype)
    assert lib.masked_attention_workspace_bytes(q, k, v, causal=True) > 0
    check(lib, q, k, v, dout, True, None, None)
    check(lib, q, k, v, dout, True, [[0, 2499, 2500]], None)      # rows that see one key, in the last part alone


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128)])
def test_what_is_masked_may_be_anything(lib, dtype, d):
    docs = [[0, 70, 90, 170]]
    n = 200
    q, k, v, dout = make(5, 1, 2, 2, n, n, d, dtype)
    for causal in (False, True):
        ref = check(lib, q, k, v, dout, causal, docs, None)
        q2, k2, v2, g2 = (x.clone() for x in (q, k, v, dout))
        for i, x in enumerate((q2, k2, v2, g2)):                   # padding behind the last document
            x[:, :, 170::3] = float("nan")
            x[:, :, 171::3] = float("inf")
            x[:, :, 172::3] = -torch.finfo(x.dtype).max
        args = dict(causal=causal, doc_offsets=ints(docs))
        out, lse = lib.masked_attention(q2, k2, v2, want_lse=True, **args)
        grads = lib.masked_attention_backward(q2, k2, v2, out, lse, g2, **args)
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
        for a, r in zip(grads, ref[2]):
            assert torch.equal(a, r)
        # a broken document leaves the others alone, in tiles that they share
        q3, k3, v3, g3 = (x.clone() for x in (q, k, v, dout))
        for x in (q3, k3, v3, g3):
            x[:, :, 75] = float("nan")
            x[:, :, 80] = float("inf")
        out, lse = lib.masked_attention(q3, k3, v3, want_lse=True, **args)
        grads = lib.masked_attention_backward(q3, k3, v3, out, lse, g3, **args)
        torch.cuda.synchronize()
        others = [i for i in range(n) if not 70 <= i < 90]
        assert torch.equal(out[:, :, others], ref[0][:, :, others]) and torch.equal(lse[:, :, others], ref[1][:, :, others])
        for a, r in zip(grads, ref[2]):
            assert torch.equal(a[:, :, others], r[:, :, others])
        assert not torch.isfinite(out[:, :, 80:90]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_value_of_infinity_reaches_the_rows_that_see_it(lib, dtype):
    q, k, v, dout = make(6, 1, 1, 1, 100, 100, 64, dtype)
    ref, _ = lib.masked_attention(q, k, v, causal=True)
    v2 = v.clone()
    v2[0, 0, 60, 3] = float("inf")
    v2[0, 0, 61, 40] = float("nan")
    out, _ = lib.masked_attention(q, k, v2, causal=True)
    torch.cuda.synchronize()
    assert torch.equal(out[:, :, :60], ref[:, :, :60])
    assert torch.isposinf(out[0, 0, 60:, 3]).all() and torch.isnan(out[0, 0, 61:, 40]).all()
    rest = [c for c in range(64) if c not in (3, 40)]
    assert torch.equal(out[0, 0, 60:][:, rest], ref[0, 0, 60:][:, rest])


def test_scores_of_any_size(lib):
    """Runaway maxima (each tile's scores above the last one's), and scores far below 0."""
    q, k, v, dout = make(7, 1, 2, 2, 300, 300, 128, "bf16")
    ramp = torch.linspace(0.1, 40.0, 300, device=DEV)[None, None, :, None]
    check(lib, q, (k.float() * ramp).to(k.dtype), v, dout, True, None, None, backward=False)
    check(lib, q, (k.float() * ramp.flip(2)).to(k.dtype), v, dout, False, None, None, backward=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_projections_and_broadcast_keys(lib, dtype):
    """q, k, v as views of one [batch, tokens, 3, heads, d] tensor; gradients into views of another; a k shared by the batch."""
    d, n, h = 64, 140, 2
    g = torch.Generator().manual_seed(8)
    qkv = torch.randn(2, n, 3, h, d, generator=g).to(DT[dtype]).to(DEV)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    dout = torch.randn(2, n, h, d, generator=g).to(DT[dtype]).to(DEV).transpose(1, 2)
    ref = check(lib, q, k, v, dout, True, None, None)
    grad = torch.full_like(qkv, 7.0)
    spare = torch.full((2, n, h + 1, d), 7.0, dtype=DT[dtype], device=DEV)
    out = spare[:, :, :h].transpose(1, 2)
    lib.masked_attention(q, k, v, causal=True, out=out)
    views = [grad[:, :, i].transpose(1, 2) for i in range(3)]
    lib.masked_attention_backward(q, k, v, ref[0], ref[1], dout, causal=True, dq=views[0], dk=views[1], dv=views[2])
    torch.cuda.synchronize()
    assert torch.equal(out, ref[0]) and (spare[:, :, h] == 7.0).all()
    for a, r in zip(views, ref[2]):
        assert torch.equal(a, r)
    one = k[:1].expand(2, h, n, d)
    check(lib, q, one, v, dout, True, None, None, backward=False)


def test_equal_calls_give_equal_bits(lib):
    q, k, v, dout = make(9, 1, 8, 2, 700, 700, 128, "bf16")
    runs = []
    for _ in range(3):
        out, lse = lib.masked_attention(q, k, v, causal=True, want_lse=True)
        runs.append((out, lse) + lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True))
    torch.cuda.synchronize()
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(r, runs[0]))


@pytest.mark.parametrize("softcap,bias", [(0.0, False), (4.0, True)])
def test_gradients_against_differences(lib, softcap, bias):
    """Central differences of the oracle's forward pass along random directions, fp32 kernels."""
    d, n = 64, 75
    q, k, v, dout = make(10, 1, 2, 1, n, n, d, "fp32", spread=1.0)
    slopes = np.array([0.1, 0.02]) if bias else None
    docs, prefix = [[0, 40, 70]], [[9, 0]]
    slo = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device=DEV)
    args = dict(causal=True, doc_offsets=ints(docs), prefix=ints(prefix), softcap=softcap, slopes=slo)
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args)
    grads = [f64(x) for x in lib.masked_attention_backward(q, k, v, out, lse, dout, **args)]
    torch.cuda.synchronize()
    see, scale = mo.visible(1, n, n, True, docs, prefix), lib.resolved_scale(d)
    base, G = [f64(x) for x in (q, k, v)], f64(dout)
    slo64 = None if slopes is None else slo.double().cpu().numpy()
    loss = lambda x: float((mo.attention(*x, see, scale, softcap, slo64)["out"] * G).sum())
    rng = np.random.default_rng(0)
    for which in range(3):
        for _ in range(3):
            u = rng.standard_normal(base[which].shape)
            step = 1e-4 / np.sqrt(u.size)
            plus, minus = ([x + (s * step * u if i == which else 0) for i, x in enumerate(base)] for s in (1, -1))
            diff = (loss(plus) - loss(minus)) / (2 * step)
            # fp32 sums of some thousand terms (2^-24 each); the differences' own error is of third order in the step
            tol = 2.0 ** -24 * 2000 * float((np.abs(grads[which]) * np.abs(u)).sum()) + 1e-6 * abs(diff)
            assert abs(diff - float((grads[which] * u).sum())) <= tol


def test_graph_replays_match_eager_calls(lib):
    q, k, v, dout = make(11, 1, 4, 2, 333, 333, 128, "bf16")
    docs = ints([[0, 200, 320]])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device=DEV)
    dq, dk, dv = (torch.empty_like(x) for x in (q, k, v))
    ws = torch.empty(max(lib.masked_attention_workspace_bytes(q, k, v, True, docs, backward=x) for x in (False, True)),
                     dtype=torch.uint8, device=DEV)

    def step():
        lib.masked_attention(q, k, v, causal=True, doc_offsets=docs, out=out, lse=lse, workspace=ws)
        lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True, doc_offsets=docs, dq=dq, dk=dk, dv=dv, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (20, 21, 22):
        for dst, src in zip((q, k, v, dout), make(seed, 1, 4, 2, 333, 333, 128, "bf16")):
            dst.copy_(src)
        step()
        torch.cuda.synchronize()
        eager = [x.clone() for x in (out, lse, dq, dk, dv)]
        for x in (out, lse, dq, dk, dv):
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, dq, dk, dv), eager))


def test_on_a_stream_of_its_own(lib):
    q, k, v, _ = make(12, 1, 4, 4, 500, 500, 128, "bf16")
    ref, _ = lib.masked_attention(q, k, v, causal=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out, _ = lib.masked_attention(q, k, v, causal=True)
    side.synchronize()
    assert torch.equal(out, ref)


def test_without_masks_as_dense_attention(lib):
    """The same function as dense_attention where nothing is masked (other kernels: bf16 weights rounded against other maxima)."""
    q, k, v, _ = make(13, 1, 3, 3, 700, 700, 128, "bf16")
    a, la = lib.masked_attention(q, k, v, want_lse=True)
    b, lb = lib.dense_attention(q, k, v, want_lse=True)
    torch.cuda.synchronize()
    ref = mo.attention(f64(q), f64(k), f64(v), mo.visible(1, 700, 700), lib.resolved_scale(128))
    bound = 2 * mo.forward_bounds(ref, 2.0 ** -7, n_terms(700, 128))
    assert np.all(np.abs(f64(a) - f64(b)) <= bound)
    assert (la - lb).abs().max() <= 2 * 2.0 ** -24 * n_terms(700, 128) * (1 + ref["zmax"])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_seen_key_of_infinity_keeps_its_weight_of_zero(lib, dtype):
    """A key whose infinite channel makes its score -inf for the rows that see it has weight 0 there, in tiles that are masked
    in part as elsewhere: out, dk, dv and the finite channels of dq are those of a mask without it, its channel of dq is NaN
    (0 * inf) for the rows that see it and finite for the others."""
    n, key, ch = 100, 30, 7
    q, k, v, dout = make(30, 1, 2, 2, n, n, 128, dtype)
    q[..., ch] = -q[..., ch].abs() - 0.5
    k[0, 0, key, ch] = float("inf")
    out, lse = lib.masked_attention(q, k, v, causal=True, want_lse=True)
    dq, dk, dv = lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True)
    torch.cuda.synchronize()
    see = mo.visible(1, n, n, True)
    see[:, :, key] = False
    q, k, v, dout, out, dq, dk, dv = (x[:, :1] for x in (q, k, v, dout, out, dq, dk, dv))
    scale = lib.resolved_scale(128)
    ref = mo.attention(f64(q), f64(k), f64(v), see, scale, dout=f64(dout))
    eps = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    assert np.all(np.abs(f64(out) - ref["out"]) <= mo.forward_bounds(ref, eps, n_terms(n, 128)))
    bounds = mo.gradient_bounds(ref, eps, n_terms(n, 128), scale)
    assert torch.isnan(dq[0, 0, key:, ch]).all()
    dq[0, 0, key:, ch] = torch.from_numpy(ref["dq"][0, 0, key:, ch]).to(dq)
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        assert np.all(np.abs(f64(got) - ref[name]) <= bounds[name]), name


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
@pytest.mark.parametrize("seed", range(6))
def test_drawn_calls(lib, seed, dtype, d):
    """Sizes, masks, caps, slopes and orders drawn by seed."""
    rng = np.random.default_rng([seed, d, dtype == "fp32"])
    b, kvh, group = int(rng.integers(1, 3)), int(rng.integers(1, 4)), int(rng.integers(1, 5))
    n = int(rng.integers(1, 400))
    m = n if rng.random() < 0.5 else int(rng.integers(1, 700))
    causal = bool(rng.random() < 0.6)
    docs = prefix = None
    if rng.random() < 0.7:                       # borders that leave padding before and behind, and may repeat
        docs = [sorted(int(x) for x in rng.integers(0, m + 1, int(rng.integers(2, 9)))) for _ in range(b)]
        docs = [x[:min(len(y) for y in docs)] for x in docs]
    if causal and rng.random() < 0.6:            # below 0 and past the end as well
        prefix = [[int(x) for x in rng.integers(-20, m + 50, 1 if docs is None else len(docs[0]) - 1)] for _ in range(b)]
    softcap = float(rng.choice([0.0, 0.0, 8.0, 30.0]))
    slopes = [float(x) for x in rng.random(kvh * group)] if rng.random() < 0.3 else None
    print(b, kvh, group, n, m, causal, docs, prefix, softcap, slopes, flush=True)
    q, k, v, dout = make(seed, b, kvh * group, kvh, n, m, d, dtype, tokens_first=bool(rng.random() < 0.5))
    check(lib, q, k, v, dout, causal, docs, prefix, softcap, slopes)


@pytest.mark.parametrize("dtype,softcap", [("bf16", 1e-3), ("bf16", 0.3), ("bf16", 1e6), ("fp32", 1e-3), ("fp32", 1e6)])
def test_caps_of_any_size(lib, dtype, softcap):
    # gradients for the large one only: 1 - tanh^2 of a capped score rounds to 0 or 2^-24, which has no relative bound
    q, k, v, dout = make(31, 1, 2, 1, 140, 140, 64, dtype)
    check(lib, q, k, v, dout, True, None, None, softcap, backward=softcap > 1)


def test_heads_that_do_not_divide_by_the_xcds(lib):
    q, k, v, dout = make(32, 1, 13, 13, 700, 700, 64, "bf16")
    check(lib, q, k, v, dout, True, None, None)


def test_more_documents_than_a_workgroup_keeps(lib):
    rng = np.random.default_rng(33)
    docs = [sorted(int(x) for x in rng.integers(0, 1501, 701)) for _ in range(2)]
    q, k, v, dout = make(33, 2, 2, 1, 1500, 1500, 64, "bf16")
    check(lib, q, k, v, dout, True, docs, [[int(x) for x in rng.integers(0, 4, 700)] for _ in range(2)])


def test_more_tiles_than_are_ranked(lib):
    """33 000 rows in documents; each document is a problem of its own, and three are compared."""
    n, d = 33000, 64
    borders = list(range(0, n, 977)) + [n]
    q, k, v, dout = make(34, 1, 1, 1, n, n, d, "bf16")
    args = dict(causal=True, doc_offsets=ints([borders]))
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args)
    grads = lib.masked_attention_backward(q, k, v, out, lse, dout, **args)
    torch.cuda.synchronize()
    scale, terms = lib.resolved_scale(d), n_terms(977, d)
    for c in (0, len(borders) // 2, len(borders) - 2):
        part = slice(borders[c], borders[c + 1])
        size = borders[c + 1] - borders[c]
        one = lambda x: f64(x[:, :, part])
        ref = mo.attention(one(q), one(k), one(v), mo.visible(1, size, size, True), scale, dout=one(dout))
        assert np.all(np.abs(one(out) - ref["out"]) <= mo.forward_bounds(ref, 2.0 ** -7, terms))
        bounds = mo.gradient_bounds(ref, 2.0 ** -7, terms, scale)
        for name, got in zip(("dq", "dk", "dv"), grads):
            assert np.all(np.abs(one(got) - ref[name]) <= bounds[name]), name


def test_tensors_past_4_gib(lib):
    """Rows a MiB apart: offsets past 32 bits, the same bits as of dense tensors."""
    n, d, apart = 4500, 128, 1 << 19
    q, k, v, dout = make(35, 1, 2, 1, n, n, d, "bf16")
    far = torch.empty(n, apart, dtype=torch.bfloat16, device=DEV)
    slot = iter(range(0, apart, d))

    def spread(heads, src=None):
        at = [next(slot) for _ in range(heads)][0]
        t = far[:, at:at + heads * d].view(n, heads, d).transpose(0, 1)[None]
        return t if src is None else t.copy_(src)
    fq, fk, fv, fg = spread(2, q), spread(1, k), spread(1, v), spread(2, dout)
    out, lse = lib.masked_attention(q, k, v, causal=True, want_lse=True)
    grads = lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True)
    fout, flse = lib.masked_attention(fq, fk, fv, causal=True, out=spread(2), want_lse=True)
    fgrads = lib.masked_attention_backward(fq, fk, fv, fout, flse, fg, causal=True, dq=spread(2), dk=spread(1), dv=spread(1))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((out, lse, *grads), (fout, flse, *fgrads)))


def test_one_row_for_all_heads(lib):
    """Inputs expanded over batch and heads (strides of 0), with a single row as well."""
    for n in (1, 70):
        q, k, v, dout = make(36, 1, 1, 1, n, 90, 128, "bf16")
        wide = [x.expand(2, 3, -1, -1) for x in (q, k, v, dout)]
        dense = [x.contiguous() for x in wide]
        out, lse = lib.masked_attention(*wide[:3], causal=True, want_lse=True)
        ref, lse_ref = lib.masked_attention(*dense[:3], causal=True, want_lse=True)
        got = lib.masked_attention_backward(*wide[:3], out, lse, wide[3], causal=True)
        want = lib.masked_attention_backward(*dense[:3], ref, lse_ref, dense[3], causal=True)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((out, lse, *got), (ref, lse_ref, *want)))


def test_two_graphs_with_one_workspace(lib):
    """Replayed one after the other, in turn; and two calls at once, with a workspace each."""
    calls = []
    for seed, (h, n, m, dtype) in ((40, (2, 3, 2500, "bf16")), (41, (3, 300, 300, "fp32"))):
        q, k, v, dout = make(seed, 1, h, 1, n, m, 64, dtype)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device=DEV)
        calls.append((q, k, v, dout, out, lse, *(torch.empty_like(x) for x in (q, k, v))))
    need = max(lib.masked_attention_workspace_bytes(*c[:3], causal=True, backward=x) for c in calls for x in (False, True))
    shared = torch.empty(need, dtype=torch.uint8, device=DEV)

    def step(c, ws):
        q, k, v, dout, out, lse, dq, dk, dv = c
        lib.masked_attention(q, k, v, causal=True, out=out, lse=lse, workspace=ws)
        lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True, dq=dq, dk=dk, dv=dv, workspace=ws)
    for c in calls:
        step(c, shared)
    torch.cuda.synchronize()
    want = [[x.clone() for x in c[4:]] for c in calls]
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(c, shared)
        graphs.append(g)
    for _ in range(3):
        for c, g in zip(calls, graphs):
            for x in c[4:]:
                x.fill_(float("nan"))
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for c, w in zip(calls, want) for a, b in zip(c[4:], w))
    streams = [torch.cuda.Stream() for _ in calls]
    for c in calls:
        for x in c[4:]:
            x.fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(calls, streams):
            with torch.cuda.stream(s):
                step(c, None)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for c, w in zip(calls, want) for a, b in zip(c[4:], w))


def test_more_documents_than_30_bits_count(lib):
    """Empty documents without end ahead of two that hold tokens: the search for a row's document passes 2^30 of them."""
    n = 130
    q, k, v, dout = make(50, 1, 2, 1, n, n, 64, "bf16")
    short = ints([[0, 70, n]])
    borders = torch.zeros(1, (1 << 30) + 100, dtype=torch.int32, device=DEV)
    borders[0, -3:] = short[0]

    def step(docs):
        out, lse = lib.masked_attention(q, k, v, causal=True, doc_offsets=docs, want_lse=True)
        return (out, lse, *lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True, doc_offsets=docs))
    want, got = step(short), step(borders)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def alike(got, want, bound):
    """Finite where the other is, within the bound; else the same infinity or NaN."""
    fin = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isfinite(got), fin)
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)])
    assert np.all(np.abs(got[fin] - want[fin]) <= bound[fin])


BORDERS = [(True, None, None), (True, [[0, 70, 90, 170]], None), (False, [[0, 100, 190]], None), (True, None, [[30]])]


@pytest.mark.parametrize("mask", BORDERS, ids=str)
@pytest.mark.parametrize("softcap", [0.0, 4.0])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_a_broken_row_of_dout_reaches_the_keys_that_it_sees(lib, dtype, d, softcap, mask):
    """Infinities and NaN in dout, in tiles that a workgroup's keys see in part and as a whole: dv takes each in its own channel,
    dk of the keys that such rows see is not finite, and nothing else changes."""
    causal, docs, prefix = mask
    n = 200
    q, k, v, dout = make(51, 1, 4, 2, n, n, d, dtype)
    clean, rows = dout.clone(), {20: float("nan"), 75: float("-inf"), 100: float("nan"), 101: float("inf"), 150: float("inf")}
    for i, (row, x) in enumerate(rows.items()):
        dout[0, i % 4, row, 5 + 9 * i], clean[0, i % 4, row, 5 + 9 * i] = x, 0.0
    args = dict(causal=causal, doc_offsets=ints(docs), prefix=ints(prefix), softcap=softcap)
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args)
    dq, dk, dv = (f64(x) for x in lib.masked_attention_backward(q, k, v, out, lse, dout, **args))
    torch.cuda.synchronize()
    see, scale = mo.visible(1, n, n, causal, docs, prefix), lib.resolved_scale(d)
    ref = mo.attention(f64(q), f64(k), f64(v), see, scale, softcap, dout=f64(clean))
    bounds = mo.gradient_bounds(ref, 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23, n_terms(2 * n, d), scale)
    for i, (row, x) in enumerate(rows.items()):                    # weights are positive: these rows see keys of finite scores
        head, seen = i % 4, see[0, row]
        ref["dv"][0, head // 2, seen, 5 + 9 * i] += x
        ref["dk"][0, head // 2, seen] = np.nan
        ref["dq"][0, head, row] = np.nan if seen.any() else 0.0
    alike(dv, ref["dv"], bounds["dv"])
    for got, name in ((dq, "dq"), (dk, "dk")):                     # inf - inf, or inf: which one is a matter of order
        alike(np.where(np.isfinite(got), got, np.nan), ref[name], bounds[name])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128)])
def test_a_value_of_infinity_leaves_dv_alone(lib, dtype, d):
    """dv is made of weights and dout; what an infinite value makes of out and delta is not in it.  An infinite query of capped
    scores (all of them the cap, slope 0) is NaN in its channel of dk."""
    n = 150
    q, k, v, dout = make(52, 1, 2, 1, n, n, d, dtype)
    ref = mo.attention(f64(q), f64(k), f64(v), mo.visible(1, n, n, True), lib.resolved_scale(d), dout=f64(dout))
    bounds = mo.gradient_bounds(ref, 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23, n_terms(2 * n, d), lib.resolved_scale(d))
    v[0, 0, 60, 3] = float("inf")
    out, lse = lib.masked_attention(q, k, v, causal=True, want_lse=True)
    dv = lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True)[2]
    torch.cuda.synchronize()
    alike(f64(dv), ref["dv"], bounds["dv"])
    q, k, v, dout = make(53, 1, 2, 1, n, n, d, dtype)
    k += torch.where(k >= 0, 0.25, -0.25).to(k.dtype)               # no score of 0 * inf
    big = q.clone()
    q[0, 1, 70, 9], big[0, 1, 70, 9] = float("inf"), 1e30            # the same capped scores
    got, want = [], []
    for x, res in ((q, got), (big, want)):
        out, lse = lib.masked_attention(x, k, v, causal=True, softcap=5.0, want_lse=True)
        res += [out, lse, *lib.masked_attention_backward(x, k, v, out, lse, dout, causal=True, softcap=5.0)]
    torch.cuda.synchronize()
    assert torch.isnan(got[3][0, 0, :71, 9]).all() and torch.isfinite(want[3]).all()
    got[3][0, 0, :71, 9] = want[3][0, 0, :71, 9]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n,m,docs,heads", [(100, 100, None, 2), (100, 1000, [[0, 920, 1000]], 2), (300, 300, [[0, 20, 300]], 300)], ids=str)
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_rows_of_scores_of_minus_infinity_alone(lib, dtype, d, bias, n, m, docs, heads):
    """Keys masked by a channel of the type's lowest value, whose scores overflow to -inf: rows that see no other key have out 0,
    lse -inf and no part in the gradients, however their keys are shared out; for the others such keys are not there."""
    q, k, v, dout = make(54, 1, heads, 1, n, m, d, dtype)
    last = docs[0][1] if docs else 10                              # the keys before it
    q[..., 4], k[..., 4] = 2.0, 0.5
    k[:, :, :last, 4] = torch.finfo(k.dtype).min
    slopes = torch.linspace(0.0, 0.5, heads, device=DEV) if bias else None
    args = dict(causal=docs is None, doc_offsets=ints(docs), slopes=slopes)
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args)
    grads = lib.masked_attention_backward(q, k, v, out, lse, dout, **args)
    torch.cuda.synchronize()
    see = mo.visible(1, n, m, docs is None, docs)
    see[:, :, :last] = False
    empty = ~see[0].any(1)
    assert empty.any() and not empty.all()
    assert torch.isneginf(lse[:, :, empty]).all() and torch.count_nonzero(out[:, :, empty]) == 0
    pick = slice(0, 2) if heads > 2 else slice(None)               # of many heads, out and dq of two are compared
    scale, slo = lib.resolved_scale(d), None if slopes is None else slopes.double().cpu().numpy()[pick]
    ref = mo.attention(f64(q)[:, pick], f64(k), f64(v), see, scale, 0.0, slo, f64(dout)[:, pick])
    eps = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
    assert np.all(np.abs(f64(out)[:, pick] - ref["out"]) <= mo.forward_bounds(ref, eps, n_terms(m, d)))
    bounds = mo.gradient_bounds(ref, eps, n_terms(max(m, 2 * n), d), scale)
    for name, got in zip(("dq", "dk", "dv"), grads):
        got = f64(got)
        if name == "dq":
            assert np.all(got[:, :, empty] == 0) and np.all(np.abs(got[:, pick] - ref[name]) <= bounds[name])
        elif heads == 2:
            assert np.all(np.abs(got - ref[name]) <= bounds[name]), name
        else:
            assert np.isfinite(got).all() and np.all(got[:, :, :last] == 0)


@pytest.mark.parametrize("heads,n,m", [(8, 1024, 20000), (1, 1, 20000), (64, 1024, 5000)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_values_under_scores_that_rise(lib, dtype, heads, n, m):
    """Values near 2^102 under scores that pass the first tile's maximum by as much as it may be stale, in every later tile or for a
    while: sums of weighted values stay in range, in one walk as in parts."""
    g = torch.Generator().manual_seed(55)
    k = torch.zeros(1, 1, m, 64)
    v = (2.0 ** 101 * (1 + torch.rand(1, 1, m, 64, generator=g))).to(DT[dtype])
    q = torch.zeros(1, heads, n, 64)
    q[..., 0] = 1.0
    for rise in (slice(64, None), slice(64, 2000), slice(1000, None, 3)):
        k.zero_()
        k[0, 0, rise, 0] = 104.5                                   # 2^18.8 times the first keys' weight, 32 keys to a lane and tile
        qd, kd, vd = (x.to(DT[dtype]).to(DEV) for x in (q, k, v))
        out, lse = lib.masked_attention(qd, kd, vd, want_lse=True)
        torch.cuda.synchronize()
        ref = mo.attention(f64(qd)[:, :1, :1], f64(kd), f64(vd), np.ones((1, 1, m), bool), lib.resolved_scale(64))
        eps = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -23
        bound = mo.forward_bounds(ref, eps, n_terms(m, 64))
        assert np.all(np.abs(f64(out) - ref["out"]) <= bound)
        assert np.abs(f64(lse) - ref["lse"]).max() <= 2.0 ** -24 * n_terms(m, 64) * (1 + ref["zmax"])


@pytest.mark.parametrize("softcap,bias", [(0.0, False), (0.0, True), (30.0, False), (6.0, False), (30.0, True)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 64)])
def test_a_row_does_not_hang_on_what_its_neighbours_hold(lib, dtype, d, softcap, bias):
    """Queries of NaN, of infinity, and fifty times as long: the other rows' results keep their bits, and so do the gradients of the
    keys that only others see."""
    n, m = 200, 700
    q, k, v, dout = make(56, 1, 2, 1, n, m, d, dtype)
    args = dict(causal=True, softcap=softcap, slopes=torch.tensor([0.05, 0.01], device=DEV) if bias else None)

    def step(x):
        out, lse = lib.masked_attention(x, k, v, want_lse=True, **args)
        return (out, lse, *lib.masked_attention_backward(x, k, v, out, lse, dout, **args))
    want = step(q)
    for row in (0, 45, 130):
        for change in (lambda x: float("nan"), lambda x: float("inf"), lambda x: 50 * x):
            broken = q.clone()
            broken[:, :, row] = change(q[:, :, row])
            got = step(broken)
            torch.cuda.synchronize()
            rows, first = [i for i in range(n) if i != row], row + m - n + 1
            for a, b in zip(got[:3], want[:3]):
                assert torch.equal(a[:, :, rows], b[:, :, rows])
            for a, b in zip(got[3:], want[3:]):
                assert torch.equal(a[:, :, first:], b[:, :, first:])


def seen_product(p, x, see):
    """p [i, j] x [j, c] over the seen pairs alone, where x may hold infinities and NaN (p is 0 where nothing is seen)."""
    r = p @ np.where(np.isfinite(x), x, 0.0)
    for j, c in zip(*np.nonzero(~np.isfinite(x))):
        r[:, c] = np.where(see[:, j], r[:, c] + p[:, j] * x[j, c], r[:, c])
    return r


def by_formula(q, k, v, g, see, scale, softcap, slopes):
    """out, lse, dq, dk, dv of one batch element, heads by heads, with inf and NaN as 64-bit arithmetic has them."""
    (h, n, d), (kvh, m) = q.shape, k.shape[:2]
    far = np.abs(np.arange(n)[:, None] + m - n - np.arange(m)[None, :])
    res = {"out": np.zeros_like(q), "lse": np.full((h, n), -np.inf), "dq": np.zeros_like(q), "dk": np.zeros_like(k), "dv": np.zeros_like(v)}
    for j in range(h):
        e = j // (h // kvh)
        s = (q[j][:, None] * k[e][None]).sum(-1) * scale
        t = np.tanh(s / softcap) if softcap else s
        z = (softcap * t if softcap else s) - (slopes[j] * far if slopes is not None else 0.0)
        z = np.where(see, z, -np.inf)
        top = z.max(1, keepdims=True) if m else np.full((n, 1), -np.inf)
        w = np.where(see, np.exp(z - np.where(np.isneginf(top), 0.0, top)), 0.0)
        total = w.sum(1, keepdims=True)
        some = total[:, 0] != 0                                    # rows with a score above -inf (or NaN)
        pair = see & some[:, None]
        p = np.where(pair, w / np.where(total == 0, 1.0, total), 0.0)
        res["lse"][j, some] = (top + np.log(total))[some, 0]
        res["out"][j, some] = seen_product(p, v[e], pair)[some]
        dp = (g[j][:, None] * v[e][None]).sum(-1)
        dz = p * (dp - (g[j] * res["out"][j]).sum(1, keepdims=True)) * (1 - t * t if softcap else 1.0)
        dz = np.where(pair, dz, 0.0)
        res["dq"][j, some] = scale * seen_product(dz, k[e], pair)[some]
        res["dk"][e] += scale * seen_product(dz.T, q[j], pair.T)
        res["dv"][e] += seen_product(p.T, g[j], pair.T)
    return res


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
@pytest.mark.parametrize("seed", range(8))
def test_drawn_calls_with_broken_elements(lib, seed, dtype, d):
    """An infinity or NaN somewhere in q, k, v or dout: what is finite by the formula is so and has its value, and what is not
    finite by the formula is not finite."""
    rng = np.random.default_rng([seed, d, dtype == "fp32", 1])
    kvh, group, n = int(rng.integers(1, 3)), int(rng.integers(1, 3)), int(rng.integers(2, 200))
    m = n if rng.random() < 0.5 else int(rng.integers(2, 300))
    causal = bool(rng.random() < 0.6)
    docs = [sorted(int(x) for x in rng.integers(0, m + 1, int(rng.integers(2, 6))))] if rng.random() < 0.6 else None
    prefix = [[int(x) for x in rng.integers(0, m + 9, len(docs[0]) - 1 if docs else 1)]] if causal and rng.random() < 0.5 else None
    softcap = float(rng.choice([0.0, 0.0, 8.0, 30.0]))
    slopes = rng.random(kvh * group).astype(np.float32) * np.float32(0.1) if rng.random() < 0.3 else None
    q, k, v, dout = tensors = make(seed, 1, kvh * group, kvh, n, m, d, dtype)
    for x in tensors:
        if rng.random() < 0.5:
            x[0, int(rng.integers(x.shape[1])), int(rng.integers(x.shape[2])), int(rng.integers(d))] = float(rng.choice([np.inf, -np.inf, np.nan]))
    args = dict(causal=causal, doc_offsets=ints(docs), prefix=ints(prefix), softcap=softcap,
                slopes=None if slopes is None else torch.from_numpy(slopes).to(DEV))
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args)
    got = dict(zip(("out", "lse", "dq", "dk", "dv"), (out, lse, *lib.masked_attention_backward(q, k, v, out, lse, dout, **args))))
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        want = by_formula(*(f64(x)[0] for x in tensors), mo.visible(1, n, m, causal, docs, prefix)[0], lib.resolved_scale(d), softcap, slopes)
    for name, x in got.items():
        x, r = f64(x)[0], want[name]
        fin = np.isfinite(r)
        assert np.array_equal(np.isfinite(x), fin), name
        # norms: far above the roundings and far below what a lost row is worth; `rest` is for results that cancel to nothing
        share, rest = (1e-2, 2.0 ** -6) if dtype == "bf16" else (1e-4, 2.0 ** -16)
        assert np.linalg.norm(x[fin] - r[fin]) <= share * np.linalg.norm(r[fin]) + rest * np.sqrt(fin.sum()), name
