"""How far masked and paged attention are from 64 bits, over whole outputs: bounds element by element have to allow for every
rounding going the same way, and would let a lost mantissa bit or a missing correction through; norms do not.

Norms of differences relative to the result's.  bf16: weights (or dz) are rounded to the type before the second product and the
result is rounded once, two roundings of equal and independent size, so sqrt(2) = 1.41 times what rounding the exact result
alone costs.  delta's mend leaves the part that weights below 0.1 have: of a unit of variance beside those two at most a tenth,
1.46.  Limit: 1.6.  fp32: a score is a sum of d products and a row one of m weights, roundings of 2^-24 that go either way, seen
through an exponential: sqrt(m + d) 2^-24 (1 + size of the scores that have weight, which lie at the row's log-sum-exp)."""
import numpy as np
import pytest
import torch

from oracle import masked_oracle as mo

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
TIMES = 1.6


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def rounded(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def off(a, b):
    return np.linalg.norm(a - b) / np.linalg.norm(b)


def limit(ref, dtype, m, d, lse):
    if dtype == "bf16":
        return TIMES * off(rounded(ref), ref)
    return 2.0 ** -24 * np.sqrt(m + d) * (1 + np.abs(lse[np.isfinite(lse)]).max())


def make(seed, h, kvh, n, m, d, dtype, spread):
    g = torch.Generator().manual_seed(seed)
    one = lambda heads, length, s=1.0: (s * torch.randn(1, heads, length, d, generator=g)).to(DT[dtype]).to(DEV)
    return one(h, n, spread), one(kvh, m), one(kvh, m), one(h, n)


# (heads, key heads, rows, keys, causal, documents, cap, slopes, spread of the queries)
CALLS = [
    (4, 2, 300, 300, True, None, 0.0, False, 1.5),
    (4, 4, 257, 257, False, [[0, 100, 240]], 0.0, False, 1.5),
    (4, 2, 200, 200, True, None, 0.0, False, 4.0),
    (2, 1, 200, 333, True, None, 20.0, False, 4.0),
    (4, 2, 200, 200, True, None, 0.0, True, 2.0),
    (2, 2, 65, 1500, True, None, 30.0, True, 1.5),
    (2, 2, 300, 300, True, None, 0.0, False, 40.0),
]


@pytest.mark.parametrize("call", CALLS, ids=str)
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_norms_of_errors(lib, call, dtype, d):
    h, kvh, n, m, causal, docs, softcap, bias, spread = call
    q, k, v, dout = make(1, h, kvh, n, m, d, dtype, spread)
    slopes = torch.linspace(0.02, 0.3, h, device=DEV) if bias else None
    args = dict(causal=causal, softcap=softcap, slopes=slopes,
                doc_offsets=None if docs is None else torch.tensor(docs, dtype=torch.int32, device=DEV))
    out, lse = lib.masked_attention(q, k, v, want_lse=True, **args)
    got = dict(zip(("out", "dq", "dk", "dv"), (out, *lib.masked_attention_backward(q, k, v, out, lse, dout, **args))))
    torch.cuda.synchronize()
    ref = mo.attention(*(f64(x) for x in (q, k, v)), mo.visible(1, n, m, causal, docs), lib.resolved_scale(d), softcap,
                       None if slopes is None else f64(slopes), f64(dout))
    for name, x in got.items():
        e, most = off(f64(x), ref[name]), limit(ref[name], dtype, m, d, ref["lse"])
        print(name, f"{e:.2e} of {most:.2e}")
        assert e <= most, name


@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("n,d", [(200, 128), (200, 64), (333, 128)])
def test_what_a_rounded_out_costs_the_gradients_is_mended(lib, n, d, softcap):
    """Rows whose weight lies on few keys: dq and dk are closer to 64 bits than those made with delta from the rounded out, which
    are made here with no other rounding than the kernels' own."""
    q, k, v, dout = make(2, 2, 2, n, n, d, "bf16", 4.0)
    out, lse = lib.masked_attention(q, k, v, causal=True, softcap=softcap, want_lse=True)
    got = [f64(x) for x in lib.masked_attention_backward(q, k, v, out, lse, dout, causal=True, softcap=softcap)]
    torch.cuda.synchronize()
    see, scale = mo.visible(1, n, n, True), lib.resolved_scale(d)
    Q, K, V, G = (f64(x) for x in (q, k, v, dout))
    ref = mo.attention(Q, K, V, see, scale, softcap, dout=G)
    plain = [np.zeros_like(ref[x]) for x in ("dq", "dk")]
    for j in range(2):
        z, gain = mo.scores(Q[0, j], K[0, j], scale, softcap)
        p, _ = mo.softmax_rows(z, see[0])
        assert np.sum(p >= 0.1) > n                                # heavy keys, in most rows
        delta = (G[0, j] * rounded(ref["out"][0, j])).sum(1, keepdims=True)
        ds = rounded(p * (G[0, j] @ V[0, j].T - delta) * gain)
        plain[0][0, j], plain[1][0, j] = rounded(scale * (ds @ K[0, j])), rounded(scale * (ds.T @ Q[0, j]))
    for name, x, unmended in zip(("dq", "dk"), got, plain):
        e, without = off(x, ref[name]), off(unmended, ref[name])
        print(name, f"{e:.2e}, not mended {without:.2e}")
        assert e <= 0.85 * without and e <= TIMES * off(rounded(ref[name]), ref[name]), name


@pytest.mark.parametrize("softcap,bias", [(0.0, False), (15.0, True)])
@pytest.mark.parametrize("heads,kvh", [(4, 2), (20, 1)])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("fp32", 128), ("fp32", 64)])
def test_norms_of_errors_over_a_cache(lib, dtype, d, heads, kvh, softcap, bias):
    lengths, page = [700, 33, 200], 16
    g = torch.Generator().manual_seed(3)
    one = lambda *s: torch.randn(*s, generator=g).to(DT[dtype])
    used = [-(-n // page) for n in lengths]
    kp, vp = (one(sum(used), page, kvh, d) for _ in range(2))
    table = torch.zeros(3, max(used), dtype=torch.int32)
    order, at = torch.randperm(sum(used), generator=g).to(torch.int32), 0
    for s, u in enumerate(used):
        table[s, :u] = order[at:at + u]
        at += u
    q = (2 * torch.randn(3, heads, d, generator=g)).to(DT[dtype])
    slopes = torch.linspace(0.01, 0.2, heads) if bias else None
    out, _ = lib.paged_attention(q.to(DEV), kp.to(DEV), vp.to(DEV), table.to(DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV),
                                 softcap=softcap, slopes=None if slopes is None else slopes.to(DEV))
    ref, lse = np.zeros((3, heads, d)), []
    for s, n in enumerate(lengths):
        k, v = (x[table[s, :used[s]].long()].reshape(-1, kvh, d)[:n].double().numpy().transpose(1, 0, 2)[None] for x in (kp, vp))
        r = mo.attention(q[s].double().numpy()[None, :, None], k, v, np.ones((1, 1, n), bool), lib.resolved_scale(d), softcap,
                         None if slopes is None else slopes.double().numpy())
        ref[s] = r["out"][0, :, 0]
        lse.append(r["lse"].ravel())
    assert off(f64(out), ref) <= limit(ref, dtype, max(lengths), d, np.concatenate(lse))
