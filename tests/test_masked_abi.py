"""What masked and paged attention refuse, before any device work; and the oracle they are tested against.  No GPU needed."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2602_01077_amd as pisa
from oracle import masked_oracle as mo

FAKE = 0x1000                    # never dereferenced: validation fails first
ODD = FAKE + 8
HUGE = 1 << 50
NONE = pisa.PisaStrides(0, 0, 0)


def masked(**kw):
    d = dict(batch=2, heads=4, kv_heads=2, q_len=100, kv_len=300, head_dim=128, dtype=pisa.PISA_BF16, causal=1, num_docs=0,
             scale=0.0, softcap=0.0, q=NONE, k=NONE, v=NONE, out=NONE)
    d.update(kw)
    return pisa.PisaMaskedShape(*(d[n] for n, _ in pisa.PisaMaskedShape._fields_))


def paged(**kw):
    d = dict(seqs=3, heads=8, kv_heads=2, head_dim=128, dtype=pisa.PISA_BF16, page_size=16, num_pages=100, max_pages=20,
             scale=0.0, softcap=0.0, k_pages=NONE, v_pages=NONE)
    d.update(kw)
    return pisa.PisaPagedShape(*(d[n] for n, _ in pisa.PisaPagedShape._fields_))


def forward(s, q=FAKE, k=FAKE, v=FAKE, docs=None, prefix=None, slopes=None, out=FAKE, lse=FAKE, ws=FAKE, size=HUGE):
    return pisa.raw().pisa_masked_attention(s, q, k, v, docs, prefix, slopes, out, lse, ws, size, None)


def backward(s, strides=None, q=FAKE, k=FAKE, v=FAKE, out=FAKE, lse=FAKE, dout=FAKE, docs=None, prefix=None, slopes=None,
             dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, size=HUGE):
    return pisa.raw().pisa_masked_attention_backward(s, strides, q, k, v, out, lse, dout, docs, prefix, slopes, dq, dk, dv, ws,
                                                     size, None)


def decode(s, q=FAKE, k=FAKE, v=FAKE, table=FAKE, lengths=FAKE, slopes=None, out=FAKE, lse=FAKE, ws=FAKE, size=HUGE):
    return pisa.raw().pisa_paged_attention(s, q, k, v, table, lengths, slopes, out, lse, ws, size, None)


def append(s, k=FAKE, v=FAKE, tokens=3, offsets=FAKE, kp=FAKE, vp=FAKE, table=FAKE, lengths=FAKE):
    return pisa.raw().pisa_paged_append(s, k, v, tokens, offsets, kp, vp, table, lengths, None)


S = pisa.PisaStrides
BAD, NOT_BUILT, SMALL = pisa.PISA_INVALID_ARG, pisa.PISA_UNSUPPORTED, pisa.PISA_WORKSPACE_TOO_SMALL


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), BAD), (dict(q_len=0), BAD), (dict(kv_len=-1), BAD), (dict(heads=5), BAD), (dict(kv_heads=0), BAD),
    (dict(head_dim=96), BAD), (dict(dtype=2), BAD), (dict(causal=2), BAD), (dict(num_docs=-1), BAD),
    (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(softcap=-1.0), BAD), (dict(softcap=float("nan")), BAD),
    (dict(softcap=float("inf")), BAD), (dict(q_len=(1 << 24) + 1), NOT_BUILT), (dict(kv_len=(1 << 24) + 1), NOT_BUILT),
    (dict(batch=40000), NOT_BUILT),
    (dict(q=S(-8, 128, 128)), BAD), (dict(k=S(76800, 38400, 64)), BAD), (dict(v=S(76800, 38400, 132)), BAD),
    (dict(k=S(0, 38400, 1 << 24)), NOT_BUILT), (dict(q=S(1 << 40, 0, 128)), NOT_BUILT),
    (dict(out=S(0, 12800, 128)), BAD), (dict(out=S(51200, 12800 - 128, 128)), BAD),
])
def test_shapes_that_masked_attention_refuses(kw, code):
    s = masked(**kw)
    assert forward(s) == code and pisa.last_error() != ""
    assert backward(s) == code
    assert pisa.raw().pisa_masked_attention_workspace_bytes(s) == 0
    assert pisa.raw().pisa_masked_attention_backward_workspace_bytes(s) == 0


def test_arguments_that_masked_attention_refuses():
    s = masked(kv_len=3000)
    assert forward(None) == BAD
    for name in ("q", "k", "v", "out"):
        assert forward(s, **{name: None}) == BAD
    for name in ("q", "k", "v", "out", "lse", "ws", "slopes", "prefix"):
        assert forward(s, **{name: ODD}) == BAD and "aligned" in pisa.last_error()
    for name in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"):
        assert backward(s, **{name: None}) == BAD
        assert backward(s, **{name: ODD}) == BAD and "aligned" in pisa.last_error()
    assert forward(s, docs=FAKE) == BAD and forward(masked(num_docs=2)) == BAD
    assert forward(masked(causal=0), prefix=FAKE) == BAD and "prefix" in pisa.last_error()
    for size, call in ((pisa.raw().pisa_masked_attention_workspace_bytes(s), forward),
                       (pisa.raw().pisa_masked_attention_backward_workspace_bytes(s), backward)):
        assert size > 0                      # 2 x 4 heads of one tile of rows: their keys are shared out; delta
        assert call(s, size=size - 1) == SMALL
        assert call(s, ws=None, size=0) == BAD
    ok = S(51200, 12800, 128)
    kv = S(768000, 384000, 128)
    assert backward(s, pisa.PisaGradStrides(S(0, 0, 128), ok, S(0, 384000, 128), kv)) == BAD and "dk" in pisa.last_error()
    assert backward(s, pisa.PisaGradStrides(ok, ok, kv, S(768000, 384000, 100))) == BAD and "dv" in pisa.last_error()


@pytest.mark.parametrize("kw,code", [
    (dict(seqs=0), BAD), (dict(heads=7), BAD), (dict(kv_heads=0), BAD), (dict(head_dim=32), BAD), (dict(dtype=3), BAD),
    (dict(page_size=0), BAD), (dict(page_size=65537), BAD), (dict(num_pages=0), BAD), (dict(max_pages=0), BAD),
    (dict(scale=float("nan")), BAD), (dict(softcap=-0.5), BAD), (dict(max_pages=1 << 27), NOT_BUILT),
    (dict(seqs=1 << 22), NOT_BUILT), (dict(k_pages=S(4096, 128, 100)), BAD), (dict(v_pages=S(4096, 0, 256)), BAD),
    (dict(v_pages=S(4096, 128, 252)), BAD),
])
def test_shapes_that_the_paged_calls_refuse(kw, code):
    s = paged(**kw)
    assert decode(s) == code and pisa.last_error() != ""
    assert append(s) == code
    assert pisa.raw().pisa_paged_attention_workspace_bytes(s) == 0


def test_arguments_that_the_paged_calls_refuse():
    s = paged()
    assert decode(None) == BAD and append(None) == BAD
    for name in ("q", "k", "v", "table", "lengths", "out"):
        assert decode(s, **{name: None}) == BAD
        assert decode(s, **{name: ODD}) == BAD and "aligned" in pisa.last_error()
    for name in ("lse", "slopes", "ws"):
        assert decode(s, **{name: ODD}) == BAD
    for name in ("k", "v", "offsets", "kp", "vp", "table", "lengths"):
        assert append(s, **{name: None}) == BAD
        assert append(s, **{name: ODD}) == BAD and "aligned" in pisa.last_error()
    assert append(s, tokens=-1) == BAD
    size = pisa.raw().pisa_paged_attention_workspace_bytes(s)
    assert size > 0 and decode(s, size=size - 1) == SMALL and decode(s, ws=None, size=0) == BAD


def test_the_binding_refuses_what_does_not_fit():
    q = torch.zeros(1, 2, 8, 64)
    with pytest.raises(ValueError):
        pisa.masked_attention(q, q, q)                                     # on the host
    with pytest.raises(ValueError):
        pisa.masked_attention(q, q[:, :, :4], q)                           # k and v unlike
    with pytest.raises(TypeError):
        pisa.masked_attention(q, q.bfloat16(), q)
    with pytest.raises(ValueError):
        pisa.masked_attention(q.transpose(2, 3), q, q)
    with pytest.raises(ValueError):
        pisa.masked_attention(q, q, q, out=torch.zeros(1, 2, 8, 128)[..., ::2])
    with pytest.raises(ValueError):
        pisa.masked_attention(q, q, q, doc_offsets=torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        pisa.masked_attention_backward(q, q, q, q, q[..., 0], q[:, :, :4])
    pages = torch.zeros(4, 16, 2, 64)
    with pytest.raises(ValueError):
        pisa.paged_attention(torch.zeros(2, 64), pages, pages, torch.zeros(2, 3), torch.zeros(2))
    with pytest.raises(TypeError):
        pisa.paged_attention(torch.zeros(2, 4, 64).bfloat16(), pages, pages, torch.zeros(2, 3), torch.zeros(2))
    with pytest.raises(ValueError):
        pisa.paged_append(pages[0], pages[0], torch.zeros(3), pages, pages, torch.zeros(2, 3), torch.zeros(2))


def test_the_structures_are_laid_out_as_in_the_header():
    assert ctypes.sizeof(pisa.PisaStrides) == 24
    assert pisa.PisaMaskedShape.q.offset == 48 and ctypes.sizeof(pisa.PisaMaskedShape) == 48 + 4 * 24
    assert pisa.PisaPagedShape.k_pages.offset == 40 and ctypes.sizeof(pisa.PisaPagedShape) == 40 + 2 * 24


def test_oracle_masks_by_hand():
    see = mo.visible(1, 5, 7, True, [[0, 4, 7]], [[2, 0]])[0].astype(int)
    assert see.tolist() == [[1, 1, 1, 0, 0, 0, 0], [1, 1, 1, 1, 0, 0, 0], [0, 0, 0, 0, 1, 0, 0], [0, 0, 0, 0, 1, 1, 0],
                            [0, 0, 0, 0, 1, 1, 1]]
    assert mo.visible(1, 3, 3, True, None, [[2]])[0].astype(int).tolist() == [[1, 1, 0], [1, 1, 0], [1, 1, 1]]
    assert mo.visible(1, 3, 2, True)[0].astype(int).tolist() == [[0, 0], [1, 0], [1, 1]]


def test_oracle_gradients_against_differences():
    rng = np.random.default_rng(0)
    q, k, v, g = (rng.standard_normal((1, h, n, 8)) for h, n in ((4, 6), (2, 9), (2, 9), (4, 6)))
    see = mo.visible(1, 6, 9, True, [[0, 5, 9]], [[2, 0]])
    slopes = np.array([0.3, 0.1, 0.0, 0.05])
    r = mo.attention(q, k, v, see, 0.4, 2.0, slopes, g)
    loss = lambda x: float((mo.attention(*x, see, 0.4, 2.0, slopes)["out"] * g).sum())
    for which, name in enumerate(("dq", "dk", "dv")):
        u = rng.standard_normal((q, k, v)[which].shape)
        up, down = ([x + (s * 1e-6 * u if i == which else 0) for i, x in enumerate((q, k, v))] for s in (1, -1))
        assert abs((loss(up) - loss(down)) / 2e-6 - float((r[name] * u).sum())) < 1e-7


@pytest.mark.parametrize("kw", [dict(softcap=2.0 ** -70), dict(softcap=2.0 ** 70), dict(softcap=1.0, scale=2.0 ** 100),
                                dict(softcap=1.0, scale=2.0 ** -100)])
def test_caps_whose_quotients_leave_the_range_are_refused(kw):
    assert forward(masked(**kw)) == NOT_BUILT and "softcap" in pisa.last_error()
    assert backward(masked(**kw)) == NOT_BUILT
    assert decode(paged(**kw)) == NOT_BUILT and "softcap" in pisa.last_error()


def test_launches_past_2_to_the_32_threads_are_refused():
    dense = S(0, 0, 0)
    big = dict(batch=1, heads=65535, kv_heads=1, q_len=128 * 256 + 1, kv_len=1, q=dense, k=dense, v=dense, out=dense)
    assert forward(masked(**big)) == NOT_BUILT and "too large" in pisa.last_error()
    s = paged()
    rows = s.kv_heads * s.head_dim
    assert append(s, tokens=(1 << 32) // rows) == NOT_BUILT
    assert decode(paged(seqs=(1 << 24) // s.heads)) == NOT_BUILT
    assert decode(paged(num_pages=(1 << 31) - 1, k_pages=S(1 << 39, 128, 256))) == NOT_BUILT


@pytest.mark.parametrize("which", ["q", "k", "v", "out", "dout"])
def test_one_row_for_all_tokens_is_refused(which):
    """Expanded over batch, heads and tokens all strides are 0, which the library reads as dense: far past the one row that is there."""
    t = {x: torch.zeros(2, 3, 70, 64) for x in ("q", "k", "v", "out", "dout")}
    t[which] = torch.zeros(1, 1, 1, 64).expand(2, 3, 70, 64)
    with pytest.raises(ValueError, match=f"{which}: one row"):
        if which != "dout":
            pisa.masked_attention(t["q"], t["k"], t["v"], out=t["out"])
        pisa.masked_attention_backward(t["q"], t["k"], t["v"], t["out"], torch.zeros(2, 3, 70), t["dout"])


def test_one_slot_for_a_whole_page_is_refused():
    table, lengths = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pages, one = torch.zeros(4, 16, 2, 64), torch.zeros(1, 1, 1, 64).expand(4, 16, 2, 64)
    for k, v, name in ((one, pages, "k_pages"), (pages, one, "v_pages")):
        with pytest.raises(ValueError, match=f"{name}: one row"):
            pisa.paged_attention(torch.zeros(2, 4, 64), k, v, table, lengths)
        with pytest.raises(ValueError, match=f"{name}: one row"):
            pisa.paged_append(torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32), k, v, table, lengths)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_workspaces_of_expanded_tensors(dtype):
    """A tensor that stands for all batch elements and heads needs the workspace of a dense one, in either memory order."""
    one = lambda n: torch.zeros(1, 1, n, 128, dtype=dtype)
    for b, h, n, m in ((2, 4, 3, 9000), (2, 4, 1, 700), (1, 24, 700, 700)):
        q, k, v = (one(x).expand(b, h, x, 128) for x in (n, m, m))
        for backward in (False, True):
            want = pisa.masked_attention_workspace_bytes(*(x.contiguous() for x in (q, k, v)), causal=True, backward=backward)
            assert pisa.masked_attention_workspace_bytes(q, k, v, causal=True, backward=backward) == want
        assert want > 0
        first = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)
        assert pisa.masked_attention_workspace_bytes(first(q), k, v, causal=True, backward=True) == want


def test_workspaces_of_refused_shapes_raise():
    q = torch.zeros(1, 5, 8, 64)
    with pytest.raises(pisa.PisaError, match="kv_heads") as e:
        pisa.masked_attention_workspace_bytes(q, q[:, :2], q[:, :2])
    assert e.value.code == BAD
    with pytest.raises(pisa.PisaError) as e:
        pisa.masked_attention_workspace_bytes(torch.zeros(1, 1, 8, 96), torch.zeros(1, 1, 8, 96), torch.zeros(1, 1, 8, 96))
    assert e.value.code == BAD
    wide = torch.zeros(1, 1, 1, 64).expand(70000, 1, 1, 64)
    with pytest.raises(pisa.PisaError, match="65535") as e:
        pisa.masked_attention_workspace_bytes(wide, wide, wide)
    assert e.value.code == NOT_BUILT
    pages, table = torch.zeros(4, 16, 2, 64), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(pisa.PisaError, match="kv_heads"):
        pisa.paged_attention_workspace_bytes(torch.zeros(2, 5, 64), pages, pages, table)
    assert pisa.paged_attention_workspace_bytes(torch.zeros(2, 4, 64), pages, pages, table) > 0
