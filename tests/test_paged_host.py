"""The calls of the cache in pages without a GPU: what they refuse before anything is enqueued, and their float64 definition
against values worked out by hand."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2603_11564_amd as D
from oracle import dapq_oracle as O
from oracle import paged_oracle as PO
from paper_2603_11564_amd import binding

T = torch.empty(1 << 12, dtype=torch.uint8)     # (never dereferenced: every call fails before)
BASE = (T.data_ptr() + 255) // 256 * 256
N = None
ERR_INVALID, ERR_UNSUPPORTED, ERR_WORKSPACE = -1, -2, -3


class At:
    """A tensor at an address."""

    def __init__(self, offset=0, size=1 << 30):
        self.address, self.size = BASE + offset, size

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.size

    def element_size(self):
        return 1


A = At()


def pages(**kw):
    a = dict(n_layers=1, batch=2, n_kv_heads=4, page_rows=16, n_pages=8, max_pages=4, format="bf16", k=A, v=A, table=A)
    raw = kw.pop("raw", {})
    a.update(kw)
    p = D.make_pages(**a)
    for name, value in raw.items():
        setattr(p, name, value)
    return p


def fp4(**kw):
    return pages(**dict(dict(format="fp4", k_scales=A, v_scales=A), **kw))


def step(**kw):
    a = dict(n_q_heads=8, total_new=2, max_new=1, lengths=A, k_strides=(0, 512, 128), v_strides=(0, 512, 128), q_strides=(0, 1024, 128), scale=0.1)
    a.update(kw)
    return D.make_step(**a)


def shape(**kw):
    a = dict(n_layers=1, batch=2, n_q_heads=8, n_kv_heads=4, n_pseudo=4, total_tokens=64, k_strides=(8192, 0, 0, 128), v_strides=(8192, 0, 0, 128),
             scale=0.1)
    a.update(kw)
    return D.make_shape(**a)


def gather(s=None, p=None, k=A, v=A, idx=A, count=A, budget=8):
    D.dapq_paged_gather(s or shape(), p or pages(), k, v, idx, count, budget, 0)


def append(p=None, s=None, k=A, v=A, positions=A, theta=5e5, pairing=0):
    D.dapq_paged_append(p or pages(), s or step(), k, v, positions, theta, pairing, 0)


def read(p=None, lengths=A, rows=8, k=A, v=A):
    D.dapq_paged_read(p or pages(), lengths, rows, k, v, 0)


def attention(p=None, s=None, q=A, out=A, work=A):
    D.dapq_paged_attention(p or pages(), s or step(), q, out, work, 0)


BAD_PAGES = [
    (dict(n_layers=0), ERR_INVALID, r"n_layers \(0\)"), (dict(batch=0), ERR_INVALID, r"batch \(0\)"),
    (dict(n_kv_heads=-1), ERR_INVALID, r"n_kv_heads \(-1\)"), (dict(n_pages=0), ERR_INVALID, r"n_pages \(0\)"),
    (dict(max_pages=0), ERR_INVALID, r"max_pages \(0\)"), (dict(head_dim=64), ERR_UNSUPPORTED, "head_dim 64"),
    (dict(raw=dict(format=2)), ERR_INVALID, r"format \(2\)"), (dict(raw=dict(format=-1)), ERR_INVALID, r"format \(-1\)"),
    (dict(page_rows=8), ERR_UNSUPPORTED, r"page_rows \(8\)"), (dict(page_rows=48), ERR_UNSUPPORTED, r"page_rows \(48\)"),
    (dict(page_rows=2048), ERR_UNSUPPORTED, r"page_rows \(2048\)"), (dict(page_rows=0), ERR_UNSUPPORTED, r"page_rows \(0\)"),
    (dict(page_rows=1024, max_pages=1 << 20), ERR_UNSUPPORTED, "2\\^30"), (dict(k=N), ERR_INVALID, "k, v and table"),
    (dict(v=N), ERR_INVALID, "k, v and table"), (dict(table=N), ERR_INVALID, "k, v and table"),
    (dict(k=At(8)), ERR_UNSUPPORTED, "16-byte aligned"), (dict(format="fp4"), ERR_INVALID, "k_scales and v_scales"),
    (dict(format="fp4", k_scales=A, v_scales=At(4)), ERR_UNSUPPORTED, "16-byte aligned"),
    (dict(n_layers=70000, n_kv_heads=1, batch=1), ERR_UNSUPPORTED, "exceeds 65535"),
    (dict(n_layers=1000, n_kv_heads=50, batch=1000), ERR_UNSUPPORTED, "2\\^24"),
]


@pytest.mark.parametrize("bad,code,message", BAD_PAGES, ids=[str(i) for i in range(len(BAD_PAGES))])
def test_bad_pages_are_refused_by_every_call(bad, code, message):
    for call in (append, read, attention, lambda p: gather(p=p)):
        with pytest.raises(D.DapqError, match=message) as e:
            call(pages(**bad))
        assert e.value.code == code
    assert D.paged_attention_workspace_bytes(pages(**bad), step()) == 0


REFUSED = [
    (lambda: gather(s=shape(batch=1)), ERR_INVALID, "differ"), (lambda: gather(s=shape(n_kv_heads=8)), ERR_INVALID, "differ"),
    (lambda: gather(s=shape(n_layers=2)), ERR_INVALID, "differ"), (lambda: gather(s=shape(head_dim=64)), ERR_UNSUPPORTED, "head_dim"),
    (lambda: gather(k=N), ERR_INVALID, "must not be NULL"), (lambda: gather(v=N), ERR_INVALID, "must not be NULL"),
    (lambda: gather(idx=N), ERR_INVALID, "must not be NULL"), (lambda: gather(count=N), ERR_INVALID, "must not be NULL"),
    (lambda: gather(budget=0), ERR_INVALID, r"budget \(0\)"), (lambda: gather(k=At(2)), ERR_UNSUPPORTED, "aligned"),
    (lambda: gather(s=shape(k_strides=(0, 0, 0, 4))), ERR_UNSUPPORTED, "k strides"),
    (lambda: gather(s=shape(batch=70000, total_tokens=140000), p=pages(batch=70000)), ERR_UNSUPPORTED, "65535"),
    (lambda: append(k=N), ERR_INVALID, "k_new"), (lambda: append(v=N), ERR_INVALID, "v_new"), (lambda: append(v=At(8)), ERR_UNSUPPORTED, "aligned"),
    (lambda: append(pairing=2), ERR_INVALID, "pairing"), (lambda: append(theta=0.0), ERR_INVALID, "theta"),
    (lambda: append(theta=float("nan")), ERR_INVALID, "theta"), (lambda: append(s=step(lengths=N)), ERR_INVALID, "lengths"),
    (lambda: append(s=step(k_strides=(0, 64, 128))), ERR_UNSUPPORTED, "k strides"),
    (lambda: append(s=step(k_strides=(0, 512, -128))), ERR_UNSUPPORTED, "k strides"),
    (lambda: append(s=step(v_strides=(4, 512, 128))), ERR_UNSUPPORTED, "v strides"),
    (lambda: append(s=step(n_q_heads=6)), ERR_INVALID, r"n_q_heads \(6\)"), (lambda: append(s=step(n_q_heads=0)), ERR_INVALID, r"n_q_heads \(0\)"),
    (lambda: append(s=step(total_new=3)), ERR_INVALID, "multiple of batch"), (lambda: append(s=step(total_new=-2)), ERR_INVALID, "negative"),
    (lambda: append(s=step(max_new=-1)), ERR_INVALID, "negative"), (lambda: append(s=step(total_new=(1 << 25) + 2)), ERR_UNSUPPORTED, "2\\^25"),
    (lambda: read(lengths=N), ERR_INVALID, "lengths"), (lambda: read(k=N), ERR_INVALID, "k_out"), (lambda: read(v=N), ERR_INVALID, "v_out"),
    (lambda: read(rows=0), ERR_INVALID, r"max_rows \(0\)"), (lambda: read(k=At(8)), ERR_UNSUPPORTED, "aligned"),
    (lambda: read(p=pages(batch=70000)), ERR_UNSUPPORTED, "65535"),
    (lambda: read(p=pages(page_rows=1024, max_pages=(1 << 20) - 1), rows=1 << 30), ERR_UNSUPPORTED, "too large"),
    (lambda: attention(q=N), ERR_INVALID, "q and out"), (lambda: attention(out=N), ERR_INVALID, "q and out"),
    (lambda: attention(work=N), ERR_INVALID, "workspace is NULL"), (lambda: attention(work=At(16)), ERR_UNSUPPORTED, "256-byte"),
    (lambda: attention(work=At(0, 128)), ERR_WORKSPACE, "workspace has 128 bytes"), (lambda: attention(q=At(8)), ERR_UNSUPPORTED, "16-byte"),
    (lambda: attention(out=At(8)), ERR_UNSUPPORTED, "16-byte"), (lambda: attention(s=step(scale=0.0)), ERR_INVALID, "scale"),
    (lambda: attention(s=step(scale=float("inf"))), ERR_INVALID, "scale"), (lambda: attention(s=step(softcap=-1.0)), ERR_INVALID, "softcap"),
    (lambda: attention(s=step(softcap=float("nan"))), ERR_INVALID, "softcap"),
    (lambda: attention(s=step(q_strides=(0, 1024, 4))), ERR_UNSUPPORTED, "q strides"), (lambda: attention(s=step(lengths=N)), ERR_INVALID, "lengths"),
]


@pytest.mark.parametrize("call,code,message", REFUSED, ids=[str(i) for i in range(len(REFUSED))])
def test_refusals(call, code, message):
    with pytest.raises(D.DapqError, match=message) as e:
        call()
    assert e.value.code == code


@pytest.mark.parametrize("scale,softcap,message", [(2.0 ** 127, 0.0, "exceeds"), (1.0, 3e38, "exceeds"), (0.1, 1e36, "must be from"), (1.0, 1e-40, "must be from"),
                                                   (2.0 ** -80, 2.0 ** 31, "must be from"), (2.0 ** 100, 2.0 ** -11, "must be from")])
def test_scales_and_caps_without_a_usable_factor_are_refused(scale, softcap, message):
    with pytest.raises(D.DapqError, match=message) as e:
        attention(s=step(scale=scale, softcap=softcap))
    assert e.value.code == ERR_UNSUPPORTED
    assert D.paged_attention_workspace_bytes(pages(), step(scale=scale, softcap=softcap)) == 0


def test_nothing_to_do_is_no_error():
    """No new tokens: nothing is enqueued (there is no GPU here), whatever the buffers."""
    for s in (step(total_new=0), step(max_new=0), step(total_new=0, cu_new=A)):
        append(s=s)
        attention(s=s)


def test_descriptors_have_the_header_s_layout():
    assert C.sizeof(binding.Pages) == 8 * 4 + 5 * 8 and C.sizeof(binding.Step) == 2 * 4 + 8 + 2 * 8 + 9 * 8 + 2 * 4
    for bad in (lambda: D.dapq_paged_read(step(), A, 8, A, A, 0), lambda: D.dapq_paged_append(pages(), pages(), A, A, A, 5e5, 0, 0),
                lambda: D.dapq_paged_gather(pages(), shape(), A, A, A, A, 8, 0), lambda: D.dapq_paged_attention(pages(), shape(), A, A, A, 0)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(D.DapqError, match=r"max_rows \(-8\)"):   # (a number that only ctypes converts)
        D.dapq_paged_read(pages(), A, C.c_int32(-8), A, A, 0)
    with pytest.raises(KeyError):
        pages(format="fp8")


def test_workspace_bytes_depend_on_no_device_data():
    """The figure is the same whatever table, lengths and cu_new hold: their addresses are not followed (here they are no memory)."""
    for p in (pages(), fp4(), pages(batch=64, max_pages=1 << 16), fp4(n_layers=8, n_kv_heads=8)):
        for s in (step(total_new=p.batch), step(total_new=64 * p.batch, max_new=64), step(total_new=5, max_new=5, cu_new=A)):
            s.lengths = 1 << 60
            p.table = 1 << 60
            n = D.paged_attention_workspace_bytes(p, s)
            assert n > 0 and n % 256 == 0


def test_workspace_bytes_follow_the_tokens_that_there_can_be():
    """max_new is a bound: without cu_new, and where it is more than all tokens, what is left of it counts."""
    p = fp4(batch=4, max_pages=1000)
    for cu in (N, A):
        few, more = (D.paged_attention_workspace_bytes(p, step(total_new=4, max_new=m, cu_new=cu)) for m in (4 if cu else 1, 1 << 30))
        assert few == more > 256
    assert D.paged_attention_workspace_bytes(p, step(total_new=0, max_new=0)) > 0


# --- the definition ---------------------------------------------------------------------------------------------------------
def group(*values):
    x = np.zeros(128)
    x[:len(values)] = values
    codes, scales = PO.fp4_quantise(x)
    return PO.fp4_values(codes, scales)[:len(values)].tolist(), int(scales[0])


def test_fp4_groups_by_hand():
    assert group(6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0) == ([6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0], 127)      # ties: the even code
    assert group(7.0, 0.3, -0.3, -6.5) == ([6.0, 0.5, -0.5, -6.0], 127)                                              # 7 is still 6
    assert group(7.03125, 0.4) == ([8.0, 0.0], 128)                                                                  # 7.03 / 2 rounds to 4
    assert group(3.5, 3.25) == ([3.0, 3.0], 126)                                                                     # 7 and 6.5 halves
    assert group(0.0, 0.0) == ([0.0, 0.0], 2)
    assert group(2.0 ** -130, 0.0) == ([0.0, 0.0], 2) and group(2.0 ** -126, 0.0)[0] == [2.0 ** -126, 0.0]
    assert group(3.3e38, 1.0) == ([6.0 * 2.0 ** 125, 0.0], 252)
    assert PO.fp4_quantise(np.array([np.inf] + [1.0] * 127))[1].tolist() == [255, 125, 125, 125]  # 7/8 < 1 <= 7/4
    codes, scales = PO.fp4_quantise(np.arange(128) * 0.0 + [1.0, -1.0] * 64)
    assert codes[0] == 0x6 | (0xE << 4) and scales[0] == 125                                                        # low half: even channel


def test_fp4_loses_at_most_half_a_step():
    x = O.bf16_bits_to_f64(O.f64_to_bf16_bits(np.random.default_rng(0).standard_normal((300, 128)) * 3))
    codes, scales = PO.fp4_quantise(x)
    back = PO.fp4_values(codes, scales)
    two = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    y = np.abs(x) / two
    half_step = np.where(y < 2, 0.25, np.where(y < 4, 0.5, 1.0))
    assert (np.abs(back - x) <= half_step * two).all() and (np.abs(x).reshape(300, 4, 32).max(-1) > 3.5 * 2.0 ** (scales.astype(float) - 127)).all()


def test_attention_by_hand():
    """Two rows with logits 0 and ln 3: weights 1/4 and 3/4; capped at 1 the second logit is tanh(ln 3) = 0.8."""
    pool = {"k": np.zeros((1, 1, 1, 16, 128), np.uint16), "v": np.zeros((1, 1, 1, 16, 128), np.uint16)}
    pool["k"][0, 0, 0, 1, 0] = O.f64_to_bf16_bits(np.array([1.0]))[0]
    pool["v"][0, 0, 0, 0, 0] = O.f64_to_bf16_bits(np.array([4.0]))[0]
    q = np.zeros((1, 2, 1, 128))
    q[0, :, 0, 0] = np.log(3.0)
    table = np.array([[0]], dtype=np.int32)
    out, _, _ = PO.attention(pool, table, [0], [0, 2], q, 1.0)
    assert np.allclose(out[0, :, 0, 0], [4.0, 1.0]) and not out[..., 1:].any()
    out, _, _ = PO.attention(pool, table, [0], [0, 2], q, 1.0, 1.0)
    assert np.isclose(out[0, 1, 0, 0], 4.0 / (1.0 + np.exp(0.8)))
    assert not PO.attention(pool, table - 1, [0], [0, 2], q, 1.0)[0].any()
