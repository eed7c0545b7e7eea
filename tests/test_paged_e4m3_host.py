"""Pages of 8 bits without a GPU: what the calls refuse, and the float64 definition of the format against values worked out by hand."""
import numpy as np
import pytest
import torch

import paper_2603_11564_amd as D
from oracle import dapq_oracle as O
from oracle import paged_oracle as PO
from test_paged_host import A, ERR_INVALID, ERR_UNSUPPORTED, At, append, attention, gather, pages, read, step


def e4m3(**kw):
    return pages(**dict(dict(format="e4m3", k_scales=A, v_scales=A), **kw))


@pytest.mark.parametrize("bad,code,message", [
    (dict(k_scales=None), ERR_INVALID, "E4M3 pages need k_scales and v_scales"), (dict(v_scales=None), ERR_INVALID, "E4M3 pages need"),
    (dict(k_scales=At(4)), ERR_UNSUPPORTED, "16-byte aligned"), (dict(v_scales=At(8)), ERR_UNSUPPORTED, "16-byte aligned"),
    (dict(v=At(8)), ERR_UNSUPPORTED, "16-byte aligned"), (dict(page_rows=24), ERR_UNSUPPORTED, r"page_rows \(24\)"),
    (dict(raw=dict(format=4)), ERR_INVALID, r"format \(4\)")])
def test_bad_pages_are_refused_by_every_call(bad, code, message):
    for call in (append, read, attention, lambda p: gather(p=p)):
        with pytest.raises(D.DapqError, match=message) as e:
            call(e4m3(**bad))
        assert e.value.code == code
    assert D.paged_attention_workspace_bytes(e4m3(**bad), step()) == 0


def test_workspace_bytes_depend_on_no_device_data():
    for p in (e4m3(), e4m3(batch=64, max_pages=1 << 16), e4m3(n_layers=8, n_kv_heads=8)):
        for s in (step(total_new=p.batch), step(total_new=64 * p.batch, max_new=64), step(total_new=5, max_new=5, cu_new=A)):
            s.lengths = 1 << 60
            p.table = 1 << 60
            n = D.paged_attention_workspace_bytes(p, s)
            assert n > 0 and n % 256 == 0


# --- the definition ---------------------------------------------------------------------------------------------------------
def group(*values):
    x = np.zeros(128)
    x[:len(values)] = values
    codes, scales = PO.e4m3_quantise(x)
    return PO.e4m3_values(codes, scales)[:len(values)].tolist(), int(scales[0])


def test_groups_by_hand():
    assert PO.E4M3_LEVELS[[0, 1, 7, 8, 15, 16, 126]].tolist() == [0.0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 15 * 2.0 ** -9, 2.0 ** -5, 448.0]
    assert group(448.0, 17.0, 19.0, -21.0, 1.0625, 1.1875) == ([448.0, 16.0, 20.0, -20.0, 1.0, 1.25], 127)           # ties: the even code
    assert group(464.0, 300.0) == ([448.0, 288.0], 127)                                                              # 464 is still 448; 300 lies above 288 by 12, below 320 by 20
    assert group(465.0, 300.0) == ([480.0, 288.0], 128)                                                              # halves: 232.5 -> 240, 150 -> 144 (by 6; 160 is off by 10)
    assert group(2.0 ** -9 * 464, 2.0 ** -18 * 1.5, 2.0 ** -19)[0] == [448 * 2.0 ** -9, 2.0 ** -17, 0.0]             # halves of the least level: to the even code
    assert group(0.0, 0.0) == ([0.0, 0.0], 10)
    assert group(2.0 ** -130, 2.0 ** -126) == ([0.0, 2.0 ** -126], 10)
    assert group(3.3e38, -3.38e38, 1.0) == ([448.0 * 2.0 ** 119, -448.0 * 2.0 ** 119, 0.0], 246)
    assert PO.e4m3_quantise(np.array([np.nan] + [1.0] * 127))[1].tolist() == [255, 119, 119, 119]                    # 232/256 < 1 <= 464/256
    codes, _ = PO.e4m3_quantise(np.arange(128) * 0.0 + [1.0, -1.0] * 64)
    assert codes[0] == 0x78 and codes[1] == 0xF8                                                                     # 256 * 2^-8


def test_loses_at_most_half_a_step():
    """2^-4 of a value (half a step of four bits), 2^-10 of the unit below 2^-6 of it; and the values are bf16 numbers as they are."""
    x = O.bf16_bits_to_f64(O.f64_to_bf16_bits(np.random.default_rng(0).standard_normal((300, 128)) * 3))
    codes, scales = PO.e4m3_quantise(x)
    back = PO.e4m3_values(codes, scales)
    unit = np.repeat(2.0 ** (scales.astype(float) - 127), 32, -1)
    assert (np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit)).all()
    assert (np.abs(x).reshape(300, 4, 32).max(-1) > 232 * 2.0 ** (scales.astype(float) - 127)).all()
    assert np.array_equal(O.bf16_bits_to_f64(O.f64_to_bf16_bits(back)), back)


def test_codes_agree_with_torch():
    """The levels are torch's e4m3."""
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    ours = PO.e4m3_values(np.arange(256).reshape(2, 128), np.full((2, 4), 127)).reshape(-1)
    assert np.array_equal(ours, t, equal_nan=True)
