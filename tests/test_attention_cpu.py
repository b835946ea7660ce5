"""Host side of the attention entry points: the table of rotary positions against its definition, and what the C entry points
refuse before anything is launched."""
import ctypes

import numpy as np
import pytest

from oracle import attention_oracle as A
from paper_2509_01229_amd import api


@pytest.mark.parametrize("scaling", [None, "linear", "ntk", "yarn"])
@pytest.mark.parametrize("rot,base", [(128, 10000.0), (64, 500000.0), (16, 10000.0)])
def test_rope_table(scaling, rot, base):
    got = api.attn_rope_table(700, rot, base, scaling, 4.0, 2048)
    want = A.rope_table(700, rot, base, scaling, 4.0, 2048)
    # FP64 angles to within 2^-52 * 700, one rounding to FP32 (below 1.2: half a unit is 2^-24)
    assert got.dtype == np.float32 and got.shape == want.shape and np.abs(got - want).max() <= 2.0 ** -24 + 1e-12
    if scaling:
        assert np.abs(want - A.rope_table(700, rot, base)).max() > 0.1


def test_rope_table_refusals():
    for bad in [dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=2048), dict(max_positions=0), dict(base=1.0), dict(base=float("nan")),
                dict(scaling="linear", factor=0.5), dict(scaling="ntk", factor=float("inf")), dict(scaling="yarn", factor=2.0)]:
        with pytest.raises(api.LiquidGemmError):
            api.attn_rope_table(**{"max_positions": 4, "rot_dim": 64, **bad})
    with pytest.raises(ValueError):
        api.attn_rope_table(4, 64, scaling="other")


def test_page_bytes():
    L = api.lib()
    assert L.kv4_page_bytes(16, 8, 128) == 8 * 16 * 136 and L.kv4_page_bytes(256, 1, 64) == 256 * 72
    for bad in [(8, 1, 128), (24, 1, 128), (512, 1, 128), (16, 0, 128), (16, 1, 96), (-16, 1, 64), (16, 5000, 64)]:
        assert L.kv4_page_bytes(*bad) == 0


P = ctypes.c_void_p(1 << 20)    # an address that is aligned and never followed
ODD = ctypes.c_void_p((1 << 20) + 8)


def _refused(f, good, changes, code):
    for i, x in changes.items():
        for value in x if isinstance(x, tuple) else (x,):
            args = list(good)
            args[i] = value
            assert f(*args) == code, (f.__name__, i, value)
            assert api.lib().w4a8_last_error()


def test_c_entries_refuse_what_they_cannot_run():
    L, bad, align = api.lib(), api.LQ_ERR_INVALID, api.LQ_ERR_ALIGN
    rope = [0, 4, 8, 2, 128, P, 1280, 128, P, 1280, 128, P, P, 100, 128, 0, P, P, 1e-6, P, 1024, 128, P, 256, 128, None]
    _refused(L.attn_qk_norm_rope, rope, {0: (2, -1), 1: (-1, 2 ** 25), 2: (0, 5000), 3: 0, 4: (96, 0, 256), 5: None, 8: None, 11: None, 12: None,
                                         13: 0, 14: (0, 8, 24, 144, -16), 18: (0.0, -1.0, float("nan"), float("inf")), 19: None, 22: None}, bad)
    _refused(L.attn_qk_norm_rope, rope, {5: ODD, 6: 1284, 7: 132, 8: ODD, 9: 4, 12: ODD, 16: ODD, 17: ODD, 19: ODD, 22: ODD, 23: 252}, align)
    write = [0, 4, 2, 128, P, 256, 128, P, 256, 128, P, P, 10, 16, None]
    _refused(L.kv4_write, write, {0: 7, 1: -1, 2: 0, 3: 80, 4: None, 7: None, 10: None, 11: None, 12: (0, -1, 2 ** 30), 13: (8, 48, 512)}, bad)
    _refused(L.kv4_write, write, {4: ODD, 5: 257, 6: 4, 7: ODD, 11: ODD, 10: ctypes.c_void_p((1 << 20) + 2)}, align)
    append = [0, 4, 8, 2, 128, P, 1536, 128, P, 1536, 128, P, 1536, 128, P, P, 100, 128, 0, None, None, 0.0, P, 1024, 128, P, P, 10, 16, None]
    _refused(L.kv4_append, append, {0: 2, 4: 32, 5: None, 8: None, 11: None, 14: None, 15: None, 16: 0, 17: 40, 19: P, 22: None, 25: None, 26: None,
                                    27: 0, 28: 17}, bad)
    _refused(L.kv4_append, append, {5: ODD, 8: ODD, 11: ODD, 12: 1540, 22: ODD, 26: ODD}, align)
    read = [0, 4, 2, 128, P, 10, 16, P, P, P, None]
    _refused(L.kv4_read, read, {0: 3, 1: -2, 3: 100, 4: None, 5: 0, 6: 20, 7: None, 8: None, 9: None}, bad)
    _refused(L.kv4_read, read, {4: ODD, 8: ODD, 9: ODD}, align)
    decode = [0, 4, 1, 8, 2, 128, P, 1024, 1024, 128, P, 10, 16, P, 5, P, 0.1, P, None, 0, None]
    _refused(L.kv4_attention, decode, {0: 9, 1: -1, 2: (0, 2 ** 30), 3: (7, 0), 4: (0, 3), 5: 32, 6: None, 10: None, 11: (0, 2 ** 28), 12: 15, 13: None,
                                       14: (0, 2 ** 28), 15: None, 16: (float("nan"), float("inf")), 17: None}, bad)
    _refused(L.kv4_attention, decode, {6: ODD, 7: 1020, 9: 100, 10: ODD, 17: ODD, 18: ODD}, align)
    prompt = [0, 2, 40, 60, 8, 2, 128, P, 1024, 128, P, 256, 128, P, 256, 128, P, P, 0.1, 1, P, None, 0, None]
    _refused(L.attn_prompt, prompt, {0: 2, 1: (-1, 2 ** 21), 2: (-1, 2 ** 29), 3: -1, 4: (0, 9), 5: 0, 6: 192, 7: None, 10: None, 13: None, 16: None,
                                     17: None, 18: float("nan"), 20: None, 11: (-8, 2 ** 25)}, bad)
    _refused(L.attn_prompt, prompt, {7: ODD, 8: 1028, 9: 4, 10: ODD, 11: 4, 12: 4, 13: ODD, 14: 4, 15: 4, 20: ODD, 21: ODD}, align)
    # nothing to do: nothing is looked at
    assert L.kv4_write(0, 0, 2, 128, *[None if x is P else x for x in write[4:]]) == 0
    assert L.kv4_attention(*[0 if i == 1 else None if x is P else x for i, x in enumerate(decode)]) == 0
    assert L.attn_prompt(*[0 if i in (1, 2) else None if x is P else x for i, x in enumerate(prompt)]) == 0
