"""What the entry points around a decoder layer's products refuse before anything is launched."""
import ctypes

import pytest

from paper_2509_01229_amd import api

P = ctypes.c_void_p(1 << 20)    # an address that is aligned and never followed
ODD = ctypes.c_void_p((1 << 20) + 8)
ODDER = ctypes.c_void_p((1 << 20) + 2)
NAN = float("nan")


def _entries():
    L = api.lib()
    norm = [0, 4, 256, P, 256, P, 256, P, 1e-6, P, P, P, P, None]
    swiglu = [1, 4, 256, P, 512, P, P, None]
    dispatch = [2, 4, 2, 8, 256, P, 256, P, P, P, P, P, P, None]
    combine = [0, 4, 2, 8, 256, P, 256, P, P, P, None]
    backward = [0, 4, 2, 8, 256, P, 256, P, 256, P, P, P, P, P, None]
    chunks = [0, 2, 40, 8, 2, 128, P, 1024, 128, P, P, 10, 16, P, 5, P, 0.1, P, None, 0, None]
    return {
        "norm": (L.w4a8_norm_quantize, norm,
                 {0: (2, -1), 1: -1, 2: (0, 252, 2 ** 25), 3: None, 5: None, 8: (0.0, -1.0, NAN, float("inf")), 9: None, 11: None, 12: None},
                 {3: ODD, 4: 260, 5: ODD, 6: 4, 7: ODD, 9: ODD, 10: ODD, 11: ODD, 12: ODD}),
        "swiglu": (L.w4a8_swiglu_quantize, swiglu, {0: 2, 1: -1, 2: (0, 4, 2 ** 25), 3: None, 5: None, 6: None}, {3: ODD, 4: 516, 5: ODD, 6: ODD}),
        "dispatch": (L.moe_dispatch, dispatch,
                     {0: (3, -1), 1: (-1, 2 ** 23), 2: (0, 65, -2), 3: (0, 257), 4: (0, 8, 250), 5: None, 7: None, 8: None, 9: None, 10: None, 11: None, 12: None},
                     {5: ODD, 6: 264, 7: ODDER, 8: ODDER, 9: ODD, 10: ODDER, 11: ODDER, 12: ODDER}),
        "combine": (L.moe_combine, combine, {0: 2, 1: (-1, 2 ** 30), 2: (0, 65), 3: -1, 4: (0, 4, 2 ** 25), 5: None, 7: None, 9: None},
                    {5: ODD, 6: 252, 7: ODDER, 8: ODDER, 9: ODD}),
        "backward": (L.moe_combine_backward, backward,
                     {0: 2, 1: (-1, 2 ** 23), 2: (0, 65), 3: -1, 4: (0, 12), 5: None, 7: None, 9: None, 10: None, 12: None, 13: None},
                     {5: ODD, 6: 4, 7: ODD, 8: 4, 9: ODDER, 10: ODDER, 11: ODDER, 12: ODD, 13: ODDER}),
        "chunks": (L.kv4_attention_chunks, chunks,
                   {0: 2, 1: (-1, 2 ** 21), 2: (-1, 2 ** 29), 3: (0, 9, 5000), 4: (0, 5000), 5: (96, 0), 6: None, 9: None, 10: None, 11: (0, 2 ** 28), 12: (8, 24),
                    13: None, 14: (0, 2 ** 28), 15: None, 16: (NAN, float("inf")), 17: None},
                   {6: ODD, 7: 1020, 8: 100, 9: ODDER, 10: ODD, 13: ODDER, 15: ODDER, 17: ODD, 18: ODD}),
    }


@pytest.mark.parametrize("which", ["norm", "swiglu", "dispatch", "combine", "backward", "chunks"])
def test_c_entries_refuse_what_they_cannot_run(which):
    call, good, invalid, unaligned = _entries()[which]
    for code, changes in ((api.LQ_ERR_INVALID, invalid), (api.LQ_ERR_ALIGN, unaligned)):
        for i, values in changes.items():
            for value in values if isinstance(values, tuple) else (values,):
                args = list(good)
                args[i] = value
                assert call(*args) == code, (which, i, value)
                assert api.lib().w4a8_last_error()


def test_nothing_to_do():
    """Empty batches succeed and look at nothing."""
    entries = _entries()
    for which, empty in (("norm", (1,)), ("swiglu", (1,)), ("combine", (1,)), ("backward", (1, 3)), ("chunks", (1,)), ("chunks", (2,))):
        call, good, _, _ = entries[which]
        assert call(*[0 if i in empty else None if x is P else x for i, x in enumerate(good)]) == 0, which


def test_chunks_workspace():
    """Workspace where few queries read many keys; none where there are many queries, or no such call."""
    size = api.lib().kv4_attention_chunks_workspace_size
    assert size(1, 17, 32, 8, 128, 64, 100) > 32768
    assert size(4, 16384, 64, 8, 128, 64, 256) == 0
    for bad in ((0, 17, 32, 8, 128, 64, 100), (1, 0, 32, 8, 128, 64, 100), (1, 17, 31, 8, 128, 64, 100), (1, 17, 32, 8, 96, 64, 100), (1, 17, 32, 8, 128, 60, 100),
                (1, 17, 32, 8, 128, 64, 0), (1, 17, 32, 8, 128, 256, 2 ** 28)):
        assert size(*bad) == 0


def test_chunks_workspace_of_many_sequences():
    """None from 65 sequences on, or where the tiles of rows may be 512 (8 kv heads, four rows each: (4 + 127) * 62 / 128 = 63 tiles, of 63 sequences 64): keys are not cut there."""
    size = api.lib().kv4_attention_chunks_workspace_size
    assert size(64, 64, 8, 1, 128, 64, 600) > 32768 and size(65, 65, 8, 1, 128, 64, 600) == 0
    assert size(62, 62, 32, 8, 128, 64, 600) > 32768 and size(63, 63, 32, 8, 128, 64, 600) == 0


def test_tensors_on_the_cpu_are_refused():
    import torch

    f, i = torch.zeros((4, 64), dtype=torch.float16), torch.zeros((4, 2), dtype=torch.int32)
    w = torch.zeros((4, 2))
    for call in (lambda: api.w4a8_norm_quantize(f), lambda: api.w4a8_swiglu_quantize(f), lambda: api.moe_dispatch(f, i, 4), lambda: api.moe_combine(f, i, w),
                 lambda: api.moe_combine_backward(f, f, i, w),
                 lambda: api.kv4_attention_chunks(f.view(4, 1, 64), torch.zeros((1, 1, 16 * 72), dtype=torch.uint8), i, i[0], i[0])):
        with pytest.raises(TypeError):
            call()
