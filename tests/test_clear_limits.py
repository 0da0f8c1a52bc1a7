"""Large calls of the recurrence in the clear that one launch can carry are not
refused (checked up to the buffers, which are absent here)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def clear():
    from paper_2608_17442_amd import clear
    return clear


def refused_for(clear, backward, **kw):
    v = dict(dtype=1, batch=1, len=64, heads=24, head_dim=64, groups=1, d_state=128)
    v.update(kw)
    d = clear._ScanDesc(**v)
    if backward:
        rc = clear._lib.fesc_clear_scan_bwd(ctypes.byref(d), *[None] * 13, 0, None)
    else:
        rc = clear._lib.fesc_clear_scan(ctypes.byref(d), *[None] * 8, 0, None)
    assert rc == -1
    return clear._lib.fesc_last_error().decode()


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw", [
    dict(batch=40000, len=64),                        # many short prompts
    dict(len=1 << 22, groups=8),                      # 2^32 entries of B
    dict(batch=4, len=1 << 20, groups=8),
])
def test_large_calls_are_taken(clear, backward, kw):
    assert "null buffer" in refused_for(clear, backward, **kw)


def test_what_no_launch_carries_is_refused(clear):
    assert "too large" in refused_for(clear, False, batch=1 << 19)
    assert "too large" in refused_for(clear, True, batch=1 << 10, len=64 << 12, heads=1)
    assert "null buffer" in refused_for(clear, False, batch=1 << 10, len=64 << 12, heads=1)


def test_small_heads_take_little_room(clear):
    """The gradient's workspace follows the states' own size, to whole tiles of 16 x 32
    entries: two directions, fp32, one state a chunk of 64 tokens."""
    for P, N in ((16, 16), (8, 32), (64, 128), (100, 33)):
        d = clear._ScanDesc(dtype=1, batch=1, len=1 << 20, heads=24, head_dim=P, groups=1, d_state=N)
        n = ctypes.c_size_t()
        assert clear._lib.fesc_clear_scan_workspace(ctypes.byref(d), 1, ctypes.byref(n)) == 0
        rows = -(-P // 16) * 16 if P <= 64 else -(-P // 64) * 64
        state = 24 * rows * (-(-N // 32) * 32) * 4
        assert n.value <= 2 * state * ((1 << 14) + 32)     # and segments' states
