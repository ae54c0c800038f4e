"""The sizes that include/kla.h allows sliding-window attention, on the host: calls within the stated number of
workgroups are taken, whatever the window, and the first one past it is refused."""
import pytest

from test_hybrid_attn_host import lib, window  # noqa: F401

MOST = 1 << 23   # workgroups


def up(a, b):
    return -(-a // b)


@pytest.mark.parametrize("W,sinks", [(1, 64), (31, 1), (100, 4), (512, 4), (1 << 20, 0)])
@pytest.mark.parametrize("T,past", [(1 << 20, 0), (100003, 5000), (777, 0), (1, 1 << 18)])
def test_calls_within_the_stated_workgroups(lib, W, sinks, T, past):
    Tk = T + past
    for Hk, H in ((1, 1), (2, 8)):
        a, b = H * up(T, 128), Hk * (up(Tk, 128) + up(T, 256))
        B = (MOST - 1) // max(a, b)
        o = dict(T=T, Tk=Tk, H=H, Hk=Hk, d=16, window=W, sinks=sinks)
        assert lib.kla_window_attn_backward_workspace(window(B=B, **o)) > 0
        assert lib.kla_window_attn_saved_bytes(window(B=B, **o)) > 0
    # one workgroup more than can be, for the keys' 128 tokens alone
    B = up(MOST, up(Tk, 128))
    assert lib.kla_window_attn_backward_workspace(window(B=B, T=T, Tk=Tk, H=1, Hk=1, d=16, window=W, sinks=sinks)) == 0
