"""Scales and caps whose factors leave the range of fp32 are refused: host-side checks, no device is touched."""
import pytest

from test_attention_abi import B, INVALID, attention  # noqa: F401


@pytest.mark.parametrize("edit", [dict(softcap=3e38), dict(softcap=2.4e38, scale=1.0), dict(softcap=1e30, scale=1e-10),
                                  dict(softcap=1e-40, scale=1e-38),
                                  dict(scale=3e38)], ids=str)
def test_factors_outside_the_normal_range_are_refused(B, edit):  # noqa: F811
    assert attention(B, **edit) == (INVALID, INVALID, 0, 0)


@pytest.mark.parametrize("edit", [dict(softcap=2.3e38, scale=4.0), dict(softcap=1e-30), dict(scale=2.3e38), dict(scale=1e-40)],
                         ids=str)
def test_factors_inside_are_taken(B, edit):  # noqa: F811
    # the workspace's size is asked for alone: nothing runs
    import ctypes as C
    s = B.make_attention_shape(2, 16, 16, 4, 2, 64)
    for n, v in edit.items():
        setattr(s, n, v)
    assert B.lib.mixlora_attention_workspace_bytes(C.byref(s), 1) > 0
