"""What linear_grad's activation argument may hold besides an activation (host only:
the dummy pointers are never read)."""

import ctypes

import pytest

import paper_2608_12573_amd as pk


def _at(n):
    return ctypes.c_void_p(n << 32)


@pytest.mark.parametrize("act,rc", [
    (0, pk.EWORKSPACE), (3, pk.EWORKSPACE), (pk.DZ_BF16, pk.EWORKSPACE), (pk.DZ_BF16 | 3, pk.EWORKSPACE),
    (4, pk.EINVAL), (pk.DZ_BF16 | 4, pk.EINVAL), (512, pk.EINVAL), (2 * pk.DZ_BF16 | pk.DZ_BF16, pk.EINVAL), (-1, pk.EINVAL),
    (-pk.DZ_BF16, pk.EINVAL)])
def test_rounded_or_not(act, rc):
    # (with a workspace of 16 bytes, which is the last thing that is looked at)
    assert pk.lib().profk_linear_grad(0, _at(1), 50, _at(2), act, _at(3), 3, 100, 100, _at(4), 50, 100, _at(5), _at(6),
                                      _at(7), _at(8), 16, None) == rc


@pytest.mark.parametrize("act", [pk.DZ_BF16, pk.DZ_BF16 | 1])
def test_the_forward_call_has_none(act):
    assert pk.lib().profk_linear(_at(1), 3, 104, 104, _at(2), 50, 104, None, act, 0, None, 50, _at(3), None, None, 0,
                                 None) == pk.EINVAL
