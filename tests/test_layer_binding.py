"""What the layer operators' Python entry points take for an argument, like the other calls': anything that stands for an integer
(numpy's integers, None for no address), and nothing else.  The library refuses each call before it touches a device: no GPU
needed."""
import numpy as np
import pytest

import paper_2205_03494_b200 as omc

A = 1 << 20
NULL = -3


class Whole:
    def __init__(self, v):
        self.v = v

    def __index__(self):
        return self.v


def calls(n):
    """Every call with n() around its integers, the first address missing."""
    return [
        (omc.mx_quantise, (n(0), n(1), n(4), n(64), n(64), n(A), n(A), n(0), n(0), n(0))),
        (omc.mx_dequantise, (n(0), n(A), n(4), n(64), n(A), n(1), n(64), n(0))),
        (omc.mx_matmul, (n(0), n(A), n(4), n(A), n(A), n(8), n(64), n(A), n(0), n(8), n(A), n(0))),
        (omc.mx_linear, (n(0), n(1), n(4), n(64), n(64), n(A), n(A), n(8), n(A), n(0), n(8), n(A), n(A), n(0))),
        (omc.layer_norm, (n(0), n(1), n(4), n(64), n(64), n(A), n(A), np.float32(1e-5), n(A), n(64), n(A), n(A), n(0))),
        (omc.layer_norm_backward, (n(0), n(64), n(A), n(64), n(1), n(4), n(64), n(A), n(A), n(A), n(A), n(64), n(A), n(A), n(A), n(0))),
    ]


@pytest.mark.parametrize("n", [int, np.int64, np.uint64, np.int32, Whole], ids=lambda n: n.__name__)
def test_integers_of_every_kind(n):
    assert omc.mx_sizes(n(4), n(64)) == (128, 1024)
    for fn, args in calls(n):
        with pytest.raises(omc.OmcError) as e:
            fn(*args)
        assert e.value.status == NULL, fn.__name__


def test_none_is_no_address():
    for fn, args in calls(int):
        with pytest.raises(omc.OmcError) as e:
            fn(None, *args[1:])
        assert e.value.status == NULL


def test_what_is_no_integer_in_range():
    for fn, args in calls(int):
        for at in range(len(args)):
            if isinstance(args[at], np.float32):
                with pytest.raises(TypeError):
                    fn(*args[:at], "x", *args[at + 1:])
                continue
            for bad, error in ((4.0, TypeError), ("4", TypeError), (1 << 64, OverflowError), (Whole(-(1 << 70)), OverflowError)):
                with pytest.raises(error):
                    fn(*args[:at], bad, *args[at + 1:])
