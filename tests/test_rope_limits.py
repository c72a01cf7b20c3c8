"""Sizes whose products do not fit 64 or 32 bits are refused before any device call: these run without a device."""
import ctypes as C

import pytest

from paper_2604_10103_b200 import binding as hf, build as hfbuild

SHAPE, P, MOST = 2, 0x10000, 2 ** 31 - 1


@pytest.mark.parametrize("kw,heads,n", [(dict(batch=MOST, tokens=MOST, head_dim=1024), 1, 1), (dict(batch=2 ** 30, tokens=2 ** 30, head_dim=16), 1, 1),
                                        (dict(batch=MOST, tokens=4, head_dim=1024), 1, 1), (dict(batch=1, tokens=1), 2 ** 30, 2), (dict(batch=1, tokens=1), MOST, 3),
                                        (dict(batch=1, tokens=1), MOST, 1)])
def test_products_of_sizes(kw, heads, n):
    hfbuild.build()
    s = hf.hf_rope_shape(**dict(dict(type=0, batch=1, tokens=4, head_dim=64, axes=1, pairing=0, inverse=0, pos_batch=0), **kw))
    s.pairs[0], s.extent[0] = 1, 4
    t = (hf.hf_rope_tensor * 3)()
    for a in t:
        a.x, a.y, a.heads, a.rotate = P, P, heads, 1
    assert hf.lib().hf_rope_axes(C.byref(s), t, n, P, P, P, None) == SHAPE and hf.lib().hf_last_error()
