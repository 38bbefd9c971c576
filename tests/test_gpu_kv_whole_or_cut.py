"""Batches for which whole items and equal ranges are estimated to take the same time, or nearly: the kernel that attends and the one that joins have to decide alike."""
import pytest

from kv_helpers import Cache, queries
from test_gpu_kv_attention import run

pytestmark = pytest.mark.gpu


# on a device of 148 SMs; the third: the estimates are equal
@pytest.mark.parametrize("dim,heads,group,lens,new", [(128, 1, 2, [3257, 1794], [453, 866]), (128, 1, 2, [2323, 3109], [283, 254]),
                                                      (128, 1, 4, [3043, 2800, 3829], [580, 263, 663]), (128, 1, 1, [3114, 1003, 3156], [285, 757, 62]),
                                                      (128, 1, 4, [3571, 2403, 2280], [567, 440, 130]), (256, 1, 1, [1554], [777]),
                                                      (256, 1, 2, [1300, 1676], [649, 234]), (256, 1, 4, [1611], [207])])
@pytest.mark.parametrize("fmt", ["mxfp4", "nvfp4", "mxint4"])
def test_estimates_that_are_nearly_equal(fmt, dim, heads, group, lens, new):
    c = Cache(fmt, lens, heads, group, dim, 64, new=new)
    run(c, queries(c))
