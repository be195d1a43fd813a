"""Between the modules before this one and those behind it: no pool of an earlier test is left for the garbage collector."""
import gc

import pytest

from paper_2510_02758_amd import kvswap as kv

pytestmark = pytest.mark.gpu


def test_no_pool_of_an_earlier_module_is_left():
    left = [x for x in gc.get_objects() if type(x) in (kv.KVPool, kv.KVBatch) and getattr(x, "h", None)]
    assert not left, "%d pools and batches, whose end would wait for the device in the middle of a later test" % len(left)
