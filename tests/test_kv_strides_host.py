"""Which strides of layers and pages a KV cache may have: every order in which no two pages' numbers share memory,
compared with the blocks themselves.  No GPU."""
import ctypes
import random

import pytest

from test_kv_host import _calls, _desc

PAGE = 2 * 64 * 16  # elements of a page of _desc


def _accepts(**kw):
    from paper_2606_17059_amd import router as R
    need = ctypes.c_int64(0)
    s = R.lib().pr_kv_workspace(ctypes.byref(_desc(**kw)), 0, 3, 5, ctypes.byref(need))
    assert s == R.PR_OK or (s == R.PR_EINVAL and "overlap" in R.pr_last_error())
    return s == R.PR_OK


@pytest.mark.parametrize("side", ["k", "v"])
@pytest.mark.parametrize("layer,page,apart", [
    (100 * PAGE, PAGE, True), (PAGE, 2 * PAGE, True),     # layers one after another; a page's layers together
    (100 * PAGE - 8, PAGE, False), (PAGE, 2 * PAGE - 8, False),
    (PAGE, PAGE, False),                                  # layer 1 of page 0 would be layer 0 of page 1
    (2 * PAGE, PAGE, False), (99 * PAGE, PAGE, False), (50 * PAGE + 8, PAGE, False),
    (3 * PAGE, 2 * PAGE, True),                           # interleaved: 0, 2, 4, ... and 3, 5, 7, ...
    (3 * PAGE + 8, 2 * PAGE, False), (5 * PAGE, 2 * PAGE + 8, False), (300 * PAGE, 2 * PAGE, True)])
def test_pages_that_share_memory_are_refused(side, layer, page, apart):
    assert _accepts(**{side + "_layer": layer, side + "_page": page}) == apart


def test_random_strides_against_the_blocks():
    """All calls refuse exactly the strides where two blocks of a page overlap."""
    rng = random.Random(3)
    met = {True: 0, False: 0}
    for _ in range(4000):
        layers, pages = rng.randint(1, 6), rng.randint(1, 7)
        unit = PAGE // 8
        a, b = (unit * rng.randint(4, 40) for _ in range(2))
        at = sorted(i * a + j * b for i in range(layers) for j in range(pages))
        apart = all(y - x >= PAGE for x, y in zip(at, at[1:]))
        met[apart] += 1
        kw = dict(layers=layers, num_pages=pages, k_layer=a, k_page=b, v_layer=PAGE * pages, v_page=PAGE)
        assert _accepts(**kw) == apart, (layers, pages, a / PAGE, b / PAGE)
    assert min(met.values()) > 500


def test_every_call_refuses_shared_pages_and_strides_past_64_bits():
    from paper_2606_17059_amd import router as R
    for d in (_desc(k_layer=PAGE), _desc(v_layer=PAGE), _desc(k_layer=1 << 62, layers=3), _desc(v_page=1 << 60)):
        for name, args in _calls(d).items():
            assert getattr(R.lib(), name)(*args) == R.PR_EINVAL, name
    big = dict(layers=1 << 20, num_pages=1 << 20, k_page=PAGE, k_layer=PAGE << 20, v_layer=PAGE, v_page=PAGE << 20)
    assert _accepts(**big)
