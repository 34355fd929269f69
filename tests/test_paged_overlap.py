"""sc_paged_append refuses places to write to that lie on themselves (an expanded axis, windows that overlap) and takes any permuted view,
with gaps or without.  B is 0 in the calls that are taken, so nothing is enqueued."""
import itertools

import pytest

from paper_2603_14303_b200 import binding
from test_paged_refusals import INVALID, _cache, _rows, append, lib  # noqa: F401  (lib: the fixture)

D, PS, H, P = 128, 16, 8, 100


@pytest.mark.parametrize("kw", [dict(page_stride=0), dict(head_stride=0), dict(row_stride=0, page_size=2), dict(head_stride=64), dict(page_stride=H * PS * D - 8),
                                dict(head_stride=PS * D - 8), dict(page_stride=D, head_stride=D), dict(row_stride=2 * D),
                                dict(page_stride=2 ** 62, num_pages=2 ** 31 - 1, head_stride=0)])
@pytest.mark.parametrize("B", [0, 2])
def test_pools_that_lie_on_themselves(lib, kw, B):  # noqa: F811
    assert append(lib, _cache(**kw), _rows(), B=B) == INVALID


@pytest.mark.parametrize("kw", [dict(qo_token=0), dict(qo_head=0), dict(qo_token=0, qo_head=0), dict(qo_head=64), dict(qo_token=128), dict(qo_token=4096 - 128),
                                dict(qo_token=2 ** 62, qo_head=0)])
@pytest.mark.parametrize("B", [0, 2])
def test_query_outputs_that_lie_on_themselves(lib, kw, B):  # noqa: F811
    assert append(lib, _cache(), _rows(**kw), B=B) == INVALID


@pytest.mark.parametrize("order", list(itertools.permutations(("page_stride", "head_stride", "row_stride"))))
@pytest.mark.parametrize("gap", [0, 16])
def test_every_order_of_the_axes_is_taken(lib, order, gap):  # noqa: F811
    size = dict(page_stride=P, head_stride=H, row_stride=PS)
    strides, at = {}, D + gap
    for axis in reversed(order):
        strides[axis] = at
        at = at * size[axis] + gap
    assert append(lib, _cache(**strides), _rows(), B=0) == binding.SC_OK


@pytest.mark.parametrize("kw", [dict(qo_token=128, qo_head=7 * 128), dict(qo_token=6144, qo_head=128), dict(qo_token=4096, qo_head=128), dict(qo_token=2 ** 62)])
def test_query_layouts_that_are_taken(lib, kw):  # noqa: F811
    assert append(lib, _cache(), _rows(**kw), B=0) == binding.SC_OK


def test_axes_of_one_entry_have_any_stride(lib):  # noqa: F811
    assert append(lib, _cache(page_stride=0, num_pages=1), _rows(), B=0) == binding.SC_OK
    assert append(lib, _cache(head_stride=0, page_heads=1), _rows(), B=0, Hkv=1, Hq=32) == binding.SC_OK
    assert append(lib, _cache(), _rows(qo_token=0), B=0, T=1) == binding.SC_OK
    assert append(lib, _cache(), _rows(qo_head=0), B=0, Hkv=8, Hq=8, T=1) == INVALID
    assert append(lib, _cache(), _rows(qo_token=0, qo_head=0, q=None, q_out=None), B=0) == binding.SC_OK   # (no queries)


def test_inputs_may_lie_on_themselves(lib):  # noqa: F811
    assert append(lib, _cache(), _rows(kv_token=0, kv_head=0, q_token=0, q_head=0), B=0) == binding.SC_OK


def test_nothing_lies_on_nothing(lib):  # noqa: F811
    assert append(lib, _cache(head_stride=0, page_stride=2 ** 20, num_pages=0), _rows(qo_token=2 ** 20, qo_head=0), B=0, T=0) == binding.SC_OK
