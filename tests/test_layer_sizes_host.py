"""Sizes at the ends of what the entry points between projections take: what is
refused, and empty batches.  Nothing here touches a GPU.
"""

import ctypes
import os

import pytest

import paper_2605_04084_amd as fasq
from test_layer_abi_host import DUMMY, _attend, _cache, _lora, _refused, _rope


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fasq.LIB_PATH):
        from paper_2605_04084_amd import _build

        _build.build()
    return fasq.lib()


@pytest.mark.parametrize("pages", [dict(), dict(pages=0, max_pages=0), dict(q=0, out=0, q_start=0, kv_len=0)])
def test_no_requests_launch_nothing(L, pages):
    """A batch of no requests has no tokens; its tables may be empty."""
    assert _attend(L, T=0, B=0, **pages) == fasq.FASQ_OK
    assert L.fasq_paged_attention_workspace_bytes(0, 0, 4, 2, 64) == 0
    _refused(_attend(L, T=3, B=0), "B must")
    assert L.fasq_paged_attention_workspace_bytes(3, 0, 4, 2, 64) == -1
    _refused(_attend(L, T=0, B=-1), "B must")


@pytest.mark.parametrize("page_size,max_pages", [(2 ** 31 - 1, 1), (2 ** 31 - 1023, 1), (16, 2 ** 27 - 1), (1, 2 ** 31 - 1023)])
def test_keys_whose_steps_would_pass_31_bits(L, page_size, max_pages):
    """The kernels step up to some hundred keys past a request's last one."""
    args = dict(cache=_cache(num_pages=1, page_size=page_size), max_pages=max_pages)
    _refused(_attend(L, **args), "2^31 - 1024")


def test_more_requests_than_a_call_takes(L):
    """Every tile looks for its request among all of them: 2^24 requests, as
    were taken before, would keep the GPU busy for hours."""
    _refused(_attend(L, T=1 << 20, B=65537), "B must")
    assert L.fasq_paged_attention_workspace_bytes(1 << 20, 65537, 4, 2, 64) == -1


@pytest.mark.parametrize("N", [2 ** 31 - 1, 2 ** 31 - 2 ** 17 + 1])
def test_features_whose_blocks_would_pass_31_bits(L, N):
    _refused(_lora(L, N=(32, N)), "projection 1: N")


@pytest.mark.parametrize("args", [dict(qos=0), dict(qoh=0), dict(qoh=63), dict(cache=_cache(head_stride=0)),
                                  dict(cache=_cache(slot_stride=32)), dict(cache=_cache(page_stride=0))])
def test_rope_outputs_whose_rows_overlap(L, args):
    """Two rows in one place: what is left there depends on which is written last."""
    _refused(_rope(L, **dict(dict(qo=DUMMY + 4096), **args)), "overlap")


@pytest.mark.parametrize("args", [dict(os=0), dict(oh=0), dict(oh=56), dict(os=8)])
def test_attention_outputs_whose_rows_overlap(L, args):
    _refused(_attend(L, **dict(dict(out=DUMMY + 4096), **args)), "overlap")


def test_attention_over_its_own_queries(L):
    """Rows that meet values that are not finite read their queries again after the output is written."""
    _refused(_attend(L, q=DUMMY, out=DUMMY), "out must not be q")
