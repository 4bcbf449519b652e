"""What infaas_sel_exec_advance and _copy refuse, on the host, and the table of the binding."""
import os

import pytest
import torch

import paper_1905_13348_amd as pkg
from paper_1905_13348_amd import binding
from test_exec_refusals import BAD_CACHE, BAD_POOLS, P, _cache, _refused, lib  # noqa: F401
from test_exec_scaled_refusals import BAD_SCALES, _scales

pytestmark = pytest.mark.skipif(not os.path.exists(pkg.library_path()), reason="library not built here")

ARRAYS = ("d_page_table", "d_seq_len", "d_page_refs", "d_seq_start", "d_token_seq", "d_token_pos", "d_taken", "d_copies")


def _table(**kw):
    t = dict(num_seqs=3, table_width=4, page_size=16, num_pages=8, max_tokens=10, **{a: P for a in ARRAYS})
    t.update(kw)
    return binding._Table(**t)


BAD_TABLE = [(dict(num_seqs=0), "sequences"), (dict(num_seqs=4097), "4097"), (dict(num_seqs=-1), "sequences"), (dict(table_width=0), "row"),
             (dict(num_pages=0), "pages"), (dict(max_tokens=0), "tokens"), (dict(page_size=0), "page size"), (dict(page_size=24), "24"),
             (dict(page_size=1 << 17), "page size"), (dict(d_page_refs=P + 4), "aligned")] + [({a: 0}, "null") for a in ARRAYS]


@pytest.mark.parametrize("bad, word", BAD_TABLE)
def test_tables(lib, bad, word):  # noqa: F811
    _refused(lib, lib.infaas_sel_exec_advance(lib.h, _table(**bad), P, None, None), "table", word)
    _refused(lib, lib.infaas_sel_exec_copy(lib.h, _cache(), None, _table(**bad), None), "table", word)


def test_null(lib):  # noqa: F811
    _refused(lib, lib.infaas_sel_exec_advance(None, _table(), P, None, None), "executor")
    _refused(lib, lib.infaas_sel_exec_advance(lib.h, None, P, None, None), "table")
    _refused(lib, lib.infaas_sel_exec_advance(lib.h, _table(), None, P, None), "advance")
    _refused(lib, lib.infaas_sel_exec_copy(None, _cache(), None, _table(), None), "executor")
    _refused(lib, lib.infaas_sel_exec_copy(lib.h, None, None, _table(), None), "cache")
    _refused(lib, lib.infaas_sel_exec_copy(lib.h, _cache(), None, None, None), "table")


@pytest.mark.parametrize("bad, word", BAD_CACHE + BAD_POOLS)
def test_caches(lib, bad, word):  # noqa: F811
    _refused(lib, lib.infaas_sel_exec_copy(lib.h, _cache(**bad), None, _table(), None), "cache", word)


@pytest.mark.parametrize("bad, word", BAD_SCALES)
def test_scales(lib, bad, word):  # noqa: F811
    _refused(lib, lib.infaas_sel_exec_copy(lib.h, _cache(), _scales(**bad), _table(), None), "scales", word)


def test_another_page_size(lib):  # noqa: F811
    _refused(lib, lib.infaas_sel_exec_copy(lib.h, _cache(page_size=32), None, _table(), None), "copy", "32")


@pytest.mark.parametrize("sizes", [(0, 1, 1, 1, 1), (4097, 1, 1, 1, 1), (1, 0, 1, 1, 1), (1, 1, 3, 1, 1), (1, 1, 1 << 17, 1, 1), (1, 1, 1, 0, 1), (1, 1, 1, 1, 0),
                                   (1, 2 ** 31, 1, 1, 1), (1, 1, 1, 2 ** 31, 1), (1, 1, 1, 1, 2 ** 31)])
def test_sizes_of_the_binding(sizes):
    with pytest.raises(ValueError):
        pkg.Table(*sizes)
