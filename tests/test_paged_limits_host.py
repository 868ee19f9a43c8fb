"""Sizes of the paged cache next to what its 32-bit counts hold (host only: nothing is launched)."""
import ctypes as C

import pytest

import paper_2507_05228_amd as cas
from test_paged_host import P, cache, lib  # noqa: F401


@pytest.mark.parametrize("max_pages", [(1 << 27) - 1, (1 << 27) - 4])
def test_lists_whose_last_step_would_pass_31_bits(lib, max_pages):  # noqa: F811
    """A walk goes in steps of up to 64 keys; the end of the last one counts in 32 bits too."""
    c = cache(n_seqs=1, page_size=16, max_pages=max_pages)
    desc = cas.PagedAttnDesc(4, 4, 1.0, cas.BF16, 0, 0)
    assert lib.cascade_paged_attn_workspace_bytes(C.byref(c), C.byref(desc)) == 0
    assert lib.cascade_paged_attn(C.byref(c), 0, C.byref(desc), P, None, P, P, None, P, 1 << 40, None) == cas.EUNSUPPORTED
    assert lib.cascade_paged_extend(C.byref(c), 1, P, P, P, P, P, None) == cas.EUNSUPPORTED
    c.max_pages = (1 << 27) - 5
    assert lib.cascade_paged_attn_workspace_bytes(C.byref(c), C.byref(desc)) > 0


@pytest.mark.parametrize("rows", [2 ** 31 - 1024, 2 ** 31 - 1])
def test_extensions_whose_last_walk_would_pass_31_bits(lib, rows):  # noqa: F811
    """Rows are walked over 1024 at a time, by threads that stop at the first row behind the last."""
    for n_shards, shard in ((1, None), (1, P), (3, P)):
        assert lib.cascade_paged_extend(C.byref(cache(n_shards=n_shards)), rows, P, shard, P, P, P, None) == cas.EUNSUPPORTED


@pytest.mark.parametrize("change", [dict(n_seqs=2 ** 31 - 1), dict(n_seqs=2 ** 31 - 4096), dict(n_seqs=1, n_shards=662, max_pages=3243933)])
def test_lists_whose_last_round_would_pass_31_bits(lib, change):  # noqa: F811
    """Sequences are taken 4096 at a time, entries of a list by 256 threads at a time."""
    c = cache(**{**dict(n_shards=1, max_pages=1), **change})
    assert c.n_seqs * c.n_shards * c.max_pages in (2 ** 31 - 1, 2 ** 31 - 4096, 2 ** 31 - 2)
    c = C.byref(c)
    assert lib.cascade_paged_extend(c, 1, P, P, P, P, P, None) == cas.EUNSUPPORTED
    assert lib.cascade_pages_free(c, 1, P, None) == cas.EUNSUPPORTED
    assert lib.cascade_pages_workspace_bytes(c) == 0
    assert lib.cascade_pages_workspace_bytes(C.byref(cache(n_shards=1, max_pages=1, n_seqs=2 ** 31 - 4097))) > 0
