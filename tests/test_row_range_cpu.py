"""Rows at positions near the ends of 64 bits are refused by every call that takes positions, as rows outside the cache
are (no GPU: validation fails before any launch)."""
import os

import pytest

import paper_2606_04511_amd.sparda as sp

FAKE = 0x7F0000000000  # aligned, never dereferenced
FAR = [2 ** 63 - 1, 2 ** 63 - 8, 2 ** 62, 8192, 8185, -1, -2 ** 63]


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(sp.library_path()):
        from paper_2606_04511_amd import build
        build.build()
    return sp.load()


def shape():
    return sp.SpardaShape(batch=2, n_kv_heads=8, group_size=4, k_total=16, t_cap=8192, nc_cap=128)


CALLS = {
    "select workspace": lambda p: sp.sparda_workspace_size(shape(), sp.SPARDA_OP_FORECAST_SELECT, 8, p),
    "tree select workspace": lambda p: sp.sparda_workspace_size(shape(), sp.SPARDA_OP_TREE_SELECT, 8, p),
    "tree attention workspace": lambda p: sp.sparda_workspace_size(shape(), sp.SPARDA_OP_TREE_ATTN, 8, p),
    "tree select": lambda p: sp.sparda_tree_select(shape(), FAKE, 8, FAKE, p, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0),
    "tree attention": lambda p: sp.sparda_tree_attn(shape(), FAKE, 8, FAKE, p, FAKE, FAKE, FAKE, FAKE, FAKE, 8, FAKE,
                                                    FAKE, 0.1, FAKE, FAKE, 1 << 40, 0),
    "select": lambda p: sp.sparda_forecast_select(shape(), FAKE, 8, p, FAKE, FAKE, FAKE, FAKE, 1 << 40, 0),
    "attention": lambda p: sp.sparda_sparse_attn(shape(), FAKE, 8, p, FAKE, FAKE, 0, FAKE, FAKE, 0.1, FAKE, FAKE, 1 << 40, 0),
    "write-back": lambda p: sp.sparda_writeback_kv(shape(), FAKE, FAKE, 8, p, FAKE, FAKE, 4, 0),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("at", FAR)
def test_rows_outside_the_cache_are_refused(name, at):
    with pytest.raises(sp.SpardaError) as ei:
        CALLS[name](at)
    assert ei.value.status == sp.SPARDA_ERR_INVALID_ARG
    assert "outside t_cap" in sp.last_error_detail()
