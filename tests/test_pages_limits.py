"""Calls of the paged cache whose workgroups one launch does not take (a launch counts its threads in 32 bits) are refused before any is made."""
import ctypes as C

import pytest

from tests.test_pages_args import AT, UNSUPPORTED, append, attend, batch, lib, pages, select  # noqa: F401


def seqs(n, new=1, width=1):
    return batch(n_seqs=n, max_new=new, n_rows=min(n * new, 2**31 - 1), width=width, table_stride=width)


def test_append(lib):  # noqa: F811
    assert append(lib, pages(), seqs(1 << 24)) == UNSUPPORTED
    assert append(lib, pages(), seqs(1 << 20, new=900, width=16)) == UNSUPPORTED  # 16 pages of a sequence


@pytest.mark.parametrize("dtype", [0, 1])
def test_attend(lib, dtype):  # noqa: F811
    assert attend(lib, pages(), seqs(1 << 21), dtype=dtype) == UNSUPPORTED                       # 8 heads of 16 rows
    assert attend(lib, pages(), seqs(1 << 18, new=1024), dtype=dtype) == UNSUPPORTED             # prompts, 512 threads to a workgroup
    assert attend(lib, pages(), seqs(1 << 20, new=65), dtype=1, heads=8, row=1024, orow=1024) == UNSUPPORTED
    assert attend(lib, pages(), seqs(1 << 17, new=16), dtype=dtype, chosen=AT, n_chosen=1) == UNSUPPORTED


def test_lists_of_more_tokens_than_positions(lib):  # noqa: F811
    assert attend(lib, pages(), batch(), chosen=AT, n_chosen=(1 << 31) // 64) == UNSUPPORTED
    assert attend(lib, pages(page_tokens=128), batch(), chosen=AT, n_chosen=2**31 - 1) == UNSUPPORTED


@pytest.mark.parametrize("units,width", [(1 << 24, 1), (1 << 23, 1025), (1 << 22, 4097), (1 << 20, 65536)])
def test_select(lib, units, width):  # noqa: F811
    assert select(lib, pages(), seqs(units // 8, width=width)) == UNSUPPORTED
    assert select(lib, pages(), seqs(units // 64, new=8, width=width), dtype=0) == UNSUPPORTED


def test_select_asks_for_no_workspace_it_cannot_use(lib):  # noqa: F811
    assert lib.tq_pages_select_workspace_bytes(C.byref(pages()), C.byref(seqs(1 << 19, width=4097))) == 0
    assert lib.tq_pages_select_workspace_bytes(C.byref(pages()), C.byref(seqs((1 << 19) - 1, width=4097))) == ((1 << 19) - 1) * 8 * 4097 * 4


def test_lists_of_rows(lib):  # noqa: F811
    n = 1 << 24
    assert lib.tq_pages_free(C.byref(pages()), C.byref(batch()), AT, n, None) == UNSUPPORTED
    assert lib.tq_pages_fork(C.byref(pages()), C.byref(batch()), AT, AT, n, None, None) == UNSUPPORTED
