"""What the paged cache's entry points refuse, before any device is touched (CPU), and the plain definition's own checks."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import pages_oracle as po

OK, INVALID, UNSUPPORTED, HIP, WORKSPACE = range(5)
AT = 1 << 20  # an aligned address that nobody reads


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2504_19874_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2504_19874_amd import build
        build.build_library(verbose=False)
    return _lib.load()


def pages(**more):
    from paper_2504_19874_amd import _lib
    p = _lib.TqPages(d=128, n_heads=8, page_tokens=64, type=0, n_pages=100, k=AT, v=AT, k_scale=AT, v_scale=AT, bounds=AT, refs=AT, workspace=AT,
                     workspace_bytes=1 << 40)
    for n, v in more.items():
        setattr(p, n, v)
    return p


def batch(**more):
    from paper_2504_19874_amd import _lib
    b = _lib.TqBatch(n_seqs=4, max_new=1, n_rows=4, width=10, table_stride=10, table=AT, lens=AT, starts=0)
    for n, v in more.items():
        setattr(b, n, v)
    return b


def append(lib, p, b, k=AT, v=AT, dtype=1, row=1024, head=128):
    return lib.tq_pages_append(p and C.byref(p), b and C.byref(b), k, v, dtype, row, head, None)


def attend(lib, p, b, q=AT, dtype=1, row=4096, head=128, heads=32, window=0, chosen=None, n_chosen=0, out=AT, orow=4096, ohead=128):
    return lib.tq_pages_attend(p and C.byref(p), b and C.byref(b), q, dtype, row, head, heads, 0.1, window, chosen, n_chosen, out, orow, ohead, None, None)


def select(lib, p, b, q=AT, dtype=1, row=4096, head=128, heads=32, first=1, last=1, chosen=AT, n=8):
    return lib.tq_pages_select(p and C.byref(p), b and C.byref(b), q, dtype, row, head, heads, first, last, chosen, n, None)


def test_struct_layouts():
    from paper_2504_19874_amd import _lib
    assert C.sizeof(_lib.TqPages) == 16 + 8 + 8 * 8 and _lib.TqPages.n_pages.offset == 16 and _lib.TqPages.workspace_bytes.offset == 80
    assert C.sizeof(_lib.TqBatch) == 56 and _lib.TqBatch.n_rows.offset == 8 and _lib.TqBatch.table_stride.offset == 24 and _lib.TqBatch.table.offset == 32


@pytest.mark.parametrize("more,want", [
    (dict(d=0), INVALID), (dict(d=96), UNSUPPORTED), (dict(d=512), UNSUPPORTED), (dict(n_heads=0), INVALID), (dict(page_tokens=0), INVALID),
    (dict(page_tokens=48), UNSUPPORTED), (dict(page_tokens=256), UNSUPPORTED), (dict(type=2), INVALID), (dict(type=-1), INVALID), (dict(n_pages=0), INVALID),
    (dict(n_pages=1 << 31), UNSUPPORTED), (dict(n_pages=1 << 26), UNSUPPORTED), (dict(n_heads=40000), UNSUPPORTED)])
def test_caches_that_every_call_refuses(lib, more, want):
    p = pages(**more)
    assert append(lib, p, batch()) == want and attend(lib, p, batch()) == want and select(lib, p, batch()) == want
    assert lib.tq_pages_reserve(C.byref(p), C.byref(batch()), None, None) == want
    assert lib.tq_pages_fork(C.byref(p), C.byref(batch()), AT, AT, 2, None, None) == want
    assert lib.tq_pages_free(C.byref(p), C.byref(batch()), AT, 2, None) == want
    assert lib.tq_pages_compact(C.byref(p), C.byref(batch()), None, None) == want
    assert lib.tq_pages_copy(C.byref(p), AT, AT, 2, None) == want
    assert lib.tq_pages_select_workspace_bytes(C.byref(p), C.byref(batch())) == 0 and lib.tq_pages_pool_workspace_bytes(C.byref(p), 4) == 0
    assert lib.tq_pages_attend_workspace_bytes(C.byref(p), C.byref(batch()), 32, 0, 0) == 0


@pytest.mark.parametrize("more", [dict(n_seqs=-1), dict(max_new=-1), dict(n_rows=-1), dict(width=-1), dict(table_stride=9)])
def test_batches_that_every_call_refuses(lib, more):
    b = batch(**more)
    assert append(lib, pages(), b) == INVALID and attend(lib, pages(), b) == INVALID and select(lib, pages(), b) == INVALID
    for f, args in (("reserve", (None,)), ("fork", (AT, AT, 2, None)), ("free", (AT, 2)), ("compact", (None,))):
        assert getattr(lib, "tq_pages_" + f)(C.byref(pages()), C.byref(b), *args, None) == INVALID


def test_null_pointers(lib):
    assert append(lib, None, batch()) == INVALID and append(lib, pages(), None) == INVALID
    assert attend(lib, None, batch()) == INVALID and attend(lib, pages(), None) == INVALID
    assert select(lib, None, batch()) == INVALID and select(lib, pages(), None) == INVALID
    for name in ("k", "v", "k_scale", "v_scale"):
        assert append(lib, pages(**{name: None}), batch()) == INVALID and attend(lib, pages(**{name: None}), batch()) == INVALID
        assert lib.tq_pages_copy(C.byref(pages(**{name: None})), AT, AT, 2, None) == INVALID
    for name in ("table", "lens"):
        b = batch(**{name: None})
        assert append(lib, pages(), b) == INVALID and attend(lib, pages(), b) == INVALID and select(lib, pages(), b) == INVALID
        assert lib.tq_pages_reserve(C.byref(pages()), C.byref(b), None, None) == INVALID
        assert lib.tq_pages_free(C.byref(pages()), C.byref(b), AT, 1, None) == INVALID
    assert append(lib, pages(), batch(), k=None) == INVALID and append(lib, pages(), batch(), v=None) == INVALID
    assert attend(lib, pages(), batch(), q=None) == INVALID and attend(lib, pages(), batch(), out=None) == INVALID
    assert select(lib, pages(), batch(), q=None) == INVALID and select(lib, pages(), batch(), chosen=None) == INVALID
    assert select(lib, pages(bounds=None), batch()) == INVALID
    none = pages(refs=None)
    assert lib.tq_pages_reserve(C.byref(none), C.byref(batch()), None, None) == INVALID
    assert lib.tq_pages_free(C.byref(none), C.byref(batch()), AT, 1, None) == INVALID
    assert lib.tq_pages_fork(C.byref(pages()), C.byref(batch()), None, AT, 1, None, None) == INVALID
    assert lib.tq_pages_copy(C.byref(pages()), None, AT, 1, None) == INVALID


def test_types_strides_alignment_and_heads(lib):
    p, b = pages(), batch()
    assert append(lib, p, b, dtype=2) == INVALID and attend(lib, p, b, dtype=-1) == INVALID and select(lib, p, b, dtype=7) == INVALID
    assert append(lib, p, b, k=AT + 8) == UNSUPPORTED and append(lib, p, b, v=AT + 2) == UNSUPPORTED
    assert append(lib, p, b, row=1028) == UNSUPPORTED and append(lib, p, b, head=132) == UNSUPPORTED and append(lib, p, b, row=-8) == INVALID
    assert append(lib, p, b, dtype=0, row=1026) == UNSUPPORTED
    assert attend(lib, p, b, q=AT + 8) == UNSUPPORTED and attend(lib, p, b, out=AT + 4) == UNSUPPORTED
    assert attend(lib, p, b, row=4100) == UNSUPPORTED and attend(lib, p, b, ohead=129) == UNSUPPORTED
    assert attend(lib, p, b, heads=12) == INVALID and attend(lib, p, b, heads=0) == INVALID and attend(lib, p, b, window=-1) == INVALID
    assert attend(lib, p, b, n_chosen=-1) == INVALID
    assert append(lib, pages(k=AT + 8), b) == UNSUPPORTED and attend(lib, pages(v_scale=AT + 2), b) == UNSUPPORTED
    assert select(lib, pages(bounds=AT + 4), b) == UNSUPPORTED
    assert select(lib, p, b, n=0) == INVALID and select(lib, p, b, n=1025) == UNSUPPORTED and select(lib, p, b, first=5, last=4) == INVALID
    assert select(lib, p, b, first=-1) == INVALID and select(lib, p, batch(width=65537, table_stride=65537)) == UNSUPPORTED


def test_sizes_beyond_a_grid(lib):
    assert append(lib, pages(), batch(n_seqs=1 << 30, max_new=1 << 20)) == UNSUPPORTED
    assert attend(lib, pages(), batch(n_seqs=1 << 30)) == UNSUPPORTED
    assert attend(lib, pages(), batch(max_new=(1 << 31) - 1)) == UNSUPPORTED
    assert select(lib, pages(), batch(n_seqs=1 << 20, max_new=1 << 10)) == UNSUPPORTED


def test_workspaces(lib):
    p, b = pages(), batch()
    need = lib.tq_pages_select_workspace_bytes(C.byref(p), C.byref(b))
    assert need >= 4 * 8 * 10 * 4
    assert select(lib, pages(workspace_bytes=need - 1), b) == WORKSPACE and select(lib, pages(workspace=None), b) == WORKSPACE
    need = lib.tq_pages_pool_workspace_bytes(C.byref(p), 3)
    for q in (pages(workspace_bytes=need - 1), pages(workspace=None)):
        assert lib.tq_pages_fork(C.byref(q), C.byref(b), AT, AT, 3, None, None) == WORKSPACE
    need = lib.tq_pages_pool_workspace_bytes(C.byref(p), 0)
    for q in (pages(workspace_bytes=need - 1), pages(workspace=None)):
        assert lib.tq_pages_reserve(C.byref(q), C.byref(b), None, None) == WORKSPACE
        assert lib.tq_pages_compact(C.byref(q), C.byref(b), None, None) == WORKSPACE
    assert lib.tq_pages_pool_workspace_bytes(C.byref(p), -1) == 0


def test_nothing_to_do_is_fine(lib):
    for b in (batch(n_seqs=0), batch(max_new=0), batch(n_rows=0)):
        assert append(lib, pages(), b, k=None, v=None) == OK and attend(lib, pages(), b, q=None, out=None) == OK and select(lib, pages(), b, q=None) == OK
    assert lib.tq_pages_free(C.byref(pages()), C.byref(batch()), None, 0, None) == OK
    assert lib.tq_pages_copy(C.byref(pages()), None, None, 0, None) == OK


def test_the_binding_takes_gpu_tensors_of_the_right_kind():
    import paper_2504_19874_amd as tq
    k = torch.zeros(4, 2, 16, 64, dtype=torch.int8)
    with pytest.raises(tq.TurboQuantError, match="GPU tensor"):
        tq.Pages(k, k, torch.ones(4, 2), torch.ones(4, 2))


# --- the definition -----------------------------------------------------------------------------------------------------------


def test_codes_are_the_nearest():
    """Every e4m3 code is its own rounding, the middle of two neighbours goes to the even one, and torch's conversion agrees."""
    codes = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert codes[-1] == 448 and np.array_equal(po.round_code(codes, "e4m3"), codes)
    middle = (codes[1:] + codes[:-1]) / 2
    assert np.array_equal(po.round_code(middle, "e4m3"), np.where(np.arange(126) % 2 == 0, codes[:-1], codes[1:]))
    x = np.random.default_rng(1).standard_normal(20000) * np.exp(np.random.default_rng(2).normal(0, 3, 20000))
    x = np.clip(x.astype(np.float32), -448, 448)
    assert np.array_equal(po.round_code(x, "e4m3"), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())
    assert np.isnan(po.round_code([np.nan], "e4m3"))[0] and po.round_code([np.nan], "int8")[0] == 0 and po.round_code([1e9], "e4m3")[0] == 448
    assert list(po.round_code([0.5, 1.5, -2.5, 200], "int8")) == [0, 2, -2, 127]


def test_scales_are_the_smallest_that_hold():
    for kind, top in po.TOP.items():
        for amax in (1e-3, 0.7, top, top * 1.0001, 3.0, 1e4):
            s = po.scale_of(amax, kind)
            assert amax / s <= top < 2 * amax / s and np.log2(s) % 1 == 0
        assert po.scale_of(0, kind) == 2.0**-40 and po.scale_of(1e30, kind) == 2.0**40


def test_tokens_one_by_one_or_at_once():
    """Appending token by token gives the codes of the last scale; only the roundings on the way may add to them."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((10, 2, 64)) * np.exp(rng.normal(0, 1, (10, 1, 1)))
    for kind in po.TOP:
        empty = lambda: {n: np.zeros((2, 2, 16, 64)) for n in "kv"} | {n: np.ones((2, 2)) for n in ("k_scale", "v_scale")}  # noqa: E731
        once, each = empty(), empty()
        po.append(once, kind, 16, x, x, [[1]], [10], [0, 10])
        for i in range(10):
            po.append(each, kind, 16, x[i:i + 1], x[i:i + 1], [[1]], [i + 1], [0, 1])
        assert np.array_equal(once["k_scale"], each["k_scale"])
        a, b = (c["k"][1] * c["k_scale"][1][:, None, None] for c in (once, each))
        step = once["k_scale"][1][:, None, None] * np.maximum(1.0 if kind == "int8" else 2.0**-9, 0 if kind == "int8" else 2.0**-3 * np.abs(once["k"][1]))
        assert (np.abs(a - b) <= step + 1e-12).all()
        assert (np.abs(a[:, :10] - x.transpose(1, 0, 2)) <= step[:, :10] / 2 * 1.0000001).all()


def test_attention_of_the_definition():
    """One key: its value; equal keys: the mean; a window and chosen places see what they say."""
    c = {"k": np.zeros((3, 1, 16, 64)), "v": np.arange(48.0).reshape(3, 1, 16, 1) * np.ones(64), "k_scale": np.ones((3, 1)), "v_scale": np.ones((3, 1))}
    q = np.ones((3, 2, 64))
    out, lse, *_ = po.attend(c, 16, q, [[2, 0, -1]], [20], [0, 3], 0.1)
    assert np.allclose(out[2], np.r_[32:48, 0:4].mean()) and np.allclose(lse[2], np.log(20)) and np.allclose(out[0], np.r_[32:48, 0:2].mean())
    assert np.allclose(po.attend(c, 16, q, [[2, 0, -1]], [20], [0, 3], 0.1, window=2)[0][2], 2.5)
    assert np.allclose(po.attend(c, 16, q, [[2, 0, -1]], [20], [0, 3], 0.1, chosen=[[[1, -1]]] * 3)[0][2], 1.5)
    out, lse, *_ = po.attend(c, 16, q, [[-1, 5]], [20], [0, 3], 0.1)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_reserve_over_more_entries_than_it_counts(lib):
    for more in (dict(n_seqs=1 << 21, max_new=2**31 - 1, width=4096, table_stride=4096), dict(n_seqs=2**31 - 1, max_new=1, width=1, table_stride=1),
                 dict(n_seqs=1 << 30, max_new=129, width=2**31 - 1, table_stride=2**31 - 1)):
        assert lib.tq_pages_reserve(C.byref(pages()), C.byref(batch(**more)), None, None) == UNSUPPORTED
