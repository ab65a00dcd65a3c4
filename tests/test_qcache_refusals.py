"""Refusals of the 8-bit cache calls: made before anything is looked up on a device, so they run here."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2508_10259_amd import capi
    return capi.load()


def _cache(**kw):
    from paper_2508_10259_amd.capi import QCache
    base = dict(k=4096, v=4096, k_scale=4096, v_scale=4096, k_bounds=4096, page_table=4096, n_pages=8, n_kv_heads=2,
                head_dim=64, rows=2, pages_per_row=4)
    base.update(kw)
    return QCache(**base)


BAD_DIMS = [dict(head_dim=96), dict(head_dim=0), dict(n_kv_heads=0), dict(n_kv_heads=1025), dict(n_pages=0),
            dict(n_pages=(1 << 28) + 1), dict(rows=0), dict(rows=65536), dict(pages_per_row=0), dict(pages_per_row=16385)]


def _append(lib, c, n_tok=4, max_new=2, ldk=128, ldv=128, dtype=2, **kw):
    return lib.ams_qcache_append(C.byref(c) if c is not None else None, 64, 64, n_tok, max_new, 4096, ldk, 4096, ldv, dtype, None)


def _attend(lib, c, n_tok=4, max_new=2, max_len=100, n_heads=4, ldq=256, ldo=256, dtype=2, scale=0.1, n_select=0,
            selected=None, ws=4096, ws_bytes=1 << 30):
    return lib.ams_qcache_attend(C.byref(c) if c is not None else None, 64, 64, n_tok, max_new, max_len, n_heads, 4096, ldq,
                                 4096, ldo, dtype, scale, n_select, selected, ws, ws_bytes, None)


@pytest.mark.parametrize("bad", BAD_DIMS)
def test_dimensions(lib, bad):
    c = _cache(**bad)
    assert _append(lib, c) == -1 and _attend(lib, c) == -1 and lib.ams_last_error()
    assert lib.ams_qcache_workspace_bytes(C.byref(c), 4, 4, 2, 100, 0) == 0


def test_null_cache(lib):
    assert _append(lib, None) == -1 and _attend(lib, None) == -1
    assert lib.ams_qcache_workspace_bytes(None, 4, 4, 2, 100, 0) == 0


@pytest.mark.parametrize("bad", [dict(n_tok=-1), dict(max_new=0), dict(dtype=3), dict(dtype=-1)])
def test_append_arguments(lib, bad):
    assert _append(lib, _cache(), **bad) == -1


@pytest.mark.parametrize("bad", [dict(n_tok=-1), dict(max_new=0), dict(max_len=0), dict(n_heads=3), dict(n_heads=0),
                                 dict(dtype=5), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(n_select=-1), dict(n_select=16385),
                                 dict(selected=64), dict(ws=None, n_select=2), dict(ws=4104),
                                 dict(n_select=2, selected=66)])
def test_attend_arguments(lib, bad):
    assert _attend(lib, _cache(), **bad) == -1


def test_attend_workspace_too_small(lib):
    assert _attend(lib, _cache(), n_select=2, ws_bytes=8) == -6


def test_no_tokens_is_no_call(lib):
    assert _append(lib, _cache(), n_tok=0) == 0 and _attend(lib, _cache(), n_tok=0) == 0
    assert lib.ams_qcache_workspace_bytes(C.byref(_cache()), 4, 0, 2, 100, 0) >= 1


def test_too_large_a_launch(lib):
    c = _cache(rows=65535, n_kv_heads=1024)
    assert _append(lib, c, n_tok=1 << 30, max_new=1 << 20) == -1
    assert _attend(lib, c, n_tok=1 << 30, max_new=1 << 20, n_heads=1024) == -1


@pytest.mark.parametrize("n_tok", [1 << 23, (1 << 23) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("n_select", [0, 1])
def test_more_queries_than_an_int_counts_tiles(lib, n_tok, n_select):
    """65,536 heads on one KV head: 2^32 tiles of 128 queries and more."""
    c = _cache(n_kv_heads=1, head_dim=128, rows=1)
    assert lib.ams_qcache_workspace_bytes(C.byref(c), 65536, n_tok, n_tok, 100, n_select) == 0
    assert _attend(lib, c, n_tok=n_tok, max_new=n_tok, n_heads=65536, ldq=1 << 23, ldo=1 << 23, n_select=n_select,
                   ws_bytes=1 << 62) == -1


@pytest.mark.parametrize("n_tok", [(1 << 31) - 63, (1 << 31) - 62, (1 << 31) - 1])
def test_append_of_as_many_tokens_as_an_int_holds(lib, n_tok):
    c = _cache(n_kv_heads=1, rows=1)
    assert _append(lib, c, n_tok=n_tok, max_new=n_tok, ldk=64, ldv=64) == -1
    assert b"too many pages" in lib.ams_last_error()


ARRAYS = [(n, None) for n in ("k", "v", "k_scale", "v_scale", "k_bounds", "page_table", "tok_off", "kv_len")] + \
    [(n, 4096 + x) for n in ("k", "v", "k_bounds") for x in (1, 4, 8)] + \
    [(n, 4096 + x) for n in ("k_scale", "v_scale", "page_table", "tok_off", "kv_len") for x in (1, 2)]


@pytest.mark.parametrize("name,at", ARRAYS)
def test_arrays_missing_or_misaligned(lib, name, at):
    call = dict(tok_off=64, kv_len=64)
    c = _cache(**({} if name in call else {name: at}))
    if name in call:
        call[name] = at
    off, lens = call["tok_off"], call["kv_len"]
    assert lib.ams_qcache_append(C.byref(c), off, lens, 4, 2, 4096, 128, 4096, 128, 2, None) == -1
    assert lib.ams_qcache_attend(C.byref(c), off, lens, 4, 2, 100, 4, 4096, 256, 4096, 256, 2, 0.1, 0, None, 4096, 1 << 30,
                                 None) == -1


@pytest.mark.parametrize("dtype,es", [(0, 4), (1, 2), (2, 2)])
def test_tensors_missing_misaligned_or_overlapping_their_next_token(lib, dtype, es):
    c = _cache()

    def append(k=4096, v=4096, ldk=128, ldv=128):
        return lib.ams_qcache_append(C.byref(c), 64, 64, 4, 2, k, ldk, v, ldv, dtype, None)

    def attend(q=4096, out=4096, ldq=256, ldo=256):
        return lib.ams_qcache_attend(C.byref(c), 64, 64, 4, 2, 100, 4, q, ldq, out, ldo, dtype, 0.1, 0, None, 4096, 1 << 30, None)
    for bad in (None, 4096 + es // 2, 4096 + es + 1):
        assert append(k=bad) == append(v=bad) == attend(q=bad) == attend(out=bad) == -1
    for bad in (0, -128, 127, (1 << 40) + 1):
        assert append(ldk=bad) == append(ldv=bad) == -1
    for bad in (0, -256, 255, (1 << 40) + 1):
        assert attend(ldq=bad) == attend(ldo=bad) == -1


@pytest.mark.parametrize("dtype,es", [(0, 4), (1, 2), (2, 2)])
def test_tensors_whose_bytes_64_bits_do_not_count(lib, dtype, es):
    """2^40 elements between tokens: 2^63 bytes and a little, and four times as many, which once counted as one token's."""
    c = _cache(n_pages=1, n_kv_heads=1, rows=1)
    for bits in (63, 65):
        a = dict(n_tok=(1 << (bits - 40)) // es + 1, max_new=1, dtype=dtype)
        big = 1 << 40
        assert _append(lib, c, ldk=big, ldv=64, **a) == _append(lib, c, ldk=64, ldv=big, **a) == -1
        assert b"2^63 bytes" in lib.ams_last_error()
        for n_select in (0, 1):
            for ldq, ldo in ((big, 64), (64, big)):
                assert _attend(lib, c, n_heads=1, ldq=ldq, ldo=ldo, n_select=n_select, **a) == -1
                assert b"2^63 bytes" in lib.ams_last_error()


def test_workspace_grows_with_splits_and_lists(lib):
    c = _cache(rows=1, pages_per_row=4096)
    one = lib.ams_qcache_workspace_bytes(C.byref(c), 4, 1, 1, 64, 0)
    long = lib.ams_qcache_workspace_bytes(C.byref(c), 4, 1, 1, 1 << 18, 0)
    listed = lib.ams_qcache_workspace_bytes(C.byref(c), 4, 1, 1, 64, 8)
    assert one == 1 < long and listed == 2 * 8 * 4


def test_rows_are_cut_into_pieces_below_512_pairs_only(lib):
    """15 rows of 32 heads leave CUs idle at the ends of ragged rows, 16 fill the GPU by themselves."""
    sizes = [lib.ams_qcache_workspace_bytes(C.byref(_cache(rows=r, n_kv_heads=32, head_dim=128, pages_per_row=512)), 32, r, 1,
                                            32000, 0) for r in (15, 16, 20, 23, 24)]
    assert sizes[0] > 1 and sizes[1:] == [1] * 4


def test_contexts_keep_room_for_the_splits_of_a_few_rows(lib):
    """16 rows of 32 heads decode in one piece each, and an extension of some of them is cut: 32 pieces a row."""
    from paper_2508_10259_amd.capi import AMS_CTX_QCACHE, ModelCfg
    cfg = C.byref(ModelCfg(1, 2048, 32, 64, 1024, 256, 256, 1e-5, 1e4, 1))
    size = [lib.ams_ctx_workspace_bytes_paged(cfg, b, 1088, 8192, 0, AMS_CTX_QCACHE) for b in (15, 16, 23, 24)]
    parts = [n * 32 * 68 * 4 * p for n, p in ((15, 33), (16, 32), (23, 25), (24, 0))]  # (1,536 - pairs) / heads pieces
    row = 17 * (2 * 64 * 2048 + 32 * 8 + 2 * 2048)  # K/V, scales and bounds of a row's pages
    for n, a, b, pa, pb in zip((1, 7, 1), size, size[1:], parts, parts[1:]):
        assert 0 <= b - a - (pb - pa) - n * row < 0.15 * n * row


def test_python_checks():
    import torch
    from paper_2508_10259_amd.qcache import QuantCache
    c = QuantCache.empty(4, 2, 64, torch.zeros(1, 2, dtype=torch.int32))
    off, lens = torch.tensor([0, 3], dtype=torch.int32), torch.tensor([3], dtype=torch.int32)
    x = torch.zeros(3, 2, 64)
    for bad in (dict(k=x[:, :1]), dict(k=x.double()), dict(k=x.transpose(1, 2)), dict(tok_off=off[:1]), dict(tok_off=off.long()),
                dict(lens=torch.zeros(2, dtype=torch.int32)), dict(v=x.half())):
        a = dict(k=x, v=x, tok_off=off, lens=lens)
        a.update(bad)
        with pytest.raises(ValueError):
            c.append(**a)
    for bad in (dict(q=x.transpose(0, 1)), dict(out=x.half()), dict(out=x[:2])):
        a = dict(q=x, tok_off=off, lens=lens)
        a.update(bad)
        with pytest.raises(ValueError):
            c.attend(**a)
    with pytest.raises(ValueError):
        c.attend_selected(x, off, lens, 0)
    with pytest.raises(ValueError):
        c.attend_selected(x, off, lens, 2, selected=torch.zeros(3, 2, 3, dtype=torch.int32))
    with pytest.raises(ValueError):
        QuantCache(c.k, c.v, c.k_scale, c.v_scale[:2], c.k_bounds, c.page_table)


def test_context_flags(lib):
    from paper_2508_10259_amd.capi import AMS_CTX_QCACHE, AMS_CTX_SHARE_PREFIX, ModelCfg
    cfg = C.byref(ModelCfg(4, 512, 4, 128, 1024, 256, 256, 1e-5, 1e4, 1))
    size = [lib.ams_ctx_workspace_bytes_paged(cfg, 16, 1024, 0, 0, f) for f in
            (0, AMS_CTX_QCACHE, AMS_CTX_SHARE_PREFIX, AMS_CTX_QCACHE | AMS_CTX_SHARE_PREFIX, 4, 7)]
    kv = 4 * 2 * 16 * 1024 * 512 * 2
    assert 0.44 * kv <= size[0] - size[1] <= 0.5 * kv and size[2] - size[3] == size[0] - size[1]
    assert size[4] == size[5] == 0
    assert lib.ams_ctx_select_pages(None, 1) == -1
