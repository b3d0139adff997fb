"""What the calls on pages refuse before anything is launched.  CPU only: the device pointers are never followed."""
import ctypes as C
import os

import pytest
import torch

P = 1 << 12                                                # stands for a device pointer; 16-byte aligned
EINVAL, ENOMEM, ENOSUP = -1, -2, -4


@pytest.fixture(scope="module")
def lib():
    import paper_2505_15380_amd as pkg
    if not os.path.exists(pkg.library_path()):
        import __graft_entry__ as g
        g.build()
    return pkg.load_library()


def pages(**kw):
    from paper_2505_15380_amd.binding import _Pages
    d = dict(dev_keys=P, dev_values=P, n_blocks=8, n_kv_heads=2, block_tokens=16, head_dim=64, dtype=1)
    d.update(kw)
    return _Pages(*[d[n] for n, _ in _Pages._fields_])


TABLES = dict(n_seqs=2, bt=16, n_blocks=8, cap=4, max_rows=2, len=P, rows=P, shared=None, owned=P, n_free=P, table=P, stack=P, owned_out=P, n_free_out=P, row_start=P,
              row_seq=P, row_pos=P, row_slot=P, status=P, stream=None)


@pytest.mark.parametrize("change, code", [
    (dict(n_seqs=0), EINVAL), (dict(max_rows=0), EINVAL), (dict(cap=0), EINVAL), (dict(n_blocks=0), EINVAL), (dict(n_seqs=4097), ENOSUP), (dict(bt=8), ENOSUP),
    (dict(bt=24), ENOSUP), (dict(bt=2048), ENOSUP), (dict(n_blocks=1 << 27), EINVAL), (dict(cap=(1 << 26) + 1), ENOSUP), (dict(max_rows=(1 << 30) + 1), ENOSUP),
] + [({k: None}, EINVAL) for k in TABLES if k not in ("shared", "stream", "n_seqs", "bt", "n_blocks", "cap", "max_rows")])
def test_block_tables_refuses(lib, change, code):
    assert lib.ssd_block_tables(*{**TABLES, **change}.values()) == code
    assert lib.ssd_last_error()


APPEND = dict(pages=None, n_rows=3, nq=4, q=P, qs=256, k=P, ks=128, v=P, vs=128, rope=P, positions=8, pos=P, slot=P, q_out=P, os=256, status=None, stream=None)


@pytest.mark.parametrize("change, code", [
    (dict(n_rows=-1), EINVAL), (dict(n_rows=(1 << 24) + 1), EINVAL), (dict(nq=-1), EINVAL), (dict(q=None), EINVAL), (dict(q_out=None), EINVAL), (dict(k=None), EINVAL),
    (dict(v=None), EINVAL), (dict(pos=None), EINVAL), (dict(slot=None), EINVAL), (dict(positions=0), EINVAL), (dict(qs=255), EINVAL), (dict(qs=260), EINVAL), (dict(os=128), EINVAL),
    (dict(ks=120), EINVAL), (dict(vs=132), EINVAL), (dict(k=P + 8), EINVAL), (dict(q=P + 2), EINVAL), (dict(os=264), EINVAL),
])
def test_rope_append_refuses(lib, change, code):
    pg = pages()
    args = {**APPEND, "pages": C.byref(pg), **change}
    assert lib.ssd_rope_append(*args.values()) == code
    assert lib.ssd_last_error()


ATTEND = dict(pages=None, nq=4, scale=0.125, n_seqs=2, n_rows=3, max_len=100, len=P, row_start=P, table=P, cap=8, shared_blocks=1, shared_table=P, shared=None, q=P, qs=256, out=P,
              os=256, ws=P, ws_bytes=1 << 30, status=None, stream=None)
LONG = dict(max_len=16000, cap=1000)                                           # keys that are read in parts: that takes a workspace


@pytest.mark.parametrize("change, code", [
    (dict(nq=3), EINVAL), (dict(nq=0), EINVAL), (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=3e38), EINVAL), (dict(n_seqs=0), EINVAL), (dict(n_seqs=(1 << 16) + 1), EINVAL),
    (dict(n_rows=-1), EINVAL), (dict(n_rows=(1 << 24) + 1), ENOSUP), (dict(max_len=0), EINVAL), (dict(len=None), EINVAL), (dict(row_start=None), EINVAL), (dict(table=None), EINVAL),
    (dict(shared_table=None), EINVAL), (dict(shared_blocks=-1), EINVAL), (dict(cap=0), EINVAL), (dict(cap=(1 << 26) + 1), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL),
    (dict(qs=100), EINVAL), (dict(os=258), EINVAL), (dict(ws=None, **LONG), EINVAL), (dict(ws=P + 4, **LONG), EINVAL), (dict(ws_bytes=0, **LONG), ENOMEM),
])
def test_paged_attention_refuses(lib, change, code):
    pg = pages()
    args = {**ATTEND, "pages": C.byref(pg), **change}
    assert lib.ssd_paged_attention(*args.values()) == code
    assert lib.ssd_last_error()


@pytest.mark.parametrize("change, code", [
    (dict(dev_keys=None), EINVAL), (dict(dev_values=None), EINVAL), (dict(dev_keys=P + 8), EINVAL), (dict(n_blocks=0), EINVAL), (dict(n_kv_heads=0), EINVAL), (dict(block_tokens=48), ENOSUP),
    (dict(block_tokens=8), ENOSUP), (dict(head_dim=96), ENOSUP), (dict(dtype=2), EINVAL), (dict(n_blocks=1 << 27), EINVAL),
])
def test_pages_are_checked_by_every_call(lib, change, code):
    pg = pages(**change)
    assert lib.ssd_rope_append(*{**APPEND, "pages": C.byref(pg)}.values()) == code
    assert lib.ssd_paged_attention(*{**ATTEND, "pages": C.byref(pg)}.values()) == code
    assert lib.ssd_paged_attention_workspace_bytes(C.byref(pg), 4, 2, 3, 100, 1) == C.c_size_t(-1).value


def test_no_rows_is_no_work(lib):
    pg = pages()
    assert lib.ssd_rope_append(*{**APPEND, "pages": C.byref(pg), "n_rows": 0}.values()) == 0
    assert lib.ssd_paged_attention(*{**ATTEND, "pages": C.byref(pg), "n_rows": 0, "ws": None, "ws_bytes": 0}.values()) == 0


def test_the_binding_refuses_what_it_can_see():
    import paper_2505_15380_amd as ssd
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    v = torch.zeros((4, 2, 64, 16), dtype=torch.bfloat16)
    for bad in (v.float(), v.transpose(2, 3), v[:3], torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), v.half()):
        with pytest.raises(ssd.SSDError):
            ssd.Pages(k, bad)
    with pytest.raises(ssd.SSDError):
        ssd.Pages(k.half(), v.half())
    pg = ssd.Pages(k, v)
    rows = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    for bad in (rows.float(), rows[:, :1], rows.transpose(0, 1), rows[:, :, :32]):
        with pytest.raises(ssd.SSDError):
            pg.rows("k", bad, 2)
    with pytest.raises(ssd.SSDError):                      # not on a GPU
        ssd.ssd_rope_append(pg, torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), rows, rows)


def test_launches_of_more_threads_than_a_grid_has_are_refused(lib):
    """2^32 threads and more; workgroups have 256, or 512."""
    many = pages(n_kv_heads=1024)
    assert lib.ssd_rope_append(*{**APPEND, "pages": C.byref(many), "n_rows": 1 << 24, "ks": 1 << 16, "vs": 1 << 16, "qs": 1 << 16, "os": 1 << 16}.values()) == ENOSUP
    args = {**ATTEND, "pages": C.byref(many), "nq": 1024, "qs": 1 << 16, "os": 1 << 16, "shared_blocks": 0, "n_seqs": 1 << 16, "n_rows": 1 << 16}
    assert lib.ssd_paged_attention(*args.values()) == ENOSUP
    assert lib.ssd_last_error()
