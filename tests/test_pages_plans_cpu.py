"""Which kernel ssd_paged_attention picks.  CPU only: nothing is launched."""
import ctypes as C
import os
import random
import re

import pytest

from tests.page_plans import BATCHES, BF16, KERNELS, name
from tests.test_kernel_resources_cpu import _code_objects, _kernels

P = 1 << 12                                                # stands for a device pointer; 16-byte aligned


@pytest.fixture(scope="module")
def lib():
    import paper_2505_15380_amd as pkg
    if not os.path.exists(pkg.library_path()):
        import __graft_entry__ as g
        g.build()
    return pkg.load_library()


def pages(dtype, hd, nkv, bt, n_blocks=1 << 16):
    from paper_2505_15380_amd.binding import _Pages
    return _Pages(P, P, n_blocks, nkv, bt, hd, 1 if dtype == BF16 else 0)


@pytest.mark.parametrize("case", BATCHES, ids=name)
def test_a_batch_reaches_its_kernel(lib, case):
    (dtype, hd, sh, own), (nq, nkv, B, per, most, sb, bt, parts_sh, parts) = case
    pg, plan = pages(dtype, hd, nkv, bt), (C.c_int * 4)()
    assert lib.ssd_paged_attention_plan(C.byref(pg), nq, B, B * per, sb * bt + most + per, sb, plan) == 0
    assert tuple(plan) == (sh, own, parts_sh, parts)


def test_every_kernel_of_the_library_has_a_batch(lib):
    import paper_2505_15380_amd as pkg
    blob = open(pkg.library_path(), "rb").read()
    names = [k[".name"] for elf in _code_objects(blob) for k in _kernels(elf)]
    there = {m.groups() for m in (re.search(r"k_paged_attentionINS_\d(BF16|F32)ELi(\d+)ELi(\d)ELi(\d)E", n) for n in names) if m}
    assert there == {("BF16" if t == BF16 else "F32", str(hd), str(sh), str(own)) for t, hd, sh, own in KERNELS}
    assert len(there) == 45


def test_plan_refuses_what_the_call_refuses(lib):
    pg, plan = pages(BF16, 64, 2, 16), (C.c_int * 4)()
    ref = C.byref(pg)
    assert lib.ssd_paged_attention_plan(ref, 14, 2, 2, 100, 0, plan) == 0
    for args in ((None, 14, 2, 2, 100, 0, plan), (ref, 13, 2, 2, 100, 0, plan), (ref, 14, 0, 2, 100, 0, plan), (ref, 14, 2, 0, 100, 0, plan), (ref, 14, 2, 2, 0, 0, plan),
                 (ref, 14, 2, 2, 100, -1, plan), (ref, 14, 2, 2, 100, 0, None)):
        assert lib.ssd_paged_attention_plan(*args) == -1
        assert lib.ssd_last_error()


def test_a_workspace_is_enough_for_every_smaller_call(lib):
    """A caller asks once, for the largest step."""
    rng = random.Random(2)
    size = lambda lo, hi: min(hi, int(lo * (hi / lo) ** rng.random() * rng.choice([1, 1, 1.3])))      # noqa: E731
    plan = (C.c_int * 4)()
    for _ in range(20000):
        nkv, group, hd, dtype, bt = rng.choice([1, 2, 4, 8]), rng.choice([1, 3, 6, 7, 8]), rng.choice([32, 64, 128]), rng.choice([BF16, BF16, 0]), rng.choice([16, 64])
        ref, nq = C.byref(pages(dtype, hd, nkv, bt)), nkv * group
        n_seqs, n_rows, max_len, sb = size(1, 2000), size(1, 30000), size(1, 60000), rng.choice([0, size(1, 1000)])
        most = lib.ssd_paged_attention_workspace_bytes(ref, nq, n_seqs, n_rows, max_len, sb)
        for _ in range(3):
            small = size(1, n_rows)
            assert lib.ssd_paged_attention_plan(ref, nq, size(1, n_seqs), small, size(1, max_len), rng.choice([0, sb, rng.randint(0, sb)]), plan) == 0
            assert plan[3] == 1 or small * nq * plan[3] * (hd + 2) * 4 <= most
    assert lib.ssd_paged_attention_workspace_bytes(ref, nq, 9, 0, 5000, 7) == 0
    assert lib.ssd_paged_attention_workspace_bytes(ref, nq, 9, 4000, 64, 0) == 0                       # one chunk of keys: nothing to cut
