"""Every kernel of ssd_paged_attention against attention in 64 bits: the batches of page_plans, ragged, some sequences outside the prefix."""
import math
import random

import pytest
import torch

from tests.page_plans import BATCHES, BF16, FP32, KERNELS, name, ragged
from tests.test_gpu_pages import U16, U32, Batch, i32, serve

pytestmark = pytest.mark.gpu

SMALLEST = [(k, bs[0]) for k, bs in KERNELS.items()]       # of every kernel


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_15380_amd as pkg
    pkg.load_library()


class Planned(Batch):
    """A batch of page_plans; every fifth sequence, where there are enough, does not have the prefix in front."""

    def __init__(self, case):
        (dtype, hd, *self.kernel), (nq, nkv, B, per, own, sb, bt, *self.parts) = case
        seqs, self.max_len = ragged(case[1])
        super().__init__(seqs, nq, nkv, hd, bt, dtype, seed=B + own, shared_blocks=sb, joins=[s % 5 != 4 for s in range(B)] if sb else None, pad=2)

    def run(self, **kw):
        import paper_2505_15380_amd as ssd
        plan = ssd.paged_attention_plan(ssd.Pages(self.keys, self.values), self.nq, len(self.rows), len(self.q) - 2, self.max_len, self.sb)
        assert plan == (*self.kernel, *self.parts)
        out = torch.full_like(self.q, 7.0)
        # (the rows behind the last one are no rows of the call)
        super().run(q=self.q[:-2], out=out[:-2], max_len=self.max_len, **kw)
        assert bool((out[-2:] == 7.0).all())
        return out[:-2]

    def mark(self):
        """1000 in one dim of the values at the edges of 64 keys, of the prefix and at the new rows: a key that is dropped, taken twice or seen too early moves that dim by far
        more than the roundings."""
        at = self.sb * self.bt
        for s, (n, r) in enumerate(zip(self.lens, self.rows)):
            p = torch.arange(n + r)
            p = p[(p % 64 == 0) | (p % 64 == 63) | (p >= n) | (p == at - 1) | (p == at)]
            d = (5 * p + p // 64) % self.hd
            blocks = self.table[s].clone()
            if self.sb and self.joins[s]:
                blocks[:self.sb] = torch.tensor(self.prefix)
            p, d, b = p.cuda(), d.cuda(), blocks[p // self.bt].cuda()
            self.values[b, :, d, p % self.bt] = 1000.0
            self.v[s][p, :, d] = 1000.0

    def oracle(self, s, scale, keep=None):
        o, e = super().oracle(s, scale, keep)
        # Tiles divide by the sum of the rounded weights p (1 + d), |d| <= u: off by sum p d (v - o) <= u (sum p |v| + |o|), the second term of which is added here.
        return o, e + (U16 * (1 + U16) * o.abs() if self.dtype == BF16 else 0)

    def block(self, s, i):
        return self.prefix[i] if self.sb and self.joins[s] and i < self.sb else int(self.table[s, i])


@pytest.mark.parametrize("case", BATCHES, ids=name)
def test_kernel(case):
    b = Planned(case)
    b.mark()
    out = b.run()
    assert b.status == 0
    b.check(out)
    assert torch.equal(out, b.run())


@pytest.mark.parametrize("case", SMALLEST, ids=name)
def test_kernel_without_some_pages(case):
    """A block of the prefix, one of a sequence's own, and all that a row sees."""
    b = Planned(case)
    n_blocks, bt = b.keys.shape[0], b.bt
    keep = [torch.ones(n + r, dtype=torch.bool, device="cuda") for n, r in zip(b.lens, b.rows)]
    bad = random.Random(1)
    if b.sb:
        gone = b.sb // 2
        b.prefix[gone] = n_blocks + 7
        for s, j in enumerate(b.joins):
            if j:
                keep[s][gone * bt:(gone + 1) * bt] = False
    for s, (n, r) in enumerate(zip(b.lens, b.rows)):
        first = b.sb if b.sb and b.joins[s] else 0
        have = -(-(n + r) // bt)
        if s % 3 == 0 and have > first:
            i = bad.randrange(first, have)
            b.table[s, i] = bad.choice([-1, -2 ** 31, n_blocks, 2 ** 31 - 1])
            keep[s][i * bt:(i + 1) * bt] = False
    alone = next((s for s, r in enumerate(b.rows) if r and not (b.sb and b.joins[s])), None)
    if alone is not None:
        b.table[alone] = -1
        keep[alone][:] = False
    out = b.run()
    b.check(out, keep=keep)
    assert b.status == 16
    if alone is not None:
        assert bool((out[b.start[alone]:b.start[alone + 1]] == 0).all())


@pytest.mark.parametrize("case", SMALLEST, ids=name)
def test_kernel_and_what_is_not_finite(case):
    """Infinities and NaN at new rows' positions are nothing to the rows before them, and come out at those that see them."""
    b = Planned(case)
    G, last = b.nq // b.nkv, b.nkv - 1
    expect = torch.zeros((b.n, b.nq, b.hd), dtype=torch.float64, device="cuda")
    seqs = [s for s, r in enumerate(b.rows) if r >= 2]
    assert seqs
    for s in seqs:
        n, r = b.lens[s], b.rows[s]
        put = [(r // 2, 3, math.inf), (r // 2, 5, math.nan), (r // 2, 8, -math.inf), (r // 2, 9, math.inf), (r - 1, 9, -math.inf), (r - 1, 31, math.inf)]
        if s % 4 == 3:                                     # a key instead
            b.keys[b.block(s, (n + r - 1) // b.bt), last, (n + r - 1) % b.bt] = math.nan
            expect[b.start[s] + r - 1, b.nq - G:] = math.nan
            continue
        if r == 2:                                         # (of two rows, the same one)
            put = [x for x in put if x[1] != 9]
        for row, d, x in put:
            b.values[b.block(s, (n + row) // b.bt), last, d, (n + row) % b.bt] = x
            expect[b.start[s] + row:b.start[s + 1], b.nq - G:, d] += x
    out = b.run().double()
    assert b.status == 0
    code = lambda t: torch.where(torch.isfinite(t), 0, t).nan_to_num(nan=1.0, posinf=2.0, neginf=3.0)      # noqa: E731
    assert torch.equal(code(out), code(expect))
    for s, r in enumerate(b.rows):
        if not r:
            continue
        o, e = b.oracle(s, b.hd ** -0.5)
        at = slice(b.start[s], b.start[s + 1])
        assert bool((((out[at] - o).abs() <= e) | (expect[at] != 0)).all()), s


@pytest.mark.parametrize("heads, seqs, sb", [((14, 2, 64), [(3000, 7), (2500, 30), (500, 90)], 0), ((12, 2, 128), [(n * 37 % 900, 8) for n in range(40)], 100),
                                             ((4, 4, 32), [(2000, 1)] * 60, 200), ((14, 2, 64), [(n % 300, 5) for n in range(250)], 300)])
def test_error_of_a_whole_result(heads, seqs, sb):
    """The norm of the error: an output is rounded once, and so is each weight.  A rounding of x by at most u |x| is a uniform one of at most half a step, which is u |x| / sqrt(3) in the root of
    the mean square or less (less by up to two, as x lies between powers of two); of one row's weights p they add up as sqrt(sum (p |v - o|)^2), or with |v| where the sum is that of the weights before they
    are rounded, since they are independent.  10 % for the spread of the
    mean over a few thousand rows, and for what is in fp32."""
    b = Batch(seqs, *heads, 16, BF16, seed=sb + len(seqs), shared_blocks=sb)
    out = b.run().double()
    err = size = 0.0
    G = b.nq // b.nkv
    for s, r in enumerate(b.rows):
        o, _ = b.oracle(s, b.hd ** -0.5)
        k, v = (t.double().repeat_interleave(G, 1).transpose(0, 1).contiguous() for t in (b.k[s], b.v[s]))
        q = b.q[b.start[s]:b.start[s + 1]].double().transpose(0, 1).contiguous()
        w = torch.bmm(q, k.transpose(1, 2).contiguous()) * b.hd ** -0.5
        p = torch.softmax(w.masked_fill(torch.arange(k.shape[1], device="cuda") > b.lens[s] + torch.arange(r, device="cuda")[:, None], -math.inf), -1)
        oo = o.transpose(0, 1).contiguous()
        # |v - o|^2 = |v|^2 - 2 v.o + |o|^2
        v2 = (v * v).sum(-1)[:, None]
        far = v2 - 2 * torch.bmm(oo, v.transpose(1, 2).contiguous()) + (oo * oo).sum(-1)[..., None]
        size += float((o * o).sum() + (p * p * torch.maximum(far, v2)).sum())
        err += float(((out[b.start[s]:b.start[s + 1]] - o) ** 2).sum())
    assert math.sqrt(err) <= 1.1 * U16 / math.sqrt(3) * math.sqrt(size)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_large_scores_pick_their_key(dtype):
    """Scores of 1e5: where the largest is apart from the next one by 200, far more than the roundings of a score (hd + 3 of 2^-24 of 1e6), its value is the result: times its
    weight, rounded (bf16: to bf16), and by its weight, the sum (a division and a product), and rounded to the type of the output."""
    b = Batch([(70, 3), (700, 20), (3, 90)], 4, 2, 64, 16, dtype, seed=9, spread=3e4)
    out = b.run()
    apart = 0
    for s in range(3):
        k, v = (t.double().repeat_interleave(2, 1).transpose(0, 1).contiguous() for t in (b.k[s], b.v[s]))
        q = b.q[b.start[s]:b.start[s + 1]].double().transpose(0, 1).contiguous()
        w = torch.bmm(q, k.transpose(1, 2).contiguous()) * 0.125
        w = w.masked_fill(torch.arange(k.shape[1], device="cuda") > b.lens[s] + torch.arange(q.shape[1], device="cuda")[:, None], -math.inf)
        top, at = w.topk(2, -1)
        clear = top[..., 0] - top[..., 1] > 200
        want = torch.gather(v, 1, at[..., :1].expand(-1, -1, 64)).transpose(0, 1)
        got = out[b.start[s]:b.start[s + 1]].double()
        clear = clear.transpose(0, 1)
        assert bool(((got - want).abs() <= want.abs() * (2.1 * U16 if dtype == BF16 else 4 * U32))[clear].all())
        apart += int(clear.sum())
    assert apart > 300


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_one_workspace_for_steps_of_all_sizes(dtype):
    """Sized for the largest, which itself needs none."""
    import paper_2505_15380_amd as ssd
    largest = Batch([(500, 64)] * 64, 14, 2, 64, 16, dtype, seed=5)
    pages = ssd.Pages(largest.keys, largest.values)
    most = ssd.paged_attention_workspace(pages, 14, 64, largest.n, 4096, 20)
    ws = torch.full((most,), 255, dtype=torch.uint8, device="cuda")
    assert ssd.paged_attention_plan(pages, 14, 64, largest.n, 564)[3] == 1
    largest.check(largest.run(ws=ws))
    cut = 0
    for seqs, sb in (([(n * 50, 1) for n in range(64)], 0), ([(n * 9, 3) for n in range(40)], 20), ([(3000, 2)], 0), ([(100, 200), (7, 1)], 3)):
        b = Batch(seqs, 14, 2, 64, 16, dtype, seed=sb, shared_blocks=sb)
        cut += ssd.paged_attention_plan(pages, 14, len(seqs), b.n, max(n + r for n, r in zip(b.lens, b.rows)), sb)[3] > 1
        out = b.run(ws=ws)
        b.check(out)
        assert torch.equal(out, b.run())
    assert cut >= 2


@pytest.mark.parametrize("dtype, heads, bt, voice, n_seqs", [(BF16, (14, 2, 64), 16, 4096, 30), (BF16, (4, 4, 32), 16, 1024, 40), (BF16, (4, 2, 128), 32, 2048, 40), (FP32, (2, 2, 64), 16, 1024, 30)])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_a_served_batch_with_a_prefix_of_its_own(dtype, heads, bt, voice, n_seqs, graph):
    """Served steps whose prefix is read once for all rows, in parts that are merged."""
    import paper_2505_15380_amd as ssd
    nq, nkv, hd = heads
    pages = ssd.Pages(torch.empty((1, nkv, bt, hd), dtype=dtype, device="cuda"), torch.empty((1, nkv, hd, bt), dtype=dtype, device="cuda"))
    sh, _, parts_sh, parts = ssd.paged_attention_plan(pages, nq, n_seqs, n_seqs * 20 + 5, voice + 6 * bt, voice // bt)
    assert sh > 0 and parts_sh > 1 and parts > 1
    serve(dtype, heads, bt, voice, n_seqs=n_seqs, steps=5, graph=graph)


@pytest.mark.parametrize("case", SMALLEST, ids=name)
def test_kernel_and_scores_of_minus_infinity(case):
    """A softmax whose scores are all -inf is NaN, as its formula is, and not the zeros of a row that has no position; with one finite score the others count for nothing."""
    b = Planned(case)
    b.q = b.q.abs() + 0.1
    G, L = b.nq // b.nkv, [n + r for n, r in zip(b.lens, b.rows)]
    keep = [torch.ones(n, dtype=torch.bool, device="cuda") for n in L]
    nothing = torch.zeros((b.n, b.nq), dtype=torch.bool, device="cuda")

    def low(s, positions):
        blocks = torch.tensor([b.block(s, int(p) // b.bt) for p in positions], dtype=torch.int64, device="cuda")
        b.keys[blocks, 0, positions.cuda() % b.bt, 1] = -math.inf
        keep[s][positions.cuda()] = False

    own = [b.sb * b.bt if b.sb and j else 0 for j in b.joins]
    for i, s in enumerate(s for s, r in enumerate(b.rows) if r):
        r = b.rows[s]
        if i % 4 == 0:                                     # all that its first rows see of its own keys; without a prefix, all that they see
            low(s, torch.arange(own[s], b.lens[s] + (r + 1) // 2))
            if not own[s]:
                nothing[b.start[s]:b.start[s] + (r + 1) // 2, :G] = True
        elif i % 4 == 1:                                   # the first 64, 128, ..: whole chunks, and parts
            low(s, torch.arange(own[s], own[s] + (b.lens[s] - own[s]) // 64 * 64))
        elif i % 4 == 2:
            low(s, torch.arange(own[s], L[s]))
            if not own[s]:
                nothing[b.start[s]:b.start[s + 1], :G] = True
    for turn in range(2 if b.sb else 1):
        if turn:                                           # and the whole prefix
            at = torch.tensor(b.prefix, device="cuda")
            b.keys[at, 0, :, 1] = -math.inf
            for s, j in enumerate(b.joins):
                if j:
                    keep[s][:own[s]] = False
                    seen = torch.arange(L[s], device="cuda") <= b.lens[s] + torch.arange(b.rows[s], device="cuda")[:, None]
                    nothing[b.start[s]:b.start[s + 1], :G] = ~(keep[s] & seen).any(-1)[:, None]
        out = b.run()
        assert b.status == 0
        assert torch.equal(torch.isnan(out).all(-1), nothing) and torch.equal(torch.isnan(out).any(-1), nothing)
        for s, r in enumerate(b.rows):
            if r:
                at = slice(b.start[s], b.start[s + 1])
                for heads, k in ((slice(0, G), keep[s]), (slice(G, None), None)):
                    o, e = b.oracle(s, b.hd ** -0.5, k)
                    assert bool((((out[at] - o).abs() <= e)[:, heads] | nothing[at, heads, None]).all()), (turn, s)
    assert bool(nothing.any())


@pytest.mark.parametrize("case", SMALLEST, ids=name)
def test_kernel_with_a_scale_of_zero(case):
    """Every position counts alike, but 0 times what is not finite is NaN: rows that see such a key, and rows whose query is one."""
    b = Planned(case)
    G = b.nq // b.nkv
    want = torch.zeros((b.n, b.nq), dtype=torch.bool, device="cuda")
    with_rows = [s for s, r in enumerate(b.rows) if r]
    for i, s in enumerate(with_rows):
        n, r, last = b.lens[s], b.rows[s], b.nkv - 1
        if i % 2 == 0:
            at = n + r // 2
            b.keys[b.block(s, at // b.bt), last, at % b.bt, 2] = math.inf if i % 4 else -math.inf
            want[b.start[s] + r // 2:b.start[s + 1], b.nq - G:] = True
        elif i % 4 == 1:
            b.q[b.start[s], 0, 7] = math.inf
            want[b.start[s], 0] = True
        else:
            b.q[b.start[s + 1] - 1, b.nq - 1, 7] = math.nan
            want[b.start[s + 1] - 1, b.nq - 1] = True
    out = b.run(scale=0.0)
    assert b.status == 0
    assert torch.equal(torch.isnan(out).all(-1), want) and torch.equal(~torch.isfinite(out).all(-1), want)
    b.q = torch.nan_to_num(b.q, nan=0.0, posinf=0.0)       # (the oracle takes every score as 0)
    for s in with_rows:
        o, e = b.oracle(s, 0.0)
        at = slice(b.start[s], b.start[s + 1])
        assert bool((((out[at] - o).abs() <= e) | want[at, :, None]).all()), s


@pytest.mark.parametrize("spread", [1e7, 1e10, 1e31])
@pytest.mark.parametrize("case", SMALLEST, ids=name)
def test_kernel_and_scores_of_any_size(case, spread):
    """Scores whose steps of 2^-24 are more than what a power of two can hold, and zeros among them: where the largest is apart from the next one by more than the roundings, its value is the
    result.  A score: hd products and their sum, the factors: (hd + 6) u of `size`, twice as they may go apart, and twice again."""
    b = Planned(case)
    b.q = (b.q * spread).to(b.dtype)
    b.keys[:, :, 1::2] = 0                                 # (every other position)
    for s in range(len(b.rows)):
        b.k[s][1::2] = 0
    out = b.run()
    assert b.status == 0 and bool(torch.isfinite(out).all())
    G, clear_rows, rows = b.nq // b.nkv, 0, 0
    for s, r in enumerate(b.rows):
        if not r:
            continue
        q = b.q[b.start[s]:b.start[s + 1]].double().transpose(0, 1).contiguous()
        k, v = (t.double().repeat_interleave(G, 1).transpose(0, 1).contiguous() for t in (b.k[s], b.v[s]))
        hidden = torch.arange(k.shape[1], device="cuda") > b.lens[s] + torch.arange(r, device="cuda")[:, None]
        w = (torch.bmm(q, k.transpose(1, 2).contiguous()) * b.hd ** -0.5).masked_fill(hidden, -math.inf)
        size = torch.bmm(q.abs(), k.abs().transpose(1, 2).contiguous()).masked_fill(hidden, 0).amax(-1) * b.hd ** -0.5
        top, at = torch.cat([w, torch.full_like(w[..., :1], -math.inf)], -1).topk(2, -1)
        clear = (top[..., 0] - top[..., 1] > 4 * (b.hd + 6) * U32 * size + 200).transpose(0, 1)
        want = torch.gather(v, 1, at[..., :1].clamp(max=k.shape[1] - 1).expand(-1, -1, b.hd)).transpose(0, 1)
        got = out[b.start[s]:b.start[s + 1]].double()
        assert bool(((got - want).abs() <= want.abs() * (2.1 * U16 if b.dtype == BF16 else 4 * U32))[clear].all()), s
        clear_rows, rows = clear_rows + int(clear.sum()), rows + clear.numel()
    assert clear_rows > 0.5 * rows


def test_scores_near_the_lowest_number_count():
    """fp32: scores of -2.2e38, and of that times log2(e) -3.2e38, are scores."""
    b = Batch([(100, 1), (0, 1), (700, 9)], 4, 2, 64, 16, FP32, seed=2)
    b.q[:], b.keys[:] = 0.0, 0.0
    b.q[..., 0], b.keys[..., 0] = 1e19, -2.2e19
    out = b.run(scale=1.0)
    for s in range(3):
        v = b.v[s].double().repeat_interleave(2, 1).cumsum(0)[b.lens[s]:]
        n = torch.arange(b.lens[s] + 1, b.lens[s] + b.rows[s] + 1, device="cuda")[:, None, None]
        size = b.v[s].double().abs().repeat_interleave(2, 1).cumsum(0)[b.lens[s]:] / n
        assert bool(((out[b.start[s]:b.start[s + 1]].double() - v / n).abs() <= size * 2 * (700 + 64) * U32).all())


@pytest.mark.parametrize("case", [c for c in SMALLEST if c[1][5]], ids=name)
def test_kernel_and_a_prefix_that_nobody_has(case):
    """Blocks of the prefix that are not in the pool are reported if some row would read them, and not if no sequence has the prefix in front."""
    (dtype, hd, *_), (nq, nkv, B, per, own, sb, bt, *_) = case
    b = Planned(case)
    b.joins = [False] * B
    for s in range(B):                                     # through their own tables, all of them
        if s % 5 != 4:
            b.table[s, :sb] = torch.tensor(b.prefix)
    b.prefix = [b.keys.shape[0] + i for i in range(sb)]
    b.check(b.run(shared=i32([0] * B)))
    assert b.status == 0
    some = next(s for s, r in enumerate(b.rows) if r and s % 5 != 4)
    b.run(shared=i32([sb if s == some else 0 for s in range(B)]))
    assert b.status == 16


@pytest.mark.parametrize("rows, bt", [(7, 16), (700, 64)])
def test_a_table_of_blocks_outside_the_pool_reaches_no_slot(rows, bt):
    """Ids that are no blocks, of which some shifted by the block size are slots of others: their rows get the slot 2^31 - 1, and an append leaves them out and says so."""
    import paper_2505_15380_amd as ssd
    wrong = [-1, 9, 1 << (32 - bt.bit_length() + 1), (1 << (32 - bt.bit_length() + 1)) + 3, -(1 << (32 - bt.bit_length() + 1)) + 2, 2 ** 31 - 1, -2 ** 31]
    B, cap = len(wrong) + 1, -(-rows // bt) + 1
    table = torch.full((B, cap), 0, dtype=torch.int32)
    for s, x in enumerate(wrong):
        table[s] = x
    table[-1] = 5
    owned = i32([cap] * B)
    assert rows * B > 4096 or rows < 10                    # (looked up by one launch, and by two)
    r = ssd.ssd_block_tables(i32([bt] * B), i32([min(rows, (cap - 1) * bt)] * B), bt, table.cuda(), owned, i32([0] * 9), i32([0]), rows * B)
    n = min(rows, (cap - 1) * bt)
    assert r["status"].item() == 0 and r["n_free"].item() == 0
    slot = r["row_slot"][:n * B].view(B, n)
    assert bool((slot[:-1] == 2 ** 31 - 1).all())
    assert slot[-1].tolist() == [5 * bt + p % bt for p in range(bt, bt + n)]
    keys, values = torch.zeros((9, 1, bt, 32), dtype=BF16, device="cuda"), torch.zeros((9, 1, 32, bt), dtype=BF16, device="cuda")
    status, k = i32([0]), torch.ones((n * (B - 1), 1, 32), dtype=BF16, device="cuda")
    ssd.ssd_rope_append(ssd.Pages(keys, values), r["row_pos"][:len(k)], r["row_slot"][:len(k)], k, k, status=status)
    assert status.item() == 16 and not bool(keys.any()) and not bool(values.any())


@pytest.mark.parametrize("change, bit", [("pool", 1), ("table", 2), ("rows", 4), ("len", 8), ("over", 8)])
def test_block_tables_of_many_rows_move_nothing_when_they_cannot(change, bit):
    """More rows than the one workgroup looks up itself: the launch behind it leaves none either."""
    import paper_2505_15380_amd as ssd
    bt, B, cap, n_blocks, max_rows = 16, 40, 30, 700, 6000
    lens, rows, owned, n_free = [20] * B, [140] * B, [2] * B, 600
    if change == "pool": n_free = 300
    if change == "table": lens[7] = cap * bt - 139
    if change == "rows": rows[3] = 600
    if change == "len": lens[39] = -1
    if change == "over": lens[0], rows[0], owned[0], n_free = 0, 0, 30, 690
    if change == "rows": cap = 60
    d = dict(table=(torch.arange(B * cap, dtype=torch.int32) % n_blocks).view(B, cap).cuda(), owned=i32(owned), free_stack=torch.arange(n_blocks, dtype=torch.int32).cuda(), n_free=i32([n_free]))
    kept = {k: v.clone() for k, v in d.items()}
    r = ssd.ssd_block_tables(i32(lens), i32(rows), bt, d["table"], d["owned"], d["free_stack"], d["n_free"], max_rows)
    assert r["status"].item() & bit
    for k, v in d.items():
        assert torch.equal(v, kept[k]), k
    assert torch.equal(r["owned"], kept["owned"]) and torch.equal(r["n_free"], kept["n_free"]) and not bool(r["row_start"].any())
    for k in ("row_seq", "row_pos", "row_slot"):
        assert bool((r[k] == -1).all())


def test_steps_without_rows():
    """Nothing is written and nothing asked for."""
    import paper_2505_15380_amd as ssd
    b = Batch([(40, 0), (7, 0)], 4, 2, 64, 16, BF16, seed=1, shared_blocks=1)
    pages, before = ssd.Pages(b.keys, b.values), b.keys.nan_to_num().clone()
    none = torch.empty((0, 4, 64), dtype=BF16, device="cuda")
    assert ssd.ssd_paged_attention(pages, none, i32(b.lens), i32([0, 0, 0]), i32(b.table), shared_table=i32(b.prefix)).shape == none.shape
    assert ssd.ssd_rope_append(pages, i32([]), i32([]), none[:, :2], none[:, :2], q=none).shape == none.shape
    padded = torch.full((5, 4, 64), 7.0, dtype=BF16, device="cuda")           # rows of the launch, of which no sequence has one
    out = padded.clone()
    ssd.ssd_paged_attention(pages, padded, i32(b.lens), i32([0, 0, 0]), i32(b.table), shared_table=i32(b.prefix), out=out, max_len=5000)
    assert torch.equal(out, padded) and torch.equal(b.keys.nan_to_num(), before)
    r = ssd.ssd_block_tables(i32(b.lens), i32([0, 0]), 16, torch.zeros((2, 9), dtype=torch.int32, device="cuda"), i32([4, 1]), i32([0] * 9), i32([2]), 3)
    assert r["status"].item() == 0 and r["row_start"].tolist() == [0, 0, 0] and r["row_slot"].tolist() == [-1] * 3 and r["owned"].tolist() == [4, 2]


@pytest.mark.parametrize("seqs, sb, hd", [([(50, 100), (700, 90)], 0, 128), ([(900, 700), (30, 900), (0, 800)], 0, 128), ([(n, 3) for n in range(30)], 60, 64),
                                          ([(n * 30, 1) for n in range(8)], 0, 32)])
def test_attention_and_append_over_a_pool_of_more_than_2_31_elements(seqs, sb, hd):
    """Tiles, streams and a prefix in blocks far apart; a third of the blocks are the pool's last."""
    import paper_2505_15380_amd as ssd
    bt, nkv = 16, 2
    n_blocks = (1 << 31) // (nkv * bt * hd) + 5000
    b = Batch(seqs, 4, nkv, hd, bt, BF16, seed=hd + sb, shared_blocks=sb, n_blocks=n_blocks)
    last = n_blocks - 1
    for s, r in enumerate(b.rows):                         # some of every sequence's blocks move to the end
        for i in range(sb, int((b.table[s] >= 0).sum()) + sb, 3):
            old = int(b.table[s, i])
            if old < 0 or last in (old, *b.prefix) or bool((b.table == last).any()):
                continue
            b.keys[last], b.values[last] = b.keys[old], b.values[old]
            b.table[s, i] = last
            last -= 1
    assert last < n_blocks - 3 and (last + 1) * nkv * bt * hd > 1 << 31
    b.check(b.run())
    assert b.status == 0
    rows = torch.randn((40, nkv, hd), device="cuda").to(BF16)
    slot = torch.arange(40) + (n_blocks - 3) * bt
    ssd.ssd_rope_append(ssd.Pages(b.keys, b.values), i32(list(range(40))), i32(slot), rows, rows)
    blk, tok = slot.cuda() // bt, slot.cuda() % bt
    assert torch.equal(b.keys[blk, :, tok], rows) and torch.equal(b.values[blk, :, :, tok], rows)
    del b
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("bt", [16, 64, 256, 1024])
@pytest.mark.parametrize("which", [0, 1, -1])
def test_one_block_of_a_sequence_is_there(dtype, bt, which):
    """The others are not: the rows that see it have its keys alone, NaN where the scores of these are -inf, and zeros where they see none; parts that begin inside a block too."""
    b = Batch([(3 * bt + 5, 3), (2 * bt + 70, 90), (2 * bt - 2, 5), (5000, 1)], 4, 2, 64, bt, dtype, seed=bt + which)
    b.q = b.q.abs() + 0.1
    keep = []
    for s, (n, r) in enumerate(zip(b.lens, b.rows)):
        have = -(-(n + r) // bt)
        i = which % have
        only = int(b.table[s, i])
        b.table[s, :] = -1
        b.table[s, i] = only
        b.keys[only, 0, :, 3] = -math.inf
        keep.append(torch.arange(n + r, device="cuda") // bt == i)
    out = b.run()
    assert b.status == 16
    for s, (n, r) in enumerate(zip(b.lens, b.rows)):
        seen = (keep[s] & (torch.arange(n + r, device="cuda") <= n + torch.arange(r, device="cuda")[:, None])).any(-1)
        got = out[b.start[s]:b.start[s + 1]]
        assert bool((torch.isnan(got[:, :2]) == seen[:, None, None]).all()) and bool((got[~seen] == 0).all())
        o, e = b.oracle(s, b.hd ** -0.5, keep[s])
        e = e + (U16 * (1 + U16) * o.abs() if dtype == BF16 else 0)
        assert bool(((got.double() - o).abs() <= e)[:, 2:].all())


@pytest.mark.parametrize("case", [c for c in SMALLEST if c[1][5]], ids=name)
def test_kernel_without_the_prefix(case):
    """No block of the prefix is in the pool, and the workspace holds NaN: every row has its own keys alone."""
    import paper_2505_15380_amd as ssd
    b = Planned(case)
    b.prefix = [b.keys.shape[0] + i for i in range(b.sb)]
    keep = [torch.arange(n + r, device="cuda") >= (b.sb * b.bt if j else 0) for n, r, j in zip(b.lens, b.rows, b.joins)]
    need = ssd.paged_attention_workspace(ssd.Pages(b.keys, b.values), b.nq, len(b.rows), b.n, b.max_len, b.sb)
    out = b.run(ws=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert b.status == 16
    b.check(out, keep=keep)
