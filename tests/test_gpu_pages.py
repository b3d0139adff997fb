"""Block tables, rotary embedding with the append, and attention with a shared prefix, alone and together, against plain forms in 64 bits.

A rounding is off by at most half a step: u = eps / 2 of the value, 2^-8 in bf16 and 2^-24 in fp32."""
import math
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2505_15380_amd as pkg
    pkg.load_library()


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


# ---------------------------------------------------------------------------------------------- block tables
class Walk:
    """The bookkeeping as a serial walk over lists."""

    def __init__(self, n_blocks, bt, cap, rng):
        ids = list(range(n_blocks))
        rng.shuffle(ids)
        self.bt, self.cap, self.free, self.table, self.n_blocks = bt, cap, ids, [], n_blocks

    def admit(self, shared=()):
        self.table.append(list(shared))

    def step(self, lens, rows, shared):
        need = [max(0, -(-(n + r) // self.bt) - s) + s for n, r, s in zip(lens, rows, shared)]
        for t, n, s in zip(self.table, need, shared):
            while len(t) > max(n, s):
                self.free.append(t.pop())
        for t, n in zip(self.table, need):
            while len(t) < n:
                t.append(self.free.pop())
        start, out = [0], []
        for s, (n, r) in enumerate(zip(lens, rows)):
            start.append(start[-1] + r)
            out += [(s, p, self.table[s][p // self.bt] * self.bt + p % self.bt) for p in range(n, n + r)]
        return start, out


def device_tables(walk, shared):
    B = len(walk.table)
    table = torch.full((B, walk.cap), -7, dtype=torch.int32)
    for s, t in enumerate(walk.table):
        table[s, :len(t)] = torch.tensor(t, dtype=torch.int32)
    stack = torch.full((walk.n_blocks,), -9, dtype=torch.int32)
    stack[:len(walk.free)] = torch.tensor(walk.free, dtype=torch.int32)
    return dict(table=table.cuda(), free_stack=stack.cuda(), owned=i32([len(t) - s for t, s in zip(walk.table, shared)]), n_free=i32([len(walk.free)]))


@pytest.mark.parametrize("B, bt, top, in_place", [(1, 16, 1, True), (1, 16, 700, False), (3, 64, 40, False), (64, 16, 1, True), (65, 32, 9, False), (300, 16, 130, True), (1024, 16, 3, False),
                                                  (1025, 16, 5, True), (4096, 16, 2, False)])
def test_block_tables_follow_the_serial_walk(B, bt, top, in_place):
    """Steps of a server: requests begin, grow, are cut back, end, and begin again in the blocks that others gave back."""
    import paper_2505_15380_amd as ssd
    rng = random.Random(1000 * B + top)
    n_sh = rng.choice([0, 3])
    reach = 12 * bt + 4 * top
    cap = n_sh + reach // bt + 2
    walk = Walk(n_sh + B * (reach // bt + 1) + 5, bt, cap, rng)
    head = [walk.free.pop() for _ in range(n_sh)]
    shared = [n_sh if rng.random() < 0.7 else 0 for _ in range(B)]
    for s in shared:
        walk.admit(head[:s])
    dev = device_tables(walk, shared)
    lens, rows = [s * bt for s in shared], [0] * B
    for step in range(4):
        for s in range(B):
            lens[s] += rows[s]
            what = rng.random()
            base = shared[s] * bt
            if what < 0.2:
                lens[s], rows[s] = rng.choice([0, base]), 0                      # over: everything of its own goes back
            elif what < 0.3:
                lens[s] = base + rng.randrange(lens[s] - base + 1) if lens[s] > base else base            # rolled back
                rows[s] = 1
            else:
                lens[s] = max(lens[s], base)
                rows[s] = rng.randint(0, top)
        max_rows = max(1, sum(rows) + rng.choice([0, 0, 3]))
        start, out = walk.step(lens, rows, shared)
        before = dev["table"].clone()
        o = None
        if in_place:
            e = lambda n: torch.full((n,), -5, dtype=torch.int32, device="cuda")      # noqa: E731
            o = dict(owned=dev["owned"], n_free=dev["n_free"], row_start=e(B + 1), row_seq=e(max_rows), row_pos=e(max_rows), row_slot=e(max_rows), status=e(1))
        r = ssd.ssd_block_tables(i32(lens), i32(rows), bt, dev["table"], dev["owned"], dev["free_stack"], dev["n_free"], max_rows,
                                 shared=i32(shared) if n_sh else None, out=o)
        dev["owned"], dev["n_free"] = r["owned"], r["n_free"]
        assert r["status"].tolist() == [0]
        assert r["n_free"].tolist() == [len(walk.free)]
        assert dev["free_stack"][:len(walk.free)].tolist() == walk.free
        assert r["owned"].tolist() == [len(t) - s for t, s in zip(walk.table, shared)]
        assert r["row_start"].tolist() == start
        rest = [-1] * (max_rows - len(out))
        for k, name in enumerate(("row_seq", "row_pos", "row_slot")):
            assert r[name].tolist() == [x[k] for x in out] + rest, name
        got, was = dev["table"].tolist(), before.tolist()
        for s, t in enumerate(walk.table):
            assert got[s][:len(t)] == t and got[s][len(t):] == was[s][len(t):], s


@pytest.mark.parametrize("change, bit", [("pool", 1), ("table", 2), ("rows", 4), ("len", 8), ("row", 8), ("owned", 8), ("shared", 8), ("free", 8), ("over", 8), ("large", 2), ("sum", 4)])
def test_block_tables_move_nothing_when_they_cannot(change, bit):
    import paper_2505_15380_amd as ssd
    bt, B, cap = 16, 5, 8
    lens, rows, owned, n_free, max_rows, shared = [20, 0, 33, 16, 5], [1, 17, 1, 2, 0], [2, 0, 5, 1, 1], 12, 30, [0] * B
    if change == "pool": n_free, owned = 1, [2, 0, 3, 1, 1]
    if change == "table": lens[1] = 127
    if change == "rows": max_rows = 20
    if change == "len": lens[2] = -1
    if change == "row": rows[3] = -2
    if change == "owned": owned[0] = -1
    if change == "shared": shared[3] = 2                   # new rows among the positions of its shared blocks
    if change == "free": n_free = 31
    if change == "over": n_free = 29                       # with the two blocks given back, more than there are
    if change == "large": lens[4], rows[4] = 0x7FFFFFFF, 0x7FFFFFFF
    if change == "sum": rows = [100, 0, 60, 0, 0]; lens = [0] * 5
    d = dict(table=torch.arange(B * cap, dtype=torch.int32).view(B, cap).cuda(), owned=i32(owned), free_stack=torch.arange(30, dtype=torch.int32).cuda(), n_free=i32([n_free]))
    kept = {k: v.clone() for k, v in d.items()}
    r = ssd.ssd_block_tables(i32(lens), i32(rows), bt, d["table"], d["owned"], d["free_stack"], d["n_free"], max_rows, shared=i32(shared))
    assert r["status"].item() & bit and r["status"].item() < 16
    for k, v in d.items():
        assert torch.equal(v, kept[k]), k
    assert torch.equal(r["owned"], kept["owned"]) and torch.equal(r["n_free"], kept["n_free"])
    assert r["row_start"].tolist() == [0] * (B + 1)
    for name in ("row_seq", "row_pos", "row_slot"):
        assert r[name].tolist() == [-1] * max_rows


# ---------------------------------------------------------------------------------------------- rotary embedding and append
def rope_table(positions, hd, base=1e4):
    f = base ** (-torch.arange(hd // 2, dtype=torch.float64) * 2.0 / hd)
    a = torch.arange(positions, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().cuda()


def turned(x, cs):
    """x [n, heads, hd], cs [n, hd / 2, 2]: what it is turned to and a bound of the error, both in 64 bits."""
    h = x.shape[2] // 2
    x, c, s = x.double(), cs[:, None, :, 0].double(), cs[:, None, :, 1].double()
    a, b = x[..., :h], x[..., h:]
    y = torch.cat([a * c - b * s, b * c + a * s], -1)
    size = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()], -1)
    return y, 2.1 * U32 * size                             # two products, or one and a fused one, and a sum: each off by u of no more than `size`


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("nq, nkv, hd, bt", [(14, 2, 64, 16), (12, 2, 128, 32), (4, 4, 32, 16), (1, 1, 64, 128), (5, 5, 128, 16), (0, 3, 64, 64)])
@pytest.mark.parametrize("n, packed, in_place", [(1, True, False), (7, True, True), (16, False, False), (67, True, False), (130, False, True)])
def test_rope_append(dtype, nq, nkv, hd, bt, n, packed, in_place):
    import paper_2505_15380_amd as ssd
    g = torch.Generator("cuda").manual_seed(n * 31 + hd + nq)
    rng = random.Random(n + hd)
    n_blocks = -(-n // bt) * 2 + 3
    first = rng.randrange(0, 5 * bt)
    # runs of positions behind each other, as prompts have them, and single ones; some rows have no position, some no slot
    pos = list(range(first, first + n))
    ids = rng.sample(range(n_blocks), n_blocks)
    slot = [ids[(p - first + first % bt) // bt] * bt + p % bt for p in pos]
    for r in range(n):
        if n > 4 and rng.random() < 0.1: slot[r] = -1
        if n > 4 and rng.random() < 0.1: pos[r] = slot[r] = -1
    rope = rope_table(first + n, hd)
    draw = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)      # noqa: E731
    keys, values = draw(n_blocks, nkv, bt, hd), draw(n_blocks, nkv, hd, bt)
    if packed:
        qkv = draw(n, (nq + 2 * nkv) * hd + 16)
        q, k, v = (t.unflatten(1, (-1, hd)) if t.shape[1] else None for t in qkv[:, :-16].split([nq * hd, nkv * hd, nkv * hd], 1))
    else:
        q, k, v = draw(n, nq, hd) if nq else None, draw(n, nkv, hd), draw(n, nkv, hd)
    q0 = q.clone() if nq else None
    k0, v0, keys0, values0 = k.clone(), v.clone(), keys.clone(), values.clone()
    status = i32([0])
    out = q if in_place and nq else torch.full((n, nq, hd), 3.0, dtype=dtype, device="cuda") if nq else None
    old = out.clone() if nq else None
    got = ssd.ssd_rope_append(ssd.Pages(keys, values), i32(pos), i32(slot), k, v, q=q, rope=rope, q_out=out, status=status)
    assert status.item() == 0
    u = U16 if dtype == BF16 else 0.0
    p = torch.tensor(pos).clamp(min=0).cuda()
    there = (torch.tensor(pos) >= 0).cuda()
    if nq:
        y, e = turned(q0, rope[p])
        assert bool((((got.double() - y).abs() <= e + u * (y.abs() + e)) | ~there[:, None, None]).all())
        assert torch.equal(got[~there], old[~there])
    y, e = turned(k0, rope[p])
    want_k, want_v, mask = keys0.double(), values0.clone(), torch.zeros_like(keys0, dtype=torch.float64)
    for r in range(n):
        if slot[r] >= 0:
            want_k[slot[r] // bt, :, slot[r] % bt] = y[r]
            mask[slot[r] // bt, :, slot[r] % bt] = e[r] + u * (y[r].abs() + e[r])
            want_v[slot[r] // bt, :, :, slot[r] % bt] = v0[r]
    assert bool(((keys.double() - want_k).abs() <= mask).all())
    assert torch.equal(values, want_v)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rope_append_without_angles_copies(dtype):
    """Bit by bit, whatever the values are."""
    import paper_2505_15380_amd as ssd
    keys = torch.zeros((4, 2, 16, 64), dtype=dtype, device="cuda")
    values = torch.zeros((4, 2, 64, 16), dtype=dtype, device="cuda")
    x = torch.randn((20, 8, 64), device="cuda").to(dtype)
    x[3, :, 40:] = math.inf
    x[5, 1, 7], x[6, 6, 60], x[7, 3, :] = math.nan, -math.inf, -0.0
    slot = torch.randperm(64)[:20]
    q = ssd.ssd_rope_append(ssd.Pages(keys, values), i32(range(20)), i32(slot), x[:, 4:6], x[:, 6:], q=x[:, :4])
    same = lambda a, b: torch.equal(a.contiguous().view(torch.int16 if dtype == BF16 else torch.int32), b.contiguous().view(torch.int16 if dtype == BF16 else torch.int32))      # noqa: E731
    assert same(q, x[:, :4])
    b, t = slot.cuda() // 16, slot.cuda() % 16
    assert same(keys[b, :, t], x[:, 4:6]) and same(values[b, :, :, t], x[:, 6:])


def test_rope_append_leaves_out_what_lies_outside():
    import paper_2505_15380_amd as ssd
    n, nkv, hd, bt = 6, 2, 64, 16
    k = torch.randn((n, nkv, hd), device="cuda").to(BF16)
    keys, values = torch.zeros((2, nkv, bt, hd), dtype=BF16, device="cuda"), torch.zeros((2, nkv, hd, bt), dtype=BF16, device="cuda")
    for pos, slot, bit in (([0, 1, 9, 3, 4, 5], [0, 1, 2, 3, 4, 5], 8), ([0, 1, 2, 3, 4, 5], [0, 1, 32, 3, 0x7FFFFFFF, 5], 16)):
        keys.zero_(), values.zero_()
        status = i32([0])
        ssd.ssd_rope_append(ssd.Pages(keys, values), i32(pos), i32(slot), k, k, rope=rope_table(8, hd), status=status)
        assert status.item() == bit
        bad = {r for r in range(n) if pos[r] >= 8 or slot[r] >= 32}
        for s in range(32):
            r = slot.index(s) if s in slot else None
            empty = r is None or r in bad
            assert bool((keys[s // bt, :, s % bt] == 0).all()) == empty
            assert empty or torch.equal(values[s // bt, :, :, s % bt], k[r])
    # no table of angles: keys as they are
    ssd.ssd_rope_append(ssd.Pages(keys, values), i32(range(n)), i32(range(n)), k, k)
    assert torch.equal(keys[0, :, :n], k.transpose(0, 1))


# ---------------------------------------------------------------------------------------------- attention
class Batch:
    """Sequences over pages in a random order, whose unwritten positions are NaN."""

    def __init__(self, seqs, nq, nkv, hd, bt, dtype, seed, shared_blocks=0, joins=None, pad=0, spread=1.5, table_pad=2, n_blocks=None):
        """seqs: (cached positions beyond the shared ones, new rows).  joins: which sequences have the prefix in front (default all)."""
        g = torch.Generator("cuda").manual_seed(seed)
        rng = random.Random(seed)
        B = len(seqs)
        self.nq, self.nkv, self.hd, self.bt, self.dtype, self.sb = nq, nkv, hd, bt, dtype, shared_blocks
        self.joins = joins if joins is not None else [True] * B
        self.lens = [n + (shared_blocks * bt if j else 0) for (n, _), j in zip(seqs, self.joins)]
        self.rows = [r for _, r in seqs]
        have = [-(-(n + r) // bt) for n, r in zip(self.lens, self.rows)]
        cap = max(have) + table_pad
        total = shared_blocks + sum(h - (shared_blocks if j else 0) for h, j in zip(have, self.joins)) + 3
        n_blocks = n_blocks or total
        ids = rng.sample(range(n_blocks), total)
        self.prefix, ids = ids[:shared_blocks], ids[shared_blocks:]
        self.keys = torch.empty((n_blocks, nkv, bt, hd), dtype=dtype, device="cuda")
        self.values = torch.empty((n_blocks, nkv, hd, bt), dtype=dtype, device="cuda")
        if n_blocks == total:
            self.keys.fill_(math.nan), self.values.fill_(math.nan)
        self.table = torch.full((B, cap), -1, dtype=torch.int64)
        draw = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)      # noqa: E731
        pk, pv = draw(shared_blocks * bt, nkv, hd), draw(shared_blocks * bt, nkv, hd)
        self.put(self.prefix, 0, pk, pv)
        self.k, self.v = [], []
        for s in range(B):
            j = shared_blocks if self.joins[s] else 0
            mine = [ids.pop() for _ in range(have[s] - j)]
            self.table[s, j:have[s]] = torch.tensor(mine, dtype=torch.int64)
            n = self.lens[s] + self.rows[s] - j * bt
            k, v = draw(n, nkv, hd), draw(n, nkv, hd)
            self.put(mine, 0, k, v)
            self.k.append(torch.cat([pk[:j * bt], k]))
            self.v.append(torch.cat([pv[:j * bt], v]))
        self.n = sum(self.rows)
        self.q = (spread * torch.randn((self.n + pad, nq, hd), generator=g, device="cuda")).to(dtype)
        self.start = [0]
        for r in self.rows:
            self.start.append(self.start[-1] + r)

    def put(self, blocks, first, k, v):
        if not len(k):
            return
        at = torch.arange(first, first + len(k), device="cuda")
        b = torch.tensor(blocks, device="cuda")[at // self.bt]
        self.keys[b, :, at % self.bt] = k
        self.values[b, :, :, at % self.bt] = v

    def run(self, **kw):
        import paper_2505_15380_amd as ssd
        status = i32([0])
        a = dict(shared_table=i32(self.prefix) if self.sb else None, shared=None if all(self.joins) else i32([self.sb if j else 0 for j in self.joins]),
                 max_len=max(n + r for n, r in zip(self.lens, self.rows)), status=status)
        a.update(kw)
        out = ssd.ssd_paged_attention(ssd.Pages(self.keys, self.values), a.pop("q", self.q), i32(self.lens), i32(self.start), i32(self.table), **a)
        self.status = status.item()
        return out

    def oracle(self, s, scale, keep=None):
        """Rows of sequence s in 64 bits and the bounds of their errors; keep: which positions there are."""
        q = self.q[self.start[s]:self.start[s + 1]].double()
        G = self.nq // self.nkv
        k, v = (t.double().repeat_interleave(G, 1).transpose(0, 1).contiguous() for t in (self.k[s], self.v[s]))      # [nq, L, hd]
        L = k.shape[1]
        seen = torch.arange(L, device="cuda") <= self.lens[s] + torch.arange(len(q), device="cuda")[:, None]
        if keep is not None:
            seen &= keep
        q = q.transpose(0, 1).contiguous()
        w = scale * torch.bmm(q, k.transpose(1, 2).contiguous())
        size = abs(scale) * torch.bmm(q.abs(), k.abs().transpose(1, 2).contiguous())
        size = size.masked_fill(~seen, 0).amax(-1)[..., None]
        w = torch.exp(w - w.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)).masked_fill(~seen, 0)
        p = w / w.sum(-1, keepdim=True)
        p = torch.where(seen.any(-1)[:, None], p, 0)
        o, a = torch.bmm(p, v), torch.bmm(p, v.abs())
        # A score: hd products and their sum, the factor, the difference from the maximum and the power of two, each off by u of no more than `size` (twice: its own and the
        # maximum's): (hd + 6) u * size, for a weight and for the sum it is divided by.  The sums over the keys, and the merges of parts: no more than L + 64 roundings of a partial sum
        # of at most `a`.  bf16: each weight is rounded once (u of it).
        e = a * (2 * (self.hd + 6) * U32 * size + 2 * (L + 64) * U32)
        if self.dtype == BF16:
            e = e + U16 * a
            e = e + U16 * (o.abs() + e)
        return o.transpose(0, 1), e.transpose(0, 1)

    def check(self, out, scale=None, keep=None):
        scale = self.hd ** -0.5 if scale is None else scale
        for s in range(len(self.rows)):
            if self.rows[s]:
                o, e = self.oracle(s, scale, None if keep is None else keep[s])
                d = (out[self.start[s]:self.start[s + 1]].double() - o).abs()
                assert bool((d <= e).all()), (s, self.lens[s], self.rows[s], float((d - e).max()), float(d.max()))


HEADS = [(14, 2, 64), (12, 2, 128), (4, 4, 32), (8, 1, 64), (1, 1, 128), (17, 1, 32), (32, 2, 128)]
BATCHES = {
    "one": ([(0, 1)], 0),
    "first tokens": ([(0, 1), (0, 2), (1, 1), (15, 1), (16, 1), (17, 1)], 0),
    "tile edges": ([(62, 1), (63, 1), (64, 1), (65, 1), (127, 2), (128, 1), (255, 1), (256, 3)], 0),
    "no rows": ([(5, 0), (40, 1), (0, 0), (0, 3), (77, 0)], 0),
    "verification": ([(300, 7), (31, 7), (129, 7)], 0),
    "decode behind a prefix": ([(0, 1), (1, 1), (16, 1), (40, 1), (333, 1)], 5),
    "verification behind a prefix": ([(n * 7 % 90, 5) for n in range(20)], 9),
    "prompts": ([(0, 70), (0, 1), (0, 131), (13, 64)], 0),
    "prompts behind a prefix": ([(0, 100), (0, 37), (3, 65)], 7),
    "long": ([(2000, 1), (3, 2), (999, 4)], 0),
    "long prefix": ([(10, 1), (0, 2), (70, 1)], 80),
}


@pytest.mark.parametrize("what", BATCHES)
@pytest.mark.parametrize("nq, nkv, hd", HEADS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention(what, nq, nkv, hd, dtype):
    seqs, sb = BATCHES[what]
    bt = {32: 16, 64: 16, 128: 32}[hd] if nq != 17 else 64
    b = Batch(seqs, nq, nkv, hd, bt, dtype, seed=len(what) * 100 + nq, shared_blocks=sb, pad=3)
    out = torch.full_like(b.q, 7.0)
    b.run(out=out)
    assert b.status == 0
    b.check(out)
    assert bool((out[b.n:] == 7.0).all())                  # rows that no sequence has
    again = torch.full_like(b.q, 7.0)
    b.run(out=again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("seqs, sb, heads", [([(1500, 300), (0, 411)], 0, (4, 2, 64)), ([(200, 1)] * 70, 40, (14, 2, 64)), ([(n % 50, 1 + n % 9) for n in range(130)], 30, (12, 2, 128)),
                                             ([(3, 1200)], 64, (6, 2, 64)), ([(64, 64), (1, 900), (700, 0), (0, 77)], 12, (8, 2, 128)), ([(5000, 2)], 0, (2, 1, 32))])
def test_attention_of_larger_batches(dtype, seqs, sb, heads):
    b = Batch(seqs, *heads, 16, dtype, seed=sb + len(seqs), shared_blocks=sb, pad=1)
    b.check(b.run())
    assert b.status == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("heads", [(4, 4, 32), (6, 3, 64), (4, 2, 128)])
@pytest.mark.parametrize("rows", [9, 23])
def test_attention_of_many_short_sequences(dtype, heads, rows):
    b = Batch([(n * 7 % 110, 1 + n % rows) for n in range(150)], *heads, 16, dtype, seed=rows, pad=2)
    b.check(b.run())
    assert b.status == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_of_thousands_of_sequences(dtype):
    """More than the 4096 that two steps of a search tell apart, most without rows."""
    rng = random.Random(1)
    b = Batch([(rng.randrange(40), rng.choice([0, 0, 1, 3])) for _ in range(4200)], 2, 1, 32, 16, dtype, seed=2, shared_blocks=1)
    out = b.run()
    assert b.status == 0
    with_rows = [s for s, r in enumerate(b.rows) if r]
    for s in with_rows[:20] + with_rows[-20:] + rng.sample(with_rows, 60):
        o, e = b.oracle(s, b.hd ** -0.5)
        assert bool(((out[b.start[s]:b.start[s + 1]].double() - o).abs() <= e).all()), s
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("bt", [16, 32, 64, 256, 1024])
def test_attention_block_sizes(bt):
    b = Batch([(bt - 1, 3), (bt, 1), (3 * bt + 5, 2)], 6, 2, 64, bt, BF16, seed=bt, shared_blocks=1)
    b.check(b.run())


@pytest.mark.parametrize("max_len", [1, 64, 100000])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_whatever_length_it_is_told(max_len, dtype):
    b = Batch([(1100, 2), (3, 30), (500, 1)], 8, 2, 64, 16, dtype, seed=max_len, shared_blocks=3)
    b.check(b.run(max_len=max_len))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_of_sequences_without_the_prefix(dtype):
    """Those that do not share it, or are shorter than it, read through their own tables."""
    joins = [True, False, True, False, True, False]
    b = Batch([(9, 3), (200, 2), (60, 1), (0, 4), (0, 5), (63, 70)], 14, 2, 64, 16, dtype, seed=3, shared_blocks=4, joins=joins)
    b.check(b.run())
    assert b.status == 0


def test_attention_of_columns_scales_and_large_scores():
    import paper_2505_15380_amd as ssd
    b = Batch([(40, 9), (100, 1)], 6, 2, 64, 16, BF16, seed=8)
    wide = torch.full((b.n, 10, 64), math.nan, dtype=BF16, device="cuda")
    wide[:, :6] = b.q
    put = torch.zeros((b.n, 640 + 64), dtype=BF16, device="cuda")
    out = put[:, 64:64 + 384].unflatten(1, (6, 64))
    b.check(b.run(q=wide[:, :6], out=out))
    assert bool((put[:, :64] == 0).all()) and bool((put[:, 448:] == 0).all())
    for scale in (0.0, -0.3, 2.0):
        b.check(b.run(scale=scale), scale=scale)
    big = Batch([(70, 3), (700, 1)], 4, 2, 64, 16, FP32, seed=9, spread=3e4)      # scores of 1e5: one key takes all
    out = big.run()
    assert bool(torch.isfinite(out).all())
    ws = torch.full((ssd.paged_attention_workspace(ssd.Pages(b.keys, b.values), 6, 2, b.n, 101),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(b.run(ws=ws, max_len=101), b.run(max_len=101))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows", [1, 40])
def test_attention_without_some_pages(dtype, rows):
    """Blocks outside the pool are left out and reported; a row that has nothing left gets zeros."""
    b = Batch([(90, rows), (33, rows), (150, rows)], 6, 2, 64, 16, dtype, seed=5 + rows, shared_blocks=2)
    n_blocks = b.keys.shape[0]
    keep = [torch.ones(n + r, dtype=torch.bool, device="cuda") for n, r in zip(b.lens, b.rows)]
    b.table[0, 4], b.table[2, 2], b.table[2, 9] = -1, n_blocks, 0x7FFFFFFF
    keep[0][64:80] = False
    keep[2][32:48] = False
    keep[2][144:160] = False
    b.check(b.run(), keep=keep)
    assert b.status == 16
    b.prefix = [-3, n_blocks + 5]
    for k in keep:
        k[:32] = False
    b.table[1] = -1
    keep[1][:] = False
    out = b.run()
    b.check(out, keep=keep)
    assert b.status == 16 and bool((out[b.start[1]:b.start[2]] == 0).all())


def test_attention_beyond_the_table_and_of_impossible_lengths():
    b = Batch([(20, 2), (40, 3), (9, 1)], 4, 2, 64, 16, BF16, seed=12, table_pad=0)
    out = torch.full_like(b.q, 7.0)
    b.lens[0], was = -5, b.lens[0]
    b.run(out=out)
    assert b.status == 8 and bool((out[:2] == 7.0).all())
    b.lens[0] = was
    b.lens[1] = 48 * 16 + 1                                # longer than the table
    out.fill_(7.0)
    b.run(out=out)
    assert b.status == 8 and bool((out[2:5] == 7.0).all())
    b.lens[1] = 46                                         # its last row stands behind the table's end
    b.run(out=out)
    assert b.status == 16 and bool(torch.isfinite(out[:2]).all())


def test_attention_is_nan_where_it_sees_nan_and_nowhere_else():
    b = Batch([(70, 4), (100, 1)], 4, 2, 64, 16, BF16, seed=14)
    good = b.run()
    blk, tok = int(b.table[0, 4]), 64 % 16
    b.keys[blk, 1, tok, 5] = math.nan                      # position 64 of the first sequence, second key head
    out = b.run()
    assert bool(torch.isnan(out[:4, 2:]).all()) and torch.equal(out[:4, :2], good[:4, :2]) and torch.equal(out[4:], good[4:])


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("seqs, sb, heads", [([(30, 5), (90, 3), (0, 1)], 0, (6, 2, 64)), ([(40, 70), (0, 131)], 0, (12, 2, 128)), ([(200, 9), (3, 2)] * 8, 6, (14, 2, 64)),
                                             ([(2000, 2), (3, 2)], 0, (4, 4, 32)), ([(62, 4), (0, 600)], 0, (2, 1, 64)), ([(900, 6)] * 3, 0, (8, 2, 64)), ([(61, 4), (127, 20)], 3, (4, 4, 32))])
def test_attention_of_rows_before_values_that_are_not_finite(dtype, seqs, sb, heads):
    """Infinities and NaN at new rows' positions are nothing to the rows before them, and come out at those that see them."""
    b = Batch(seqs, *heads, 16, dtype, seed=sb + len(seqs), shared_blocks=sb)
    G = heads[0] // heads[1]
    expect = torch.zeros((b.n, heads[0], heads[2]), dtype=torch.float64, device="cuda")
    for s, (n, r) in enumerate(zip(b.lens, b.rows)):
        if r < 2:
            continue
        put = {(r // 2, 3): math.inf, (r // 2, 5): math.nan, (r // 2, 8): -math.inf, (r // 2, 9): math.inf}
        put.update({(r - 1, 9): -math.inf, (r - 1, 31): math.inf})                 # (of two rows, the same one)
        for (row, d), x in put.items():
            b.values[int(b.table[s, (n + row) // 16]), heads[1] - 1, d, (n + row) % 16] = x
            expect[b.start[s] + row:b.start[s + 1], heads[0] - G:, d] += x
    out = b.run().double()
    plain = torch.where(expect == 0, out, 0)
    assert bool(torch.isfinite(plain).all())
    for s in range(len(b.rows)):
        o, e = b.oracle(s, b.hd ** -0.5)
        at = slice(b.start[s], b.start[s + 1])
        assert bool((((out[at] - o).abs() <= e) | (expect[at] != 0)).all()), s
    differs = torch.where(expect == 0, 0, out).nan_to_num(nan=1.0, posinf=2.0, neginf=3.0) != expect.nan_to_num(nan=1.0, posinf=2.0, neginf=3.0)
    assert not bool(differs.any())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("seqs, sb, heads", [([(30, 5), (90, 3)], 0, (6, 2, 64)), ([(40, 70), (0, 131)], 0, (12, 2, 128)), ([(200, 9), (3, 2)] * 8, 6, (14, 2, 64)), ([(62, 4), (0, 600)], 0, (4, 4, 32))])
def test_attention_of_rows_before_keys_that_are_not_finite(dtype, seqs, sb, heads):
    """A key of NaN makes NaN of the rows that see it, in the heads that read it, and nothing of others."""
    b = Batch(seqs, *heads, 16, dtype, seed=sb + 3 * len(seqs), shared_blocks=sb)
    G = heads[0] // heads[1]
    seen = torch.zeros((b.n, heads[0], 1), dtype=torch.bool, device="cuda")
    for s, (n, r) in enumerate(zip(b.lens, b.rows)):
        row = r // 2
        b.keys[int(b.table[s, (n + row) // 16]), 0, (n + row) % 16] = math.nan
        b.keys[int(b.table[s, (n + r - 1) // 16]), 0, (n + r - 1) % 16, 1:] = math.inf
        seen[b.start[s] + row:b.start[s + 1], :G] = True
    out = b.run().double()
    assert bool((torch.isnan(out) == seen).all())
    for s in range(len(b.rows)):
        o, e = b.oracle(s, b.hd ** -0.5)
        at = slice(b.start[s], b.start[s + 1])
        assert bool((((out[at] - o).abs() <= e) | seen[at]).all()), s


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("seqs, sb, heads", [([(30, 2), (90, 1), (700, 3)], 0, (6, 2, 64)), ([(20, 70), (900, 90)], 4, (4, 2, 64)), ([(3, 1)] * 70, 2, (4, 4, 32))])
def test_attention_of_rows_that_begin_behind_others(dtype, seqs, sb, heads):
    """The first sequence's rows need not be the first rows."""
    b = Batch(seqs, *heads, 16, dtype, seed=11 + sb, shared_blocks=sb, pad=2)
    b.q = torch.cat([torch.full_like(b.q[:19], math.nan), b.q])
    b.start = [x + 19 for x in b.start]
    out = torch.full_like(b.q, 7.0)
    b.run(out=out)
    assert b.status == 0
    b.check(out)
    assert bool((out[:19] == 7.0).all()) and bool((out[19 + b.n:] == 7.0).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_over_a_pool_of_more_than_2_31_elements(dtype):
    """Blocks far apart in a pool whose offsets take more than 32 bits of elements."""
    n_blocks = (1 << 31) // (2 * 16 * 128) + 1000
    b = Batch([(50, 3), (700, 1)], 4, 2, 128, 16, dtype, seed=31, shared_blocks=2, n_blocks=n_blocks)
    assert int(b.table.max()) * 2 * 16 * 128 > 1 << 30
    last = n_blocks - 1
    if last not in b.prefix and not bool((b.table == last).any()):
        old = int(b.table[0, 2])
        b.table[0, 2] = last
        b.keys[last], b.values[last] = b.keys[old], b.values[old]
    # (of the unwritten positions of a block nothing is known here: they were never set)
    b.check(b.run())
    del b
    torch.cuda.empty_cache()


# ---------------------------------------------------------------------------------------------- together
def serve(dtype, heads, bt, voice, n_seqs, steps, stream=None, graph=False, pad=5):
    """A batch behind one prefix: prompts of different lengths, then single tokens and verifications, a request that ends and one that begins
    again; every step is tables, append, attention.  Against contiguous keys and values in 64 bits."""
    import paper_2505_15380_amd as ssd
    nq, nkv, hd = heads
    rng = random.Random(voice + n_seqs)
    g = torch.Generator("cuda").manual_seed(voice)
    sb, cap = voice // bt, voice // bt + 12
    n_blocks = sb + n_seqs * 12
    keys = torch.full((n_blocks, nkv, bt, hd), math.nan, dtype=dtype, device="cuda")
    values = torch.full((n_blocks, nkv, hd, bt), math.nan, dtype=dtype, device="cuda")
    pages = ssd.Pages(keys, values)
    rope = rope_table(voice + 12 * bt, hd)
    max_rows = n_seqs * 20 + pad
    z = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")      # noqa: E731
    dev = dict(lens=z(n_seqs), rows=z(n_seqs), table=z(n_seqs * cap).view(n_seqs, cap).fill_(-1), owned=z(n_seqs), free_stack=torch.arange(n_blocks - 1, -1, -1, dtype=torch.int32).cuda(),
               n_free=i32([n_blocks]), shared=i32([sb] * n_seqs))
    out = dict(owned=dev["owned"], n_free=dev["n_free"], row_start=z(n_seqs + 1), row_seq=z(max_rows), row_pos=z(max_rows), row_slot=z(max_rows), status=z(1))
    qkv = torch.zeros((max_rows, (nq + 2 * nkv) * hd), dtype=dtype, device="cuda")
    q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([nq * hd, nkv * hd, nkv * hd], 1))
    att = torch.zeros((max_rows, nq, hd), dtype=dtype, device="cuda")
    prefix = z(max(1, sb))
    need = ssd.paged_attention_workspace(pages, nq, n_seqs, max_rows, voice + 12 * bt, sb)
    ws = torch.empty(max(1, need), dtype=torch.uint8, device="cuda")

    def step():
        ssd.ssd_block_tables(dev["lens"], dev["rows"], bt, dev["table"], dev["owned"], dev["free_stack"], dev["n_free"], max_rows, shared=dev["shared"], out=out)
        ssd.ssd_rope_append(pages, out["row_pos"], out["row_slot"], k, v, q=q, rope=rope, q_out=q, status=out["status"])
        ssd.ssd_paged_attention(pages, q, dev["lens"], out["row_start"], dev["table"], shared_table=prefix if sb else None, shared=dev["shared"], max_len=voice + 6 * bt, out=att,
                                ws=ws, status=out["status"])

    # the voice prompt is a sequence of its own, whose blocks the others then share
    pk, pv = torch.zeros((0, nkv, hd), dtype=dtype, device="cuda"), torch.zeros((0, nkv, hd), dtype=dtype, device="cuda")
    if sb:
        first = ssd.ssd_block_tables(z(1), i32([voice]), bt, prefix.view(1, sb), z(1), dev["free_stack"], dev["n_free"], voice)
        dev["n_free"].copy_(first["n_free"])
        a = torch.randn((2, voice, nkv, hd), generator=g, device="cuda").to(dtype)
        ssd.ssd_rope_append(pages, first["row_pos"], first["row_slot"], a[0], a[1], rope=rope)
        blocks = prefix.long()
        pk = keys[blocks].transpose(1, 2).reshape(-1, nkv, hd)
        pv = values[blocks].permute(0, 3, 1, 2).reshape(-1, nkv, hd)
    have = [[pk, pv] for _ in range(n_seqs)]
    captured = None
    if graph:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
    lens = [voice] * n_seqs
    for t in range(steps):
        rows = [rng.choice([0, 1, 1, 1, 5, 16 if t == 0 else 1]) for _ in range(n_seqs)]
        for s in range(n_seqs):
            if t and rng.random() < 0.2:                   # over, and another request in its place
                lens[s], have[s] = voice, [pk, pv]
            elif t and rng.random() < 0.2 and lens[s] > voice:                 # rejected drafts
                lens[s] -= rng.randint(1, min(4, lens[s] - voice))
                have[s] = [x[:lens[s]] for x in have[s]]
        dev["lens"].copy_(i32(lens)), dev["rows"].copy_(i32(rows))
        qkv.copy_(torch.randn(qkv.shape, generator=g, device="cuda"))
        att.fill_(7.0)
        raw = [x.clone() for x in (q, k, v)]
        (captured.replay if graph else step)()
        n = sum(rows)
        assert out["status"].item() == 0
        assert bool((att[n:] == 7.0).all()) and torch.equal(q[n:], raw[0][n:])
        start = 0
        b = Batch.__new__(Batch)
        b.nq, b.nkv, b.hd, b.dtype, b.q, b.lens, b.rows, b.start, b.k, b.v = nq, nkv, hd, dtype, q, lens, rows, [0], [], []
        for s in range(n_seqs):
            r = rows[s]
            pos = torch.arange(lens[s], lens[s] + r)
            u = U16 if dtype == BF16 else 0.0
            slots = out["row_slot"][start:start + r].long()
            kept = keys[slots // bt, :, slots % bt]
            for got, raw_ in ((q[start:start + r], raw[0]), (kept, raw[1])):
                y, e = turned(raw_[start:start + r], rope[pos.cuda()])
                assert bool(((got.double() - y).abs() <= e + u * (y.abs() + e)).all())
            have[s] = [torch.cat([have[s][0], kept]), torch.cat([have[s][1], raw[2][start:start + r]])]
            b.k.append(have[s][0]), b.v.append(have[s][1])
            start += r
            b.start.append(start)
        b.check(att)
        lens = [n_ + r for n_, r in zip(lens, rows)]
    held = sum(-(-n_ // bt) - sb for n_ in lens)
    assert dev["n_free"].item() <= n_blocks - sb - held + n_seqs


@pytest.mark.parametrize("dtype, heads, bt, voice", [(BF16, (14, 2, 64), 16, 0), (BF16, (14, 2, 64), 16, 160), (BF16, (12, 2, 128), 32, 96), (FP32, (4, 4, 32), 16, 32)])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_a_served_batch(dtype, heads, bt, voice, graph):
    serve(dtype, heads, bt, voice, n_seqs=9, steps=6, graph=graph)


def test_steps_on_another_stream():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        serve(BF16, (4, 2, 64), 16, 48, n_seqs=5, steps=3)
    torch.cuda.current_stream().wait_stream(s)


def test_attention_over_a_cache_that_a_model_filled():
    """The pages of an ssd_kv cache: what a prefill left there, read by the call that stands alone."""
    import paper_2505_15380_amd as ssd
    import synth_inputs as si
    shape = si.model_shape("mini_bf16")
    model = ssd.Model(shape, ssd.upload_weights(shape, si.make_weights(shape, 150)), 256)
    kv = ssd.KVCache(model, 2, 64, 32, 16, 16, 1)
    lens = [45, 130]
    for s, n in enumerate(lens):
        ssd.ssd_prefill(model, kv, s, torch.from_numpy(si.make_prefix(shape, 2, n - 1, 70 + s)).cuda())
    b = Batch.__new__(Batch)
    b.nq, b.nkv, b.hd, b.dtype = shape["n_q_heads"], shape["n_kv_heads"], shape["head_dim"], BF16
    b.q = torch.randn((2, b.nq, b.hd), generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(BF16)
    b.lens, b.rows, b.start = [n - 1 for n in lens], [1, 1], [0, 1, 2]
    table = torch.full((2, 16), -1, dtype=torch.int32)
    for layer in range(shape["n_layers"]):
        b.k, b.v = [], []
        for s, n in enumerate(lens):
            st = kv.state(s)
            assert st["len"] == n
            table[s, :st["n_owned"]] = torch.tensor(st["table"], dtype=torch.int32)
            k, v = kv.gather(s, layer, n)
            b.k.append(torch.from_numpy(k).cuda()), b.v.append(torch.from_numpy(v).cuda())
        b.check(ssd.ssd_paged_attention(kv.pages(layer), b.q, i32(b.lens), i32(b.start), table.cuda()))


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_calls_side_by_side_and_two_graphs(dtype):
    """Two batches on two streams at once, then two captured calls replayed in turn with other work between, their lengths changed in place."""
    import paper_2505_15380_amd as ssd
    pair = [Batch([(900, 3), (20, 2), (333, 1)], 6, 2, 64, 16, dtype, seed=1, shared_blocks=8), Batch([(1500, 1), (64, 5)], 4, 2, 128, 32, dtype, seed=2)]
    args = [(ssd.Pages(b.keys, b.values), b.q, i32(b.lens), i32(b.start), i32(b.table)) for b in pair]
    kw = [dict(shared_table=i32(b.prefix) if b.sb else None, max_len=2000) for b in pair]
    plain = [ssd.ssd_paged_attention(*a, **k) for a, k in zip(args, kw)]
    for b, out in zip(pair, plain):
        b.check(out)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i in (0, 1):
            with torch.cuda.stream(streams[i]):
                outs[i].append(ssd.ssd_paged_attention(*args[i], **kw[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, plain[i]) for i in (0, 1) for o in outs[i])
    graphs, held = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for i in (0, 1):
        out = torch.empty_like(plain[i])
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            ssd.ssd_paged_attention(*args[i], out=out, **kw[i])
        held.append(out)
    for turn in range(4):
        lens = [torch.tensor(b.lens, dtype=torch.int32) - 7 * turn * torch.tensor([n > b.sb * b.bt + 60 for n in b.lens], dtype=torch.int32) for b in pair]
        for i in (0, 1):
            args[i][2].copy_(lens[i])
            held[i].fill_(math.nan)
        for i in (0, 1):
            graphs[i].replay()
        torch.ones(1 << 16, device="cuda").sum()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert torch.equal(held[i], ssd.ssd_paged_attention(*args[i], **kw[i])), (turn, i)
