"""The cache path of one step of a served batch, operator by operator, as work that can be timed and compared.

  tables   ssd_block_tables: block tables, row offsets and slots of a step, from the requests' lengths
  append   ssd_rope_append: queries and keys rotated, keys and values put into their slots
  attend   ssd_paged_attention: every row against its sequence's pages, the prefix that the batch shares read once for all

Head layouts are those of the model shapes in synth_inputs (14/2 x 64, 12/2 x 128, 6/2 x 64, 4/2 x 128, and 4/4 x 32 in fp32).  A batch's lengths
and row counts are spread evenly over the case's range and dealt out by the seed, so that its work depends on the case alone."""
import math

import torch

own = False

BF16, FP32 = torch.bfloat16, torch.float32
HEADS = {"half": (14, 2, 64), "one_half": (12, 2, 128), "mini": (6, 2, 64), "mini128": (4, 2, 128), "tiny": (4, 4, 32)}


def listed():
    return [
        # one token for each of 64 streams of any age: every decoding step has this call
        dict(name="tables_decode_64", op="tables", B=64, rlo=1, rhi=1, lo=256, hi=4096, bt=16, shared=0, done=0),
        # a busy server: prompts in pieces beside short continuations, requests that are over give their blocks back
        dict(name="tables_mixed_960", op="tables", B=960, rlo=1, rhi=160, lo=128, hi=2048, bt=16, shared=8, done=60),
        # the rows of 16 verifications with six drafts each, in a launch with room for a few more
        dict(name="append_verify_112", op="append", heads="half", n=112, pad=16, dtype="bf16", bt=16, reach=4096),
        # a long prompt of the larger model
        dict(name="append_prompt_4099", op="append", heads="one_half", n=4099, pad=0, dtype="bf16", bt=16, reach=4099),
        # fp32 storage
        dict(name="append_fp32_517", op="append", heads="tiny", n=517, pad=3, dtype="fp32", bt=16, reach=1100),
        # one stream, one token: all latency
        dict(name="attend_one_1024", op="attend", heads="half", B=1, rlo=1, rhi=1, shared=0, lo=1023, hi=1023, dtype="bf16", bt=16),
        # sixteen verifications of any age that share nothing
        dict(name="attend_verify_16x7", op="attend", heads="half", B=16, rlo=7, rhi=7, shared=0, lo=256, hi=4096, dtype="bf16", bt=16),
        # 64 sentences in one voice, a token each: the voice prompt is most of every prefix
        dict(name="attend_shared_64x1", op="attend", heads="half", B=64, rlo=1, rhi=1, shared=4096, lo=1, hi=1024, dtype="bf16", bt=16),
        # the same as verifications of the larger model
        dict(name="attend_shared_61x8_d128", op="attend", heads="one_half", B=61, rlo=8, rhi=8, shared=2048, lo=64, hi=1501, dtype="bf16", bt=16),
        # a long document read by many: 1280 rows against the same 16384 positions
        dict(name="attend_shared_256x5", op="attend", heads="half", B=256, rlo=5, rhi=5, shared=16384, lo=1, hi=500, dtype="bf16", bt=32),
        # ragged prompts behind a common instruction
        dict(name="attend_prompts_7", op="attend", heads="half", B=7, rlo=100, rhi=2001, shared=1024, lo=0, hi=0, dtype="bf16", bt=16),
        # fp32 storage, small heads without groups
        dict(name="attend_fp32_33x4", op="attend", heads="tiny", B=33, rlo=1, rhi=7, shared=160, lo=0, hi=401, dtype="fp32", bt=16),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["tables", "append", "attend", "attend"])
    bt = rng.choice([16, 16, 32, 64])
    if op == "tables":
        while True:
            B, rhi = _log_int(rng, 1, 2048), _log_int(rng, 1, 4096)
            if B * rhi <= 160000:
                break
        lo = rng.choice([0, 1, 100])
        return dict(op=op, B=B, rlo=rng.choice([1, rhi]), rhi=rhi, lo=lo, hi=lo + _log_int(rng, 1, 2000), bt=bt, shared=rng.choice([0, 0, _log_int(rng, 1, 100)]),
                    done=rng.randint(0, B // 8))
    heads = rng.choice(sorted(HEADS))
    dtype = "fp32" if heads == "tiny" else "bf16"
    if op == "append":
        n = _log_int(rng, 1, 4099)
        return dict(op=op, heads=heads, n=n, pad=rng.choice([0, rng.randint(1, 30)]), dtype=dtype, bt=bt, reach=n + _log_int(rng, 1, 4000))
    while True:
        B, rhi = _log_int(rng, 1, 256), _log_int(rng, 1, 2001)
        shared = rng.choice([0, _log_int(rng, 1, 1024), _log_int(rng, 1, 1024)]) * bt
        lo = rng.choice([0, 1, 50])
        hi = lo + _log_int(rng, 1, 4000)
        c = dict(op=op, heads=heads, B=B, rlo=rng.choice([1, rhi]), rhi=rhi, shared=shared, lo=lo, hi=hi, dtype=dtype, bt=bt)
        nq, nkv, hd = HEADS[heads]
        reach = shared + hi + rhi
        if shared <= 16384 and B * reach * nkv * hd <= 256 * 16889 * 2 * 64 and B * rhi * nq * reach <= 200e6 and sum(_spread(c["rlo"], rhi, B)) <= 8000:
            return c


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread."""
    return [lo + (hi - lo) * (2 * i + 1) // (2 * n) for i in range(n)] if n > 1 else [hi]


def _counts(case, seed):
    """Cached positions and new rows of each sequence: the case's, in the seed's order."""
    B = case["B"]
    g = torch.Generator().manual_seed(seed)
    lens = torch.tensor(_spread(case["lo"], case["hi"], B))[torch.randperm(B, generator=g)]
    rows = torch.tensor(_spread(case["rlo"], case["rhi"], B))[torch.randperm(B, generator=g)]
    return lens, rows, g


def prepare(case, seed):
    return {"tables": _prepare_tables, "append": _prepare_append, "attend": _prepare_attend}[case["op"]](case, seed)


def _prepare_tables(case, seed):
    """A server's state between two steps: lengths and new rows, who holds which blocks, and the stack of free ones."""
    B, bt, shared = case["B"], case["bt"], case["shared"]
    lens, rows, g = _counts(case, seed)
    lens = lens + shared * bt                                   # the common prefix is in front of every sequence
    owned = (lens + bt - 1) // bt - shared
    over = torch.randperm(B, generator=g)[:case["done"]]        # requests that are over: they hold blocks and need none
    cap = (case["hi"] + case["rhi"]) // bt + shared + 2
    n_rows = sum(_spread(case["rlo"], case["rhi"], B))
    lens[over], rows[over] = shared * bt, 0
    n_blocks = int(owned.sum()) + n_rows // bt + B + shared + 7
    ids = torch.randperm(n_blocks, generator=g)
    table = torch.full((B, cap), -1, dtype=torch.int64)
    table[:, :shared] = ids[:shared]
    held = (torch.arange(cap) >= shared) & (torch.arange(cap) < shared + owned[:, None])
    table[held] = ids[shared:shared + int(owned.sum())]
    free = ids[shared + int(owned.sum()):]
    stack = torch.zeros(n_blocks, dtype=torch.int64)
    stack[:len(free)] = free
    i32 = lambda t: t.to(torch.int32).cuda()                    # noqa: E731
    s = dict(op="tables", lens=i32(lens), rows=i32(rows), owned=i32(owned), table=i32(table), stack=i32(stack), n_free=i32(torch.tensor([len(free)])),
             shared=i32(torch.full((B,), shared)), bt=bt, max_rows=n_rows)
    s["out"] = dict(owned=torch.zeros_like(s["owned"]), n_free=torch.zeros_like(s["n_free"]), row_start=i32(torch.zeros(B + 1)), status=i32(torch.zeros(1)),
                    **{k: i32(torch.zeros(n_rows)) for k in ("row_seq", "row_pos", "row_slot")})
    return s


def _rope_table(positions, hd):
    """cos and sin of every position's angles, [positions, hd / 2, 2], evaluated in 64 bits and rounded once."""
    f = 1.0e6 ** (-torch.arange(hd // 2, dtype=torch.float64, device="cuda") * 2.0 / hd)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _prepare_append(case, seed):
    """The rows that a QKV projection left behind each other, their positions and slots; rows behind the last one have slot -1."""
    nq, nkv, hd = HEADS[case["heads"]]
    n, pad, bt = case["n"], case["pad"], case["bt"]
    dt = BF16 if case["dtype"] == "bf16" else FP32
    g = torch.Generator().manual_seed(seed)
    gg = torch.Generator("cuda").manual_seed(seed)
    first = int(torch.randint(0, case["reach"] - n + 1, (1,), generator=g))
    pos = torch.arange(first, first + n)
    blocks = -(-case["reach"] // bt)
    table = torch.randperm(blocks, generator=g)
    slot = table[pos // bt] * bt + pos % bt
    none = torch.full((pad,), -1)
    # one block more than the pages have, behind them: the plain form's rows without a slot go there
    keys = torch.randn((blocks + 1, nkv, bt, hd), generator=gg, device="cuda").to(dt)
    values = torch.randn((blocks + 1, nkv, hd, bt), generator=gg, device="cuda").to(dt)
    qkv = torch.randn((n + pad, (nq + 2 * nkv) * hd), generator=gg, device="cuda").to(dt)
    s = dict(op="append", qkv=qkv, pos=torch.cat([pos, none]).to(torch.int32).cuda(), slot=torch.cat([slot, none]).to(torch.int32).cuda(), keys=keys, values=values, bt=bt,
             heads=(nq, nkv, hd), rope=_rope_table(case["reach"], hd), q_out=torch.zeros((n + pad, nq, hd), dtype=dt, device="cuda"), status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    return s


def _prepare_attend(case, seed):
    """Pages in any order, queries of every row, and the batch's tables as ssd_block_tables leaves them."""
    nq, nkv, hd = HEADS[case["heads"]]
    B, bt, shared = case["B"], case["bt"], case["shared"]
    dt = BF16 if case["dtype"] == "bf16" else FP32
    lens, rows, g = _counts(case, seed)
    gg = torch.Generator("cuda").manual_seed(seed)
    lens = lens + shared
    have = (lens + rows + bt - 1) // bt
    sb = shared // bt
    cap = int(have.max())
    n_blocks = sb + int((have - sb).sum()) + 3
    ids = torch.randperm(n_blocks, generator=g)
    table = torch.full((B, cap), -1, dtype=torch.int64)
    table[:, :sb] = ids[:sb]
    mine = (torch.arange(cap) >= sb) & (torch.arange(cap) < have[:, None])
    table[mine] = ids[sb:sb + int(mine.sum())]
    n = int(rows.sum())
    start = torch.cat([torch.zeros(1, dtype=torch.int64), rows.cumsum(0)])
    seq = torch.repeat_interleave(torch.arange(B), rows)
    pad = 2 if n > 8 else 0                                     # rows of the launch that no sequence has
    i32 = lambda t: t.to(torch.int32).cuda()                    # noqa: E731
    draw_ = lambda *shape: torch.randn(shape, generator=gg, device="cuda")      # noqa: E731
    return dict(op="attend", heads=(nq, nkv, hd), bt=bt, sb=sb, q=(1.5 * draw_(n + pad, nq, hd)).to(dt), keys=draw_(n_blocks, nkv, bt, hd).to(dt),
                values=draw_(n_blocks, nkv, hd, bt).to(dt), lens=i32(lens), row_start=i32(start), table=i32(table), prefix=i32(table[0, :sb]), max_len=int((lens + rows).max()),
                max_rows=int(rows.max()), row_seq=seq.cuda(), row_off=(torch.arange(n) - start[:-1][seq]).cuda(), out=torch.zeros((n + pad, nq, hd), dtype=dt, device="cuda"),
                status=torch.zeros(1, dtype=torch.int32, device="cuda"))


def run(s):
    if own:
        return {"tables": _own_tables, "append": _own_append, "attend": _own_attend}[s["op"]](s)
    return {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend}[s["op"]](s)


def _own_tables(s):
    import paper_2505_15380_amd as ssd
    o = ssd.ssd_block_tables(s["lens"], s["rows"], s["bt"], s["table"], s["owned"], s["stack"], s["n_free"], s["max_rows"], shared=s["shared"], out=s["out"])
    return [s["table"], s["stack"], o["owned"], o["n_free"], o["row_start"], o["row_seq"], o["row_pos"], o["row_slot"], o["status"]]


def _plain_tables(s):
    lens, rows, owned, shared, table, stack = (s[k].long() for k in ("lens", "rows", "owned", "shared", "table", "stack"))
    bt, n, cap = s["bt"], stack.numel(), table.shape[1]
    need = ((lens + rows + bt - 1) // bt - shared).clamp(min=0)
    give, take = (owned - need).clamp(min=0), (need - owned).clamp(min=0)
    top = s["n_free"].long()
    at = torch.arange(cap, device=table.device) - shared[:, None]                                     # which of its own blocks an entry is
    gone = (at >= need[:, None]) & (at < owned[:, None])
    place = top + (give.cumsum(0) - give)[:, None] + owned[:, None] - 1 - at
    stack = torch.cat([stack, stack[:1]]).index_put((torch.where(gone, place, n).reshape(-1),), table.reshape(-1))[:n]
    top = top + give.sum()
    new = (at >= owned[:, None]) & (at < need[:, None])
    nth = (take.cumsum(0) - take)[:, None] + at - owned[:, None]
    table = torch.where(new, stack[(top - 1 - nth).clamp(0, n - 1)], table)
    start = torch.cat([torch.zeros_like(rows[:1]), rows.cumsum(0)])
    r = torch.arange(s["max_rows"], device=table.device)
    seq = torch.searchsorted(start[1:], r, right=True).clamp(max=len(rows) - 1)
    there = r < start[-1]
    pos = lens[seq] + r - start[seq]
    slot = table[seq, (pos // bt).clamp(max=cap - 1)] * bt + pos % bt
    none = torch.full_like(r, -1)
    i32 = lambda t: t.to(torch.int32)                           # noqa: E731
    return [i32(table), i32(stack), i32(need), i32(top - take.sum()), i32(start), i32(torch.where(there, seq, none)), i32(torch.where(there, pos, none)),
            i32(torch.where(there, slot, none)), torch.zeros_like(s["n_free"])]


def _qkv(s):
    nq, nkv, hd = s["heads"]
    n = s["qkv"].shape[0]
    q, k, v = s["qkv"].split([nq * hd, nkv * hd, nkv * hd], 1)
    return q.view(n, nq, hd), k.view(n, nkv, hd), v.view(n, nkv, hd)


def _own_append(s):
    import paper_2505_15380_amd as ssd
    q, k, v = _qkv(s)
    pages = ssd.Pages(s["keys"][:-1], s["values"][:-1])
    ssd.ssd_rope_append(pages, s["pos"], s["slot"], k, v, q=q, rope=s["rope"], q_out=s["q_out"], status=s["status"])
    return [s["q_out"], s["keys"][:-1], s["values"][:-1], s["status"]]


def _plain_append(s):
    q, k, v = _qkv(s)
    nq, nkv, hd = s["heads"]
    there = (s["slot"] >= 0)[:, None, None]
    cs = s["rope"][s["pos"].clamp(min=0).long()]
    c, d = cs[:, None, :, 0], cs[:, None, :, 1]
    x = torch.cat([q, k], 1).float()
    a, b = x[..., :hd // 2], x[..., hd // 2:]
    x = torch.cat([a * c - b * d, b * c + a * d], -1).to(q.dtype)
    slot = torch.where(s["slot"] < 0, (s["keys"].shape[0] - 1) * s["bt"], s["slot"]).long()
    s["q_out"].copy_(torch.where(there, x[:, :nq], s["q_out"]))
    s["keys"][slot // s["bt"], :, slot % s["bt"]] = x[:, nq:]
    s["values"][slot // s["bt"], :, :, slot % s["bt"]] = v
    return [s["q_out"], s["keys"][:-1], s["values"][:-1], s["status"]]


def _own_attend(s):
    import paper_2505_15380_amd as ssd
    pages = ssd.Pages(s["keys"], s["values"])
    ssd.ssd_paged_attention(pages, s["q"], s["lens"], s["row_start"], s["table"], shared_table=s["prefix"], max_len=s["max_len"], out=s["out"], status=s["status"])
    return [s["out"], s["status"]]


def _plain_attend(s):
    nq, nkv, hd = s["heads"]
    B, cap = s["table"].shape
    R, L = s["max_rows"], cap * s["bt"]
    n = s["row_seq"].numel()
    start, lens = s["row_start"].long(), s["lens"].long()
    pages = s["table"].clamp(min=0).long()
    k = s["keys"][pages].permute(0, 2, 1, 3, 4).reshape(B, nkv, L, hd).float()
    v = s["values"][pages].permute(0, 2, 1, 4, 3).reshape(B, nkv, L, hd).float()
    i = torch.arange(R, device=k.device)
    q = s["q"][(start[:-1, None] + i).clamp(max=n - 1)].float()                                      # [B, R, nq, hd]
    q = q.view(B, R, nkv, nq // nkv, hd).permute(0, 2, 1, 3, 4).reshape(B, nkv, R * (nq // nkv), hd)
    w = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(hd))
    hidden = torch.arange(L, device=k.device) > (lens[:, None] + i)[..., None]                        # [B, R, L]
    w = w.view(B, nkv, R, nq // nkv, L).masked_fill_(hidden[:, None, :, None], -math.inf)
    w = (w - w.amax(-1, keepdim=True)).exp_()
    w = w.div_(w.sum(-1, keepdim=True)).view(B, nkv, R * (nq // nkv), L)
    o = torch.matmul(w, v).view(B, nkv, R, nq // nkv, hd).permute(0, 2, 1, 3, 4).reshape(B, R, nq, hd)
    s["out"][:n] = o[s["row_seq"], s["row_off"]].to(s["out"].dtype)
    return [s["out"], s["status"]]


def work(case):
    if case["op"] == "tables":
        B, bt = case["B"], case["bt"]
        n = sum(_spread(case["rlo"], case["rhi"], B))
        moved = n // bt + B                                     # ids taken or given back
        return {"bytes": 28 * B + 8 * moved + 12 * n, "flops": 0}
    nq, nkv, hd = HEADS[case["heads"]]
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "append":
        return {"bytes": case["n"] * (2 * (nq + 2 * nkv) * hd * e + hd * 4 + 8), "flops": case["n"] * (nq + nkv) * hd * 3}
    rows, lens = _spread(case["rlo"], case["rhi"], case["B"]), _spread(case["lo"], case["hi"], case["B"])
    n, own_keys = sum(rows), sum(rows) + sum(lens)
    # (rows and lengths are dealt out apart from each other: a row sees its sequence's mean length and half of its rows)
    seen = n * (case["shared"] + sum(lens) / len(lens)) + sum(r * (r + 1) / 2 for r in rows)
    return {"bytes": (case["shared"] + own_keys) * nkv * hd * 2 * e + 2 * n * nq * hd * e, "flops": 4 * seen * nq * hd}


def exact(case, seed):
    """From the definitions, in 64 bits, a sequence or a head at a time."""
    s = prepare(case, seed)
    if case["op"] == "tables":
        return None                                             # whole numbers all of them
    nq, nkv, hd = HEADS[case["heads"]]
    bt = case["bt"]
    if case["op"] == "append":
        n = case["n"]
        x = s["qkv"][:n].double().view(n, nq + 2 * nkv, hd)
        z = torch.view_as_complex(torch.stack([x[:, :nq + nkv, :hd // 2], x[:, :nq + nkv, hd // 2:]], -1))
        z = z * torch.view_as_complex(s["rope"].double())[s["pos"][:n].long()][:, None]
        rot = torch.cat([z.real, z.imag], -1)
        q_out, keys, values = s["q_out"].double(), s["keys"][:-1].double(), s["values"][:-1].double()
        q_out[:n] = rot[:, :nq]
        keys = keys.transpose(1, 2).contiguous().view(-1, nkv, hd)
        values = values.permute(0, 3, 1, 2).contiguous().view(-1, nkv, hd)
        keys[s["slot"][:n].long()] = rot[:, nq:]
        values[s["slot"][:n].long()] = x[:, nq + nkv:]
        return [q_out, keys.view(-1, bt, nkv, hd).transpose(1, 2).contiguous(), values.view(-1, bt, nkv, hd).permute(0, 2, 3, 1).contiguous(), None]
    out = s["out"].double()
    lens, start = s["lens"].tolist(), s["row_start"].tolist()
    for b in range(case["B"]):
        a, e = start[b], start[b + 1]
        length = lens[b] + e - a
        at = torch.arange(length, device="cuda")
        block = s["table"][b].long()[at // bt]
        k, v = s["keys"][block, :, at % bt].double(), s["values"][block, :, :, at % bt].double()      # [length, nkv, hd]
        seen = at <= lens[b] + torch.arange(e - a, device="cuda")[:, None]
        for h in range(nq):
            w = s["q"][a:e, h].double() @ k[:, h // (nq // nkv)].t() / math.sqrt(hd)
            w = torch.softmax(w.masked_fill(~seen, -math.inf), -1)
            out[a:e, h] = w @ v[:, h // (nq // nkv)]
    return [out, None]
