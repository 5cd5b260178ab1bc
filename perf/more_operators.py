"""The operators of a batch of requests that share one pool of Key-Value blocks held in 8 bits, as they are timed: tables of the batch's rows and
blocks built on the GPU from the requests' lengths, rows written into the pool and read back, and attention of each request's last tokens over its
blocks where they lie.

Shapes are the repository's workloads (paper_2508_06447_amd/inputs.py): 32 query and 8 key-value heads of 128 or 28 and 4 in bf16, 4 and 2 heads of 64
in float32; blocks of 16, 64 and 128 tokens; requests from one token to 131072.  Key states have a few channels that are eight times as large as the
others, and queries half follow keys of their own request, so that the softmax is neither flat nor a single key.

A batch: request r holds lens[r] tokens and adds n_new[r]; the added tokens of all requests, one behind the other, are the rows of the step.  Block b of
a request's tokens lies in slot block_table[r, b] of the pool, or nowhere (-1: dropped or swapped out, and not attended to).  row_slot names a row's place
in the pool: slot * block + its row of the block.

A slot of blocks of B tokens with H kv heads of d: the Keys' codes [H, B, d] (a byte each: sign, four bits of exponent with bias 7, three of mantissa,
largest 448, 127 not a number), the Values', and per head the bytes e + 127 of the Keys and of the Values [H, 2]; a code stands for its value times
2^e, e the smallest in [-117, 119] for which no magnitude of the head's rows in the block is above 448 * 2^e.  Rows that join a block keep the larger
of its exponent and their own; where it grows, the rows that are there are rounded again.
"""
from __future__ import annotations

import math
import random

import torch

own = False

HEADS = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (4, 2, 64)}     # query heads, kv heads, head size
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
MOST_TOKENS = 131072                    # of a request, for the width of a block table


def listed():
    return [
        # the next token of 256 requests, some of which begin a block with it
        dict(name="map_step_256", kind="map", requests=256, longest=8192, new=1, block=64),
        # 37 prompts that come in together, 32768 tokens at most, in a batch padded to a fixed number of rows
        dict(name="map_prompts_37", kind="map", requests=37, longest=0, new=1700, block=64),
        # the Key and Value states of 24 prompts of up to 2400 tokens, as slices of the projections' joint output
        dict(name="write_prompts_24", kind="write", family="llama", dtype="bf16", block=64, requests=24, longest=0, new=2400),
        # one token each for 256 requests, into blocks that are partly filled
        dict(name="write_step_256", kind="write", family="llama", dtype="bf16", block=16, requests=256, longest=8192, new=1),
        # chunks of a few float32 prompts that begin and end inside a block
        dict(name="write_chunks_fp32", kind="write", family="small", dtype="fp32", block=24, requests=5, longest=301, new=149),
        # the 154 retained blocks of a 32k prompt become rows again, for a follow-up prompt
        dict(name="read_9856", kind="read", family="llama", dtype="bf16", block=64, tokens=9856),
        # a small float32 request, its last block short
        dict(name="read_small_fp32", kind="read", family="small", dtype="fp32", block=16, tokens=509),
        # one token each for 256 requests of 64 to 8192 tokens
        dict(name="attn_step_256", kind="attn", family="llama", dtype="bf16", block=64, requests=256, longest=8192, new=1, kept=1.0),
        # one token behind a 128k prompt
        dict(name="attn_one_131072", kind="attn", family="llama", dtype="bf16", block=128, requests=1, longest=131072, new=1, kept=1.0),
        # the smallest call: one token of a small float32 request
        dict(name="attn_one_509_fp32", kind="attn", family="small", dtype="fp32", block=16, requests=1, longest=509, new=1, kept=1.0),
        # a follow-up prompt of odd length over the tokens that a pruned prompt left, seven query heads per kv head
        dict(name="attn_follow_up_1511", kind="attn", family="qwen", dtype="bf16", block=64, requests=1, longest=9856, new=1511, kept=1.0),
        # drafts of up to five tokens checked for 48 requests of which a third of the blocks is retained
        dict(name="attn_drafts_48", kind="attn", family="llama", dtype="bf16", block=64, requests=48, longest=32768, new=5, kept=0.3),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["map", "write", "write", "read", "attn", "attn", "attn", "attn"])
    block = rng.choice([16, 64, 64, 128, _log(rng, 8, 160)])
    if kind == "map":
        requests = _log(rng, 1, 512)
        new = rng.choice([1, 1, _log(rng, 1, max(1, 32768 // requests))])
        return dict(kind=kind, requests=requests, longest=rng.choice([0, _log(rng, 1, 8192)]), new=new, block=block)
    family = rng.choice(["llama", "llama", "qwen", "small"])
    dtype = "fp32" if family == "small" else rng.choice(["bf16", "bf16", "bf16", "fp32"])
    c = dict(kind=kind, family=family, dtype=dtype, block=block)
    most = 2048 if family == "small" else 32768 if dtype == "bf16" else 8192
    if kind == "read":
        return dict(c, tokens=_log(rng, 1, most))
    if kind == "write":
        requests = _log(rng, 1, 256)
        new = rng.choice([1, _log(rng, 1, max(1, most // requests))])
        return dict(c, requests=requests, longest=rng.choice([0, _log(rng, 1, 4096)]), new=new)
    shape = rng.choice(["one", "step", "drafts", "follow-up"])
    if shape == "one":
        c.update(requests=1, longest=_log(rng, 1, most), new=1)
    elif shape == "step":
        requests = _log(rng, 2, 256)
        c.update(requests=requests, longest=_log(rng, 1, min(most, (1 << 18) // requests)), new=1)
    elif shape == "drafts":
        requests = _log(rng, 1, 48)
        c.update(requests=requests, longest=_log(rng, 1, min(most, (1 << 18) // requests)), new=_log(rng, 2, 16))
    else:
        c.update(requests=rng.choice([1, 1, 2, 3]), longest=rng.choice([0, _log(rng, 1, 4096)]), new=_log(rng, 16, 1024))
    return dict(c, kept=rng.choice([1.0, 1.0, 0.3]))


def _lengths(case):
    """Tokens that each request holds and adds: the longest and a spread over the logarithm of what is shorter.  A function of the case alone."""
    rng = random.Random(case["requests"] * 1000003 + case["longest"] * 101 + case["new"])
    before, new = [], []
    for i in range(case["requests"]):
        most = case["longest"]
        before.append(most if i == 0 or most < 2 else _log(rng, max(1, most // 128), most))
        new.append(case["new"] if i == 0 or case["new"] < 2 else _log(rng, max(1, case["new"] // 8), case["new"]))
    if case["kind"] == "map" and case["requests"] > 3 and case["new"] == 1:
        new[2] = 0                                               # a request that rests in this step
    return before, new


def _blocks(tokens, block):
    return -(-tokens // block)


def _pads(rows):
    return -(-rows // 64) * 64                                   # rows of a batch of fixed size


def _kept_blocks(case):
    """Per request, which of its blocks lie in the pool: the first, those of the last and of the added tokens, and a fraction of the others."""
    before, new = _lengths(case)
    rng = random.Random(case["requests"] * 7919 + case["longest"])
    out = []
    for b, n in zip(before, new):
        nb = _blocks(b + n, case["block"])
        sure = max(0, b - 1) // case["block"]
        out.append([i == 0 or i >= sure or case["kept"] == 1.0 or rng.random() < case["kept"] for i in range(nb)])
    return out


def _in_sight(case):
    """Tokens in the pool, pairs of a query and a key that it sees."""
    before, new = _lengths(case)
    tokens = pairs = 0
    for b, n, kept in zip(before, new, _kept_blocks(case)):
        B = case["block"]
        for i, k in enumerate(kept):
            if not k:
                continue
            lo, hi = i * B, min((i + 1) * B, b + n)
            tokens += hi - lo
            old = max(0, min(hi, b) - lo)
            pairs += old * n
            fresh = hi - max(lo, b)                              # added tokens of this block: token b + j is seen by n - j queries
            if fresh > 0:
                j0 = max(lo, b) - b
                pairs += sum(n - j for j in range(j0, j0 + fresh))
    return tokens, pairs


def work(case):
    if case["kind"] == "map":
        before, new = _lengths(case)
        rows, taken = sum(new), sum(_blocks(b + n, case["block"]) - _blocks(b, case["block"]) for b, n in zip(before, new))
        return {"bytes": 16 * case["requests"] + 8 * _pads(rows) + 8 * taken, "flops": 8 * case["requests"] + 4 * rows}
    Hq, Hkv, d = HEADS[case["family"]]
    es = 2 if case["dtype"] == "bf16" else 4
    row8, row = 2 * Hkv * d, 2 * Hkv * d * es
    if case["kind"] == "read":
        return {"bytes": case["tokens"] * (row8 + row), "flops": case["tokens"] * 2 * Hkv * d}
    if case["kind"] == "write":
        before, new = _lengths(case)
        B = case["block"]
        back = sum(_blocks(b + n, B) - b // B for b, n in zip(before, new)) * B
        return {"bytes": sum(new) * (row + row8 + 4) + back * (row8 + row), "flops": 3 * sum(new) * 2 * Hkv * d}
    tokens, pairs = _in_sight(case)
    return {"bytes": tokens * row8 + 2 * sum(_lengths(case)[1]) * Hq * d * es, "flops": 4 * Hq * d * pairs}


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.host = torch.Generator()
        self.host.manual_seed(seed)

    def normal(self, *shape, std=1.0):
        return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.g)

    def large(self, d):
        """Channels of the Keys that are larger than the others."""
        f = torch.ones(d)
        f[torch.randperm(d, generator=self.host)[:max(1, d // 32)]] = 8.0
        return f.cuda()

    def order(self, n):
        return torch.randperm(n, generator=self.host).to(torch.int32)


# ---- the format, in 32 bits
def _exponent_byte(most):
    """e + 127 of the smallest e in [-117, 119] with most <= 448 * 2^e; most: float32, finite."""
    bits = most.contiguous().view(torch.int32)
    return (((bits + 0x1FFFFF) >> 23) - 8).clamp(10, 246)


def _power(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _round8(y):
    """The nearest value of the format, ties to the even one, 448 for what is above."""
    a = y.abs().clamp(max=448.0)
    low = (a.view(torch.int32) & 0x7F800000).view(torch.float32).clamp(min=2.0 ** -6)     # the power of two below, 2^-6 at least
    return torch.copysign(torch.round(a / low * 8.0) * low / 8.0, y)


def _code(value):
    """The byte of a value of the format."""
    a = value.abs()
    small = (a * 512.0).to(torch.int32)
    code = torch.where(a < 2.0 ** -6, small, (a.view(torch.int32) >> 20) - 960)
    return (code + 128 * (value.view(torch.int32) < 0).to(torch.int32)).to(torch.uint8)


def _grid(device):
    """The values of the 256 codes."""
    c = torch.arange(128, dtype=torch.int32, device=device)
    v = torch.where(c < 8, c.to(torch.float32) / 512.0, ((c + 960) << 20).view(torch.float32))
    v[127] = math.nan
    return torch.cat((v, -v))


def _slot_bytes(block, heads, d):
    return -(-(2 * heads * block * d + 2 * heads) // 16) * 16


def _sections(pool, block, heads, d):
    """Views of pool[slots, bytes]: codes [2, slots, heads, block, d] as (Keys, Values), and exponent bytes [slots, heads, 2]."""
    c = heads * block * d
    k, v = (pool[:, i * c:(i + 1) * c].view(-1, heads, block, d) for i in (0, 1))
    return k, v, pool[:, 2 * c:2 * c + 2 * heads].view(-1, heads, 2)


def _fill(pool, slots, rows, block):
    """Puts rows [blocks * block, heads, d] of Keys and Values into the slots."""
    heads, d = rows[0].shape[1:]
    sections = _sections(pool, block, heads, d)
    for i, x in enumerate(rows):
        x = x.unflatten(0, (-1, block)).transpose(1, 2)          # [blocks, heads, block, d]
        byte = _exponent_byte(x.abs().amax((2, 3)))
        sections[i][slots] = _code(_round8(x / _power(byte)[:, :, None, None]))
        sections[2][slots, :, i] = byte.to(torch.uint8)


def _values(codes, byte):
    """What codes [.., heads, block, d] with bytes [.., heads] stand for, in float32."""
    return _grid(codes.device)[codes.to(torch.int32)] * _power(byte)[..., None, None]


def _table(case, g, slots_of):
    """block_table [requests, blocks of the longest] of the requests' lists of slots, -1 elsewhere."""
    wide = max(len(s) for s in slots_of)
    t = torch.full((len(slots_of), wide + 1), -1, dtype=torch.int32)
    for r, s in enumerate(slots_of):
        t[r, :len(s)] = torch.tensor(s, dtype=torch.int32)
    return t.cuda()


def prepare(case, seed):
    g = _Draw(seed)
    st = {"case": case}
    if own:
        import paper_2508_06447_amd as slim
        st["slim"] = slim
    block = case["block"]
    if case["kind"] == "read":
        Hq, Hkv, d = HEADS[case["family"]]
        nb = _blocks(case["tokens"], block)
        st["pool"] = torch.zeros(nb + 3, _slot_bytes(block, Hkv, d), dtype=torch.uint8, device="cuda")
        st["slots"] = g.order(nb + 3)[:nb].cuda()
        k, v = g.normal(nb * block, Hkv, d) * g.large(d), g.normal(nb * block, Hkv, d)
        _fill(st["pool"], st["slots"].to(torch.int64), (k, v), block)
        st["k_out"] = torch.empty(case["tokens"], Hkv, d, dtype=DTYPE[case["dtype"]], device="cuda")
        st["v_out"] = torch.empty_like(st["k_out"])
        return st
    before, new = _lengths(case)
    rows, R = sum(new), case["requests"]
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    if case["kind"] == "map":
        had = [_blocks(b, block) for b in before]
        need = sum(_blocks(b + n, block) for b, n in zip(before, new))
        st["n_slots"] = need + 40
        order = g.order(st["n_slots"]).tolist()
        slots_of, at = [], 0
        for h in had:
            slots_of.append(order[at:at + h])
            at += h
        wide = _blocks(max(b + n for b, n in zip(before, new)), block)
        st["block_table"] = torch.full((R, wide + 1), -1, dtype=torch.int32)
        for r, s in enumerate(slots_of):
            st["block_table"][r, :len(s)] = torch.tensor(s, dtype=torch.int32)
        st["block_table"] = st["block_table"].cuda()
        st["free_slots"] = torch.tensor([0, 0, 0] + order[at:], dtype=torch.int32).cuda()      # three entries are taken already
        st["used"] = torch.tensor([3], dtype=torch.int32, device="cuda")
        st["lens"], st["n_new"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (before, new))
        st["n_rows"] = _pads(rows)
        for name, size in (("lens_out", R), ("row_start", R + 1), ("row_pos", st["n_rows"]), ("row_slot", st["n_rows"]), ("info", 4)):
            st[name] = torch.empty(size, dtype=torch.int32, device="cuda")
        return st
    Hq, Hkv, d = HEADS[case["family"]]
    dtype, size = DTYPE[case["dtype"]], _slot_bytes(block, Hkv, d)
    if case["kind"] == "write":
        # only the blocks that the rows reach: request r's are slots[at_r ..], the first of which may hold rows already
        reach = [_blocks(b + n, block) - b // block for b, n in zip(before, new)]
        total = sum(reach)
        slots = g.order(total + 3)[:total]
        st["slots"] = slots.cuda()
        st["pool"] = torch.zeros(total + 3, size, dtype=torch.uint8, device="cuda")
        large = g.large(d)
        there = torch.zeros(R * block, 1, 1)                     # 1 for rows that the first blocks hold
        place, at = torch.empty(rows, dtype=torch.int64), 0
        for r in range(R):
            there[r * block:r * block + before[r] % block] = 1.0
            p = before[r] % block + torch.arange(new[r])
            place[start[r]:start[r + 1]] = at * block + p
            at += reach[r]
        st["place"] = place.cuda()                               # of a row among the blocks that are read back
        first = torch.tensor([sum(reach[:r]) for r in range(R)])
        st["first"] = first.cuda()
        row = slots.to(torch.int64)[place // block] * block + place % block
        st["row_slot"] = row.to(torch.int32).cuda()
        k, v = g.normal(R * block, Hkv, d) * large, g.normal(R * block, Hkv, d)
        _fill(st["pool"], st["slots"][st["first"]].to(torch.int64), (0.5 * k * there.cuda(), v * there.cuda()), block)
        st["had"] = torch.tensor([b % block > 0 for b in before]).cuda()
        st["old"] = tuple(x[st["slots"][st["first"]].to(torch.int64)].clone() for x in _sections(st["pool"], block, Hkv, d))
        joint = g.normal(rows, Hq + 2 * Hkv, d)
        joint[:, Hq:Hq + Hkv] *= large
        joint = joint.to(dtype)
        st["k"], st["v"] = joint[:, Hq:Hq + Hkv], joint[:, Hq + Hkv:]
        st["k_out"] = torch.empty(total * block, Hkv, d, dtype=dtype, device="cuda")
        st["v_out"] = torch.empty_like(st["k_out"])
        return st
    kept = _kept_blocks(case)
    total = sum(sum(k) for k in kept)
    order, at = g.order(total + 3).tolist(), 0
    slots_of = []
    for k in kept:
        mine = iter(order[at:at + sum(k)])
        slots_of.append([next(mine) if x else -1 for x in k])
        at += sum(k)
    st["block_table"] = _table(case, g, slots_of)
    st["pool"] = torch.randint(0, 126, (total + 3, size), generator=g.g, device="cuda", dtype=torch.uint8)      # what free slots and unused rows hold
    st["q"] = torch.empty(rows, Hq, d, dtype=dtype, device="cuda")
    large = g.large(d)
    step = max(1, (1 << 18) // block)
    for r, s in enumerate(slots_of):
        mine = [x for x in s if x >= 0]
        for lo in range(0, len(mine), step):
            part = torch.tensor(mine[lo:lo + step], device="cuda")
            k, v = g.normal(len(part) * block, Hkv, d) * large, g.normal(len(part) * block, Hkv, d)
            _fill(st["pool"], part, (k, v), block)
        seen = min(block, k.shape[0], before[r] + new[r])
        pick = torch.randint(0, seen, (new[r],), generator=g.host).cuda()
        st["q"][start[r]:start[r + 1]] = 0.25 * k[pick].repeat_interleave(Hq // Hkv, dim=1) + g.normal(new[r], Hq, d, std=0.5)
    st["start"], st["before"], st["new"], st["slots_of"] = start, before, new, slots_of
    st["row_start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
    st["lens"] = torch.tensor([b + n for b, n in zip(before, new)], dtype=torch.int32, device="cuda")
    st["out"] = torch.empty_like(st["q"])
    if own:
        st["workspace"] = torch.empty(max(256, slim.batch_attn_kv8_workspace_bytes(rows, R, Hq, Hkv, d, dtype)), dtype=torch.uint8, device="cuda")
    return st


def run(state):
    case = state["case"]
    if not own:
        return {"map": _plain_map, "write": _plain_write, "read": _plain_read, "attn": _plain_attn}[case["kind"]](state, case)
    slim, block = state["slim"], case["block"]
    if case["kind"] == "map":
        out = slim.slim_batch_map(state["lens"], state["n_new"], block, state["block_table"], state["free_slots"], state["n_slots"], state["n_rows"],
                                  used=state["used"], lens_out=state["lens_out"], row_start=state["row_start"], row_pos=state["row_pos"],
                                  row_slot=state["row_slot"], info=state["info"])
        return (*out, state["block_table"])
    if case["kind"] == "attn":
        return slim.slim_batch_attn_kv8(state["q"], state["row_start"], state["lens"], state["block_table"], state["pool"], block, HEADS[case["family"]][1],
                                        out=state["out"], workspace=state["workspace"])
    tokens = state["k_out"].shape[0]
    if case["kind"] == "write":
        slim.slim_kv8_write(state["k"], state["v"], state["pool"], block, state["row_slot"])
    return slim.slim_kv8_read(state["pool"], block, tokens, state["slots"], k_out=state["k_out"], v_out=state["v_out"])


# ---- plain forms
def _plain_map(st, case):
    """(lens_out, row_start, row_pos, row_slot, info, block_table)."""
    B, n = case["block"], st["n_rows"]
    lens, new = st["lens"].to(torch.int64), st["n_new"].to(torch.int64)
    had, need = (lens + B - 1) // B, (lens + new + B - 1) // B
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    row_start = torch.cat((zero, torch.cumsum(new, 0)))
    first = torch.cumsum(need - had, 0) - (need - had) + st["used"]            # of a request's new blocks in the list of free slots
    b = torch.arange(st["block_table"].shape[1], device="cuda")[None]
    fresh = (b >= had[:, None]) & (b < need[:, None])
    at = torch.where(fresh, first[:, None] + b - had[:, None], 0)
    table = torch.where(fresh, st["free_slots"][at], st["block_table"])
    t = torch.arange(n, device="cuda")
    r = (t[:, None] >= row_start[None, 1:]).sum(1)
    pad = r >= lens.shape[0]
    r = torch.where(pad, 0, r)
    pos = torch.where(pad, 0, lens[r] + t - row_start[r])
    slot = table[r, torch.where(pad, 0, pos // B)].to(torch.int64)
    row_slot = torch.where(pad | (slot < 0), -1, slot * B + pos % B)
    taken = (need - had).sum()
    info = torch.stack((row_start[-1], taken, zero[0], st["used"][0] + taken))
    return tuple(x.to(torch.int32) for x in (lens + new, row_start, pos, row_slot, info, table))


def _plain_write(st, case):
    """The blocks that the rows reach, as rows: what was there, rounded again where the exponent has grown, and the new rows; zeros behind them."""
    B = case["block"]
    nb = st["slots"].shape[0]
    out = []
    for i, x in enumerate((st["k"], st["v"])):
        codes, byte = st["old"][i], st["old"][2][:, :, i].to(torch.int32)
        wide = torch.zeros(nb * B, *x.shape[1:], device="cuda")
        wide[st["place"]] = x.to(torch.float32)
        wide = wide.view(nb, B, *x.shape[1:])
        mine = _exponent_byte(wide.abs().amax((1, 3)))                           # [blocks, heads]
        byte = torch.where(st["had"][:, None], byte, 10)
        mine[st["first"]] = torch.maximum(mine[st["first"]], byte)
        power = _power(mine)[:, None, :, None]
        new = _round8(wide / power) * power
        old = _values(codes, byte).transpose(1, 2)                               # [requests, block, heads, d]
        now = power[st["first"]]
        new[st["first"]] += torch.where(st["had"][:, None, None, None], _round8(old / now) * now, 0.0)
        out.append(new.flatten(0, 1).to(x.dtype))
    return tuple(out)


def _plain_read(st, case):
    Hq, Hkv, d = HEADS[case["family"]]
    k, v, e = _sections(st["pool"], case["block"], Hkv, d)
    at = st["slots"].to(torch.int64)
    return tuple(_values(c[at], e[at, :, i]).transpose(1, 2).flatten(0, 1)[:case["tokens"]].to(st["k_out"].dtype) for i, c in enumerate((k, v)))


def _plain_attn(st, case):
    Hq, Hkv, d = HEADS[case["family"]]
    G, B = Hq // Hkv, case["block"]
    kc, vc, e = _sections(st["pool"], B, Hkv, d)
    grid = _grid("cuda")
    out = torch.empty_like(st["q"])
    for r, slots in enumerate(st["slots_of"]):
        before, n, lo = st["before"][r], st["new"][r], st["start"][r]
        at = st["block_table"][r, :len(slots)].to(torch.int64)
        there = at >= 0
        token = (torch.arange(len(slots), device="cuda")[:, None] * B + torch.arange(B, device="cuda"))[there].flatten()
        at = at[there]
        p = before + torch.arange(n, device="cuda")
        k, v = ((grid[c[at].to(torch.int32)] * _power(e[at, :, i])[:, :, None, None]).transpose(0, 1).flatten(1, 2) for i, c in enumerate((kc, vc)))
        k, v = k.contiguous(), torch.where((token < before + n)[None, :, None], v, 0.0)
        for i0 in range(0, n, 512):
            i1 = min(n, i0 + 512)
            q = st["q"][lo + i0:lo + i1].to(torch.float32).view(i1 - i0, Hkv, G, d).transpose(0, 1).reshape(Hkv, -1, d)
            s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(Hkv, i1 - i0, G, -1) / math.sqrt(d)
            s = s.masked_fill_((token[None, :] > p[i0:i1, None])[None, :, None], -math.inf)
            s = torch.exp(s - s.amax(-1, keepdim=True))
            s = s / s.sum(-1, keepdim=True)
            o = torch.matmul(s.view(Hkv, (i1 - i0) * G, -1), v).view(Hkv, i1 - i0, G, d)
            out[lo + i0:lo + i1] = o.transpose(0, 1).reshape(i1 - i0, Hq, d).to(out.dtype)
    return out


# ---- from the definitions, in 64 bits
def _exact_grid():
    v = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (x - 10) for x in range(1, 16) for m in range(8)]
    return torch.tensor(v[:127], dtype=torch.float64, device="cuda")


def _exact_round(y):
    grid = _exact_grid()
    a = y.abs()
    up = torch.bucketize(a, grid).clamp(max=126)                  # the first value that is not below
    down = (up - 1).clamp(min=0)
    above, below = grid[up] - a, a - grid[down]
    pick = torch.where((above < below) | ((above == below) & (up % 2 == 0)), up, down)
    return torch.sign(y) * grid[pick]


def _exact_exponent(most):
    """The smallest e in [-117, 119] with most <= 448 * 2^e: counted up from the fraction."""
    m, x = torch.frexp(most / 448.0)                              # most / 448 = m 2^x, m in [0.5, 1)
    e = torch.where(m == 0.5, x - 1, x)
    return torch.where(most == 0, torch.full_like(e, -117), e.clamp(-117, 119)).to(torch.int64)


def _exact_power(e):
    """2^e: its bits, as the power function need not be exact."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_of_codes(c, byte):
    c = c.to(torch.int64)
    grid = torch.cat((_exact_grid(), torch.tensor([math.nan], dtype=torch.float64, device="cuda")))
    value = grid[c % 128] * torch.where(c >= 128, -1.0, 1.0).to(torch.float64)
    return value * _exact_power(byte.to(torch.int64) - 127)[..., None, None]


def exact(case, seed):
    st = prepare(case, seed)
    B = case["block"]
    if case["kind"] == "map":
        lens, new, table = st["lens"].tolist(), st["n_new"].tolist(), st["block_table"].tolist()
        free, used = st["free_slots"].tolist(), int(st["used"][0])
        start, pos, slot, at = [0], [], [], used
        for r, (b, n) in enumerate(zip(lens, new)):
            for x in range(_blocks(b, B), _blocks(b + n, B)):
                table[r][x] = free[at]
                at += 1
            for p in range(b, b + n):
                pos.append(p)
                slot.append(-1 if table[r][p // B] < 0 else table[r][p // B] * B + p % B)
            start.append(start[-1] + n)
        pad = st["n_rows"] - len(pos)
        parts = ([b + n for b, n in zip(lens, new)], start, pos + [0] * pad, slot + [-1] * pad, [start[-1], at - used, 0, at], table)
        return tuple(torch.tensor(x, dtype=torch.int32, device="cuda") for x in parts)
    Hq, Hkv, d = HEADS[case["family"]]
    if case["kind"] == "read":
        k, v, e = _sections(st["pool"], B, Hkv, d)
        out = []
        for i, c in enumerate((k, v)):
            rows = [_exact_of_codes(c[s], e[s, :, i]).transpose(0, 1) for s in st["slots"].tolist()]
            out.append(torch.cat(rows)[:case["tokens"]])
        return tuple(out)
    if case["kind"] == "write":
        place, first, had = st["place"].tolist(), st["first"].tolist(), st["had"].tolist()
        rows_of = [[] for _ in range(st["slots"].shape[0])]
        for t, p in enumerate(place):
            rows_of[p // B].append((p % B, t))
        owner = {b: r for r, b in enumerate(first)}
        out = []
        for i, x in enumerate((st["k"], st["v"])):
            whole = torch.zeros(len(rows_of), B, Hkv, d, dtype=torch.float64, device="cuda")
            for b, pairs in enumerate(rows_of):
                r = owner.get(b)
                t0, r0 = pairs[0][1], pairs[0][0]
                mine = x[t0:t0 + len(pairs)].to(torch.float64)
                e = _exact_exponent(mine.abs().amax((0, 2)))
                if r is not None and had[r]:
                    byte = st["old"][2][r, :, i]
                    e = torch.maximum(e, byte.to(torch.int64) - 127)
                    unit = _exact_power(e)[None, :, None]
                    old = _exact_of_codes(st["old"][i][r], byte).transpose(0, 1)[:r0]
                    whole[b, :r0] = _exact_round(old / unit) * unit
                unit = _exact_power(e)[None, :, None]
                whole[b, r0:r0 + len(pairs)] = _exact_round(mine / unit) * unit
            out.append(whole.flatten(0, 1))
        return tuple(out)
    G, scale = Hq // Hkv, 1.0 / math.sqrt(d)
    kc, vc, e = _sections(st["pool"], B, Hkv, d)
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for r, slots in enumerate(st["slots_of"]):
        last, n, lo = st["before"][r] + st["new"][r], st["new"][r], st["start"][r]
        where = [(b, s) for b, s in enumerate(slots) if s >= 0]
        at = torch.tensor([s for _, s in where], device="cuda")
        token = torch.cat([torch.arange(b * B, (b + 1) * B) for b, _ in where]).cuda()
        use = token < last
        token = token[use]
        for g in range(Hkv):
            k, v = (_exact_of_codes(c[at, g:g + 1], e[at, g:g + 1, i]).flatten(0, 2)[use] for i, c in enumerate((kc, vc)))
            for i0 in range(0, n, 256):
                i1 = min(n, i0 + 256)
                q = st["q"][lo + i0:lo + i1, g * G:(g + 1) * G].to(torch.float64).reshape(-1, d)
                a = (torch.mm(q, k.t().contiguous()) * scale).view(i1 - i0, G, -1)
                p = last - n + torch.arange(i0, i1, device="cuda")
                a = a.masked_fill((token[None] > p[:, None])[:, None], -math.inf)
                weight = torch.softmax(a, -1).view((i1 - i0) * G, -1)
                out[lo + i0:lo + i1, g * G:(g + 1) * G] = torch.mm(weight, v).view(i1 - i0, G, d)
    return out
