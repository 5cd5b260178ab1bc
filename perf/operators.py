"""The operators that work on a prompt's Key-Value cache once the prefill is done, as they are timed: blocks of the cache written in 4 bits and
read back, a decoded token's attention over the blocks as they lie in their slots, and causal attention with a sliding window and visible first
tokens for prompts, follow-up prompts and single tokens.

Shapes are the repository's workloads (paper_2508_06447_amd/inputs.py): 32 query and 8 key-value heads of 128 or 28 and 4 in bf16, 4 and 2 heads of
64 in float32; prompts of up to 131072 tokens in blocks of 16, 64 and 128.  Key states have a few channels that are eight times as large as the
others, as rotated keys of trained models have, and half of a query head's states follow its kv head's keys, so that the softmax is neither flat
nor a single key.

A cached row is held in groups of 32 channels: one power of two 2^e per group, with the largest magnitude in [3.5, 7) of it, and per channel the nearest of 0, 0.5, 1,
1.5, 2, 3, 4, 6 times it, ties to the even code, with a sign.  One slot holds of a block of B tokens and H kv heads, heads first, tokens next: the Keys'
codes [H, B, d / 2] (channel 2 i in the low half of byte i), the Values' codes, the Keys' e + 127 [H, B, d / 32], the Values'.
"""
from __future__ import annotations

import math

import torch

own = False

HEADS = {"llama": (32, 8, 128), "qwen": (28, 4, 128), "small": (4, 2, 64)}     # query heads, kv heads, head size
DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
SINKS = 64                              # first tokens that a long answer keeps in sight: the first block


def listed():
    return [
        # a prompt's blocks as they leave the prefill, into slots that lie in no order, and read back whole
        dict(name="write_32768", kind="write", family="llama", dtype="bf16", block=64, first=0, tokens=32768),
        # a chunk of a prompt that begins and ends inside a block
        dict(name="write_chunk_1511", kind="write", family="qwen", dtype="bf16", block=128, first=2983, tokens=1511),
        # one more token behind 9856 others; its block is read back
        dict(name="write_one_token", kind="write", family="llama", dtype="bf16", block=64, first=9860, tokens=1),
        # a follow-up prompt: the 154 retained blocks of a 32k prompt become rows again
        dict(name="read_154_of_512", kind="read", family="llama", dtype="bf16", block=64, tokens=32768, blocks=154),
        # the small float32 cache, whole, its last block short
        dict(name="read_small_fp32", kind="read", family="small", dtype="fp32", block=16, tokens=509, blocks=32),
        # one decoded token: 8k active prompt tokens and a short answer
        dict(name="decode_128_slots", kind="decode", family="llama", dtype="bf16", block=64, slots=128, response=17),
        # the whole of a 128k prompt behind a longer answer
        dict(name="decode_2048_slots", kind="decode", family="llama", dtype="bf16", block=64, slots=2048, response=301),
        # numbers checked in float32, seven query heads per kv head, blocks that end inside a tile
        dict(name="decode_fp32_37_slots", kind="decode", family="qwen", dtype="fp32", block=80, slots=37, response=5),
        # a 32k prompt with a window of 4096 tokens and the first block in sight
        dict(name="sliding_prompt_32768", kind="sliding", family="llama", dtype="bf16", queries=32768, keys=32768, window=4096, sinks=SINKS),
        # a follow-up prompt of odd length over the retained tokens, all of them in sight
        dict(name="sliding_follow_up_1511", kind="sliding", family="qwen", dtype="bf16", queries=1511, keys=9856 + 1511, window=9856 + 1511, sinks=0),
        # one decoded token with a dense cache
        dict(name="sliding_token", kind="sliding", family="llama", dtype="bf16", queries=1, keys=32768, window=4096, sinks=SINKS),
        # the small float32 prompt, a window that is no multiple of anything
        dict(name="sliding_small_fp32", kind="sliding", family="small", dtype="fp32", queries=512, keys=512, window=101, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "decode", "decode", "sliding", "sliding", "sliding"])
    family = rng.choice(["llama", "llama", "qwen", "small" if kind != "decode" else "qwen"])
    dtype = "fp32" if family == "small" else rng.choice(["bf16", "bf16", "bf16", "fp32"]) if kind != "sliding" else "bf16"
    c = dict(kind=kind, family=family, dtype=dtype)
    if kind == "sliding":
        keys = _log(rng, 64, 2048) if family == "small" else _log(rng, 64, 32768)
        queries = rng.choice([1, _log(rng, 1, min(keys, 64)), _log(rng, 1, keys), keys])
        c.update(queries=queries, keys=keys, window=min(_log(rng, 1, 4096), keys), sinks=rng.choice([0, 1, 4, SINKS, _log(rng, 1, 300)]))
        if family != "small" and rng.random() < 0.3 and queries <= 2048:
            c["window"] = keys
        return c
    c["block"] = rng.choice([16, 64, 64, 128, _log(rng, 16, 160)])
    most = 2048 if family == "small" else 32768 if dtype == "bf16" else 8192
    if kind == "write":
        tokens = _log(rng, 1, most)
        c.update(first=rng.choice([0, _log(rng, 1, 16384)]), tokens=tokens)
    elif kind == "read":
        tokens = _log(rng, 1, most)
        nb = -(-tokens // c["block"])
        c.update(tokens=tokens, blocks=rng.choice([nb, rng.randint(1, nb)]))
    else:
        slots = _log(rng, 1, (131072 if dtype == "bf16" else 16384) // c["block"])
        c.update(slots=slots, response=rng.choice([0, 1, _log(rng, 1, 1500)]))
    return c


def _visible(case):
    """Keys that any query of the case sees, and pairs of a query and a key that it sees."""
    n, m, w, s = case["keys"], case["queries"], case["window"], case["sinks"]
    pairs = 0
    for p0 in range(n - m, n, 65536):
        p = torch.arange(p0, min(n, p0 + 65536), dtype=torch.int64)
        near = torch.clamp(p + 1, max=w)
        pairs += int((near + torch.minimum(torch.clamp(p + 1 - near, min=0), torch.tensor(s))).sum())
    first = max(0, n - m - w + 1)
    return n - first + min(s, first), pairs


def work(case):
    Hq, Hkv, d = HEADS[case["family"]]
    es = 2 if case["dtype"] == "bf16" else 4
    row4 = 2 * Hkv * (d // 2 + d // 32)                        # a token's Key and Value states in 4 bits
    row = 2 * Hkv * d * es
    if case["kind"] == "write":
        back = case["first"] + case["tokens"] - case["first"] // case["block"] * case["block"]
        return {"bytes": case["tokens"] * (row + row4) + back * (row4 + row), "flops": 4 * case["tokens"] * Hkv * d}
    if case["kind"] == "read":
        n = _rows_of(case["tokens"], case["block"], case["blocks"])
        return {"bytes": n * (row4 + row), "flops": 2 * n * Hkv * d}
    if case["kind"] == "decode":
        n = _prompt_in_slots(case)
        return {"bytes": n * row4 + case["response"] * row + 2 * Hq * d * es, "flops": 4 * Hq * d * (n + case["response"])}
    keys, pairs = _visible(case)
    return {"bytes": keys * row + 2 * case["queries"] * Hq * d * es, "flops": 4 * Hq * d * pairs}


def _rows_of(tokens, block, blocks):
    """Tokens in `blocks` blocks, the last and perhaps short one among them."""
    return tokens - (-(-tokens // block) - blocks) * block


def _spare(slots):
    return slots // 16                                         # slots of the pool that are free


def _prompt_tokens(case):
    return (case["slots"] + 3) * case["block"] - case["block"] // 3


def _prompt_in_slots(case):
    """Prompt tokens that lie in slots: the last, short block of the prompt is among them."""
    return (case["slots"] - _spare(case["slots"])) * case["block"] - case["block"] // 3


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.host = torch.Generator()
        self.host.manual_seed(seed)

    def normal(self, *shape, std=1.0):
        return torch.empty(*shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.g)

    def keys(self, n, heads, d):
        k = self.normal(n, heads, d)
        k[:, :, torch.randperm(d, generator=self.host)[:max(1, d // 32)].cuda()] *= 8.0
        return k

    def queries(self, n, k, group):
        """Half noise, half the keys of the same kv head, picked at random."""
        pick = torch.randint(0, k.shape[0], (n,), generator=self.host).cuda()
        return 0.25 * k[pick].repeat_interleave(group, dim=1) + self.normal(n, k.shape[1] * group, k.shape[2], std=0.5)

    def order(self, n):
        return torch.randperm(n, generator=self.host).to(torch.int32)


def _groups(x):
    """Codes (as whole numbers below 16) and e + 127 of the groups of 32 along the last axis."""
    g = x.to(torch.float32).unflatten(-1, (-1, 32))
    most = g.abs().amax(-1, keepdim=True)
    bits = (most.view(torch.int32) + (1 << 21)) >> 23          # a magnitude from 1.75 times a power of two on counts as the next power
    byte = (bits - 2).clamp(2, 252)
    y = g.abs() * ((254 - byte) << 23).view(torch.float32)
    code = sum((y > t).to(torch.int32) if open_ else (y >= t).to(torch.int32) for t, open_ in
               ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)))
    code = code + 8 * (g < 0).to(torch.int32)
    return code.flatten(-2), byte.squeeze(-1)


def _values(code, byte):
    """What codes [.., d] and e + 127 [.., d / 32] stand for, in float32."""
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=code.device)
    scale = (byte.to(torch.int32) << 23).view(torch.float32)
    return (grid[code.to(torch.int64)].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _sections(pool, block, heads, d):
    """The four parts of every slot of pool[slots, bytes]: codes [slots, heads, block, d / 2] and e + 127 [slots, heads, block, d / 32] of Keys and Values."""
    c, s, out, at = heads * block * (d // 2), heads * block * (d // 32), [], 0
    for size, last in ((c, d // 2), (c, d // 2), (s, d // 32), (s, d // 32)):
        out.append(pool[:, at:at + size].view(pool.shape[0], heads, block, last))
        at += size
    return out


def _slot_bytes(block, heads, d):
    return -(-heads * block * (d + d // 16) // 16) * 16


def _fill(pool, rows, slots, block, heads, d):
    """Puts rows (k, v) [blocks * block, heads, d] into the slots of their blocks."""
    kc, vc, ks, vs = _sections(pool, block, heads, d)
    for x, codes, scales in ((rows[0], kc, ks), (rows[1], vc, vs)):
        code, byte = _groups(x.unflatten(0, (-1, block)).transpose(1, 2))
        codes[slots] = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
        scales[slots] = byte.to(torch.uint8)


def _unpacked(codes, scales):
    code = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    return _values(code, scales)


def prepare(case, seed):
    Hq, Hkv, d = HEADS[case["family"]]
    dtype, g = DTYPE[case["dtype"]], _Draw(seed)
    st = {"case": case}
    if case["kind"] == "sliding":
        k = g.keys(case["keys"], Hkv, d)
        st["q"] = g.queries(case["queries"], k, Hq // Hkv).to(dtype)
        st["k"], st["v"] = k.to(dtype), g.normal(case["keys"], Hkv, d).to(dtype)
        st["out"] = torch.empty_like(st["q"])
        if own:
            import paper_2508_06447_amd as slim
            st["slim"] = slim
            st["workspace"] = torch.empty(max(256, slim.sliding_attn_workspace_bytes(case["queries"], case["keys"], Hq, Hkv, d, case["window"],
                                                                                    case["sinks"], dtype)), dtype=torch.uint8, device="cuda")
        return st
    block = case["block"]
    size = _slot_bytes(block, Hkv, d)
    if own:
        import paper_2508_06447_amd as slim
        st["slim"] = slim
    if case["kind"] == "write":
        nb = -(-(case["first"] + case["tokens"]) // block)
        n0 = case["first"] // block * block                     # the blocks that the chunk reaches, and their rows that are there already
        there = torch.cat((g.keys(block, Hkv, d), g.normal(block, Hkv, d))).to(dtype)
        st["pool"] = torch.zeros(nb + 1, size, dtype=torch.uint8, device="cuda")
        st["slot_of_block"] = g.order(nb + 1)[:nb].cuda()
        st["k"], st["v"] = g.keys(case["tokens"], Hkv, d).to(dtype), g.normal(case["tokens"], Hkv, d).to(dtype)
        _fill(st["pool"], (there[:block], there[block:]), st["slot_of_block"][n0 // block:n0 // block + 1].to(torch.int64), block, Hkv, d)
        st["old"] = _sections(st["pool"][int(st["slot_of_block"][n0 // block])].clone()[None], block, Hkv, d)
        st["blocks"] = torch.arange(n0 // block, nb, dtype=torch.int32, device="cuda")
        rows = case["first"] + case["tokens"] - n0
    elif case["kind"] == "read":
        nb = -(-case["tokens"] // block)
        st["pool"] = torch.zeros(nb + 1, size, dtype=torch.uint8, device="cuda")
        st["slot_of_block"] = g.order(nb + 1)[:nb].cuda()
        _fill(st["pool"], (g.keys(nb * block, Hkv, d), g.normal(nb * block, Hkv, d)), st["slot_of_block"].to(torch.int64), block, Hkv, d)
        some = g.order(nb - 1)[:case["blocks"] - 1].sort().values if case["blocks"] > 1 else torch.empty(0, dtype=torch.int32)
        st["blocks"] = torch.cat((some, torch.tensor([nb - 1], dtype=torch.int32))).cuda()
        rows = _rows_of(case["tokens"], block, case["blocks"])
    else:
        ns, R = case["slots"], case["response"]
        used = ns - _spare(ns)
        nb = -(-_prompt_tokens(case) // block)
        block_of_slot = torch.full((ns,), -1, dtype=torch.int32)
        blocks = torch.cat((g.order(nb - 1)[:used - 1], torch.tensor([nb - 1], dtype=torch.int32)))
        at = g.order(ns)[:used].to(torch.int64)
        block_of_slot[at] = blocks
        st["block_of_slot"] = block_of_slot.cuda()
        st["pool"] = torch.randint(0, 250, (ns, size), generator=g.g, device="cuda", dtype=torch.uint8)      # what free slots and unused rows hold
        k, v = g.keys(used * block, Hkv, d), g.normal(used * block, Hkv, d)
        _fill(st["pool"], (k, v), at.cuda(), block, Hkv, d)
        st["q"] = g.queries(1, k, Hq // Hkv)[0].to(dtype)
        st["k_response"], st["v_response"] = g.keys(R, Hkv, d).to(dtype), g.normal(R, Hkv, d).to(dtype)
        st["out"] = torch.empty_like(st["q"])
        if own:
            need = slim.load_library().slim_decode_attn_workspace_bytes(ns, R, Hq)
            st["workspace"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
        return st
    st["k_out"] = torch.empty(rows, Hkv, d, dtype=dtype, device="cuda")
    st["v_out"] = torch.empty_like(st["k_out"])
    return st


def run(state):
    case = state["case"]
    if own:
        slim = state["slim"]
        if case["kind"] == "sliding":
            return slim.slim_sliding_attn(state["q"], state["k"], state["v"], case["window"], case["sinks"], out=state["out"], workspace=state["workspace"])
        if case["kind"] == "decode":
            return slim.slim_decode_attn_kv4(state["q"], state["pool"], state["block_of_slot"], case["block"], _prompt_tokens(case), state["k_response"].shape[1],
                                             state["k_response"] if case["response"] else None, state["v_response"] if case["response"] else None,
                                             out=state["out"], workspace=state["workspace"])
        total = case["tokens"]
        if case["kind"] == "write":
            total += case["first"]
            slim.slim_kv4_write(state["k"], state["v"], state["pool"], case["block"], state["slot_of_block"], first_token=case["first"])
        return slim.slim_kv4_read(state["pool"], case["block"], total, state["slot_of_block"], state["blocks"], k_out=state["k_out"], v_out=state["v_out"])
    return {"write": _plain_write, "read": _plain_read, "decode": _plain_decode, "sliding": _plain_sliding}[case["kind"]](state, case)


def _plain_write(state, case):
    """What the blocks that the chunk reaches stand for afterwards: the rows of the first one that were there already, and the chunk's."""
    part = case["first"] % case["block"]
    old = state["old"]
    out = []
    for x, codes, scales in ((state["k"], old[0], old[2]), (state["v"], old[1], old[3])):
        there = _unpacked(codes[0, :, :part], scales[0, :, :part]).transpose(0, 1)
        out.append(torch.cat((there, _values(*_groups(x)))).to(x.dtype))
    return tuple(out)


def _plain_read(state, case):
    Hq, Hkv, d = HEADS[case["family"]]
    slots = state["slot_of_block"][state["blocks"].to(torch.int64)].to(torch.int64)
    kc, vc, ks, vs = _sections(state["pool"], case["block"], Hkv, d)
    rows = state["k_out"].shape[0]
    return tuple(_unpacked(c[slots], s[slots]).transpose(1, 2).flatten(0, 1)[:rows].to(state["k_out"].dtype) for c, s in ((kc, ks), (vc, vs)))


def _softmax(s):
    p = torch.exp(s - s.amax(-1, keepdim=True))
    return p / p.sum(-1, keepdim=True)


def _plain_decode(state, case):
    Hq, Hkv, d = HEADS[case["family"]]
    block, of = case["block"], state["block_of_slot"]
    kc, vc, ks, vs = _sections(state["pool"], block, Hkv, d)
    token = of[:, None] * block + torch.arange(block, device="cuda")
    seen = ((of[:, None] >= 0) & (token < _prompt_tokens(case))).flatten()
    seen = torch.cat((seen, torch.ones(case["response"], dtype=torch.bool, device="cuda")))
    k, v = (torch.cat((_unpacked(c, s).transpose(1, 2).flatten(0, 1), r.to(torch.float32))).transpose(0, 1)
            for c, s, r in ((kc, ks, state["k_response"]), (vc, vs, state["v_response"])))
    q = state["q"].to(torch.float32).view(Hkv, Hq // Hkv, d)
    p = _softmax((torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)).masked_fill_(~seen, -math.inf))
    return torch.matmul(p, v.contiguous()).view(Hq, d).to(state["q"].dtype)


def _plain_sliding(state, case):
    """Query tiles against the stretch of keys that their windows cover; the first keys beside it where a window has left them behind."""
    Hq, Hkv, d = HEADS[case["family"]]
    m, n, w, s, G = case["queries"], case["keys"], case["window"], min(case["sinks"], case["keys"]), Hq // Hkv
    tile = min(m, 256)
    tiles, off = -(-m // tile), n - m
    long = w - 1 + tile                                          # keys of a tile's stretch
    q = torch.zeros(tiles * tile, Hq, d, device="cuda")
    q[:m] = state["q"].to(torch.float32)
    q = q.view(tiles, tile, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(tiles, Hkv, G * tile, d)

    def stretch(x):
        # the stretch of tile t begins with key off + t * tile - (w - 1); what lies outside the keys is zero, and not seen
        wide = torch.zeros(Hkv, d, off + tiles * tile + w - 1, device="cuda")
        wide[:, :, w - 1:w - 1 + n] = x.to(torch.float32).permute(1, 2, 0)
        return wide[:, :, off:].unfold(2, long, tile).permute(2, 0, 1, 3)            # [tiles, Hkv, d, long]

    at = torch.arange(tiles, device="cuda")[:, None, None] * tile + off
    p = at + torch.arange(tile, device="cuda")[None, :, None]
    j = at - (w - 1) + torch.arange(long, device="cuda")[None, None, :]
    near = (j >= 0) & (j <= p) & (j > p - w) & (j < n)
    first = torch.arange(s, device="cuda")[None, None, :]
    far = first <= p - w
    k0, v0 = (x[:s].to(torch.float32).transpose(0, 1)[None].expand(tiles, -1, -1, -1) for x in (state["k"], state["v"]))
    score = torch.cat((torch.matmul(q, stretch(state["k"]).contiguous()), torch.matmul(q, k0.transpose(2, 3).contiguous())), -1)
    seen = torch.cat((near, far), -1)[:, None, None]             # [tiles, 1, 1, tile, keys]
    score = (score / math.sqrt(d)).view(tiles, Hkv, G, tile, long + s)
    score = score.masked_fill_(~seen, -math.inf)
    score -= torch.clamp(score.amax(-1, keepdim=True), min=-3e38)                   # (rows behind the last query may see nothing)
    score = score.exp_()
    total = score.sum(-1, keepdim=True).view(tiles, Hkv, G * tile, 1)
    score = score.view(tiles, Hkv, G * tile, long + s)
    out = torch.matmul(score[..., :long], stretch(state["v"]).transpose(2, 3).contiguous()) + torch.matmul(score[..., long:], v0.contiguous())
    out = (out / total).view(tiles, Hkv, G, tile, d).permute(0, 3, 1, 2, 4).reshape(tiles * tile, Hq, d)[:m]
    return out.to(state["q"].dtype)


# ---- from the definitions, in 64 bits
def _exact_values(x):
    """The nearest of sixteen multiples of a group's power of two."""
    g = x.to(torch.float64).unflatten(-1, (-1, 32))
    most = g.abs().amax(-1, keepdim=True)
    mantissa, exponent = torch.frexp(most)                       # most = mantissa * 2^exponent, mantissa in [0.5, 1)
    e = torch.where(most == 0, torch.full_like(exponent, -125), torch.clamp(exponent - 3 + (mantissa >= 0.875).to(exponent.dtype), -125, 125))
    unit = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), e.to(torch.float64))
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)
    y = (g / unit).abs()
    up = torch.bucketize(y, grid).clamp(max=7)                   # the first value that is not below y
    down = (up - 1).clamp(min=0)
    above, below = grid[up] - y, y - grid[down]
    pick = torch.where((above < below) | ((above == below) & (up % 2 == 0)), up, down)
    return (torch.sign(g) * grid[pick] * unit).flatten(-2)


def _exact_unpacked(codes, scales):
    c = codes.to(torch.int64)
    two = torch.empty(*c.shape[:-1], 2 * c.shape[-1], dtype=torch.int64, device=c.device)
    two[..., 0::2], two[..., 1::2] = c % 16, c // 16
    size = two % 8
    sub = size < 2                                               # below one: halves; else 1 + half the low bit times a power of two
    value = torch.where(sub, 0.5 * size, (1 + 0.5 * (size % 2)) * torch.pow(2.0, (size // 2 - 1).to(torch.float64)))
    value = torch.where(two >= 8, -value, value)
    power = torch.pow(2.0, scales.to(torch.float64) - 127).repeat_interleave(32, dim=-1)
    return value * power


def exact(case, seed):
    st = prepare(case, seed)
    Hq, Hkv, d = HEADS[case["family"]]
    G = Hq // Hkv
    if case["kind"] == "write":
        part, out = case["first"] % case["block"], []
        for x, c, s in ((st["k"], 0, 2), (st["v"], 1, 3)):
            old = _exact_unpacked(st["old"][c][0], st["old"][s][0]).permute(1, 0, 2)[:part]
            out.append(torch.cat((old, _exact_values(x))))
        return tuple(out)
    if case["kind"] == "read":
        parts, block = _sections(st["pool"], case["block"], Hkv, d), case["block"]
        out = []
        for c, s in ((0, 2), (1, 3)):
            rows = []
            for b in st["blocks"].tolist():
                slot = int(st["slot_of_block"][b])
                rows.append(_exact_unpacked(parts[c][slot], parts[s][slot]).permute(1, 0, 2)[:min(block, case["tokens"] - b * block)])
            out.append(torch.cat(rows))
        return tuple(out)
    scale = 1.0 / math.sqrt(d)
    if case["kind"] == "decode":
        parts, block = _sections(st["pool"], case["block"], Hkv, d), case["block"]
        of = st["block_of_slot"].tolist()
        ks, vs = [], []
        for lo in range(0, len(of), 64):
            kd, vd = (_exact_unpacked(parts[c][lo:lo + 64], parts[s][lo:lo + 64]) for c, s in ((0, 2), (1, 3)))
            for i, b in enumerate(of[lo:lo + 64]):
                rows = min(block, _prompt_tokens(case) - b * block)
                if b >= 0:
                    ks.append(kd[i, :, :rows])
                    vs.append(vd[i, :, :rows])
        ks.append(st["k_response"].to(torch.float64).permute(1, 0, 2))
        vs.append(st["v_response"].to(torch.float64).permute(1, 0, 2))
        k, v, q = torch.cat(ks, 1), torch.cat(vs, 1), st["q"].to(torch.float64)
        out = torch.empty(Hq, d, dtype=torch.float64, device="cuda")
        for h in range(Hq):
            weight = torch.softmax((k[h // G] * q[h]).sum(-1) * scale, 0)
            out[h] = (weight[:, None] * v[h // G]).sum(0)
        return out
    m, n, w, s = case["queries"], case["keys"], case["window"], case["sinks"]
    out = torch.empty(m, Hq, d, dtype=torch.float64, device="cuda")
    step = 512
    for i0 in range(0, m, step):
        i1 = min(m, i0 + step)
        p = torch.arange(n - m + i0, n - m + i1, device="cuda")
        low, high = max(0, n - m + i0 - w + 1), n - m + i1
        j = torch.cat((torch.arange(0, min(s, low), device="cuda"), torch.arange(low, high, device="cuda")))
        hidden = (j[None] > p[:, None]) | ((j[None] <= p[:, None] - w) & (j[None] >= s))
        for g in range(Hkv):
            k, v = st["k"][j, g].to(torch.float64), st["v"][j, g].to(torch.float64)
            q = st["q"][i0:i1, g * G:(g + 1) * G].to(torch.float64).reshape(-1, d)
            a = torch.mm(q, k.t().contiguous()) * scale
            a = a.view(i1 - i0, G, -1).masked_fill(hidden[:, None], -math.inf)
            out[i0:i1, g * G:(g + 1) * G] = torch.mm(torch.softmax(a, -1).view((i1 - i0) * G, -1), v).view(i1 - i0, G, d)
    return out
