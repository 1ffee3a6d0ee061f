"""The operators around a decode step over the hierarchical codec's cache, over the
sizes that serving gives them.

A case is a dict of plain values.  `kind` names the operator:

  attn    attention over the cache as lynx_hkv_encode leaves it, read straight
          from its 4-bit planes (anchors, or the single 4-bit code) or from
          its merged 8-bit codes, with the BF16 tokens behind it
          (lynx_attn_hier)
  rope    the norm of every query and key head, the rotation by its token's
          position, and V, from the rows of one fused projection to the rows
          that attention and the append read (lynx_qk_norm_rope)
  blocks  the step's plan: blocks for the new tokens of every sequence out of a
          free stack, block table, slots, positions and rows of the tokens, and
          the blocks given back once the drafts are dropped (lynx_blocks_extend,
          lynx_blocks_release)

Contexts: `batch` sequences of `tokens` tokens, or spread over
[min_tokens, tokens], the last `empty` of them without any; block_tokens 0 is
one block per sequence, anything else a paged pool under a random block table.
K channels are normal, 1% of them 8 times larger.

`own` chooses who computes: this file's plain form, in elementary torch
operations, or the framework's calls.
"""
import math
import random

import torch

own = False

D = 128
PAGE, CHUNK = 256, 32  # tokens of the codec's pages and chunks
BIASED, CENTRED, INT4 = 0, 1, 2

# No drawn case does more than the largest listed one of its kind.
MOST_TOKEN_HEADS = 4 * 65536 * 8     # tokens of all sequences x kv heads
MOST_ROW_TOKENS = 32768 * 8 * 80     # the same x query rows of a kv head
MOST_ROPE_HEADS = 16384 * 48         # tokens x heads of Q, K and V
MOST_STEP_TOKENS = 131072            # tokens of a step's plan


def listed():
    return [
        # a small model's layer at 4K context, one token of one user: latency alone
        dict(name="attn-4k-b1", kind="attn", batch=1, q_heads=8, kv_heads=4, tokens=4096, min_tokens=0, empty=0, block_tokens=0,
             drafts=1, tail=0, variant=INT4, full=False, alpha=255.0),
        # drafting on the anchors while the residual is on its way: a ragged paged batch, 21 tokens generated so far
        dict(name="attn-paged-b16-tail21", kind="attn", batch=16, q_heads=32, kv_heads=8, tokens=8192, min_tokens=1024, empty=1,
             block_tokens=16, drafts=1, tail=21, variant=CENTRED, full=False, alpha=255.0),
        # a 70B-shaped layer over four long contexts held in 4 bits: the largest
        dict(name="attn-64k-b4", kind="attn", batch=4, q_heads=64, kv_heads=8, tokens=65536, min_tokens=0, empty=0,
             block_tokens=0, drafts=1, tail=0, variant=INT4, full=False, alpha=255.0),
        # verification of 20 drafts over the merged codes, one long context
        dict(name="attn-full-32k-k20", kind="attn", batch=1, q_heads=32, kv_heads=8, tokens=32768, min_tokens=0, empty=0,
             block_tokens=0, drafts=20, tail=20, variant=CENTRED, full=True, alpha=255.0),
        # a chunk of 33 queries, seven heads a kv head, blocks that chunks and pages straddle
        dict(name="attn-paged-b3-k33", kind="attn", batch=3, q_heads=28, kv_heads=4, tokens=6001, min_tokens=2000, empty=0,
             block_tokens=48, drafts=33, tail=40, variant=INT4, full=False, alpha=15.0),
        # one token of one user
        dict(name="rope-1", kind="rope", tokens=1, q_heads=32, kv_heads=8, rotary=128, pairs=False, norm=True, values=True,
             spread=False),
        # a decode step of a batch, padded, half of each head rotated in neighbouring pairs
        dict(name="rope-61-padded", kind="rope", tokens=61, q_heads=64, kv_heads=8, rotary=64, pairs=True, norm=True,
             values=True, spread=True),
        # a chunk of odd length, no norm, V left where it is
        dict(name="rope-2999", kind="rope", tokens=2999, q_heads=28, kv_heads=4, rotary=128, pairs=False, norm=False,
             values=False, spread=False),
        # a long prompt
        dict(name="rope-16384", kind="rope", tokens=16384, q_heads=32, kv_heads=8, rotary=128, pairs=False, norm=True,
             values=True, spread=False),
        # one user, one token
        dict(name="blocks-b1", kind="blocks", batch=1, tokens=32768, block_tokens=16, most=1, rows=1, short=False),
        # a batch's drafts
        dict(name="blocks-b64-k8", kind="blocks", batch=64, tokens=16384, block_tokens=16, most=8, rows=512, short=False),
        # a busy server: prompts in chunks next to single tokens, more asked than there are blocks
        dict(name="blocks-b500-chunks", kind="blocks", batch=500, tokens=8192, block_tokens=32, most=4096, rows=131072,
             short=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "rope", "rope", "blocks"])
    if kind == "rope":
        q_heads, kv_heads = rng.choice([(8, 4), (32, 8), (64, 8), (28, 4), (16, 16), (5, 1)])
        return dict(kind=kind, tokens=_log_int(rng, 1, MOST_ROPE_HEADS // (q_heads + 2 * kv_heads)), q_heads=q_heads,
                    kv_heads=kv_heads, rotary=rng.choice([16, 32, 48, 64, 96, 112, 128, 128, 128]), pairs=rng.random() < 0.4,
                    norm=rng.random() < 0.75, values=rng.random() < 0.75, spread=rng.random() < 0.4)
    if kind == "blocks":
        batch = _log_int(rng, 1, 2000)
        most = _log_int(rng, 1, 4096)
        return dict(kind=kind, batch=batch, tokens=_log_int(rng, 1, 32768), block_tokens=rng.choice([1, 16, 16, 32, 48, 128]),
                    most=most, rows=min(MOST_STEP_TOKENS, max(1, int(batch * most * rng.choice([0.4, 1.0])))),
                    short=rng.random() < 0.4)
    q_heads, kv_heads = rng.choice([(8, 4), (32, 8), (32, 8), (64, 8), (28, 4), (20, 1)])
    c = dict(kind=kind, batch=_log_int(rng, 1, 32), q_heads=q_heads, kv_heads=kv_heads)
    c["drafts"] = 1 if rng.random() < 0.5 else _log_int(rng, 2, 64)
    c["tail"] = rng.choice([0, c["drafts"], rng.randint(c["drafts"], 64)])
    rows = c["drafts"] * q_heads // kv_heads
    most = min(MOST_TOKEN_HEADS, MOST_ROW_TOKENS // rows) // (kv_heads * c["batch"])
    c["tokens"] = _log_int(rng, 100, max(101, min(131072, most)))
    c["min_tokens"] = max(1, c["tokens"] // rng.randint(2, 8)) if c["batch"] > 1 and rng.random() < 0.7 else 0
    c["empty"] = rng.choice([0, 0, 1]) if c["batch"] > 1 else 0
    c["block_tokens"] = rng.choice([0, 0, 16, 16, 24, 32, 48, 64, 256])
    c["variant"] = rng.choice([BIASED, CENTRED, CENTRED, INT4, INT4])
    c["full"] = c["variant"] != INT4 and rng.random() < 0.5
    c["alpha"] = rng.choice([1.0, 15.0, 255.0, 255.0])
    return c


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

def _host(case, what):
    """Choices that are part of the case, not of the seed."""
    return random.Random(what + repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    lo, hi, r = case["min_tokens"], case["tokens"], _host(case, "lengths")
    lens = [r.randint(lo, hi) if lo else hi - r.randint(0, min(hi, 128) - 1) for _ in range(case["batch"])]
    return lens[: len(lens) - case["empty"]] + [0] * case["empty"]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _levels(alpha, variant, full):
    """The signed level of every plane byte's code ([256], merged) or of every
    nibble ([16], the 4-bit planes), in 64 bits."""
    n = torch.arange(256 if full else 16, dtype=torch.float64, device="cuda")
    a = torch.floor(n / 16) if full else n
    r = n - 16 * a
    r = torch.where(r >= 8, r - 16, r)                      # the correction, two's complement
    V = torch.where(a >= 8, 15 - a, a)                      # the sign-aware anchor
    if variant == BIASED:
        code = (16 * V - r if full else 16 * V).clamp(0, 127)
    elif variant == CENTRED:
        code = 16 * V + 8 + r if full else 16 * V + 7.5
    else:
        code = V
    level = torch.expm1(code / (7 if variant == INT4 else 127) * math.log1p(alpha)) / alpha
    return torch.where(a >= 8, -level, level)


def _cache(case, g, seed, capacity):
    """A filled cache of `capacity` tokens a sequence: planes [blocks][heads][block
    tokens][row bytes], page and chunk metadata, block table."""
    B, H, bt = case["batch"], case["kv_heads"], case["block_tokens"] or capacity
    per = -(-capacity // bt)
    order = torch.randperm(B * per, generator=torch.Generator().manual_seed(seed)) if per > 1 else torch.arange(B)
    la, out = math.log1p(case["alpha"]), {}
    wide = torch.ones(H * D, device="cuda")
    wide[torch.randperm(H * D, generator=g, device="cuda")[: max(1, H * D // 100)]] = 8.0
    for name in "kv":
        plane = torch.empty(B * per, H, bt, D if case["full"] else D // 2, dtype=torch.uint8, device="cuda")
        for part in plane.view(-1).split(1 << 26):
            # values of a chunk over its largest: the code is uniform in the transform
            def code(m):
                x = (torch.randn(part.shape, generator=g, device="cuda") / 2.2).clamp_(-1.0, 1.0)
                i = (torch.log1p(case["alpha"] * x.abs()) / la * m).round_().to(torch.int32)
                return i, x < 0
            def nibble(i, neg):
                v = i if case["variant"] == INT4 else (i + 7 >> 4).clamp(max=7) if case["variant"] == BIASED else i >> 4
                return torch.where(neg, 15 - v, v), v
            if case["full"]:
                i, neg = code(127)
                q, v = nibble(i, neg)
                res = (16 * v - i).clamp(-8, 7) if case["variant"] == BIASED else i - 16 * v - 8
                part.copy_(q * 16 + (res & 15))
            else:
                m = 7 if case["variant"] == INT4 else 127
                part.copy_(nibble(*code(m))[0] + 16 * nibble(*code(m))[0])
        pages, chunks = (B, H, -(-capacity // PAGE), D), (B, H, -(-capacity // CHUNK), D)
        u = lambda shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
        size = wide.view(1, H, 1, D) if name == "k" else 1.0
        out.update({name: plane, name + "_gmin": -(u(pages) * 0.8 + 2.6) * size, name + "_gscale": (u(pages) * 1.2 + 5.4) * size,
                    name + "_mu": u(chunks) * 0.1 + 0.45, name + "_sigma": u(chunks) * 0.15 + 0.28})
    return dict(out, table=order.to(torch.int32).view(B, per).cuda())


META = ("k_gmin", "k_gscale", "k_mu", "k_sigma", "v_gmin", "v_gscale", "v_mu", "v_sigma")


def _prepare_attn(case, seed):
    g, B, H, Hq, k, n = _gen(seed), case["batch"], case["kv_heads"], case["q_heads"], case["drafts"], case["tail"]
    lens = _lengths(case)
    capacity = max(max(lens), 1)
    s = _cache(case, g, seed, capacity)
    s.update(case=case, lens=_ints(lens), longest=max(lens), q=_normal(g, B, k, Hq, D),
             k_tail=_normal(g, B, n, H, D) if n else None, v_tail=_normal(g, B, n, H, D) if n else None,
             out=torch.empty(B, k, Hq, D, dtype=torch.bfloat16, device="cuda"))
    if own:  # the handles and the workspace that a program keeps
        from paper_2607_01831_amd import lynx
        s["layout"] = lynx.Layout(num_kv_heads=H, block_tokens=s["k"].shape[2], max_blocks_per_seq=s["table"].shape[1],
                                  num_blocks=s["k"].shape[0], max_tokens=capacity)
        s["meta"] = lynx.HMeta(*(s[x] for x in META))
        s["ws"] = lynx.workspace(s["layout"], B, Hq, k, max(lens), tree=False)
    return s


def _prepare_rope(case, seed):
    g, r, N, Hq, H = _gen(seed), random.Random(seed), case["tokens"], case["q_heads"], case["kv_heads"]
    qkv = _normal(g, N, (Hq + 2 * H) * D)
    # runs of positions, one a sequence, somewhere in a long context
    positions, rows, n_rows = [], None, N
    while len(positions) < N:
        run = min(N - len(positions), r.randint(1, 8 if N < 256 else 4096))
        first = r.randint(0, 131071 - run)
        positions += range(first, first + run)
    if case["spread"]:  # a padded batch: every ninth token is not there, the others go to rows of their own
        n_rows = N + N // 4
        rows = r.sample(range(n_rows), N)
        positions = [-1 if i % 9 == 5 else p for i, p in enumerate(positions)]
    s = dict(case=case, positions=_ints(positions), rows=None if rows is None else _ints(rows), qkv=qkv)
    s["q"], s["k"], s["v"] = (qkv[:, a * D:b * D].unflatten(1, (-1, D)) for a, b in ((0, Hq), (Hq, Hq + H), (Hq + H, Hq + 2 * H)))
    s["w"] = [1 + 0.2 * torch.randn(D, generator=g, device="cuda").to(torch.bfloat16) for _ in "qk"] if case["norm"] else [None] * 2
    half = case["rotary"] // 2
    s["inv_freq"] = (500000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().cuda()
    s["outs"] = [torch.zeros(n_rows, h, D, dtype=torch.bfloat16, device="cuda") for h in (Hq, H, H)]
    if not case["values"]:
        s["v"], s["outs"][2] = None, None
    return s


EPS = 1e-6


def _step(case):
    """Lengths and counts of a step's plan."""
    r, B = _host(case, "step"), case["batch"]
    lens = [r.randint(0, case["tokens"]) for _ in range(B)]
    counts = [1 if r.random() < 0.6 else r.randint(0, case["most"]) for _ in range(B)]
    return lens, counts


def _prepare_blocks(case, seed):
    (lens, counts), B, bt = _step(case), case["batch"], case["block_tokens"]
    per = -(-(case["tokens"] + case["most"]) // bt)
    held = [-(-n // bt) for n in lens]
    asked = sum(-(-(n + c) // bt) for n, c in zip(lens, counts)) - sum(held)
    free = asked // 2 if case["short"] else asked + 7
    ids = torch.randperm(sum(held) + max(free, 1), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((B, per), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = ids[at:at + n]
        at += n
    stack = torch.full((len(ids),), -1, dtype=torch.int32)
    stack[:free] = ids[at:at + free]
    rows = case["rows"]
    s = dict(case=case, lens=_ints(lens), counts=_ints(counts), table=table.cuda(), stack=stack.cuda(),
             state=_ints([free, 0]), capacity=per * bt, n_blocks=len(ids))
    for name, n in (("granted", B), ("starts", B + 1), ("seq_of", rows), ("positions", rows), ("slots", rows), ("rows", rows)):
        s[name] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["after"] = torch.empty(B, dtype=torch.int32, device="cuda")
    if own:  # the cache's geometry, which a program keeps
        from paper_2607_01831_amd import lynx
        s["layout"] = lynx.Layout(num_kv_heads=8, block_tokens=bt, max_blocks_per_seq=per, num_blocks=len(ids),
                                  max_tokens=per * bt)
    return s


def prepare(case, seed):
    return {"attn": _prepare_attn, "rope": _prepare_rope, "blocks": _prepare_blocks}[case["kind"]](case, seed)


# ----------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------

def _whole(s, name, T, to):
    """K or V of all sequences [B][heads][T][128] as the cache defines them."""
    case = s["case"]
    x = s[name][s["table"].long()]  # [B][blocks][heads][block tokens][row]
    B, nb, H, bt, row = x.shape
    x = x.permute(0, 2, 1, 3, 4).reshape(B, H, nb * bt, row)[:, :, :T]
    if not case["full"]:
        x = torch.stack([x & 15, x >> 4], -1).flatten(-2)
    x = _levels(case["alpha"], case["variant"], case["full"]).to(to)[x.int()]
    chunk, page = (lambda y, n: s[name + y].to(to).repeat_interleave(n, 2)[:, :, :T])("_sigma", CHUNK), PAGE
    x = x.mul_(chunk).add_(s[name + "_mu"].to(to).repeat_interleave(CHUNK, 2)[:, :, :T])
    return x.mul_(s[name + "_gscale"].to(to).repeat_interleave(page, 2)[:, :, :T]).add_(
        s[name + "_gmin"].to(to).repeat_interleave(page, 2)[:, :, :T])


def _attn(s):
    case, T, n = s["case"], s["longest"], s["case"]["tail"]
    B, k, Hq, _ = s["q"].shape
    H, G = case["kv_heads"], Hq // case["kv_heads"]
    K, V = (_whole(s, x, T, torch.float32) for x in "kv")
    seen = (torch.arange(T, device="cuda") < s["lens"].unsqueeze(1)).view(B, 1, 1, T).expand(B, 1, k * G, T)
    if n:
        K, V = (torch.cat([x, s[y].float().transpose(1, 2)], 2) for x, y in ((K, "k_tail"), (V, "v_tail")))
        # query i of k sees the tail's first n - k + i + 1 tokens
        sees = torch.arange(n, device="cuda") <= torch.arange(k, device="cuda").repeat_interleave(G).unsqueeze(1) + (n - k)
        seen = torch.cat([seen, sees.view(1, 1, k * G, n).expand(B, 1, k * G, n)], 3)
    rows = s["q"].float().view(B, k, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, k * G, D)
    x = (rows @ K.transpose(2, 3)).mul_(1 / math.sqrt(D)).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ V) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(o.view(B, H, k, G, D).permute(0, 2, 1, 3, 4).reshape(B, k, Hq, D))
    return s["out"]


def _turned(x, w, cos, sin, case):
    """One tensor's heads [N][heads][128] normed and rotated, in the tables' precision."""
    x = x.to(cos.dtype)
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.to(cos.dtype)
    turn, rest = x[..., :case["rotary"]], x[..., case["rotary"]:]
    a, b = (turn[..., ::2], turn[..., 1::2]) if case["pairs"] else turn.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    turn = torch.stack([a, b], -1).flatten(-2) if case["pairs"] else torch.cat([a, b], -1)
    return torch.cat([turn, rest], -1)


def _rope(s, to=torch.float32):
    case = s["case"]
    angle = s["positions"].double().unsqueeze(1) * s["inv_freq"].double()
    cos, sin = (x.to(to).unsqueeze(1) for x in (angle.cos(), angle.sin()))
    new = [_turned(s["q"], s["w"][0], cos, sin, case), _turned(s["k"], s["w"][1], cos, sin, case), s["v"]]
    there = (s["positions"] >= 0).nonzero(as_tuple=True)[0]
    at = there if s["rows"] is None else s["rows"].long()[there]
    put = lambda page, x: page.index_copy_(0, at, x[there].to(page.dtype))  # noqa: E731
    return [None if x is None else put(page, x) for page, x in zip(s["outs"], new)]


def _blocks(s):
    case, lens, bt = s["case"], s["lens"].long(), s["case"]["block_tokens"]
    counts = torch.minimum(s["counts"].long().clamp(0, case["most"]), s["capacity"] - lens)
    held = (lens + bt - 1) // bt
    need = (lens + counts + bt - 1) // bt - held
    upto = need.cumsum(0)
    fits = ((need == 0) | (upto <= s["state"][0])) & (counts.cumsum(0) <= case["rows"])
    granted = torch.where(fits, counts, 0)
    starts = torch.nn.functional.pad(granted.cumsum(0), (1, 0))
    n = torch.arange(case["rows"], device="cuda")
    b = torch.searchsorted(starts[1:], n, right=True).clamp(max=len(lens) - 1)
    live = n < starts[-1]
    i = n - starts[b]
    pos = lens[b] + i
    block, first = pos // bt, held[b]
    taken = s["state"][0] - 1 - (upto - need)[b] - (block - first)
    old = s["table"].long()[b, block.clamp(max=s["table"].shape[1] - 1)]
    ids = torch.where(block < first, old, s["stack"].long()[taken.clamp(0, s["n_blocks"] - 1)])
    masked = lambda x: torch.where(live, x, -1).to(torch.int32)  # noqa: E731
    out = dict(granted=granted.to(torch.int32), starts=starts.to(torch.int32), seq_of=masked(b), positions=masked(pos),
               slots=masked(ids * bt + pos % bt), rows=masked(b * case["most"] + i))
    new = (live & (block >= first)).nonzero(as_tuple=True)[0]
    s["table"][b[new], block[new]] = ids[new].to(torch.int32)
    s["state"][0] -= torch.where(fits, need, 0).sum().to(torch.int32)
    # the drafts dropped: the blocks behind the lengths go back, the first sequence's first on top
    after = lens + granted
    keep, end = (lens + bt - 1) // bt, (after + bt - 1) // bt
    j = torch.arange(s["table"].shape[1], device="cuda")
    back = (j >= keep.unsqueeze(1)) & (j < end.unsqueeze(1))
    which = s["table"][back]
    total = which.shape[0]
    s["stack"][s["state"][0] + total - 1 - torch.arange(total, device="cuda")] = which
    s["table"].masked_fill_(back, -1)
    s["state"][0] += total
    return dict(out, table=s["table"], stack=s["stack"], free=s["state"])


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------

def _call(s):
    from paper_2607_01831_amd import lynx
    case = s["case"]
    if case["kind"] == "attn":
        lynx.lynx_attn_hier(s["layout"], case["batch"], case["q_heads"], case["drafts"], s["longest"], s["lens"], s["table"],
                            case["full"], s["k"], s["v"], case["alpha"], case["variant"], s["meta"], s["q"], s["k_tail"],
                            s["v_tail"], s["out"], None, s["ws"])
        return s["out"]
    if case["kind"] == "rope":
        lynx.lynx_qk_norm_rope(s["q"], s["k"], s["v"], s["positions"], s["rows"], *s["w"], EPS, s["inv_freq"], case["pairs"],
                               1.0, *s["outs"])
        return s["outs"]
    lynx.lynx_blocks_extend(s["layout"], case["batch"], case["most"], s["lens"], s["counts"], s["table"], s["stack"],
                            s["state"], s["granted"], s["starts"], s["seq_of"], s["positions"], s["slots"], s["rows"])
    torch.add(s["lens"], s["granted"], out=s["after"])
    lynx.lynx_blocks_release(s["layout"], case["batch"], s["after"], s["lens"], s["table"], s["stack"], s["state"])
    return dict({x: s[x] for x in ("granted", "starts", "seq_of", "positions", "slots", "rows", "table", "stack")},
                free=s["state"])


def run(s):
    if own:
        return _call(s)
    return {"attn": _attn, "rope": _rope, "blocks": _blocks}[s["case"]["kind"]](s)


def work(case):
    if case["kind"] == "rope":
        N, Hq, H = case["tokens"], case["q_heads"], case["kv_heads"]
        live = N - len(range(5, N, 9)) if case["spread"] else N
        heads = Hq + H * (2 if case["values"] else 1)
        return {"bytes": live * (heads * D * 4 + (8 if case["spread"] else 4)) + 2 * case["rotary"] + 4 * D,
                "flops": live * (Hq + H) * D * (7 if case["norm"] else 3)}
    if case["kind"] == "blocks":
        lens, counts = _step(case)
        new = sum(-(-(n + c) // case["block_tokens"]) - -(-n // case["block_tokens"]) for n, c in zip(lens, counts))
        new = new // 2 if case["short"] else new
        # lengths and counts, granted counts and starts; the token arrays; blocks off the stack into the table and back
        return {"bytes": 16 * case["batch"] + 16 * case["rows"] + 24 * new, "flops": 8 * case["rows"]}
    lens, H, B = _lengths(case), case["kv_heads"], case["batch"]
    rows, n, k = case["drafts"] * case["q_heads"], case["tail"], case["drafts"]
    chunks, pages = sum(-(-x // CHUNK) for x in lens), sum(-(-x // PAGE) for x in lens)
    return {"bytes": H * (2 * sum(lens) * (D if case["full"] else D // 2) + 16 * D * (chunks + pages)) + 4 * B * (rows + n * H) * D,
            "flops": 4 * D * (rows * sum(lens) + B * case["q_heads"] * sum(n - k + i + 1 for i in range(k if n else 0)))}


# ----------------------------------------------------------------------------
# the same in 64 bits
# ----------------------------------------------------------------------------

def _exact_side(s, b, kv, T, name):
    """K or V of sequence b's head kv, token by token block, in 64 bits."""
    case, bt = s["case"], s[name].shape[2]
    raw = torch.cat([s[name][i, kv] for i in s["table"][b].tolist()])[:T].to(torch.int64)
    if not case["full"]:
        wide = torch.empty(T, D, dtype=torch.int64, device="cuda")
        wide[:, 0::2], wide[:, 1::2] = raw % 16, raw // 16
        raw = wide
    x = _levels(case["alpha"], case["variant"], case["full"])[raw]
    t = torch.arange(T, device="cuda")
    part = lambda what, n: s[name + what][b, kv].double()[t // n]  # noqa: E731
    return part("_gmin", PAGE) + part("_gscale", PAGE) * (part("_mu", CHUNK) + part("_sigma", CHUNK) * x)


def _exact_attn(s):
    case, lens, n = s["case"], s["lens"].tolist(), s["case"]["tail"]
    B, k, Hq, _ = s["q"].shape
    G = Hq // case["kv_heads"]
    out = torch.zeros(B, k, Hq, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        T = lens[b]
        if T + n == 0:
            continue
        for kv in range(case["kv_heads"]):
            K, V = (_exact_side(s, b, kv, T, x) for x in "kv")
            if n:
                K, V = torch.cat([K, s["k_tail"][b, :, kv].double()]), torch.cat([V, s["v_tail"][b, :, kv].double()])
            for i in range(k):
                upto = T + (n - k + i + 1 if n else 0)
                if not upto:
                    continue
                x = s["q"][b, i, kv * G:(kv + 1) * G].double() @ K[:upto].t().contiguous() / math.sqrt(D)
                out[b, i, kv * G:(kv + 1) * G] = torch.softmax(x, 1) @ V[:upto]
    return out


def _exact_rope(s):
    """Rotation as the product with e^(i angle)."""
    case, half = s["case"], s["case"]["rotary"] // 2
    pages = [None if x is None else x.double() for x in s["outs"]]
    there = [i for i, p in enumerate(s["positions"].tolist()) if p >= 0]
    where = there if s["rows"] is None else [s["rows"].tolist()[i] for i in there]
    if not there:
        return pages
    angle = s["positions"][there].double()[:, None] * s["inv_freq"].double()[None]
    phase = torch.polar(torch.ones_like(angle), angle)[:, None]
    for x, w, page in ((s["q"], s["w"][0], pages[0]), (s["k"], s["w"][1], pages[1])):
        x = x[there].double()
        if w is not None:
            x = x / (x.square().sum(-1, keepdim=True) / D + EPS).sqrt() * w.double()
        first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["pairs"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(x[..., first], x[..., second]) * phase
        x[..., first], x[..., second] = z.real, z.imag
        page[where] = x
    if s["v"] is not None:
        pages[2][where] = s["v"][there].double()
    return pages


def exact(case, seed):
    if case["kind"] == "blocks":
        return None  # whole numbers
    return _exact_rope(prepare(case, seed)) if case["kind"] == "rope" else _exact_attn(prepare(case, seed))
