"""The operators that follow a tree of drafted tokens through the cache, over the
sizes that serving gives them.

A case is a dict of plain values.  `kind` names the operator:

  tree     verification attention: the nodes of a token tree over the merged
           8-bit cache and over their own ancestors' BF16 K and V
           (lynx_attn_verify_tree)
  greedy,  acceptance of the tree's longest path that the target model's own
  sample   choices follow, greedy or drawn (lynx_spec_accept_tree_greedy,
           lynx_spec_accept_tree_sample)
  append   tokens quantized into the cache as they are kept (lynx_kv_append),
           and the groups they fall into read back
  dequant  a range of every sequence read back as BF16 (lynx_kv_dequant)

Contexts: `batch` sequences of `tokens` tokens, or spread over
[min_tokens, tokens]; block_tokens 0 is one block per sequence, anything else a
paged pool under a random block table.  Trees: `nodes` nodes in levels of
`width`, each node's parent one of the level above; -2 marks a node that is
not there (`absent` of them at the end of every second sequence: a padded
batch).  K channels are normal, 1% of them 8 times larger.

`own` chooses who computes: this file's plain form, in elementary torch
operations, or the framework's calls.
"""
import math
import random

import torch

own = False

D = 128
GROUP = 128  # tokens per K quantization group
RING = 256   # BF16 K rows kept per sequence behind the cache's end

# No drawn case does more than the largest listed one of its kind.
MOST_TREE = 64 * 8 * 8 * 2 * 65536     # rows of a kv head x token-heads
MOST_TOKEN_HEADS = 2 * 65536 * 8       # tokens of all sequences x kv heads
MOST_SCORES = 16 * 64 * 128256         # rows x vocabulary, greedy
MOST_PROBS = 16 * 33 * 128256          # the same, drawn


def listed():
    return [
        # a small model's layer at 4K context and a handful of nodes: latency alone
        dict(name="tree-4k-n8", kind="tree", batch=1, q_heads=8, kv_heads=4, tokens=4096, min_tokens=0, block_tokens=0,
             nodes=8, width=3, absent=0),
        # continuous batching, ragged and paged, an odd number of nodes, padded trees
        dict(name="tree-paged-b16-n25", kind="tree", batch=16, q_heads=32, kv_heads=8, tokens=8192, min_tokens=1024,
             block_tokens=16, nodes=25, width=6, absent=4),
        # a 70B-shaped layer, the widest tree, two long contexts: the largest
        dict(name="tree-64k-b2-n64", kind="tree", batch=2, q_heads=64, kv_heads=8, tokens=65536, min_tokens=0,
             block_tokens=0, nodes=64, width=10, absent=0),
        # one user, a 32000-entry vocabulary
        dict(name="greedy-b1-n24", kind="greedy", batch=1, nodes=24, width=5, absent=0, kept=3, vocab=32000),
        # a busy server over the Llama-3 vocabulary, wide trees
        dict(name="greedy-b16-n63", kind="greedy", batch=16, nodes=63, width=10, absent=7, kept=4, vocab=128256),
        # drawn choices, a vocabulary of odd length
        dict(name="sample-b2-n12", kind="sample", batch=2, nodes=12, width=4, absent=0, kept=2, vocab=50257),
        # drawn choices for a batch
        dict(name="sample-b16-n32", kind="sample", batch=16, nodes=32, width=6, absent=5, kept=4, vocab=128256),
        # plain decoding at 32K: one token a step
        dict(name="append-32k-1", kind="append", batch=1, kv_heads=8, tokens=32768, min_tokens=0, block_tokens=0,
             most=1, nodes=0),
        # the accepted paths of a batch's trees, ragged and paged
        dict(name="append-paged-b16-path", kind="append", batch=16, kv_heads=8, tokens=8192, min_tokens=1024,
             block_tokens=16, most=25, nodes=25),
        # chunked prefill: chunks of up to 4096 tokens behind whole chunks
        dict(name="append-chunk-b4-4096", kind="append", batch=4, kv_heads=8, tokens=8192, min_tokens=2048,
             block_tokens=16, most=4096, nodes=0),
        # the open groups of a batch, before its first append
        dict(name="dequant-paged-b16-128", kind="dequant", batch=16, kv_heads=8, tokens=8192, min_tokens=1024,
             block_tokens=16, most=128),
        # whole long prefixes back to BF16, for attention that reads BF16 pages
        dict(name="dequant-64k-b2", kind="dequant", batch=2, kv_heads=8, tokens=65536, min_tokens=0, block_tokens=0,
             most=65536),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "greedy", "sample", "append", "append", "dequant"])
    if kind in ("greedy", "sample"):
        n, vocab = _log_int(rng, 1, 64 if kind == "greedy" else 32), _log_int(rng, 1000, 152064)
        most = (MOST_SCORES if kind == "greedy" else MOST_PROBS) // ((n + 1) * vocab)
        c = dict(kind=kind, batch=_log_int(rng, 1, max(1, min(64, most))), nodes=n, width=rng.randint(1, 12), vocab=vocab)
        c["absent"] = rng.randint(0, n // 4)
        c["kept"] = rng.randint(0, min(5, max(0, 16 * 5 * 128256 // (c["batch"] * vocab) - 1)))
        return c
    q_heads, kv_heads = rng.choice([(8, 4), (32, 8), (32, 8), (64, 8), (28, 4)])
    c = dict(kind=kind, batch=_log_int(rng, 1, 32), kv_heads=kv_heads)
    most = MOST_TOKEN_HEADS // kv_heads
    if kind == "tree":
        n = _log_int(rng, 1, 64)
        c.update(q_heads=q_heads, nodes=n, width=rng.randint(1, 12), absent=rng.randint(0, n // 4))
        most = min(most // 2, MOST_TREE // (n * (q_heads // kv_heads) * kv_heads))
    c["tokens"] = _log_int(rng, 200, max(201, min(131072, most // c["batch"])))
    c["min_tokens"] = max(1, c["tokens"] // rng.randint(2, 8)) if c["batch"] > 1 and rng.random() < 0.7 else 0
    c["block_tokens"] = rng.choice([0, 16, 16, 32, 48, 64])
    if kind == "append":
        c["nodes"] = _log_int(rng, 1, 64) if rng.random() < 0.5 else 0
        # (a path's tokens come from its tree; without one a chunk may be long)
        c["most"] = c["nodes"] or _log_int(rng, 1, min(4096, c["tokens"], MOST_TOKEN_HEADS // (8 * kv_heads * c["batch"])))
    if kind == "dequant":
        c["most"] = _log_int(rng, 1, c["tokens"])
    return c


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

def _host(case, what):
    """Choices that are part of the case, not of the seed."""
    return random.Random(what + repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _lengths(case):
    lo, hi, r = case["min_tokens"], case["tokens"], _host(case, "lengths")
    return [r.randint(lo, hi) if lo else hi - r.randint(0, min(hi, GROUP) - 1) for _ in range(case["batch"])]


def _appended(case):
    """Lengths before and tokens appended.  A chunk longer than the kept rows
    comes behind whole groups, as chunks of a prompt do."""
    lens, r = _lengths(case), _host(case, "counts")
    if case["nodes"]:
        return lens, [r.randint(1, min(8, case["most"])) for _ in lens]
    if case["most"] > GROUP:
        lens = [n // GROUP * GROUP for n in lens]
    return lens, [case["most"] - r.randint(0, case["most"] // 4) for _ in lens]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _parents(case, seed):
    """Parents [batch][nodes], node i's before i; the seed's own tree for every sequence."""
    r = random.Random(seed)
    out = []
    for b in range(case["batch"]):
        row = []
        for i in range(case["nodes"]):
            above = range((i // case["width"] - 1) * case["width"], i // case["width"] * case["width"])
            row.append(r.choice(above) if i >= case["width"] else -1)
        for i in range(case["nodes"] - (case["absent"] if b % 2 else 0), case["nodes"]):
            row[i] = -2
        out.append(row)
    return out


def _cache(case, g, seed, capacity):
    """A filled cache of `capacity` tokens a sequence: code planes
    [blocks][heads][block tokens][128], metadata, block table."""
    B, H, bt = case["batch"], case["kv_heads"], case["block_tokens"] or capacity
    per = -(-capacity // bt)
    order = torch.randperm(B * per, generator=torch.Generator().manual_seed(seed)) if per > 1 else torch.arange(B)
    codes = []
    for _ in range(2):
        x = torch.empty(B * per, H, bt, D, dtype=torch.uint8, device="cuda")
        for part in x.view(-1).split(1 << 27):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda").mul_(42).add_(127.5).round_().clamp_(0, 255))
        codes.append(x)
    wide = torch.ones(H * D, device="cuda")
    wide[torch.randperm(H * D, generator=g, device="cuda")[: max(1, H * D // 100)]] = 8.0
    scales = [torch.rand(*shape, generator=g, device="cuda") * 0.004 + 0.022
              for shape in ((B, H, -(-capacity // GROUP), D), (B, H, capacity))]
    scales[0] *= wide.view(1, H, 1, D)
    return dict(k_codes=codes[0], v_codes=codes[1], k_scale=scales[0], k_zero=-127.5 * scales[0], v_scale=scales[1],
                v_zero=-127.5 * scales[1], table=order.to(torch.int32).view(B, per).cuda(), wide=wide.view(H, D))


def _choices(kind, scores, uniforms):
    """The target's choice in every row: the first of the largest scores, or the
    draw whose weights are floor(p 2^40)."""
    V = scores.shape[-1]
    if kind == "greedy":
        at = torch.arange(V, device="cuda", dtype=torch.int32)
        return torch.where(scores == scores.amax(-1, keepdim=True), at, V).amin(-1).to(torch.int32)
    upto = (scores.clamp(0.0, 1.0) * 2.0 ** 40).to(torch.int64).cumsum_(-1)
    total = upto[..., -1]
    u = (uniforms.double() * 2.0 ** 32).floor().clamp(0, 2.0 ** 32 - 1).to(torch.int64)
    # floor(total u / 2^32) in 64-bit pieces
    high, low = total >> 32, total & 0xFFFFFFFF
    t = high * u + ((low * (u >> 16) + (low * (u & 0xFFFF) >> 16)) >> 16)
    token = (upto <= t.unsqueeze(-1)).sum(-1)
    return torch.where(total > 0, token, -1).to(torch.int32)


def _decision(case, seed):
    """Scores or probabilities of every row, the tree, its tokens and uniforms.
    Tokens agree with the target's choices along one path of `kept` nodes."""
    g, r = _gen(seed), random.Random(seed + 1)
    B, n, V = case["batch"], case["nodes"], case["vocab"]
    parents = _parents(case, seed)
    scores = torch.empty(B, n + 1, V, device="cuda")
    for b in range(B):  # logits come out of a BF16 product
        scores[b] = (torch.randn(n + 1, V, generator=g, device="cuda") * 3.0).to(torch.bfloat16)
        if case["kind"] == "sample":
            scores[b] = torch.softmax(scores[b], -1)
    uniforms = torch.rand(B, n + 1, generator=g, device="cuda")
    choice = torch.stack([_choices(case["kind"], scores[b], uniforms[b]) for b in range(B)]).cpu().tolist()
    tokens = [[r.randrange(V) for _ in range(n)] for _ in range(B)]
    for b in range(B):
        for i in range(n):  # no other node agrees by chance
            if parents[b][i] >= -1 and tokens[b][i] == choice[b][parents[b][i] + 1]:
                tokens[b][i] = (tokens[b][i] + 1) % V
        there = [i for i in range(n) if parents[b][i] >= -1]
        deep = min(case["kept"], -(-len(there) // case["width"]))
        at = r.choice([i for i in there if i // case["width"] == deep - 1]) if deep else -1
        while at >= 0:
            tokens[b][at] = choice[b][parents[b][at] + 1]
            at = parents[b][at]
    return dict(scores=scores, uniforms=uniforms, tokens=_ints(tokens), parents=_ints(parents))


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("greedy", "sample"):
        s = _decision(case, seed)
        B, n = case["batch"], case["nodes"]
        s.update(case=case, accepted=torch.empty(B, dtype=torch.int32, device="cuda"),
                 path=torch.empty(B, n, dtype=torch.int32, device="cuda"),
                 next=torch.empty(B, dtype=torch.int32, device="cuda"))
        if own:  # the workspace that a program keeps
            from paper_2607_01831_amd import lynx
            s["ws"] = lynx.spec_tree_workspace(B, n, case["vocab"])
        return s
    g, B, H = _gen(seed), case["batch"], case["kv_heads"]
    lens, counts = _appended(case) if kind == "append" else (_lengths(case), None)
    capacity = max(case["tokens"], max(lens)) + (case["most"] if kind == "append" else 0)
    s = _cache(case, g, seed, capacity)
    s.update(case=case, lens=_ints(lens), longest=max(lens), capacity=capacity)
    if kind == "tree":
        n, Hq = case["nodes"], case["q_heads"]
        s.update(q=_normal(g, B, n, Hq, D), k_new=_normal(g, B, n, H, D), v_new=_normal(g, B, n, H, D),
                 parents=_ints(_parents(case, seed)), out=torch.empty(B, n, Hq, D, dtype=torch.bfloat16, device="cuda"))
    else:
        most = case["most"]
        if kind == "append":
            n = case["nodes"] or most
            s.update(counts=_ints(counts), k_new=(torch.randn(B, n, H, D, generator=g, device="cuda") * s["wide"]).bfloat16(),
                     v_new=_normal(g, B, n, H, D),
                     k_open=(torch.randn(B, RING, H, D, generator=g, device="cuda") * s["wide"]).bfloat16(), path=None)
            if case["nodes"]:
                r = random.Random(seed + 2)
                s["path"] = _ints([sorted(r.sample(range(n), c)) + [-1] * (most - c) for c in counts])
            starts = [x // GROUP * GROUP for x in lens]
            spans = [x + c - f for x, c, f in zip(lens, counts, starts)]
            most = -(-max(spans) // GROUP) * GROUP
        else:
            r = _host(case, "spans")
            spans = [min(x, most - r.randint(0, most // 4)) for x in lens]
            starts = [r.randint(0, x - c) for x, c in zip(lens, spans)]
            if most == GROUP:  # the open groups
                starts, spans = [x // GROUP * GROUP for x in lens], [x % GROUP for x in lens]
        pages = [torch.zeros(B, most, H, D, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        s.update(starts=_ints(starts), spans=_ints(spans), most=most, pages=pages)
    if own:  # the handles and the workspace that a program keeps
        from paper_2607_01831_amd import lynx
        blocks, bt = s["k_codes"].shape[0], s["k_codes"].shape[2]
        s["layout"] = lynx.Layout(num_kv_heads=H, block_tokens=bt, max_blocks_per_seq=s["table"].shape[1],
                                  num_blocks=blocks, max_tokens=capacity)
        s["meta"] = lynx.Meta(s["k_scale"], s["k_zero"], s["v_scale"], s["v_zero"])
        if kind == "tree":
            s["ws"] = lynx.workspace(s["layout"], B, case["q_heads"], case["nodes"], s["longest"])
    return s


# ----------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------

def _paths(parents):
    """Ancestors-or-self [B][n][n] of the nodes that are there, and which those
    are [B][n]: a node whose parent is not one of -1 .. i - 1 is not, nor is
    anything below it."""
    B, n = parents.shape
    at = torch.arange(n, device="cuda")
    linked = (parents >= -1) & (parents < at)
    step = (parents.unsqueeze(-1) == at) & linked.unsqueeze(-1)
    reach = torch.linalg.matrix_power(step.float() + torch.eye(n, device="cuda"), max(1, n)) > 0
    there = ~(reach & ~linked.unsqueeze(1)).any(-1)
    return reach & there.unsqueeze(-1), there


def _accept(s):
    kind, tokens, parents = s["case"]["kind"], s["tokens"], s["parents"]
    B, n = tokens.shape
    V = s["scores"].shape[-1]
    at = torch.arange(n, device="cuda")
    choice = _choices(kind, s["scores"], s["uniforms"])
    reach, there = _paths(parents)
    agrees = there & (tokens == choice.gather(1, (parents.clamp(-1, n - 1) + 1).long())) & (tokens >= 0) & (tokens < V)
    twin = (parents.unsqueeze(1) == parents.unsqueeze(2)) & (at.unsqueeze(0) < at.unsqueeze(1)) & agrees.unsqueeze(1)
    agrees = agrees & ~twin.any(-1)  # of siblings with one token the first
    kept = there & ~(reach & ~agrees.unsqueeze(1)).any(-1)
    accepted = kept.sum(1).to(torch.int32)
    path = torch.where(kept, at, n).sort(1).values  # a path's nodes go up
    last = torch.where(kept, at, -1).amax(1) + 1
    return {"accepted": accepted, "path": torch.where(path < n, path, -1).to(torch.int32),
            "next": choice.gather(1, last.unsqueeze(1)).squeeze(1)}


def _logical(planes, table, length):
    """Rows [B][heads][length][128] of the sequences."""
    x = planes[table.long()]  # [B][blocks][heads][block tokens][128]
    B, nb, H, bt, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, H, nb * bt, d)[:, :, :length]


def _tree(s):
    case, q, T = s["case"], s["q"], s["longest"]
    B, n, Hq, _ = q.shape
    H, G = case["kv_heads"], Hq // case["kv_heads"]
    ks, kz = (s[x].repeat_interleave(GROUP, 2)[:, :, :T] for x in ("k_scale", "k_zero"))
    K = _logical(s["k_codes"], s["table"], T).float() * ks + kz
    V = _logical(s["v_codes"], s["table"], T).float() * s["v_scale"][:, :, :T, None] + s["v_zero"][:, :, :T, None]
    K = torch.cat([K, s["k_new"].float().transpose(1, 2)], 2)
    V = torch.cat([V, s["v_new"].float().transpose(1, 2)], 2)
    reach, there = _paths(s["parents"])
    inside = (torch.arange(T, device="cuda") < s["lens"].unsqueeze(1)).unsqueeze(1) & there.unsqueeze(2)
    seen = torch.cat([inside, reach], 2).repeat_interleave(G, 1).unsqueeze(1)  # rows node-major, heads inside
    rows = q.float().view(B, n, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, n * G, D)
    x = (rows @ K.transpose(2, 3)).mul_(1 / math.sqrt(D)).masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ V) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(o.view(B, H, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D))
    return s["out"]


def _place(s, starts, most):
    """Tokens starts .. starts + most - 1 of every sequence: their positions and
    plane rows [B][most], and their places in the cache's arrays."""
    pos = s["starts"].unsqueeze(1).long() + torch.arange(most, device="cuda")
    bt = s["k_codes"].shape[2]
    at = pos.clamp(max=s["capacity"] - 1)
    return pos, s["table"].long().gather(1, at // bt), at % bt, torch.arange(pos.shape[0], device="cuda").unsqueeze(1)


def _read(s):
    """The range of every sequence as BF16 [B][most][heads][128]."""
    pos, block, row, b = _place(s, s["starts"], s["most"])
    at = pos.clamp(max=s["capacity"] - 1)
    inside = (torch.arange(s["most"], device="cuda") < s["spans"].unsqueeze(1))[..., None, None]
    for codes, scale, zero, page in ((s["k_codes"], s["k_scale"][b, :, at // GROUP], s["k_zero"][b, :, at // GROUP], s["pages"][0]),
                                     (s["v_codes"], s["v_scale"][b, :, at].unsqueeze(-1), s["v_zero"][b, :, at].unsqueeze(-1),
                                      s["pages"][1])):
        x = codes[block, :, row].float() * scale + zero
        page.copy_(torch.where(inside, x.to(torch.bfloat16), page))
    return {"k": s["pages"][0], "v": s["pages"][1]}


def _codes(x, lo, hi):
    """Codes, scales and zeros of values whose groups span [lo, hi]."""
    lo, span = lo + 0.0, (hi + 0.0) - (lo + 0.0)
    inv = torch.where(span > 0, 255.0 / span, 0.0)
    return ((x - lo) * inv).round().clamp(0, 255).to(torch.uint8), torch.where(span > 0, span / 255.0, 0.0), lo


def _append(s):
    """The groups that the appended tokens fall into, quantized from the kept
    BF16 rows and the new ones."""
    B, most = s["lens"].shape[0], s["most"]
    pos, block, row, b = _place(s, s["starts"], most)
    i = pos - s["lens"].unsqueeze(1)  # number among the new tokens
    live = i < s["counts"].unsqueeze(1)
    fresh = (i >= 0) & live
    n = i.clamp(0, s["case"]["most"] - 1)
    if s["path"] is not None:
        n = s["path"].long().gather(1, n).clamp(min=0)
    k = torch.where((i < 0)[..., None, None], s["k_open"][b, pos % RING], s["k_new"][b, n]).float()
    grouped = k.view(B, most // GROUP, GROUP, -1, D)
    there = live.view(B, most // GROUP, GROUP, 1, 1)
    lo = torch.where(there, grouped, math.inf).amin(2, keepdim=True)
    hi = torch.where(there, grouped, -math.inf).amax(2, keepdim=True)
    codes, scale, zero = _codes(grouped, lo, hi)
    where = live.nonzero(as_tuple=True)
    s["k_codes"][block[where], :, row[where]] = codes.view(B, most, -1, D)[where]
    touched = there[:, :, 0, 0, 0].nonzero(as_tuple=True)
    group = s["starts"].long()[touched[0]] // GROUP + touched[1]
    s["k_scale"][touched[0], :, group] = scale[:, :, 0][touched]
    s["k_zero"][touched[0], :, group] = zero[:, :, 0][touched]
    where = fresh.nonzero(as_tuple=True)
    v = s["v_new"][b, n].float()
    codes, scale, zero = _codes(v, v.amin(-1, keepdim=True), v.amax(-1, keepdim=True))
    s["v_codes"][block[where], :, row[where]] = codes[where]
    s["v_scale"][where[0], :, pos[where]] = scale[..., 0][where]
    s["v_zero"][where[0], :, pos[where]] = zero[..., 0][where]
    # the rows of the last group begun and of the one before it stay in BF16
    end = (s["lens"] + s["counts"]).unsqueeze(1)
    where = (fresh & (pos >= end // GROUP * GROUP - GROUP)).nonzero(as_tuple=True)
    s["k_open"][where[0], pos[where] % RING] = s["k_new"][b, n][where]
    return _state(s, _read(s))


def _state(s, pages):
    return {**pages, "k_open": s["k_open"], "k_scale": s["k_scale"], "k_zero": s["k_zero"], "v_scale": s["v_scale"],
            "v_zero": s["v_zero"]}


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------

def _call(s):
    from paper_2607_01831_amd import lynx
    case = s["case"]
    kind, B = case["kind"], case["batch"]
    if kind == "greedy":
        lynx.lynx_spec_accept_tree_greedy(s["scores"], s["tokens"], s["parents"], s["accepted"], s["path"], s["next"],
                                          s["ws"])
    elif kind == "sample":
        lynx.lynx_spec_accept_tree_sample(s["scores"], s["tokens"], s["parents"], s["uniforms"], s["accepted"], s["path"],
                                          s["next"], s["ws"])
    if kind in ("greedy", "sample"):
        return {"accepted": s["accepted"], "path": s["path"], "next": s["next"]}
    L, m = s["layout"], s["meta"]
    if kind == "tree":
        lynx.lynx_attn_verify_tree(L, B, case["q_heads"], case["nodes"], s["longest"], s["lens"], s["table"], s["k_codes"],
                                   s["v_codes"], m, s["q"], s["k_new"], s["v_new"], s["parents"], s["out"], s["ws"])
        return s["out"]
    if kind == "append":
        lynx.lynx_kv_append(L, B, case["most"], s["lens"], s["counts"], s["path"], s["table"], s["k_new"], s["v_new"],
                            s["k_open"], s["k_codes"], s["v_codes"], None, None, None, None, m)
    lynx.lynx_kv_dequant(L, B, s["most"], s["starts"], s["spans"], s["table"], s["k_codes"], s["v_codes"], m, *s["pages"])
    pages = {"k": s["pages"][0], "v": s["pages"][1]}
    return _state(s, pages) if kind == "append" else pages


def run(s):
    if own:
        return _call(s)
    kind = s["case"]["kind"]
    if kind == "tree":
        return _tree(s)
    if kind in ("greedy", "sample"):
        return _accept(s)
    return _append(s) if kind == "append" else _read(s)


def work(case):
    kind = case["kind"]
    if kind in ("greedy", "sample"):
        # the choices along the path alone decide
        deep = [min(case["kept"], -(-(case["nodes"] - x) // case["width"])) for x in (0, case["absent"])]
        n = sum(deep[b % 2] + 1 for b in range(case["batch"])) * case["vocab"]
        return {"bytes": 4 * n, "flops": n}
    H, B = case["kv_heads"], case["batch"]
    row = 2 * (D + 4) * H  # codes of K and V of a token with V's scalars
    if kind == "tree":
        lens, n, rows = _lengths(case), case["nodes"], case["nodes"] * case["q_heads"]
        groups = sum(-(-x // GROUP) for x in lens)
        return {"bytes": sum(lens) * row + groups * 1024 * H + 4 * B * (rows + n * H) * D,
                "flops": 4 * D * rows * (sum(lens) + B * min(n, -(-n // case["width"])))}
    if kind == "append":
        lens, counts = _appended(case)
        rows = sum((x % GROUP) + c for x, c in zip(lens, counts))  # K tokens of the groups touched
        new, groups = sum(counts), sum(-(-(x % GROUP + c) // GROUP) for x, c in zip(lens, counts))
        keep = sum(min(c, GROUP + (x + c) % GROUP) for x, c in zip(lens, counts))
        write = H * (rows * 2 * D + new * 2 * D + rows * D + new * (D + 8) + groups * 1024 + keep * 2 * D)
        # read back: K and V of the groups touched
        return {"bytes": write + rows * (row + 4 * D * H) + groups * 1024 * H, "flops": 6 * H * D * (rows + new)}
    lens, r = _lengths(case), _host(case, "spans")
    spans = [min(x, case["most"] - r.randint(0, case["most"] // 4)) for x in lens]
    if case["most"] == GROUP:
        spans = [x % GROUP for x in lens]
    groups = sum(-(-x // GROUP) for x in spans)
    return {"bytes": sum(spans) * (row + 4 * D * H) + groups * 1024 * H, "flops": 4 * sum(spans) * H * D}


# ----------------------------------------------------------------------------
# the same in 64 bits
# ----------------------------------------------------------------------------

def _whole(s, b, length, name):
    """K or V of sequence b's first `length` tokens as the cache defines them."""
    planes, bt = s[name + "_codes"], s[name + "_codes"].shape[2]
    blocks = s["table"][b].tolist()
    codes = torch.cat([planes[i] for i in blocks], 1)[:, :length].double()  # [heads][length][128]
    if name == "v":
        return codes * s["v_scale"][b, :, :length, None].double() + s["v_zero"][b, :, :length, None].double()
    out = torch.empty_like(codes)
    for t in range(0, length, GROUP):
        out[:, t:t + GROUP] = (codes[:, t:t + GROUP] * s["k_scale"][b, :, t // GROUP, None].double()
                               + s["k_zero"][b, :, t // GROUP, None].double())
    return out


def _exact_tree(s):
    case, lens, parents = s["case"], s["lens"].tolist(), s["parents"].tolist()
    B, n, Hq, _ = s["q"].shape
    G = Hq // case["kv_heads"]
    out = torch.zeros(B, n, Hq, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        above = {-1: []}
        for i, p in enumerate(parents[b]):
            if p in above and p < i:
                above[i] = above[p] + [i]
        K, V = _whole(s, b, lens[b], "k"), _whole(s, b, lens[b], "v")
        nodes = [i for i in range(n) if i in above]
        bars = torch.ones(len(nodes), n, dtype=torch.bool, device="cuda")
        for at, i in enumerate(nodes):
            bars[at, above[i]] = False
        bars = torch.cat([torch.zeros(len(nodes), lens[b], dtype=torch.bool, device="cuda"), bars], 1)
        for h in range(Hq if nodes else 0):
            kv = h // G
            keys = torch.cat([K[kv], s["k_new"][b, :, kv].double()])
            values = torch.cat([V[kv], s["v_new"][b, :, kv].double()])
            x = s["q"][b, nodes, h].double() @ keys.t().contiguous() / math.sqrt(D)
            out[b, nodes, h] = torch.softmax(x.masked_fill(bars, -math.inf), 1) @ values
    return out


def _exact_pages(s, K, V):
    """Ranges of every sequence from its whole K and V [tokens][heads][128]."""
    pages = [torch.zeros(s["pages"][0].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    for b, (f, c) in enumerate(zip(s["starts"].tolist(), s["spans"].tolist())):
        pages[0][b, :c], pages[1][b, :c] = K[b][f:f + c], V[b][f:f + c]
    return {"k": pages[0], "v": pages[1]}


def _exact_append(s):
    case = s["case"]
    ring = s["k_open"].double()
    meta = {x: s[x].double() for x in ("k_scale", "k_zero", "v_scale", "v_zero")}
    Ks, Vs = [], []
    for b, (T, c) in enumerate(zip(s["lens"].tolist(), s["counts"].tolist())):
        f = T // GROUP * GROUP
        src = s["path"][b, :c].tolist() if s["path"] is not None else list(range(c))
        raw = torch.cat([s["k_open"][b, [t % RING for t in range(f, T)]], s["k_new"][b, src]]).double()
        new = s["v_new"][b, src].double()
        K, V = _whole(s, b, T, "k").transpose(0, 1), _whole(s, b, T, "v").transpose(0, 1)
        pieces = []
        for t in range(0, raw.shape[0], GROUP):
            x = raw[t:t + GROUP]
            lo, step = x.amin(0), (x.amax(0) - x.amin(0)) / 255
            meta["k_scale"][b, :, (f + t) // GROUP], meta["k_zero"][b, :, (f + t) // GROUP] = step, lo
            pieces.append(lo + step * torch.where(step > 0, (x - lo) / step, 0.0).round())
        Ks.append(torch.cat([K[:f]] + pieces))
        lo, step = new.amin(2, keepdim=True), (new.amax(2, keepdim=True) - new.amin(2, keepdim=True)) / 255
        meta["v_scale"][b, :, T:T + c], meta["v_zero"][b, :, T:T + c] = step[..., 0].t(), lo[..., 0].t()
        Vs.append(torch.cat([V, lo + step * torch.where(step > 0, (new - lo) / step, 0.0).round()]))
        for i in range(c):
            if T + i >= (T + c) // GROUP * GROUP - GROUP:
                ring[b, (T + i) % RING] = s["k_new"][b, src[i]].double()
    return {**_exact_pages(s, Ks, Vs), "k_open": ring, **meta}


def exact(case, seed):
    if case["kind"] in ("greedy", "sample"):
        return None  # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "tree":
        return _exact_tree(s)
    if case["kind"] == "append":
        return _exact_append(s)
    ends = [f + c for f, c in zip(s["starts"].tolist(), s["spans"].tolist())]
    return _exact_pages(s, *[[_whole(s, b, n, x).transpose(0, 1) for b, n in enumerate(ends)] for x in "kv"])
