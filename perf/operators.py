"""Scoring a token tree with the target model: the cache operators of a decoding iteration, as cases that can be timed.

Between the draft step and verification the target model scores all nodes of every sequence's tree in one
pass.  In each of its layers the nodes' keys and values are rotated by position and appended to a paged cache
(`append`), and every node attends to the prefix that the whole batch shares, to its own sequence's
context and to its ancestors in the tree (`attend`).  After the tree walk the entries of the accepted path move
up to the end of the context, in all layers at once (`accept`).  A case names

    op          "append", "attend", "accept"
    batch       sequences
    nodes       tree nodes per sequence; 1: a single token, as in decoding without drafts
    k           children per node (1: a chain, which is how a chunk of a prompt comes)
    kv_heads, group, dim    heads of the cache, query heads per head of the cache, head size
    page        tokens per page of the cache
    layout      "nhd": a token's heads lie together in a page; "hnd": a head's tokens do
    dtype       "bf16" or "fp16"
    shortest, longest       lengths of the sequences' own contexts, spread evenly between
    shared      tokens of the prefix that all sequences share
    rotated     dimensions of a head that are rotated
    pairs       "split": dimension i goes with i + rotated / 2; "next": 2i with 2i + 1
    layers      layers that `accept` moves
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name=None, op="attend", batch=1, nodes=1, k=2, kv_heads=8, group=4, dim=128, page=16, layout="nhd",
          dtype="bf16", shortest=1, longest=1000, shared=0, rotated=128, pairs="split", layers=1):
    c = dict(op=op, batch=batch, nodes=nodes, k=k, kv_heads=kv_heads, group=group, dim=dim, page=page, layout=layout,
             dtype=dtype, shortest=shortest, longest=longest, shared=shared, rotated=rotated, pairs=pairs, layers=layers)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one user, one new token: latency is all that counts
        _case("append_one_token", "append", 1, 1, longest=1000, shortest=1000),
        # a busy server: 256 sequences with the trees of the headline verification
        _case("append_tree_batch256", "append", 256, 31, shortest=16, longest=200, shared=100000),
        # a chunk of the prompts of eight sequences, heads of 64 of which half is rotated, pairs of neighbours
        _case("append_prompt_fp16", "append", 8, 1000, 1, 4, 7, 64, 64, "hnd", "fp16", 1, 500, 0, 32, "next"),
        # one user at a terminal: 7 nodes, a context of ordinary length
        _case("attend_one_sequence", "attend", 1, 7, shortest=1500, longest=1500),
        # decoding without drafts: a serving batch of ragged lengths
        _case("attend_decode_batch64", "attend", 64, 1, shortest=1000, longest=8192),
        # trees of 31 nodes for a serving batch, no prefix in common
        _case("attend_tree_batch64", "attend", 64, 31, shortest=500, longest=4000),
        # the same trees behind a long system prompt
        _case("attend_tree_shared", "attend", 64, 31, page=64, shortest=100, longest=1000, shared=8192),
        # many short requests behind one prompt, small heads, single tokens
        _case("attend_decode_shared_fp16", "attend", 256, 1, dim=64, page=32, layout="hnd", dtype="fp16", shortest=1,
              longest=1000, shared=5000),
        # two very long contexts, 15 nodes, five query heads per head of the cache
        _case("attend_long_context", "attend", 2, 15, group=5, page=128, layout="hnd", shortest=100000, longest=131001),
        # a chunk of four prompts: a chain of 500 nodes behind what is in the cache already
        _case("attend_prompt_chunk", "attend", 4, 500, 1, shortest=1, longest=4000),
        # one user's accepted path, all layers of the model
        _case("accept_one_sequence", "accept", 1, 7, shortest=500, longest=500, layers=32),
        # a serving batch's accepted paths
        _case("accept_batch128", "accept", 128, 31, shortest=16, longest=100, layers=32),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(("append", "attend", "attend", "attend", "accept"))
    k = rng.choice((1, 2, 2, 3))
    nodes = rng.choice((1, _spread(rng, 2, 63), _spread(rng, 2, 63), _spread(rng, 64, 500) if k == 1 else 31))
    dim = rng.choice((64, 128, 128))
    kv_heads, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 5, 7, 8))
    page, layout, dtype = rng.choice((8, 16, 32, 64, 128)), rng.choice(("nhd", "hnd")), rng.choice(("bf16", "bf16", "fp16"))
    rotated, pairs = rng.choice((dim, dim, dim // 2)), rng.choice(("split", "next"))
    if op == "append":
        batch = min(_spread(rng, 1, 256), max(1, 250000000 // (nodes * (group + 2) * kv_heads * dim * 8)))
        return _case(None, op, batch, nodes, k, kv_heads, group, dim, page, layout, dtype, 0, _spread(rng, 1, 200),
                     rng.choice((0, _spread(rng, 100, 100000))), rotated, pairs)
    if op == "accept":
        layers = _spread(rng, 1, 32)
        batch = min(_spread(rng, 1, 128), max(1, 12000000 // ((100 + nodes) * kv_heads * dim * layers // 32)))
        return _case(None, op, batch, max(2, nodes), k, kv_heads, 1, dim, page, layout, dtype, 0, _spread(rng, 1, 100), layers=layers)
    longest = _spread(rng, 1, 32000)
    shared = rng.choice((0, 0, _spread(rng, 1, 8192)))
    batch = _spread(rng, 1, 256)
    batch = min(batch, 300000 // (longest + nodes) * 8 // kv_heads,
                int(250e9) // (4 * dim * kv_heads * group * nodes * (longest + shared + nodes)))
    return _case(None, op, max(1, batch), nodes, k, kv_heads, group, dim, page, layout, dtype, rng.randint(0, longest), longest, shared)


def _lens(case):
    b, lo, hi = case["batch"], case["shortest"], case["longest"]
    return [hi - (hi - lo) * i // max(1, b - 1) for i in range(b)]


def _parents(case):
    return [-1] + [(n - 1) // case["k"] for n in range(1, case["nodes"])]


def _tables(case):
    """Depth of every node, and for every node the set of nodes that it sees (its ancestors and itself) as bits of 32-bit words."""
    n, parents = case["nodes"], _parents(case)
    depth, sees = np.zeros(n, np.int32), np.eye(n, dtype=bool)
    for i in range(1, n):
        depth[i] = depth[parents[i]] + 1
        sees[i] |= sees[parents[i]]
    bits = np.zeros((n, 32 * -(-n // 32)), np.uint8)
    bits[:, :n] = sees
    return depth, np.packbits(bits, axis=1, bitorder="little").view(np.int32)


def _paths(case):
    """What the tree walk leaves for each sequence: the nodes of the accepted path, then -1."""
    rng, kids = random.Random(case["nodes"] * 1000 + case["batch"]), {}
    depth = _tables(case)[0]
    for i, p in enumerate(_parents(case)):
        kids.setdefault(p, []).append(i)
    rows = []
    for _ in range(case["batch"]):
        path = [0]
        while path[-1] in kids and rng.random() < 0.7:
            path.append(rng.choice(kids[path[-1]]))
        rows.append(path + [-1] * (int(depth.max()) + 1 - len(path)))
    return rows


def _cache(case, pages, gen, layers=None):
    shape = (pages, case["kv_heads"], case["page"]) if case["layout"] == "hnd" else (pages, case["page"], case["kv_heads"])
    shape = (() if layers is None else (layers,)) + shape + (case["dim"],)
    t = torch.empty(shape, dtype=TYPES[case["dtype"]], device="cuda").normal_(generator=gen)
    return t.transpose(-3, -2) if case["layout"] == "hnd" else t


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    dt, b, n, ps = TYPES[case["dtype"]], case["batch"], case["nodes"], case["page"]
    hk, d = case["kv_heads"], case["dim"]
    lens = np.array(_lens(case), np.int64)[rng.permutation(b)]
    need = -(-(lens + n) // ps)
    at_shared = -(-case["shared"] // ps) if case["op"] == "attend" else 0
    total = int(need.sum()) + at_shared
    ids = rng.permutation(total).astype(np.int32)
    table = np.full((b, int(need.max())), -1, np.int32)
    table[np.arange(table.shape[1]) < need[:, None]] = ids[at_shared:]
    depth, mask = _tables(case)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    layers = case["layers"] if case["op"] == "accept" else None
    s = dict(case=case, lens=dev(lens.astype(np.int32)), pages=dev(table), kc=_cache(case, total, gen, layers),
             vc=_cache(case, total, gen, layers))
    if case["op"] == "accept":
        s["path"] = dev(np.array(_paths(case), np.int32)[rng.permutation(b)])
        return s
    normal = lambda *shape: torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=gen)  # noqa: E731
    s["q"] = (normal(b, n, hk * case["group"], d) * 2).to(dt)   # (scores of a spread that attention has in earnest)
    if case["op"] == "append":
        s["k"], s["v"] = normal(b, n, hk, d).to(dt), normal(b, n, hk, d).to(dt)
        r = case["rotated"]
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()
        s["depth"] = dev(depth)
    else:
        s["mask"], s["shared_pages"] = dev(mask), dev(ids[:at_shared])
    return s


# ---- the plain forms -----------------------------------------------------------------------------------------

def _slots(s, at):
    """Page and place in it of each sequence's slots `at` [B][...]; a slot that no page holds goes to a page that is there."""
    ps, table = s["case"]["page"], s["pages"]
    flat = at.reshape(at.shape[0], -1)
    page = torch.gather(table, 1, (flat // ps).clamp(max=table.shape[1] - 1)).reshape(at.shape)
    return page.clamp(min=0).long(), at % ps


def _rotate(x, position, inv_freq, pairs):
    # (the angle of a far position needs more than 32 bits)
    angle = position.double()[..., None] * inv_freq.double()
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    r = 2 * inv_freq.numel()
    a, rest = x[..., :r].float(), x[..., r:].float()
    if pairs == "next":
        x0, x1 = a[..., 0::2], a[..., 1::2]
        y = torch.stack((x0 * cos - x1 * sin, x0 * sin + x1 * cos), -1).flatten(-2)
    else:
        x0, x1 = a[..., : r // 2], a[..., r // 2:]
        y = torch.cat((x0 * cos - x1 * sin, x0 * sin + x1 * cos), -1)
    return torch.cat((y, rest), -1).to(x.dtype)


def _plain_append(s):
    case = s["case"]
    lens, nodes = s["lens"].long()[:, None], torch.arange(case["nodes"], device="cuda")
    position = case["shared"] + lens + s["depth"].long()
    page, place = _slots(s, lens + nodes)
    s["kc"][page, place] = _rotate(s["k"], position, s["inv_freq"], case["pairs"])
    s["vc"][page, place] = s["v"]
    return dict(q=_rotate(s["q"], position, s["inv_freq"], case["pairs"]), k_cache=s["kc"], v_cache=s["vc"],
                status=torch.zeros_like(s["lens"]))


def _plain_attend(s):
    case, q, lens = s["case"], s["q"], s["lens"].long()
    b, n, hk, g, d = case["batch"], case["nodes"], case["kv_heads"], case["group"], case["dim"]
    longest = case["longest"] + n
    slot = torch.arange(longest, device="cuda")
    page, place = _slots(s, slot.expand(b, longest))
    there = slot < (lens + n)[:, None]
    k = s["kc"][page, place].float().permute(0, 2, 3, 1)                                                   # B, Hk, D, L
    v = torch.where(there[:, :, None, None], s["vc"][page, place].float(), 0.0).permute(0, 2, 1, 3)        # B, Hk, L, D
    node = slot - lens[:, None]                                                                            # B, L
    at = node.clamp(0, n - 1)
    word = s["mask"].t()[at // 32]                                                                         # B, L, N
    in_tree = ((word >> (at % 32)[:, :, None]) & 1).bool() & ((node >= 0) & (node < n))[:, :, None]
    sees = (in_tree | (node < 0)[:, :, None]).permute(0, 2, 1)                                             # B, N, L
    x = q.float().reshape(b, n, hk, g, d).permute(0, 2, 1, 3, 4)                                           # B, Hk, N, G, D
    scale = 1.0 / math.sqrt(d)
    score = (x.reshape(b, hk, n * g, d) @ k).reshape(b, hk, n, g, longest) * scale
    score = torch.where(sees[:, None, :, None, :], score, -math.inf)
    top = score.amax(-1)
    if case["shared"]:
        prefix = torch.arange(case["shared"], device="cuda")
        sp, so = s["shared_pages"][prefix // case["page"]].long(), prefix % case["page"]
        ks, vs = s["kc"][sp, so].float(), s["vc"][sp, so].float()                                         # Ls, Hk, D
        xs = x.permute(1, 0, 2, 3, 4).reshape(hk, b * n * g, d)
        score_s = (xs @ ks.permute(1, 2, 0)).reshape(hk, b, n, g, -1).transpose(0, 1) * scale
        top = torch.maximum(top, score_s.amax(-1))
    ref = torch.where(top == -math.inf, 0.0, top)[..., None]
    p = torch.exp(score - ref)
    total = p.sum(-1)
    out = (p.reshape(b, hk, n * g, longest) @ v).reshape(b, hk, n, g, d)
    if case["shared"]:
        p = torch.exp(score_s - ref)
        total = total + p.sum(-1)
        out = out + (p.transpose(0, 1).reshape(hk, b * n * g, -1) @ vs.transpose(0, 1)).reshape(hk, b, n, g, d).transpose(0, 1)
    out = torch.where((total > 0)[..., None], out / total[..., None], 0.0)
    lse = ref[..., 0] + torch.log(total)
    back = (0, 2, 1, 3)
    return dict(out=out.permute(0, 2, 1, 3, 4).reshape(b, n, hk * g, d).to(q.dtype), lse=lse.permute(back).reshape(b, n, hk * g),
                status=torch.zeros_like(s["lens"]))


def _plain_accept(s):
    lens, path = s["lens"].long()[:, None], s["path"].long()
    place = torch.arange(path.shape[1], device="cuda").expand_as(path)
    kept = (path >= 0).cumprod(1)
    source = torch.where(kept > 0, path, place)      # (what is not kept stays where it is)
    src, dst = _slots(s, lens + source), _slots(s, lens + place)
    s["kc"][:, dst[0], dst[1]] = s["kc"][:, src[0], src[1]]
    s["vc"][:, dst[0], dst[1]] = s["vc"][:, src[0], src[1]]
    return dict(lens=s["lens"] + kept.sum(1).int(), k_cache=s["kc"], v_cache=s["vc"], status=torch.zeros_like(s["lens"]))


# ---- the framework's calls -----------------------------------------------------------------------------------

def _own_append(s):
    import paper_2411_05289_b200 as sh
    case = s["case"]
    r = sh.spechub_cache_append(s["q"], s["k"], s["v"], s["kc"], s["vc"], s["pages"], s["lens"], s["depth"], s["inv_freq"],
                                pos_offset=case["shared"], interleaved=case["pairs"] == "next")
    return dict(q=r["q"], k_cache=s["kc"], v_cache=s["vc"], status=r["status"])


def _own_attend(s):
    import paper_2411_05289_b200 as sh
    case = s["case"]
    if not case["shared"]:
        return sh.spechub_tree_attention(s["q"], s["kc"], s["vc"], s["pages"], s["lens"], s["mask"])
    return sh.spechub_tree_attention(s["q"], s["kc"], s["vc"], s["pages"], s["lens"], s["mask"],
                                     shared_pages=s["shared_pages"], shared_len=case["shared"])


def _own_accept(s):
    import paper_2411_05289_b200 as sh
    r = sh.spechub_cache_accept(s["kc"], s["vc"], s["pages"], s["lens"], s["path"])
    return dict(lens=r["lens"], k_cache=s["kc"], v_cache=s["vc"], status=r["status"])


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_append(state) if op == "append" else _own_attend(state) if op == "attend" else _own_accept(state)
    return _plain_append(state) if op == "append" else _plain_attend(state) if op == "attend" else _plain_accept(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    b, n, hk, g, d = case["batch"], case["nodes"], case["kv_heads"], case["group"], case["dim"]
    rows = b * n
    if case["op"] == "append":
        return {"bytes": 4.0 * rows * (g + 2) * hk * d, "flops": 3.0 * rows * (g + 1) * hk * case["rotated"]}
    if case["op"] == "accept":
        moved = sum(1 for path in _paths(case) for at, node in enumerate(path) if node > at)
        return {"bytes": 8.0 * moved * hk * d * case["layers"] + 4.0 * sum(len(path) for path in _paths(case)), "flops": 0.0}
    keys = sum(_lens(case)) + rows + case["shared"]
    pairs = n * (sum(_lens(case)) + b * case["shared"]) + b * int(_tables(case)[0].sum() + n)
    return {"bytes": 4.0 * keys * hk * d + rows * hk * g * (4.0 * d + 4.0), "flops": 4.0 * pairs * hk * g * d}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    ps, n = case["page"], case["nodes"]
    lens, table = s["lens"].tolist(), s["pages"].tolist()
    zeros = torch.zeros_like(s["lens"])
    if case["op"] == "accept":
        kc, vc = s["kc"].clone(), s["vc"].clone()
        grown = []
        for b, path in enumerate(s["path"].tolist()):
            for to, node in enumerate(path):
                if node < 0:
                    break
                i, j = lens[b] + node, lens[b] + to
                for new, old in ((kc, s["kc"]), (vc, s["vc"])):
                    new[:, table[b][j // ps], j % ps] = old[:, table[b][i // ps], i % ps]
            grown.append(lens[b] + sum(node >= 0 for node in path))
        return dict(lens=torch.tensor(grown, dtype=torch.int32), k_cache=kc.float(), v_cache=vc.float(), status=zeros)
    if case["op"] == "append":
        kc, vc, qs = s["kc"].double(), s["vc"].double(), s["q"].double()
        r = case["rotated"]
        first = torch.arange(r // 2) * 2 if case["pairs"] == "next" else torch.arange(r // 2)
        second = first + 1 if case["pairs"] == "next" else first + r // 2
        first, second = first.cuda(), second.cuda()
        freq, depth = s["inv_freq"].double(), s["depth"].double()
        for b in range(case["batch"]):
            # the rotation as a product of complex numbers
            turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), (case["shared"] + lens[b] + depth)[:, None] * freq)
            k = s["k"][b].double()
            for x in (k, qs[b]):
                z = torch.complex(x[..., first], x[..., second]) * turn[:, None, :]
                x[..., first], x[..., second] = z.real, z.imag
            slot = torch.arange(lens[b], lens[b] + n, device="cuda")
            page = s["pages"][b].long()[slot // ps]
            kc[page, slot % ps] = k
            vc[page, slot % ps] = s["v"][b].double()
        return dict(q=qs, k_cache=kc, v_cache=vc, status=zeros)
    b, hk, g, d = case["batch"], case["kv_heads"], case["group"], case["dim"]
    parents = _parents(case)
    ancestors = np.eye(n, dtype=bool)
    for i in range(1, n):
        ancestors[i] |= ancestors[parents[i]]
    ancestors = torch.from_numpy(ancestors).cuda()
    flat = lambda cache, pages, count: cache[pages.long()].flatten(0, 1)[:count].double().transpose(0, 1)  # noqa: E731
    ks, vs = (flat(c, s["shared_pages"], case["shared"]) for c in (s["kc"], s["vc"]))
    out = torch.empty((b, n, hk * g, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((b, n, hk * g), dtype=torch.float64, device="cuda")
    for i in range(b):
        count = lens[i] + n
        k, v = (flat(c, s["pages"][i, : -(-count // ps)], count) for c in (s["kc"], s["vc"]))
        k, v = torch.cat((ks, k), 1), torch.cat((vs, v), 1)                      # Hk, L, D
        x = s["q"][i].double().reshape(n, hk, g, d).permute(1, 2, 0, 3)          # Hk, G, N, D
        score = x.reshape(hk, g * n, d) @ k.transpose(1, 2) / math.sqrt(d)
        score.view(hk, g, n, -1)[..., case["shared"] + lens[i]:].masked_fill_(~ancestors, -math.inf)
        total = torch.logsumexp(score, -1)
        o = torch.exp(score - total[..., None]) @ v
        out[i] = o.reshape(hk, g, n, d).permute(2, 0, 1, 3).reshape(n, hk * g, d)
        lse[i] = total.reshape(hk, g, n).permute(2, 0, 1).reshape(n, hk * g)
    return dict(out=out, lse=lse, status=zeros)
