"""Work on a paged K/V cache behind its attention, as measurable cases: drafted tokens that form a tree, and the eviction of keys.

A case is a dict of plain values; "op" names the operator:
  tree    tr_paged_attn_tree: attention of drafted tokens, each on the keys in front of the drafts and on its own branch
  weigh   tr_cache_weigh: the attention weight that every cached key gets from the new tokens, added to what it had
  select  tr_cache_select: the keys of every sequence and K/V head that stay, by weight, with the first and the last ones
  keep    tr_cache_keep: the kept keys moved together in their pages (an eviction's, or the accepted path of a tree)
"seqs" sequences have "new" new tokens each ("prompt" > 0: the first one that many; "idle": every fifth one none) and up to "kv" keys, the
new ones among them; "ragged" is the share of "kv" by which the lengths differ.  "shift" moves the new tokens' positions away from the last keys, as on
a device that holds a part of the cache.  "cache" is bf16 or fp8; "page" keys lie in a page; "layout" says whether a page holds its keys head by
head or token by token.  A tree of drafts is either "branches" chains side by side, or has "arity" children at every token.
"""
import math

import torch

own = False

GOLDEN = 0.6180339887498949


def listed():
    base = {"prompt": 0, "idle": False, "ragged": 0.0, "shift": 0, "layout": "head"}
    tree = dict(base, op="tree", branches=0, arity=0)
    weigh = dict(base, op="weigh", causal=True, fresh=True)
    return [
        # eight drafts of one short chat: nothing but latency
        dict(tree, name="tree_one_short", seqs=1, new=8, arity=2, kv=108, Hq=8, Hkv=2, D=64, page=16, cache="bf16"),
        # a verification step of a server: 25 drafts of each of 16 sequences on an 8-bit cache
        dict(tree, name="tree_16x25_fp8", seqs=16, new=25, arity=2, kv=4097, ragged=0.5, Hq=32, Hkv=8, D=128, page=32, cache="fp8"),
        # larger trees of four sequences behind longer texts
        dict(tree, name="tree_4x64_8k", seqs=4, new=64, arity=3, kv=8256, ragged=0.2, Hq=32, Hkv=8, D=128, page=64, cache="bf16"),
        # eight continuations of one long text, 64 tokens each, looked over as one tree
        dict(tree, name="tree_branches_30k_fp8", seqs=1, new=512, branches=8, kv=30512, Hq=32, Hkv=8, D=128, page=128, cache="fp8"),
        # a decode step of one short chat
        dict(weigh, name="weigh_one_short", seqs=1, new=1, kv=100, Hq=8, Hkv=2, D=64, page=16, cache="bf16"),
        # a decode step of a full server: 64 sequences of very different lengths, 8-bit cache in small pages
        dict(weigh, name="weigh_decode_64_fp8", seqs=64, new=1, kv=16384, ragged=0.95, Hq=32, Hkv=8, D=128, page=16, cache="fp8"),
        # one prompt's first chunk among decoding sequences, head dim 64 without grouped heads
        dict(weigh, name="weigh_mixed_d64", seqs=16, new=1, prompt=700, kv=4000, ragged=0.8, Hq=24, Hkv=24, D=64, page=16, cache="bf16", layout="token"),
        # the largest: the last chunk of a 32K prompt weighs all keys
        dict(weigh, name="weigh_chunk_at_30k", seqs=1, new=2048, kv=32768, Hq=32, Hkv=8, D=128, page=64, cache="bf16"),
        # every sequence of a server back from 4600 keys to 4096
        {"name": "select_64x4k", "op": "select", "seqs": 64, "kv": 4608, "ragged": 0.02, "Hkv": 8, "page": 64, "budget": 4096, "first": 4, "last": 256, "zeros": 0.1},
        # one long text cut down to what fits
        {"name": "select_one_32k", "op": "select", "seqs": 1, "kv": 32768, "ragged": 0.0, "Hkv": 8, "page": 64, "budget": 4099, "first": 4, "last": 1024, "zeros": 0.5},
        # the eviction of the 64 sequences, with the keys' weights
        {"name": "keep_64x4k_fp8", "op": "keep", "seqs": 64, "kv": 4608, "ragged": 0.02, "Hkv": 8, "D": 128, "page": 64, "cache": "fp8", "layout": "head",
         "budget": 4096, "path": 0, "weights": True},
        # accepted paths of the trees of 16 sequences, the same ones for all heads
        {"name": "keep_paths_bf16", "op": "keep", "seqs": 16, "kv": 4097, "ragged": 0.5, "Hkv": 8, "D": 128, "page": 32, "cache": "bf16", "layout": "token",
         "budget": 7, "path": 25, "weights": False},
    ]


def _between(rng, lo, hi):
    """A whole number between lo and hi, spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    D = rng.choice((64, 128))
    Hkv, group = rng.choice(((2, 4), (8, 4), (8, 8), (8, 1), (24, 1), (4, 7), (1, 16)))
    common = {"Hkv": Hkv, "page": rng.choice((16, 32, 48, 64, 128, 256)), "ragged": rng.choice((0.0, 0.3, 0.95))}
    pages = {"D": D, "cache": rng.choice(("bf16", "fp8")), "layout": rng.choice(("head", "token"))}
    op = rng.choice(("tree", "tree", "weigh", "weigh", "select", "keep"))
    if op == "select":
        seqs = _between(rng, 1, 64)
        kv = _between(rng, 20, min(65536, 600000 // seqs))
        first, last = rng.choice((0, 4)), rng.choice((0, kv // 10))
        return dict(common, op=op, seqs=seqs, kv=kv, budget=first + last + _between(rng, 1, kv), first=first, last=last, zeros=rng.choice((0.0, 0.1, 0.7)))
    if op == "keep":
        seqs = _between(rng, 1, 64)
        if rng.random() < 0.4:
            path = _between(rng, 2, 64)
            return dict(common, **pages, op=op, seqs=seqs, kv=path + _between(rng, 1, 4000), budget=_between(rng, 1, path), path=path, weights=rng.random() < 0.5)
        kv = _between(rng, 20, min(32768, 150000 // seqs))
        return dict(common, **pages, op=op, seqs=seqs, kv=kv, budget=rng.randrange(1, kv), path=0, weights=rng.random() < 0.5)
    case = dict(common, **pages, op=op, Hq=Hkv * group, idle=rng.random() < 0.2, shift=0, prompt=0)
    if op == "tree":
        seqs = _between(rng, 1, 32)
        new = _between(rng, 2, min(512, 1024 // seqs))
        shape = {"branches": 0, "arity": rng.randrange(1, 5)} if rng.random() < 0.6 else {"branches": rng.randrange(1, new + 1), "arity": 0}
        case.update(shape, seqs=seqs, new=new, kv=new + _between(rng, 1, min(30000, 60000 // seqs)))
    else:
        case.update(causal=rng.random() < 0.85, fresh=rng.random() < 0.85)
        kind = rng.choice(("decode", "drafts", "chunk", "mixed"))
        if kind == "decode":
            seqs = _between(rng, 1, 64)
            case.update(seqs=seqs, new=1, kv=_between(rng, 1, min(32768, 400000 // seqs)))
        elif kind == "drafts":
            seqs = _between(rng, 1, 32)
            case.update(seqs=seqs, new=rng.randrange(2, 17), kv=_between(rng, 20, min(16384, 100000 // seqs)))
        elif kind == "chunk":
            seqs = _between(rng, 1, 4)
            new = _between(rng, 17, 2048 // seqs)
            case.update(seqs=seqs, new=new, kv=new + _between(rng, 1, 16384 // seqs))
        else:
            seqs, prompt = _between(rng, 2, 24), _between(rng, 17, 512)
            case.update(seqs=seqs, new=rng.choice((1, 1, 3)), prompt=prompt, kv=prompt + _between(rng, 1, 4000), idle=False)
    if rng.random() < 0.25:
        case["shift"] = rng.choice((-1, 1)) * _between(rng, 1, case["kv"])
    return case


def _lengths(case):
    """(keys, new tokens) of every sequence."""
    n, new, kv = case["seqs"], max(case.get("new", 0), case.get("path", 0)), case["kv"]
    q = [0 if case.get("idle") and i % 5 == 3 else new for i in range(n)]
    if case.get("prompt"):
        q[0] = case["prompt"]
    return [max(q[i], 1, int(kv * (1 - case["ragged"] * (i * GOLDEN % 1)))) for i in range(n)], q


def _parent(case, i):
    """Of drafted token i, -1: it follows the text."""
    return i - case["branches"] if case["branches"] else (i - 1) // case["arity"] if i else -1


def _ancestors(case):
    """[new][new]: whether drafted token i sees token j: itself and what is above it."""
    n = case["new"]
    sees = torch.zeros((n, n), dtype=torch.bool)
    for i in range(n):
        if _parent(case, i) >= 0:
            sees[i] = sees[_parent(case, i)]
        sees[i, i] = True
    return sees


def _quantised(x):
    """Rows x as (e4m3, e8m0): the smallest power of two that brings a row's largest value down to 448 or less."""
    x = x.float()
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)
    k = torch.where(a == 0, 0, torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126))
    return (x * (127 - k << 23).view(torch.float32).unsqueeze(-1)).to(torch.float8_e4m3fn), (k + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)   # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)   # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    op, n, H, ps = case["op"], case["seqs"], case["Hkv"], case["page"]
    kv, q = _lengths(case)
    used = [-(-x // ps) for x in kv]
    pages, width = sum(used) + 3, max(used)
    ids = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int32)
    counts = ints(used)
    column = torch.arange(width, device="cuda")
    at = (counts.cumsum(0) - counts)[:, None] + column
    s = {"case": case, "table": torch.where(column < counts[:, None], ids[at.clamp(max=pages - 1)], -1).to(torch.int32).contiguous(), "kv_len": ints(kv)}
    s["weights"] = None
    if op in ("weigh", "select") or case.get("weights"):   # what earlier tokens left: few keys have most of it, some nothing
        s["weights"] = (2 * normal(pages, H, ps)).exp_().masked_fill_(uniform(pages, H, ps) < case.get("zeros", 0.1), 0.0)
        if op == "weigh":   # (about as much as the new ones bring)
            s["weights"].mul_(0.1 * case["Hq"] * sum(q) / H / sum(kv))
    if op != "select":
        D = case["D"]

        def pool(*tail):   # what earlier tokens left, in every slot
            x = normal(*((pages, H, ps) if case["layout"] == "head" else (pages, ps, H)), *tail)
            return x if case["layout"] == "head" else x.transpose(1, 2)
        for name in ("k", "v"):
            x = pool(D).bfloat16()
            s[name + "_pages"], e = _quantised(x) if case["cache"] == "fp8" else (x, None)
            s[name + "_scales"] = e if e is None else e.contiguous()
    if op in ("tree", "weigh"):
        starts = [0]
        for x in q:
            starts.append(starts[-1] + x)
        s["q_start"], s["tokens"], s["most"] = ints(starts), starts[-1], max(q)
        s["q"] = normal(1, s["tokens"], case["Hq"], D).bfloat16().transpose(1, 2)
        s["scale"] = D ** -0.5
        s["q_pos"] = s["kv_len"] - (s["q_start"][1:] - s["q_start"][:-1]) + case["shift"] if case["shift"] else None
    if op == "tree":
        words = -(-case["new"] // 32)
        sees = torch.zeros((case["new"], words * 32), dtype=torch.int64)
        sees[:, :case["new"]] = _ancestors(case)
        bits = (sees.view(-1, words, 32) << torch.arange(32)).sum(-1)
        s["tree"] = torch.where(bits >= 2 ** 31, bits - 2 ** 32, bits).to(torch.int32).cuda().repeat(sum(x > 0 for x in q), 1)
        s["out"] = torch.zeros((1, s["tokens"], case["Hq"], D), dtype=torch.bfloat16, device="cuda").transpose(1, 2)
        s["lse"] = torch.zeros((1, case["Hq"], s["tokens"]), device="cuda")
    elif op == "weigh":
        s["lse"] = torch.zeros((1, case["Hq"], s["tokens"]), device="cuda")   # what the attention on the same keys has left
        token, used = _tokens(s)
        x = _scores(s, token, _causal(s))
        s["lse"][0][:, token[used]] = torch.logsumexp(x, -1).permute(1, 2, 0, 3).reshape(case["Hq"], n, s["most"])[:, used]
    elif op == "select":
        s["keys"], s["count"] = torch.zeros((n, H, case["budget"]), dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    elif case["path"]:   # of each tree one path, some of them empty
        taken = torch.rand((n, case["path"]), generator=g, device="cuda").topk(case["budget"], dim=1).indices.sort(-1).values
        s["start"] = s["kv_len"] - case["path"]
        s["count"] = torch.randint(0, case["budget"] + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
        s["keys"] = (s["start"][:, None] + taken).to(torch.int32)[:, None].contiguous()
    else:
        there = torch.arange(width * ps, device="cuda") < s["kv_len"][:, None, None]
        s["start"], s["count"] = None, s["kv_len"].clamp(max=case["budget"])
        best = torch.where(there, uniform(n, H, width * ps), -1.0).topk(case["budget"], dim=-1).indices
        column = torch.arange(case["budget"], device="cuda")
        s["keys"] = torch.where(column < s["count"][:, None, None], best, 2 ** 30).sort(-1).values.to(torch.int32).contiguous()
    return s


def run(state):
    return {"tree": _tree, "weigh": _weigh, "select": _select, "keep": _keep}[state["case"]["op"]](state)


def _bits(t):
    return t.view(torch.uint8) if t.element_size() == 1 else t


def _place(s, keys):
    """Page and slot of keys [seqs, ...]."""
    ps = s["case"]["page"]
    page = s["table"].gather(1, (keys.flatten(1) // ps).clamp(min=0, max=s["table"].shape[1] - 1)).view(keys.shape)
    return page.clamp(min=0).long(), keys % ps


def _rows(s, name):
    """K or V of all keys that the table has room for, in 32 bits: [seqs, Hkv, keys, D]."""
    pages, scales = s[name + "_pages"], s[name + "_scales"]
    page, slot = _place(s, torch.arange(s["table"].shape[1] * s["case"]["page"], device="cuda").expand(s["case"]["seqs"], -1))
    x = _bits(pages)[page, :, slot]   # [seqs, keys, Hkv, D]
    if scales is None:
        return x.float().transpose(1, 2)
    e = scales.view(torch.uint8)[page, :, slot].int()
    return (x.view(pages.dtype).float() * (e << 23).view(torch.float32).unsqueeze(-1)).transpose(1, 2)


def _tokens(s):
    """[seqs, most]: the token that is the t-th new one of a sequence, and whether there is one."""
    t = torch.arange(s["most"], device="cuda")
    return (s["q_start"][:-1, None] + t).clamp(max=max(s["tokens"] - 1, 0)).long(), t < (s["q_start"][1:] - s["q_start"][:-1])[:, None]


def _keys(s):
    """[seqs, keys]: key numbers relative to the first new token's, and whether there is such a key."""
    keys = torch.arange(s["table"].shape[1] * s["case"]["page"], device="cuda").expand(s["case"]["seqs"], -1)
    count = s["q_start"][1:] - s["q_start"][:-1]
    pos = s["kv_len"] - count if s["q_pos"] is None else s["q_pos"]
    return keys - pos[:, None], keys < s["kv_len"][:, None]


def _causal(s):
    ahead, there = _keys(s)
    seen = there[:, None, :].expand(-1, s["most"], -1)
    return seen & (ahead[:, None, :] <= torch.arange(s["most"], device="cuda")[:, None]) if s["case"]["causal"] else seen


def _scores(s, token, seen):
    """[seqs, Hkv, group, most, keys] in 32 bits, -inf where a token does not see a key."""
    c = s["case"]
    n, D, Hkv, group = c["seqs"], c["D"], c["Hkv"], c["Hq"] // c["Hkv"]
    q = s["q"][0][:, token].float()   # [Hq, n, t, D]
    q = q.view(Hkv, group, n, s["most"], D).permute(2, 0, 1, 3, 4).reshape(n, Hkv, group * s["most"], D)
    x = torch.matmul(q, _rows(s, "k").transpose(2, 3)).mul_(s["scale"]).view(n, Hkv, group, s["most"], -1)
    return x.masked_fill_(~seen[:, None, None], float("-inf"))


def _tree(s):
    c = s["case"]
    if own:
        import paper_2412_20501_amd as tr
        if "workspace" not in s:
            s["workspace"] = torch.empty(tr.tr_paged_attn_tree_workspace_bytes(s["q"], s["k_pages"], s["table"]), dtype=torch.uint8, device="cuda")
        tr.tr_paged_attn_tree(s["q"], s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["q_start"], s["tree"], s["scale"], s["out"], s["lse"],
                              s["k_scales"], s["v_scales"], s["q_pos"], s["workspace"])
        return s["out"], s["lse"]
    n, D, Hkv, group = c["seqs"], c["D"], c["Hkv"], c["Hq"] // c["Hkv"]
    token, used = _tokens(s)
    ahead, there = _keys(s)
    words = s["tree"][token]   # [n, t, words]
    draft = ahead.clamp(min=0, max=s["most"] - 1)
    seen = words.gather(2, (draft // 32)[:, None].expand(-1, s["most"], -1)) >> (draft % 32)[:, None] & 1
    seen = there[:, None] & ((ahead < 0)[:, None] | ((ahead < (s["q_start"][1:] - s["q_start"][:-1])[:, None])[:, None] & (seen == 1)))
    x = _scores(s, token, seen)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top.clamp(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, Hkv, group * s["most"], -1), _rows(s, "v")).view(n, Hkv, group, s["most"], D) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log())[..., 0]
    s["out"][0][:, token[used]] = o.permute(1, 2, 0, 3, 4).reshape(c["Hq"], n, s["most"], D)[:, used].to(s["out"].dtype)
    s["lse"][0][:, token[used]] = lse.permute(1, 2, 0, 3).reshape(c["Hq"], n, s["most"])[:, used]
    return s["out"], s["lse"]


def _weigh(s):
    c = s["case"]
    if own:
        import paper_2412_20501_amd as tr
        tr.tr_cache_weigh(s["q"], s["lse"], s["k_pages"], s["table"], s["kv_len"], s["q_start"], c["causal"], s["scale"], s["weights"], c["fresh"],
                          s["k_scales"], s["q_pos"])
        return s["weights"]
    n, Hkv, group = c["seqs"], c["Hkv"], c["Hq"] // c["Hkv"]
    token, used = _tokens(s)
    lse = s["lse"][0][:, token].view(Hkv, group, n, s["most"]).permute(2, 0, 1, 3)
    live = used[:, None, None] & lse.isfinite()
    x = _scores(s, token, _causal(s)).sub_(torch.where(live, lse, float("inf")).unsqueeze(-1)).exp_()
    added = x.sum((2, 3))   # [n, Hkv, keys]
    ahead, there = _keys(s)
    count = s["q_start"][1:] - s["q_start"][:-1]
    page, slot = _place(s, torch.arange(there.shape[1], device="cuda").expand(n, -1))
    page, slot, there_at = page[there], slot[there], added.transpose(1, 2)[there]
    old = s["weights"][page, :, slot]
    if c["fresh"]:
        old = torch.where(((ahead >= 0) & (ahead < count[:, None]))[there][:, None], 0.0, old)
    s["weights"][page, :, slot] = old + there_at
    return s["weights"]


def _select(s):
    c = s["case"]
    if own:
        import paper_2412_20501_amd as tr
        tr.tr_cache_select(s["weights"], s["table"], s["kv_len"], c["first"], c["last"], s["keys"], s["count"])
        return s["keys"], s["count"]
    keys = torch.arange(s["table"].shape[1] * c["page"], device="cuda").expand(c["seqs"], -1)
    page, slot = _place(s, keys)
    length = s["kv_len"][:, None]
    w = s["weights"][page, :, slot].transpose(1, 2)   # [seqs, Hkv, keys]
    w = torch.where(((keys < c["first"]) | (keys >= length - c["last"]))[:, None], float("inf"), w)
    w = torch.where((keys < length)[:, None], w, float("-inf"))
    best = w.sort(dim=-1, descending=True, stable=True).indices[..., :c["budget"]]
    s["count"].copy_(s["kv_len"].clamp(max=c["budget"]))
    there = torch.arange(best.shape[-1], device="cuda") < s["count"][:, None, None]
    best = torch.where(there, best, 2 ** 30).sort(-1).values
    s["keys"][..., :best.shape[-1]] = torch.where(there, best.to(torch.int32), s["keys"][..., :best.shape[-1]])
    return s["keys"], s["count"]


def _keep(s):
    c = s["case"]
    if own:
        import paper_2412_20501_amd as tr
        tr.tr_cache_keep(s["k_pages"], s["v_pages"], s["table"], s["kv_len"], s["keys"], s["count"], s["start"], s["k_scales"], s["v_scales"], s["weights"])
    else:
        n, H, N = c["seqs"], c["Hkv"], s["keys"].shape[-1]
        column = torch.arange(N, device="cuda")
        there = (column < s["count"][:, None, None]).expand(n, H, N)
        source = s["keys"].expand(n, H, N).clamp(max=c["kv"])
        to = ((0 if s["start"] is None else s["start"][:, None, None]) + column).expand(n, H, N)
        head = torch.arange(H, device="cuda")[None, :, None].expand(n, H, N)[there]
        (page, slot), (to_page, to_slot) = ([x[there] for x in _place(s, y)] for y in (source, to))
        for name in ("k_pages", "v_pages", "k_scales", "v_scales", "weights"):
            if s[name] is not None:
                x = _bits(s[name])
                x[to_page, head, to_slot] = x[page, head, slot]
    return {x: s[x] for x in ("k_pages", "v_pages", "k_scales", "v_scales", "weights")}


def work(case):
    kv, q = _lengths(case)
    H, D = case["Hkv"], case.get("D", 0)
    row = (D + 1 if case.get("cache") == "fp8" else 2 * D) * H   # K or V of a key
    if case["op"] == "select":
        return {"bytes": 4 * H * sum(kv) + 4 * H * sum(min(x, case["budget"]) for x in kv), "flops": H * sum(kv)}
    if case["op"] == "keep":   # a half of the shortest paths, and nearly all of an eviction's keys, move
        rows = case["seqs"] * case["budget"] / 2 if case["path"] else sum(min(x, case["budget"]) if x > case["budget"] else 0 for x in kv)
        return {"bytes": int(2 * rows * (2 * row + (4 * H if case["weights"] else 0) + 2 * H)), "flops": 0}
    keys = pairs = 0
    above = float(_ancestors(case).sum()) / case["new"] if case["op"] == "tree" else 0
    for x, n in zip(kv, q):
        pos = x - n + case["shift"]
        seen = lambda t: min(x, max(0, pos + t))   # noqa: E731,B023
        if case["op"] == "tree":
            keys += seen(n) if n else 0
            pairs += n * seen(0) + (above * (seen(n) - seen(0)) if case["shift"] <= 0 else 0)
        elif case["causal"]:
            keys += seen(n) if n else 0
            pairs += sum(seen(t + 1) for t in range(n))
        else:
            keys += x if n else 0
            pairs += n * x
    if case["op"] == "tree":
        return {"bytes": 2 * keys * row + sum(q) * case["Hq"] * (4 * D + 4), "flops": int(4 * D * case["Hq"] * pairs)}
    return {"bytes": keys * (row + 8 * H) + sum(q) * case["Hq"] * (2 * D + 4), "flops": int((2 * D + 2) * case["Hq"] * pairs)}


def _power(k):
    """2 ** k in 64 bits, by its bits (pow and ldexp round)."""
    return (k.long() + 1023 << 52).view(torch.float64)


def exact(case, seed):
    if case["op"] == "select":
        return None   # whole numbers
    s = prepare(case, seed)
    kv, q = _lengths(case)
    ps, table = case["page"], s["table"].long().cpu()

    def place(b, c):
        return table[b, c // ps].cuda(), (c % ps).cuda()

    if case["op"] == "keep":
        found = {}
        keys, count = s["keys"].cpu().long(), s["count"].tolist()
        start = [0] * case["seqs"] if s["start"] is None else s["start"].tolist()
        for name in ("k_pages", "v_pages", "k_scales", "v_scales", "weights"):
            found[name] = None
            if s[name] is None:
                continue
            old = s[name].double()
            new = old.clone()
            for b in range(case["seqs"]):
                to = place(b, start[b] + torch.arange(count[b]))
                for h in range(case["Hkv"]):
                    page, slot = place(b, keys[b, min(h, keys.shape[1] - 1), :count[b]])
                    new[to[0], h, to[1]] = old[page, h, slot]
            found[name] = new
        return found

    def values(name, b, h):
        page, slot = place(b, torch.arange(kv[b]))
        pages = s[name + "_pages"][:, h]
        x = _bits(pages)[page, slot]
        if s[name + "_scales"] is None:
            return x.double()
        return x.view(pages.dtype).double() * _power(s[name + "_scales"].view(torch.uint8)[page, h, slot].long() - 127).unsqueeze(-1)

    group, at = case["Hq"] // case["Hkv"], 0
    above = _ancestors(case).cuda() if case["op"] == "tree" else None
    out, lse = (s["out"].double(), s["lse"].double()) if case["op"] == "tree" else (None, s["lse"].double())
    weights = s["weights"].double() if case["op"] == "weigh" else None
    for b in range(case["seqs"]):
        n = q[b]
        if not n:
            continue
        pos = kv[b] - n + case["shift"]
        c, t = torch.arange(kv[b], device="cuda"), torch.arange(n, device="cuda")
        if case["op"] == "tree":
            shown = (c < pos).expand(n, kv[b]).clone()
            lo, hi = max(pos, 0), min(pos + n, kv[b])
            if lo < hi:
                shown[:, lo:hi] = above[:n, lo - pos:hi - pos]
        else:
            shown = c <= (pos + t)[:, None] if case["causal"] else torch.ones((n, kv[b]), dtype=torch.bool, device="cuda")
        page, slot = place(b, torch.arange(kv[b]))
        for h in range(case["Hkv"]):
            K = values("k", b, h)
            if case["op"] == "weigh":
                total = weights[page, h, slot]
                if case["fresh"]:
                    total[max(pos, 0):max(min(pos + n, kv[b]), 0)] = 0
            else:
                V = values("v", b, h)
            for j in range(h * group, (h + 1) * group):
                x = (s["q"][0, j, at:at + n].double() @ K.T * s["scale"]).masked_fill(~shown, -math.inf)
                if case["op"] == "tree":
                    z = torch.logsumexp(x, -1)
                    out[0, j, at:at + n] = torch.exp(x - z.clamp(min=-1e300)[:, None]) @ V
                    lse[0, j, at:at + n] = z
                else:
                    z = lse[0, j, at:at + n]
                    total = total + torch.exp(x - torch.where(z.isfinite(), z, math.inf)[:, None]).sum(0)
            if case["op"] == "weigh":
                weights[page, h, slot] = total
        at += n
    return (out, lse) if case["op"] == "tree" else weights
