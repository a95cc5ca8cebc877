"""Cases of the paged key / value cache: what a program that serves sequences with a loop of its own calls of
`paper_2510_23264_amd`.

A case names one operator, the shape of the batch and its sizes:

  append   kv_append of new tokens' keys (rotated on the way) and values to their sequences' pages, their queries rotated beside
  attend   kv_attention of the new tokens' queries over their sequences' pages: the next token, a piece of a prompt, or a tree
           of drafted tokens that see their ancestors
  keep     kv_append of a drafted tree, then kv_keep of the path that was accepted: its rows move together

The plain forms compute the same from the formulas with elementary torch operations, sequences padded to the longest.  A batch's
lengths follow from the case alone (`shape` is their seed), everything else from the seed of `prepare`.  Values: queries and keys
normal with a few large channels, as trained models have them, at scores that spread by one to two; values normal.  Head counts are
those of this repository's workloads, grouped as eight keys' heads for 32 queries' where that is said, and odd ones.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
MAX_FLOPS = 4.0 * 128 * 32 * 8192 * 8193 / 2         # of the largest listed case with flops: a prompt of 8192 tokens
MAX_BYTES = 131072 * 8 * 128 * 2 * 2                 # of the longest listed context
MAX_PADDED = 1 << 31                                 # scores of the padded plain form


def listed():
    return [
        # the next token of a few sequences: launches are all of it
        dict(name="append_4_tokens", op="append", batch=4, new=1, longest=6000, ragged=True, shape=1, heads=8, group=4, d=128, rot=128,
             page=16, type="bf16", layout="half", scaling="bands", theta=500000.0, queries=True),
        # a long prompt's projections on their way into the cache
        dict(name="append_8192_tokens", op="append", batch=1, new=8192, longest=8192, ragged=False, shape=2, heads=8, group=4, d=128, rot=128,
             page=64, type="bf16", layout="half", scaling="none", theta=10000.0, queries=True),
        # ragged prompts of the GPT-2-small shape in fp32, a quarter of each head turned, pages of an odd size
        dict(name="append_ragged_f32", op="append", batch=7, new=1000, longest=3000, ragged=True, shape=3, heads=12, group=1, d=64, rot=16,
             page=24, type="f32", layout="interleaved", scaling="linear", theta=10000.0, queries=False),
        # the next token of one short sequence of the GPT-2-small shape in the engine's own fp32: latency
        dict(name="attend_token_short", op="attend", batch=1, new=1, longest=200, ragged=False, shape=4, heads=12, group=1, d=64, page=16,
             type="f32", tree=0),
        # the next token of a full batch whose contexts differ much in length
        dict(name="attend_64_tokens", op="attend", batch=64, new=1, longest=16384, ragged=True, shape=5, heads=8, group=4, d=128, page=16,
             type="bf16", tree=0),
        # the next token of one very long context
        dict(name="attend_token_131072", op="attend", batch=1, new=1, longest=131072, ragged=False, shape=6, heads=8, group=4, d=128, page=64,
             type="bf16", tree=0),
        # a long prompt: the matrix cores are all of it
        dict(name="attend_prompt_8192", op="attend", batch=1, new=8192, longest=8192, ragged=False, shape=7, heads=8, group=4, d=128, page=64,
             type="bf16", tree=0),
        # pieces of prompts behind cached prefixes of differing length, the GPT-2-small shape's heads
        dict(name="attend_ragged_prompts", op="attend", batch=9, new=1500, longest=4096, ragged=True, shape=8, heads=12, group=1, d=64, page=16,
             type="f16", tree=0),
        # a piece of two prompts in fp32, a head of 80 and pages of an odd size
        dict(name="attend_piece_f32", op="attend", batch=2, new=333, longest=2100, ragged=True, shape=9, heads=5, group=3, d=80, page=24,
             type="f32", tree=0),
        # drafted trees of 64 tokens are verified for eight sequences
        dict(name="attend_trees", op="attend", batch=8, new=64, longest=8000, ragged=True, shape=10, heads=8, group=4, d=128, page=16,
             type="bf16", tree=64),
        # a few sequences' drafts of 26 tokens, of which up to five are kept
        dict(name="keep_4", op="keep", batch=4, new=26, longest=3000, ragged=True, shape=11, heads=8, group=4, d=128, rot=128, page=16,
             type="bf16", layout="half", scaling="none", theta=10000.0, queries=False, depth=5),
        # the drafts of a full batch, 64 tokens each, up to eight kept
        dict(name="keep_192", op="keep", batch=192, new=64, longest=600, ragged=True, shape=12, heads=12, group=1, d=64, rot=64, page=32,
             type="f16", layout="half", scaling="none", theta=10000.0, queries=False, depth=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "keep"])
    d = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, 128, 192, 256])
    c = dict(op=op, batch=_log(rng, 1, 256), longest=_log(rng, 1, 131072), ragged=rng.random() < 0.7, shape=rng.randrange(1 << 30),
             heads=rng.choice([1, 2, 4, 5, 8, 8, 12, 16]), group=rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 16]), d=d,
             page=rng.choice([1, 8, 16, 16, 24, 32, 64, 64, 100, 256]), type=rng.choice(list(TYPES)))
    if op == "append":
        c["new"] = _log(rng, 1, 8192)
    elif op == "keep":
        c["new"] = rng.randint(2, 80)
        c["depth"] = rng.randint(1, 10)
    else:
        kind = rng.choice(["token", "token", "prompt", "prompt", "tree"])
        c["tree"] = rng.randint(2, 150) if kind == "tree" else 0
        c["new"] = 1 if kind == "token" else _log(rng, 2, 8192) if kind == "prompt" else c["tree"]
    if op != "attend":
        c.update(rot=d if rng.random() < 0.6 else 2 * rng.randint(1, d // 2), layout=rng.choice(["half", "interleaved"]),
                 scaling=rng.choice(["none", "linear", "bands"]), theta=rng.choice([10000.0, 500000.0, 1e6]), queries=op == "append" and rng.random() < 0.7)
    c["longest"] = max(c["longest"], c["new"])
    while _cost(c) > 1:
        if c["batch"] > 1:
            c["batch"] = max(1, c["batch"] * 2 // 3)
        elif c["longest"] > c["new"]:
            c["longest"] = max(c["new"], c["longest"] * 2 // 3)
        else:
            c["new"] = c["new"] * 2 // 3
            c["longest"] = c["new"]
            if c.get("tree"):
                c["tree"] = c["new"]
    return c


def _cost(c):
    """The largest of a case's needs as parts of what a case may take."""
    w = work(c)
    padded = c["batch"] * c["heads"] * (c["group"] * c["new"] if c["op"] == "attend" else 0) * c["longest"]
    held = c["batch"] * c["longest"] * c["heads"] * c["d"] * BYTES[c["type"]] * 2
    return max(w["flops"] / MAX_FLOPS, w["bytes"] / MAX_BYTES, padded / MAX_PADDED, held / (2 * MAX_BYTES))


def _batch(c):
    """New tokens and lengths (new ones included) of each sequence."""
    rng = random.Random(c["shape"])
    new, lengths = [], []
    for b in range(c["batch"]):
        n = c["new"]
        if c["ragged"] and n > 1 and not c.get("tree") and c["op"] != "keep":
            n = rng.randint(1, n)
        length = c["longest"] if not c["ragged"] else max(n, _log(rng, max(1, c["longest"] / 100), c["longest"]))
        new.append(n)
        lengths.append(length)
    return new, lengths


def _parents(c):
    """The drafted tree of a case: a token's parent is one of the eight in front of it, -1 for the first."""
    rng = random.Random(c["shape"] + 1)
    return [-1] + [rng.randrange(max(0, i - 8), i) for i in range(1, c["new"])]


def _depths(parents):
    depth = []
    for p in parents:
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return depth


def _paths(c):
    """The accepted nodes of each sequence's tree, from the root down: the root at least, `depth` at most."""
    rng, parents = random.Random(c["shape"] + 2), _parents(c)
    paths = []
    for _ in range(c["batch"]):
        path, most = [0], rng.randint(1, c["depth"])
        while len(path) < most:
            after = [i for i, p in enumerate(parents) if p == path[-1]]
            if not after:
                break
            path.append(rng.choice(after))
        paths.append(path)
    return paths


def work(case):
    c = case
    new, lengths = _batch(c)
    e = BYTES[c["type"]]
    row = c["heads"] * c["d"] * e
    if c["op"] == "attend":
        if c["tree"]:
            pairs = sum(l - n for n, l in zip(new, lengths)) * c["new"] + c["batch"] * sum(v + 1 for v in _depths(_parents(c)))
        else:
            pairs = sum(n * (l - n) + n * (n + 1) // 2 for n, l in zip(new, lengths))
        return {"bytes": 2 * sum(lengths) * row + 2 * sum(new) * row * c["group"], "flops": 4.0 * c["d"] * c["heads"] * c["group"] * pairs}
    tokens = sum(new)
    moved = tokens * (2 + (c["group"] if c["queries"] else 0)) + (sum(len(p) for p in _paths(c)) * 2 if c["op"] == "keep" else 0)
    return {"bytes": 2 * moved * row + 8 * tokens, "flops": 0}


# ------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _inputs(c, seed):
    """A dict: the cache's two halves [pages][heads][page][d] filled with what the sequences hold, the batch (int32: starts, lengths, pages of
    each sequence in an order of no meaning, -1 behind its last), and what the operator takes."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    t, heads, d, page = TYPES[c["type"]], c["heads"], c["d"], c["page"]
    new, lengths = _batch(c)
    held = [-(-v // page) for v in lengths]
    order = torch.randperm(sum(held) + 3, generator=g, device="cuda").to(torch.int32)
    pages = torch.full((c["batch"], max(held)), -1, dtype=torch.int32, device="cuda")
    before = torch.tensor([0] + held, device="cuda").cumsum(0)
    at = torch.arange(max(held), device="cuda")
    there = at < torch.tensor(held, device="cuda")[:, None]
    pages[there] = order[(before[:-1, None] + at)[there]]
    starts = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    big = torch.where(torch.rand(d, generator=g, device="cuda") < 0.05, 3.0, 1.0)
    s = dict(k=(_normal(g, len(order), heads, page, d) * big).to(t), v=_normal(g, len(order), heads, page, d).to(t),
             starts=starts, lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), pages=pages)
    tokens = sum(new)
    owner = torch.repeat_interleave(torch.arange(c["batch"], device="cuda"), torch.tensor(new, device="cuda"))
    index = torch.arange(tokens, device="cuda") - starts[owner] + (s["lengths"] - torch.tensor(new, device="cuda"))[owner]
    if c["op"] == "attend":
        s["q"] = (_normal(g, tokens, heads * c["group"], d) * (1.5 / big.square().mean().sqrt())).to(t)
        if c["tree"]:
            s["tree"] = _tree_words(c).repeat(c["batch"], 1).cuda()
        return s
    # rows of a projection: queries, keys and values of a token side by side
    rows = (_normal(g, tokens, heads * (c["group"] + 2), d)).to(t)
    s["q"], s["new_k"], s["new_v"] = rows.split([heads * c["group"], heads, heads], dim=1)
    s["positions"] = index
    if c["op"] == "keep":
        depth = torch.tensor(_depths(_parents(c)), device="cuda")
        s["positions"] = (s["lengths"].long() - c["new"])[owner] + depth.repeat(c["batch"])
        paths = _paths(c)
        s["paths"] = torch.tensor([p + [-1] * (c["depth"] - len(p)) for p in paths], dtype=torch.int32, device="cuda")
    return s


def _tree_words(c):
    """int64 [tokens][words]: bit j % 64 of word j // 64 says that a node sees node j, itself and its ancestors."""
    parents, seen = _parents(c), []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    words = -(-len(parents) // 64)
    signed = lambda w: w - (1 << 64) if w >> 63 else w                    # noqa: E731
    return torch.tensor([[signed(m >> 64 * k & (1 << 64) - 1) for k in range(words)] for m in seen], dtype=torch.int64)


def _frequencies(c):
    """Radians a position, in 64 bits."""
    f = [c["theta"] ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]
    if c["scaling"] == "linear":
        f = [v / 4 for v in f]
    if c["scaling"] == "bands":
        g = [min(1.0, max(0.0, (8192 * v / (2 * math.pi) - 1.0) / 3.0)) for v in f]
        f = [v * (w + (1 - w) / 8) for v, w in zip(f, g)]
    return f


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case, longest_new=max(_batch(case)[0]), longest=max(_batch(case)[1]))
    if case["op"] != "attend":
        state["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    if own:
        import paper_2510_23264_amd as P
        state["P"] = P
        state["cache"] = P.KvCache(state["k"], state["v"])
        state["batch"] = P.KvBatch(state["starts"], state["lengths"], state["pages"])
        if case["op"] != "attend":
            factor = {"none": 1.0, "linear": 4.0, "bands": 8.0}[case["scaling"]]
            state["table"] = P.rotary_table(case["rot"], theta=case["theta"], scaling=case["scaling"], factor=factor, original=8192, turns=(1.0, 4.0))
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    c, P, cache, batch = state["case"], state["P"], state["cache"], state["batch"]
    if c["op"] == "attend":
        return P.kv_attention(state["q"], cache, batch, tree=state.get("tree"))
    q = P.kv_append(cache, batch, state["new_k"], state["new_v"], positions=state["positions"], table=state["table"], layout=c["layout"],
                    q=state["q"] if c["queries"] else None)
    if c["op"] == "append":
        return q, cache.keys, cache.values
    return P.kv_keep(cache, batch, state["paths"]), cache.keys, cache.values


def _run_plain(state):
    return {"append": _append, "attend": _attend, "keep": _keep}[state["case"]["op"]](state)


def _turn(x, angle, layout):
    x, r, cos, sin = x.float(), 2 * angle.shape[1], angle.cos().float()[:, None], angle.sin().float()[:, None]
    if layout == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat((a * cos - b * sin, a * sin + b * cos), dim=-1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack((a * cos - b * sin, a * sin + b * cos), dim=-1).flatten(-2)
    return torch.cat((turned, x[..., r:]), dim=-1)


def _places(state, owner, index):
    """Page and place in the page of a sequence's rows."""
    page = state["case"]["page"]
    return state["pages"][owner, index // page].long(), index % page


def _owners(state):
    new = state["starts"].diff()
    return torch.repeat_interleave(torch.arange(len(new), device=new.device), new.long(), output_size=len(state["new_k"])), new


def _append(state):
    c = state["case"]
    owner, new = _owners(state)
    index = torch.arange(len(owner), device=owner.device) - state["starts"][owner] + (state["lengths"] - new)[owner]
    page, place = _places(state, owner, index)
    angle = state["positions"].double()[:, None] * state["frequencies"]
    state["k"][page, :, place] = _turn(state["new_k"], angle, c["layout"]).to(state["k"].dtype)
    state["v"][page, :, place] = state["new_v"]
    q = _turn(state["q"], angle, c["layout"]).to(state["q"].dtype) if c["queries"] else None
    return q, state["k"], state["v"]


def _keep(state):
    _append(state)
    new, paths = state["starts"].diff(), state["paths"]
    base, (owner, i) = state["lengths"] - new, torch.nonzero(paths >= 0, as_tuple=True)
    source = _places(state, owner, base[owner] + paths[owner, i])
    target = _places(state, owner, base[owner] + i)
    state["k"][target[0], :, target[1]] = state["k"][source[0], :, source[1]]
    state["v"][target[0], :, target[1]] = state["v"][source[0], :, source[1]]
    return base + (paths >= 0).sum(1).to(torch.int32), state["k"], state["v"]


def _attend(state):
    c, q, starts, lengths = state["case"], state["q"], state["starts"].long(), state["lengths"].long()
    batch, heads, group, d = c["batch"], c["heads"], c["group"], c["d"]
    new, i, j = starts.diff(), torch.arange(state["longest_new"], device=q.device), torch.arange(state["longest"], device=q.device)
    held = j < lengths[:, None]
    page, place = _places(state, torch.arange(batch, device=q.device)[:, None], torch.where(held, j, 0))
    # [batch][heads][longest][d], and the queries of a group below each other
    k = state["k"][page, :, place].float().permute(0, 2, 3, 1).contiguous()
    v = (state["v"][page, :, place].float() * held[:, :, None, None]).permute(0, 2, 1, 3).contiguous()
    there = i < new[:, None]
    row = torch.where(there, starts[:-1, None] + i, 0)
    rows = q[row].float().view(batch, len(i), heads, group, d).permute(0, 2, 3, 1, 4).reshape(batch, heads, group * len(i), d)
    s = torch.matmul(rows, k).view(batch, heads, group, len(i), len(j)) * d ** -0.5
    ahead = j - (lengths - new)[:, None]                                   # which new token a key is, negative for those before
    if c["tree"]:
        words, place = state["tree"][row], ahead.clamp(min=0)
        seen = words.gather(2, (place // 64)[:, None].clamp(max=words.shape[2] - 1).expand(-1, len(i), -1)) >> (place % 64)[:, None] & 1
        seen = (ahead < 0)[:, None] | (seen != 0)
    else:
        seen = ahead[:, None] <= i[:, None]
    seen = (seen & held[:, None])[:, None, None]
    top = s.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(s - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = p.sum(-1, keepdim=True)
    p = (p / torch.where(total == 0, 1.0, total)).view(batch, heads, group * len(i), len(j))
    o = torch.matmul(p, v).view(batch, heads, group, len(i), d).permute(0, 3, 1, 2, 4).reshape(batch, len(i), heads * group, d)
    return o[there].to(q.dtype)


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    c, s = case, _inputs(case, seed)
    new, lengths = _batch(c)
    page = c["page"]

    def rows_of(cache, b, lo, hi):
        """Rows lo .. hi - 1 of sequence b: [hi - lo][heads][d]."""
        parts = []
        for at in range(lo // page, -(-hi // page)):
            whole = cache[int(table[b][at])].transpose(0, 1)
            parts.append(whole[max(0, lo - at * page):min(page, hi - at * page)])
        return torch.cat(parts)

    table = s["pages"].tolist()
    if c["op"] == "attend":
        out, at = [], 0
        bits = _tree_words(c).tolist() if c["tree"] else None
        for b in range(c["batch"]):
            n, length = new[b], lengths[b]
            base = length - n
            ks, vs = rows_of(s["k"], b, 0, length), rows_of(s["v"], b, 0, length)
            if bits is None:
                hidden = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1)
            else:
                hidden = torch.tensor([[bits[i][j // 64] >> j % 64 & 1 == 0 for j in range(n)] for i in range(n)], device="cuda")
            hidden = hidden.repeat_interleave(c["group"], dim=0)
            each = []
            for h in range(c["heads"]):
                k, v, q = ks[:, h].double(), vs[:, h].double(), s["q"][at:at + n, h * c["group"]:(h + 1) * c["group"]].double()
                z = q.reshape(n * c["group"], c["d"]) @ k.t().contiguous() / math.sqrt(c["d"])
                z[:, base:][hidden] = -math.inf
                each.append((torch.softmax(z, dim=1) @ v).view(n, c["group"], c["d"]))
            out.append(torch.cat(each, dim=1))
            at += n
        return torch.cat(out)

    f = _frequencies(c)

    def turned(x):
        y = x.double().clone()
        for i, w in enumerate(f):
            ia, ib = (i, i + c["rot"] // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
            z = torch.complex(x[..., ia].double(), x[..., ib].double()) * torch.polar(
                torch.ones(len(x), dtype=torch.float64, device="cuda"), s["positions"].double() * w)[:, None]
            y[..., ia], y[..., ib] = z.real, z.imag
        return y

    k, v, new_k = s["k"].double(), s["v"].double(), turned(s["new_k"])
    owner = torch.tensor([b for b, n in enumerate(new) for _ in range(n)], device="cuda")
    index = torch.tensor([lengths[b] - n + i for b, n in enumerate(new) for i in range(n)], device="cuda")
    k[s["pages"][owner, index // page].long(), :, index % page] = new_k
    v[s["pages"][owner, index // page].long(), :, index % page] = s["new_v"].double()
    if c["op"] == "append":
        return turned(s["q"]) if c["queries"] else None, k, v
    paths, after = _paths(c), []
    for b, path in enumerate(paths):
        base = lengths[b] - new[b]
        at = [(table[b][(base + x) // page], (base + x) % page) for x in path]
        rows = [(k[p, :, o].clone(), v[p, :, o].clone()) for p, o in at]
        for i, (x, y) in enumerate(rows):
            k[table[b][(base + i) // page], :, (base + i) % page] = x
            v[table[b][(base + i) // page], :, (base + i) % page] = y
        after.append(base + len(path))
    return torch.tensor(after, dtype=torch.int32, device="cuda"), k, v
