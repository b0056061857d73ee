"""Serving on a restored cache: attention over a shared prefix, new tokens into pages, and the pages' own life, as cases
that can be timed and checked.

A case is one pass of a serving program over a pool of pages (one cache of [2][blocks][block][heads][dim] a layer, a table
of pages and a length a row, a count of holders a page):

  attend   kvc_attend_paged: the queries of a batch whose rows share their first tokens, one layer
  append   kvc_append_paged: keys and values of new tokens to their slots, one layer
  samples  kvc_pages_free, _fork, _grow: last turn's samples go, every prompt is forked anew, each fork gets room for a token
  copy     kvc_pages_copy: whole pages of all layers
  compact  kvc_pages_compact: the pages in use move to the lowest places, tables and counts follow

Rows: row 0 holds the shared prefix (attend), or the rows of a case come one after the other (the others).  Sizes are those
of the models whose tiles this repository packs, of their tensor-parallel shards, and of the blocks its tests page by.
"""
import math

import torch

own = False  # false: the plain forms; true: the library's kernels

DEV = "cuda"
TORCH_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}

# layers, query heads, KV heads, head_dim
MODELS = {
    "llama8b": (32, 32, 8, 128),
    "yi34b": (60, 56, 8, 128),
    "lwm7b": (32, 32, 32, 128),
    "llama70b": (80, 64, 8, 128),
}


def _case(op, model, dtype="f16", tp=1, block=16, layers=None, **more):
    L, Q, H, D = MODELS[model]
    return dict({"op": op, "layers": L if layers is None else layers, "q_heads": Q // tp, "heads": H // tp, "head_dim": D,
                 "dtype": dtype, "block": block}, **more)


def _attend(model, requests, prefix, own_tokens, new=1, **more):
    """own_tokens: of the longest row beyond the prefix; new: queries of the row with most of them."""
    return _case("attend", model, layers=1, requests=requests, prefix=prefix, own_tokens=max(own_tokens, new), new=new, **more)


def listed():
    cases = [
        # a chat's four samples behind a system prompt, a few tokens in: the call is over as soon as it has begun
        ("attend_four_short", _attend("llama8b", 4, 1000, 60)),
        # a document of 32K tokens, fetched once, and 64 conversations about it: a decoding step
        ("attend_64_of_32k", _attend("llama8b", 64, 32768, 500)),
        # one of eight tensor-parallel shards, a single KV head, odd lengths, more of the rows' own than is shared
        ("attend_shard_odd", _attend("llama70b", 33, 12345, 2001, dtype="bf16", tp=8, block=32)),
        # eight questions of up to 317 tokens about a 32K-token document arrive at once: the first pass over them
        ("attend_questions", _attend("yi34b", 8, 32768, 317, new=317, dtype="bf16")),
        # the step's new keys and values of 64 conversations
        ("append_step", _case("append", "llama8b", layers=1, requests=64, old_tokens=900, new=1)),
        # the keys and values of prompts of up to 1000 tokens
        ("append_prompts", _case("append", "yi34b", "bf16", layers=1, requests=16, old_tokens=100, new=1000, block=64)),
        # one prompt, four samples
        ("samples_of_one", _case("samples", "llama8b", prompts=1, samples=4, tokens=1001)),
        # 32 prompts of up to 397 tokens, eight samples each
        ("samples_of_32", _case("samples", "llama8b", prompts=32, samples=8, tokens=397)),
        # a few pages that a scheduler moves out of the way
        ("copy_three", _case("copy", "llama70b", "bf16", tp=8, pages=3, blocks=200)),
        # 150 pages of all 60 layers
        ("copy_150", _case("copy", "yi34b", "bf16", pages=150, blocks=400)),
        # a shard's pool, one third in use
        ("compact_shard", _case("compact", "llama70b", "bf16", tp=8, block=32, blocks=501, used=167, rows=12)),
        # a pool of 1300 pages, 40 % of them in use, spread all over
        ("compact_1300", _case("compact", "llama8b", blocks=1300, used=520, rows=64)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    op = rng.choices(["attend", "append", "samples", "copy", "compact"], [5, 1, 2, 1, 2])[0]
    model, dtype = rng.choice(sorted(MODELS)), rng.choice(["f16", "bf16"])
    tp, block = rng.choice([1, 1, 2, 4, 8]), rng.choice([8, 16, 16, 32, 64])
    of = {"dtype": dtype, "tp": tp, "block": block}
    page = 2 * 2 * block * MODELS[model][0] * MODELS[model][2] // tp * MODELS[model][3]  # bytes, all layers
    if op == "attend":
        most = _cost(listed()[3])
        while True:
            new = rng.choices([1, rng.randint(2, 8), _log(rng, 9, 1000)], [6, 2, 3])[0]
            c = _attend(model, _log(rng, 1, 128), 0 if rng.random() < 0.1 else _log(rng, 50, 32768), _log(rng, 1, 3000), new, **of)
            scores = sum(_new_tokens(c)) * c["q_heads"] * (c["prefix"] + c["own_tokens"])
            padded = c["requests"] * c["new"] * c["q_heads"] * c["own_tokens"]
            rows = c["requests"] * c["own_tokens"] * c["heads"] * c["head_dim"]
            if _cost(c) <= most and max(scores, padded) <= 5 << 29 and rows <= 1 << 29:  # (what the plain form holds)
                return c
    if op == "append":
        return _case(op, model, layers=1, requests=_log(rng, 1, 64), old_tokens=_log(rng, 1, 2000), new=rng.choice([1, _log(rng, 2, 500)]), **of)
    if op == "samples":
        prompts, samples, tokens = _log(rng, 1, 24), _log(rng, 1, 8), _log(rng, 1, 2000)
        while _samples_blocks(prompts, samples, tokens, block) * page > 3 << 30:
            prompts, tokens = max(1, prompts // 2), max(1, tokens // 2)
        return _case(op, model, prompts=prompts, samples=samples, tokens=tokens, **of)
    blocks = max(16, min(_log(rng, 24, 3000), (3 << 30) // page))
    if op == "copy":
        return _case(op, model, pages=max(1, min(_log(rng, 1, 400), blocks // 2)), blocks=blocks, **of)
    used = rng.randint(1, blocks)
    return _case(op, model, blocks=blocks, used=used, rows=_log(rng, 1, min(used, 100)), **of)


# ------------------------------------------------------------------ sizes that follow from a case


def _spread(n, low, high):
    """n whole numbers from high down to about low."""
    return [high - (high - low) * i // n for i in range(n)]


def _new_tokens(c):
    return _spread(c["requests"], 1, c["new"])


def _own_tokens(c):
    """Tokens of each row beyond the prefix, the new ones among them."""
    return [max(new, o) for new, o in zip(_new_tokens(c), _spread(c["requests"], 1, c["own_tokens"]))]


def _pages(tokens, block):
    return -(-tokens // block)


def _samples_blocks(prompts, samples, tokens, block):
    shared = sum(_pages(t, block) for t in _spread(prompts, 1, tokens))
    return 2 * (shared + 3 * prompts * samples) + 8


def work(c):
    token = 2 * c["heads"] * c["head_dim"] * 2  # bytes of a token's keys and values in one layer
    if c["op"] == "attend":
        new, owned = _new_tokens(c), _own_tokens(c)
        seen = sum(n * (c["prefix"] + o) - n * (n - 1) // 2 for n, o in zip(new, owned))
        rows = sum(new) * c["q_heads"]
        return {"bytes": (c["prefix"] + sum(owned)) * token + rows * (2 * c["head_dim"] * 2 + 4),
                "flops": 4 * seen * c["q_heads"] * c["head_dim"]}
    if c["op"] == "append":
        return {"bytes": 2 * sum(_new_tokens(c)) * token, "flops": 0}
    token *= c["layers"]
    page = token * c["block"]
    if c["op"] == "samples":  # the part of a page that each fork copies, and the counts of all pages
        part = sum(t % c["block"] for t in _spread(c["prompts"], 1, c["tokens"])) * c["samples"]
        shared = sum(t // c["block"] for t in _spread(c["prompts"], 1, c["tokens"])) * c["samples"]
        blocks = _samples_blocks(c["prompts"], c["samples"], c["tokens"], c["block"])
        return {"bytes": 2 * part * token + 4 * (2 * blocks + 4 * shared), "flops": 0}
    if c["op"] == "copy":
        return {"bytes": 2 * c["pages"] * page, "flops": 0}
    return {"bytes": 2 * _moved(c) * page + 4 * 3 * c["blocks"], "flops": 0}


def _moved(c):
    return c["used"] * (c["blocks"] - c["used"]) // c["blocks"]


# ------------------------------------------------------------------ inputs


def _generators(seed):
    g, h = torch.Generator(device=DEV), torch.Generator()
    g.manual_seed(seed)
    h.manual_seed(seed)
    return g, h


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _normal(shape, g, dtype):
    """Normal values, each channel with a deviation of its own: log-uniform in [0.3, 2]."""
    x = torch.randn(shape, generator=g, device=DEV)
    sigma = torch.exp(torch.empty(shape[-2:], device=DEV).uniform_(math.log(0.3), math.log(2.0), generator=g))
    return x.mul_(sigma).to(TORCH_DTYPE[dtype])


def _paged(c, rows, blocks, h):
    """Tables of rows of so many pages, on pages in random order; the pages that are left."""
    order = torch.randperm(blocks, generator=h).tolist()
    length = max(1, max(rows, default=1))
    tables, at = [], 0
    for n in rows:
        tables.append(order[at:at + n] + [-1] * (length - n))
        at += n
    return tables, order[at:]


def prepare(case, seed):
    c, (g, h) = case, _generators(seed)
    s = {"case": c, "block": c["block"]}
    make = {"attend": _prepare_attend, "append": _prepare_append, "samples": _prepare_samples, "copy": _prepare_copy, "compact": _prepare_compact}
    make[c["op"]](c, s, g, h)
    s["layers"] = torch.tensor([x.data_ptr() for x in s["cache"]], dtype=torch.int64, device=DEV)
    if own:
        _handles(s)
    return s


def _shuffled(values, h):
    return [values[i] for i in torch.randperm(len(values), generator=h).tolist()]


def _batch(s, new, h):
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"], s["n_new"], s["most_new"] = _i32(starts), starts[-1], max(new)


def _prepare_attend(c, s, g, h):
    b, P, H, D = c["block"], c["prefix"], c["heads"], c["head_dim"]
    both = _shuffled(list(zip(_new_tokens(c), _own_tokens(c))), h)  # the rows' order is the seed's
    new, lens = [n for n, _ in both], [P + o for _, o in both]
    shared = P // b
    rows = [_pages(P, b)] + [_pages(n, b) - shared for n in lens]
    blocks = sum(rows) + sum(rows) // 4 + 1
    tables, _ = _paged(c, rows, blocks, h)
    length = max(_pages(n, b) for n in lens + [P])
    tables = [(t if i == 0 else tables[0][:shared] + t[:rows[i]]) for i, t in enumerate(tables)]
    s["tables"] = _i32([(t + [-1] * length)[:length] for t in tables])
    s["lens"], s["refs"] = _i32([P] + lens), None
    s["cache"] = _normal((1, 2, blocks, b, H, D), g, c["dtype"])
    if P % b:  # what a fork copies: the prompt's last page, filled in part, is each row's own
        at = s["tables"][1:, shared].long()
        s["cache"][0, :, at, :P % b] = s["cache"][0, :, tables[0][shared]][:, None, :P % b]
    _batch(s, new, h)
    s["rows"] = _i32(list(range(1, len(new) + 1)))
    s["q"] = _normal((s["n_new"], c["q_heads"], D), g, c["dtype"])
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((s["n_new"], c["q_heads"]), device=DEV)
    s["most_tokens"], s["scale"] = max(lens), 1.0 / math.sqrt(D)


def _prepare_append(c, s, g, h):
    b, H, D = c["block"], c["heads"], c["head_dim"]
    both = _shuffled(list(zip(_new_tokens(c), reversed(_spread(c["requests"], 0, c["old_tokens"])))), h)
    new, lens = [n for n, _ in both], [n + o for n, o in both]
    rows = [_pages(n, b) for n in lens]
    blocks = sum(rows) + sum(rows) // 4 + 1
    s["tables"], s["lens"], s["refs"] = _i32(_paged(c, rows, blocks, h)[0]), _i32(lens), None
    s["cache"] = _normal((1, 2, blocks, b, H, D), g, c["dtype"])
    _batch(s, new, h)
    s["rows"] = _i32(list(range(len(new))))
    s["qkv"] = _normal((s["n_new"], c["q_heads"] + 2 * H, D), g, c["dtype"])  # what the layer's projection gives, in one piece


def _bits(c, blocks, g):
    return torch.randint(-32768, 32768, (c["layers"], 2, blocks, c["block"], c["heads"] * c["head_dim"]), generator=g, device=DEV, dtype=torch.int16)


def _prepare_samples(c, s, g, h):
    b, prompts, each = c["block"], c["prompts"], c["samples"]
    tokens = _shuffled(_spread(prompts, 1, c["tokens"]), h)
    n = prompts * each
    blocks = _samples_blocks(prompts, each, c["tokens"], b)
    parents = [i // each for i in range(n)]
    # the last turn's samples: two pages of their own each, and all whole pages of a prompt
    last = _shuffled(parents, h)
    tables, _ = _paged(c, [_pages(t, b) for t in tokens] + [2] * n, blocks, h)
    length = max(_pages(t, b) for t in tokens) + 3
    refs, lens = [0] * blocks, list(tokens)
    for i, p in enumerate(last):
        shared = tokens[p] // b
        tables[prompts + i] = tables[p][:shared] + tables[prompts + i][:2]
        lens.append((shared + 1) * b + 1)
    for t, k in zip(tables, lens):
        for page in t[:_pages(k, b)]:
            refs[page] += 1
    s["tables"] = _i32([(t + [-1] * length)[:length] for t in tables])
    s["lens"], s["refs"] = _i32(lens), _i32(refs)
    s["parents"], s["children"] = _i32(parents), _i32(list(range(prompts, prompts + n)))
    s["cache"] = _bits(c, blocks, g)


def _prepare_copy(c, s, g, h):
    order = torch.randperm(c["blocks"], generator=h)[:2 * c["pages"]].to(torch.int32).to(DEV)
    s["src"], s["dst"] = order[:c["pages"]].contiguous(), order[c["pages"]:].contiguous()
    s["tables"], s["lens"], s["refs"] = _i32([[0]]), _i32([0]), None
    s["cache"] = _bits(c, c["blocks"], g)


def _prepare_compact(c, s, g, h):
    b, n, rows = c["block"], c["used"], c["rows"]
    high = _moved(c)  # so many of the pages in use lie beyond the place of the last one after the call
    low = torch.randperm(n, generator=h)[:n - high].tolist()
    pages = _shuffled(low + [n + i for i in torch.randperm(c["blocks"] - n, generator=h)[:high].tolist()], h)
    cut = [n * i // rows for i in range(rows + 1)]
    tables = [pages[i:j] for i, j in zip(cut, cut[1:])]
    refs = [0] * c["blocks"]
    tables += [t[:len(t) // 2] for t in tables[:rows // 2]]  # forks that hold the first half of another row's pages
    length = max(1, max(len(t) for t in tables))
    for t in tables:
        for page in t:
            refs[page] += 1
    more = torch.randint(0, b, (len(tables),), generator=h).tolist()
    lens = [len(t) * b - (k if t and i < rows else 0) for i, (t, k) in enumerate(zip(tables, more))]
    s["tables"] = _i32([(t + [-1] * length)[:length] for t in tables])
    s["lens"], s["refs"] = _i32(lens), _i32(refs)
    s["new_tables"], s["new_refs"], s["map"] = torch.empty_like(s["tables"]), torch.empty_like(s["refs"]), torch.empty_like(s["refs"])
    s["cache"] = _bits(c, c["blocks"], g)


# ------------------------------------------------------------------ one pass


def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


# The library's calls.


def _handles(s):
    """What a program that serves from a pool keeps: its descriptor, and the workspaces of its calls."""
    import paper_2602_09725_amd as kvc

    c, ptr = s["case"], lambda name: None if s.get(name) is None else s[name].data_ptr()  # noqa: E731
    dtype = kvc.KVC_F16 if c["dtype"] == "f16" else kvc.KVC_BF16
    n_rows, length = s["tables"].shape
    s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    s["pool"] = kvc.Pool(c["layers"], c["heads"], c["head_dim"], dtype, s["cache"].shape[2], c["block"], n_rows, length, ptr("layers"),
                         ptr("tables"), ptr("lens"), ptr("refs"), ptr("err"))
    size = 0
    if "starts" in s:
        one_each = s["most_new"] == 1
        s["batch"] = kvc.Batch(s["rows"].numel(), s["n_new"], s["most_new"], ptr("rows"), None if one_each else ptr("starts"))
    if c["op"] == "attend":
        strides = (c["q_heads"] * c["head_dim"], c["head_dim"])
        s["attention"] = kvc.Attention(c["q_heads"], s["scale"], s["most_tokens"], c["prefix"], 0, strides, strides)
        size = kvc.attention_workspace(s["pool"], s["batch"], s["attention"])
    elif c["op"] in ("samples", "compact"):
        size = kvc.pages_workspace(s["pool"])
    s["workspace"] = torch.empty(size, dtype=torch.uint8, device=DEV)
    s["kvc"] = kvc


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_attend(s):
    w = s["workspace"]
    s["kvc"].kvc_attend_paged(s["pool"], s["batch"], s["attention"], 0, s["q"].data_ptr(), s["out"].data_ptr(), s["lse"].data_ptr(),
                              w.data_ptr(), w.numel(), _stream())
    return {"out": s["out"], "lse": s["lse"]}


def _own_append(s):
    c, x = s["case"], s["qkv"]
    k, v = x[:, c["q_heads"]:], x[:, c["q_heads"] + c["heads"]:]
    s["kvc"].kvc_append_paged(s["pool"], s["batch"], 0, k.data_ptr(), v.data_ptr(), x.stride(0), _stream())
    return {"cache": s["cache"]}


def _own_samples(s):
    kvc, pool, w, n, at = s["kvc"], s["pool"], s["workspace"], s["children"].numel(), _stream()
    children, room = s["children"].data_ptr(), (w.data_ptr(), w.numel())
    kvc.kvc_pages_free(pool, children, n, at)
    kvc.kvc_pages_fork(pool, s["parents"].data_ptr(), children, n, *room, at)
    kvc.kvc_pages_grow(pool, children, None, n, *room, at)
    return _pool_state(s)


def _own_copy(s):
    s["kvc"].kvc_pages_copy(s["pool"], s["src"].data_ptr(), s["dst"].data_ptr(), s["src"].numel(), _stream())
    return {"cache": s["cache"]}


def _own_compact(s):
    w = s["workspace"]
    s["kvc"].kvc_pages_compact(s["pool"], s["map"].data_ptr(), s["new_tables"].data_ptr(), s["new_refs"].data_ptr(), w.data_ptr(),
                               w.numel(), _stream())
    return {"map": s["map"], "tables": s["new_tables"], "refs": s["new_refs"], "cache": s["cache"]}


# The plain forms.


def _pool_state(s):
    return {"tables": s["tables"], "lens": s["lens"], "refs": s["refs"], "cache": s["cache"]}


def _tokens(s):
    """Of every new token: its request, its place among the request's, its row's length, and its position."""
    starts = s["starts"].long()
    t = torch.arange(s["n_new"], device=DEV)
    r = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[r]
    length = s["lens"].long()[s["rows"].long()[r]]
    return r, i, length - (starts[r + 1] - starts[r]) + i


def _plain_attend(s):
    c, b = s["case"], s["block"]
    P, H, D, n = c["prefix"], c["heads"], c["head_dim"], s["n_new"]
    G, R, m, S = c["q_heads"] // H, s["rows"].numel(), s["most_new"], s["most_tokens"] - P
    r, i, at = _tokens(s)
    kv = s["cache"][0].flatten(1, 2)  # [2][slots][H][D]
    q = (s["q"].float() * s["scale"]).view(n, H, G, D)

    def slots(table, positions):
        return table.gather(-1, positions // b).clamp(min=0).long() * b + positions % b

    # the prefix, once for all: [H][n G][P]
    positions = torch.arange(P, device=DEV)
    shared = kv[:, slots(s["tables"][0], positions)].float().permute(0, 2, 1, 3).contiguous()  # [2][H][P][D]
    near = torch.matmul(q.permute(1, 0, 2, 3).reshape(H, n * G, D), shared[0].transpose(1, 2).contiguous()).view(H, n, G, P)
    near = near.masked_fill((positions > at[:, None])[None, :, None, :], -math.inf)
    # each row's own tokens, all rows as long as the longest: [R][H][m G][S]
    ours = P + torch.arange(S, device=DEV).expand(R, S)
    last = s["tables"].shape[1] * b - 1
    k, v = kv[:, slots(s["tables"][s["rows"].long()], ours.clamp(max=last))].float().permute(0, 1, 3, 2, 4).contiguous()  # [R][H][S][D]
    padded = torch.zeros((R, m, H, G, D), device=DEV)
    padded[r, i] = q
    far = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(R, H, m * G, D), k.transpose(2, 3).contiguous())
    far = far.view(R, H, m, G, S).permute(0, 2, 1, 3, 4)[r, i].permute(1, 0, 2, 3)  # [H][n][G][S]
    far = far.masked_fill((ours[r] > at[:, None])[None, :, None, :], -math.inf)
    # one softmax over both
    scores = torch.cat([near, far], dim=-1)
    most = scores.amax(dim=-1, keepdim=True)
    most = torch.where(most == -math.inf, torch.zeros_like(most), most)
    p = torch.exp(scores.sub_(most))
    total = p.sum(dim=-1, keepdim=True)
    of_prefix = torch.matmul(p[..., :P].reshape(H, n * G, P), shared[1]).view(H, n, G, D)
    padded = torch.zeros((R, m, H, G, S), device=DEV)
    padded[r, i] = p[..., P:].permute(1, 0, 2, 3)
    of_own = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(R, H, m * G, S), v)
    of_own = of_own.view(R, H, m, G, D).permute(0, 2, 1, 3, 4)[r, i].permute(1, 0, 2, 3)
    out = (of_prefix + of_own) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (most + torch.log(total)).squeeze(-1)
    return {"out": out.permute(1, 0, 2, 3).reshape(n, H * G, D).to(TORCH_DTYPE[c["dtype"]]), "lse": lse.permute(1, 0, 2).reshape(n, H * G).contiguous()}


def _plain_append(s):
    c, b = s["case"], s["block"]
    H = c["heads"]
    r, _, at = _tokens(s)
    slot = s["tables"][s["rows"].long()[r], at // b].long() * b + at % b
    k, v = s["qkv"][:, c["q_heads"]:].split(H, dim=1)
    kv = s["cache"][0].flatten(1, 2)
    kv[0, slot], kv[1, slot] = k, v
    return {"cache": s["cache"]}


def _free_pages(refs):
    return torch.nonzero(refs == 0).flatten().to(torch.int32)


def _plain_samples(s):
    b, tables, lens, refs, cache = s["block"], s["tables"], s["lens"], s["refs"], s["cache"]
    parents, children = s["parents"].long(), s["children"].long()
    column = torch.arange(tables.shape[1], device=DEV)
    # free
    held = column < ((lens[children] + b - 1) // b)[:, None]
    pages = tables[children][held].long()
    refs.index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    # fork
    n = lens[parents].long()
    rows, whole = tables[parents], (column < (n // b)[:, None])
    pages = rows[whole].long()
    refs.index_add_(0, pages, torch.ones_like(pages, dtype=torch.int32))
    part = n % b > 0
    source = rows.gather(1, (n // b).clamp(max=tables.shape[1] - 1)[:, None])[part, 0].long()
    fresh = _free_pages(refs)[:source.numel()]
    into = rows[part]
    into.scatter_(1, (n[part] // b)[:, None], fresh[:, None])
    rows[part] = into
    used = torch.where(column < ((n + b - 1) // b)[:, None], rows, tables[children])
    tables[children], lens[children] = used, n.to(torch.int32)
    refs[fresh.long()] = 1
    filled = (torch.arange(b, device=DEV) < (n[part] % b)[:, None])[None, None, :, :, None]
    cache[:, :, fresh.long()] = torch.where(filled, cache[:, :, source], cache[:, :, fresh.long()])
    # grow, by a token each
    n = lens[children].long()
    new = n % b == 0
    fresh = _free_pages(refs)[:int(new.sum())]
    tables[children[new], (n // b)[new]] = fresh
    refs[fresh.long()] = 1
    lens[children] = (n + 1).to(torch.int32)
    return _pool_state(s)


def _plain_copy(s):
    s["cache"][:, :, s["dst"].long()] = s["cache"][:, :, s["src"].long()]
    return {"cache": s["cache"]}


def _plain_compact(s):
    b, tables, lens, refs, cache = s["block"], s["tables"], s["lens"], s["refs"], s["cache"]
    page = torch.arange(refs.numel(), device=DEV)
    used = refs > 0
    n = int(used.sum())
    source, place = page[n:][used[n:]], page[:n][~used[:n]]
    to = torch.where(used, page, torch.full_like(page, -1))
    to[source] = place
    cache[:, :, place] = cache[:, :, source]
    held = torch.arange(tables.shape[1], device=DEV) < ((lens + b - 1) // b)[:, None]
    new_tables = torch.where(held, to[tables.clamp(min=0).long()].to(torch.int32), tables)
    new_refs = torch.zeros_like(refs)
    new_refs[to[used]] = refs[used]
    return {"map": to.to(torch.int32), "tables": new_tables, "refs": new_refs, "cache": cache}


_PLAIN = {"attend": _plain_attend, "append": _plain_append, "samples": _plain_samples, "copy": _plain_copy, "compact": _plain_compact}
_OWN = {"attend": _own_attend, "append": _own_append, "samples": _own_samples, "copy": _own_copy, "compact": _own_compact}


# ------------------------------------------------------------------ from the definition, in 64 bits


def exact(case, seed):
    """Attention request by request over the whole of its row, prefix and all, head by head; appended values token by token.
    The other passes move bits."""
    if case["op"] not in ("attend", "append"):
        return None
    c, s = case, prepare(case, seed)
    b, H = c["block"], c["heads"]
    G = c["q_heads"] // H
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    if case["op"] == "append":
        cache, tables, x = s["cache"].double(), s["tables"].tolist(), s["qkv"].double()
        for row, (first, end) in enumerate(zip(starts, starts[1:])):
            for t in range(first, end):
                at = lens[row] - end + t
                cache[0, :, tables[row][at // b], at % b] = x[t, c["q_heads"]:].view(2, H, -1)
        return {"cache": cache}
    out = torch.zeros((s["n_new"], c["q_heads"], c["head_dim"]), dtype=torch.float64, device=DEV)
    lse = torch.full((s["n_new"], c["q_heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for request, row in enumerate(s["rows"].tolist()):
        first, end, n = starts[request], starts[request + 1], lens[row]
        pages = s["tables"][row, :_pages(n, b)].long()
        for head in range(H):
            keys = s["cache"][0, 0, pages, :, head].reshape(-1, c["head_dim"])[:n].double()
            values = s["cache"][0, 1, pages, :, head].reshape(-1, c["head_dim"])[:n].double()
            heads = slice(head * G, head * G + G)
            query = s["q"][first:end, heads].double()
            score = torch.einsum("qgd,kd->qgk", query, keys) * s["scale"]
            seen = torch.arange(n, device=DEV)[None] <= n - (end - first) + torch.arange(end - first, device=DEV)[:, None]
            score = score.masked_fill(~seen[:, None], -math.inf)
            norm = torch.logsumexp(score, dim=-1)
            share = torch.where(norm[..., None] == -math.inf, torch.zeros_like(score), torch.exp(score - norm[..., None]))
            out[first:end, heads] = torch.einsum("qgk,kd->qgd", share, values)
            lse[first:end, heads] = norm
    return {"out": out, "lse": lse}
