"""Serving on a cache held in 4 bits, as cases that can be timed and checked.

The pages of such a pool hold K and V as 4-bit codes, a pair {scale, mn} in the pool's 16-bit type for each token and head.
A case is one pass of a program that serves from them:

  attend   kvc_attend_paged: the queries of a batch whose rows share their first tokens, one layer
  write    kvc_append_paged, kvc_read_paged: new tokens are quantized as they are written, and read back as what they are now,
           for the pass over the prompt that has them at hand; one layer
  read     kvc_read_paged: whole rows back into 16-bit tensors, one layer
  convert  kvc_pages_convert: pages between a 16-bit pool and a 4-bit one, all layers; "back": from 4 bits only, "both": to 4
           bits and into other pages of the 16-bit pool again

Sizes are those of the models whose tiles this repository packs, of their tensor-parallel shards, and of the blocks that its
tests page by.  Rows: row 0 holds the shared prefix (attend), or the rows of a case come one after the other.

A page of one layer and kind, for H heads of D elements and blocks of b tokens, in 32-bit words:
  codes [H][b / 4][D / 8][4]: word w of a token holds its elements 8 w .. 8 w + 7, the even ones in the low half from bit 0
  on, the odd ones in the high half; tokens 4 i .. 4 i + 3 of a block lie side by side
  pairs [H][b]: scale in the low half, mn in the high one
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
    "narrow": (12, 12, 4, 64),
    "ragged": (6, 6, 2, 40),
    "wide": (18, 16, 8, 256),
}


def _case(op, model, dtype="f16", tp=1, block=16, layers=1, **more):
    L, Q, H, D = MODELS[model]
    return dict({"op": op, "layers": layers or L, "q_heads": Q // tp, "heads": H // tp, "head_dim": D, "dtype": dtype, "block": block}, **more)


def _attend(model, requests, prefix, own_tokens, new=1, **more):
    """own_tokens: of the longest row beyond the prefix; new: queries of the row with most of them."""
    return _case("attend", model, requests=requests, prefix=prefix, own_tokens=max(own_tokens, new), new=new, **more)


def listed():
    cases = [
        # a chat's four samples behind a system prompt, a few tokens in: the call is over as soon as it has begun
        ("attend_four_short", _attend("llama8b", 4, 1000, 60)),
        # a document of 32K tokens, fetched once, and 64 conversations about it: a decoding step
        ("attend_64_of_32k", _attend("llama8b", 64, 32768, 500)),
        # a decoding step of 24 long conversations that share nothing, every query head with a KV head of its own
        ("attend_24_long", _attend("lwm7b", 24, 0, 16001)),
        # one of eight tensor-parallel shards, a single KV head, odd lengths, more of the rows' own than is shared
        ("attend_shard_odd", _attend("llama70b", 33, 12345, 2001, dtype="bf16", tp=8, block=32)),
        # eight questions of up to 317 tokens about a 32K-token document arrive at once: the first pass over them
        ("attend_questions", _attend("yi34b", 8, 32768, 317, new=317, dtype="bf16")),
        # a wide head, prompts of up to 700 tokens in one piece, nothing before them
        ("attend_prompts_wide", _attend("wide", 5, 0, 701, new=701, dtype="bf16", block=32)),
        # the step's new keys and values of 64 conversations
        ("write_step", _case("write", "llama8b", requests=64, old_tokens=900, new=1)),
        # the keys and values of prompts of up to 1000 tokens
        ("write_prompts", _case("write", "yi34b", "bf16", requests=16, old_tokens=100, new=1000, block=64)),
        # a draft of a few hundred tokens looked at again
        ("read_one", _case("read", "llama70b", "bf16", tp=8, rows=1, tokens=333)),
        # the rows of a batch for a layer that wants them in 16 bits
        ("read_32", _case("read", "llama8b", rows=32, tokens=8001)),
        # a restored prompt of 200 tokens is put into 4 bits, and what it stands for is looked at
        ("convert_short", _case("convert", "llama70b", "bf16", tp=8, layers=0, pages=13, blocks=40, way="both")),
        # 4000 tokens of all 60 layers come back to 16 bits
        ("convert_250", _case("convert", "yi34b", "bf16", layers=0, pages=250, blocks=520, way="back")),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, low, high):
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    op = rng.choices(["attend", "write", "read", "convert"], [5, 2, 1, 2])[0]
    model, dtype = rng.choice(sorted(MODELS)), rng.choice(["f16", "bf16"])
    heads = MODELS[model][2]
    tp, block = rng.choice([t for t in (1, 1, 2, 4, 8) if heads % t == 0 and MODELS[model][1] % t == 0]), rng.choice([8, 16, 16, 20, 32, 64])
    of = {"dtype": dtype, "tp": tp, "block": block}
    most = max(_cost(c) for c in listed())
    while True:
        if op == "attend":
            new = rng.choices([1, rng.randint(2, 8), _log(rng, 9, 1000)], [6, 2, 3])[0]
            prefix, requests = 0 if rng.random() < 0.2 else _log(rng, 50, 32768), _log(rng, 1, 128)
            c = _attend(model, requests, prefix, _log(rng, 1, 16000 if prefix == 0 else 3000), new, **of)
            scores = sum(_new_tokens(c)) * c["q_heads"] * (c["prefix"] + c["own_tokens"])
            padded = c["requests"] * c["new"] * c["q_heads"] * c["own_tokens"]
            rows = c["requests"] * c["own_tokens"] * c["heads"] * c["head_dim"]
            fits = max(scores, padded) <= 5 << 29 and rows <= 13 << 27  # (what the plain form holds)
        elif op == "write":
            c = _case(op, model, requests=_log(rng, 1, 64), old_tokens=_log(rng, 1, 2000), new=rng.choice([1, _log(rng, 2, 1000)]), **of)
            fits = c["requests"] * (c["old_tokens"] + c["new"]) * c["heads"] * c["head_dim"] <= 1 << 28
        elif op == "read":
            c = _case(op, model, rows=_log(rng, 1, 64), tokens=_log(rng, 1, 16000), **of)
            fits = c["rows"] * c["tokens"] * c["heads"] * c["head_dim"] <= 1 << 29
        else:
            blocks = _log(rng, 12, 600)  # room for the pages twice, and for three that nobody asks for
            c = _case(op, model, layers=0, pages=_log(rng, 1, (blocks - 3) // 2), blocks=blocks, way=rng.choice(["both", "back"]), **of)
            fits = 2 * c["layers"] * blocks * block * c["heads"] * c["head_dim"] <= 5 << 28
        if fits and _cost(c) <= most:
            return c


# ------------------------------------------------------------------ sizes that follow from a case


def _spread(n, low, high):
    """n whole numbers from high down to about low."""
    return [high - (high - low) * i // n for i in range(n)]


def _new_tokens(c):
    return _spread(c["requests"], 1, c["new"])


def _own_tokens(c):
    """Tokens of each row beyond the prefix, the new ones among them."""
    return [max(new, o) for new, o in zip(_new_tokens(c), _spread(c["requests"], 1, c["own_tokens"]))]


def _read_tokens(c):
    return _spread(c["rows"], 1, c["tokens"])


def _pages(tokens, block):
    return -(-tokens // block)


def work(c):
    held = 2 * c["heads"] * (c["head_dim"] // 2 + 4)  # bytes of a token's keys and values in one layer, in 4 bits
    wide = 2 * c["heads"] * c["head_dim"] * 2  # and in 16
    if c["op"] == "attend":
        new, owned = _new_tokens(c), _own_tokens(c)
        seen = sum(n * (c["prefix"] + o) - n * (n - 1) // 2 for n, o in zip(new, owned))
        rows = sum(new) * c["q_heads"]
        return {"bytes": (c["prefix"] + sum(owned)) * held + rows * (2 * c["head_dim"] * 2 + 4),
                "flops": 4 * seen * c["q_heads"] * c["head_dim"]}
    if c["op"] == "write":  # tokens come, codes are kept, what they stand for goes out
        return {"bytes": sum(_new_tokens(c)) * (wide + held + wide), "flops": 0}
    if c["op"] == "read":
        return {"bytes": sum(_read_tokens(c)) * (held + wide), "flops": 0}
    tokens = c["pages"] * c["block"] * c["layers"]
    return {"bytes": tokens * (held + wide + (wide if c["way"] == "both" else 0)), "flops": 0}


# ------------------------------------------------------------------ codes, in elementary operations


def _hold(x):
    """Pages' tokens x [..][b][H][D], of a 16-bit type -> their words [..][H b (D / 8 + 1)], int32.
    mn is the least of a token's head, scale a fifteenth of the rest, rounded up to the type; a code is the nearest step."""
    *lead, b, H, D = x.shape
    f = x.float()
    mn = f.amin(dim=-1) + 0.0
    step = ((f.amax(dim=-1) - mn).double() / 15).float()
    scale = step.to(x.dtype)
    scale = torch.where(scale.float() < step, (scale.view(torch.int16) + 1).view(x.dtype), scale)  # (the next one: they are not negative)
    inv = torch.where(scale == 0, 0.0, 1 / scale.double()).float()
    code = ((f - mn[..., None]) * inv[..., None]).round().clamp(max=15).to(torch.int32)
    del f
    code = code.view(*lead, b // 4, 4, H, D // 8, 8)
    word = torch.zeros(code.shape[:-1], dtype=torch.int32, device=x.device)
    for i, shift in enumerate(_SHIFTS):
        word |= code[..., i] << shift
    n = len(lead)
    word = word.permute(*range(n), n + 2, n, n + 3, n + 1).reshape(*lead, -1)
    pair = torch.stack([scale, mn.to(x.dtype)], dim=-1).view(torch.int32).squeeze(-1).transpose(-1, -2).reshape(*lead, -1)
    return torch.cat([word, pair], dim=-1)


_SHIFTS = [4 * (i // 2) + 16 * (i % 2) for i in range(8)]


def _values(words, b, H, D, dtype):
    """Words of pages [..][H b (D / 8 + 1)] -> what their codes stand for, [..][b][H][D] in 32 bits."""
    *lead, _ = words.shape
    n, cut = len(lead), H * b * D // 8
    code = words[..., :cut].reshape(*lead, H, b // 4, D // 8, 4, 1) >> torch.tensor(_SHIFTS, dtype=torch.int32, device=words.device) & 15
    code = code.permute(*range(n), n + 1, n + 3, n, n + 2, n + 4).reshape(*lead, b, H, D)
    pair = words[..., cut:].contiguous().view(TORCH_DTYPE[dtype]).view(*lead, H, b, 2).transpose(-3, -2).float()
    return code.float() * pair[..., :1] + pair[..., 1:]  # (the product of a code and a scale is exact)


def _narrow(x, dtype):
    """Rounded once to the type; what a rounded-up scale has pushed beyond its largest number is that number."""
    most = torch.finfo(TORCH_DTYPE[dtype]).max
    return x.clamp(-most, most).to(TORCH_DTYPE[dtype])


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


def _held_pages(c, blocks, g):
    """A layer's pages of normal values, in 4 bits: int32 [2][blocks][words]."""
    return torch.stack([_hold(_normal((blocks, c["block"], c["heads"], c["head_dim"]), g, c["dtype"])) for _ in range(2)])


def _paged(rows, blocks, h):
    """Tables of rows of so many pages, on pages in random order."""
    order = torch.randperm(blocks, generator=h).tolist()
    length = max(1, max(rows, default=1))
    tables, at = [], 0
    for n in rows:
        tables.append(order[at:at + n] + [-1] * (length - n))
        at += n
    return tables


def _shuffled(values, h):
    return [values[i] for i in torch.randperm(len(values), generator=h).tolist()]


def _batch(s, new):
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s["starts"], s["n_new"], s["most_new"] = _i32(starts), starts[-1], max(new)


def prepare(case, seed):
    c, (g, h) = case, _generators(seed)
    s = {"case": c, "block": c["block"]}
    {"attend": _prepare_attend, "write": _prepare_write, "read": _prepare_read, "convert": _prepare_convert}[c["op"]](c, s, g, h)
    if own:
        _handles(s)
    return s


def _prepare_attend(c, s, g, h):
    b, P, H, D = c["block"], c["prefix"], c["heads"], c["head_dim"]
    both = _shuffled(list(zip(_new_tokens(c), _own_tokens(c))), h)  # the rows' order is the seed's
    new, lens = [n for n, _ in both], [P + o for _, o in both]
    shared = P // b
    rows = [_pages(P, b)] + [_pages(n, b) - shared for n in lens]
    blocks = sum(rows) + sum(rows) // 16 + 1
    tables = _paged(rows, blocks, h)
    length = max(_pages(n, b) for n in lens + [P])
    tables = [(t if i == 0 else tables[0][:shared] + t[:rows[i]]) for i, t in enumerate(tables)]
    s["tables"], s["lens"] = _i32([(t + [-1] * length)[:length] for t in tables]), _i32([P] + lens)
    s["held"] = _held_pages(c, blocks, g)[None]
    if P % b:  # what a fork copies: the prompt's last page, filled in part, is each row's own
        slots = torch.arange(P % b, device=DEV)
        codes, pairs = _words_at(c, (_i32([t[shared] for t in tables]).long()[:, None] * b + slots).flatten())
        for flat in (x.view(-1) for x in s["held"][0]):
            for at in (codes, pairs):
                at = at.unflatten(0, (len(tables), -1))
                flat[at[1:]] = flat[at[:1]].expand_as(at[1:])
    _batch(s, new)
    s["rows"] = _i32(list(range(1, len(new) + 1)))
    s["q"] = _normal((s["n_new"], c["q_heads"], D), g, c["dtype"])
    s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty((s["n_new"], c["q_heads"]), device=DEV)
    s["most_tokens"], s["scale"] = max(lens), 1.0 / math.sqrt(D)


def _prepare_write(c, s, g, h):
    b, H, D = c["block"], c["heads"], c["head_dim"]
    both = _shuffled(list(zip(_new_tokens(c), reversed(_spread(c["requests"], 0, c["old_tokens"])))), h)
    new, lens = [n for n, _ in both], [n + o for n, o in both]
    rows = [_pages(n, b) for n in lens]
    blocks = sum(rows) + sum(rows) // 4 + 1
    s["tables"], s["lens"] = _i32(_paged(rows, blocks, h)), _i32(lens)
    s["held"] = _held_pages(c, blocks, g)[None]
    _batch(s, new)
    s["rows"] = _i32(list(range(len(new))))
    s["qkv"] = _normal((s["n_new"], c["q_heads"] + 2 * H, D), g, c["dtype"])  # what the layer's projection gives, in one piece
    s["k"], s["v"] = (torch.empty((s["n_new"], H, D), dtype=TORCH_DTYPE[c["dtype"]], device=DEV) for _ in range(2))


def _prepare_read(c, s, g, h):
    b, H, D = c["block"], c["heads"], c["head_dim"]
    lens = _shuffled(_read_tokens(c), h)
    rows = [_pages(n, b) for n in lens]
    blocks = sum(rows) + sum(rows) // 16 + 1
    s["tables"], s["lens"] = _i32(_paged(rows, blocks, h)), _i32(lens)
    s["held"] = _held_pages(c, blocks, g)[None]
    _batch(s, lens)
    s["rows"] = _i32(list(range(len(lens))))
    s["k"], s["v"] = (torch.empty((s["n_new"], H, D), dtype=TORCH_DTYPE[c["dtype"]], device=DEV) for _ in range(2))


def _prepare_convert(c, s, g, h):
    b, H, D, n = c["block"], c["heads"], c["head_dim"], c["pages"]
    wide = torch.stack([torch.stack([_normal((c["blocks"], b, H, D), g, c["dtype"]) for _ in range(2)]) for _ in range(c["layers"])])
    order = torch.randperm(c["blocks"], generator=h)[:2 * n].to(torch.int32)
    s["wide"], s["source"], s["place"] = wide, order[:n].to(DEV), order[n:].to(DEV)
    s["in_held"] = torch.randperm(n + 3, generator=h)[:n].to(torch.int32).to(DEV)
    s["held"] = torch.stack([_hold(x[:, :n + 3].contiguous()) for x in wide])
    s["tables"], s["lens"] = _i32([[0]]), _i32([0])


# ------------------------------------------------------------------ one pass


def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["op"]](s)


# The library's calls.


def _handles(s):
    """What a program that serves from a pool keeps: its descriptor, and the workspace of its calls."""
    import paper_2602_09725_amd as kvc

    c, ptr = s["case"], lambda x: x.data_ptr()  # noqa: E731
    dtype = kvc.KVC_F16 if c["dtype"] == "f16" else kvc.KVC_BF16
    n_rows, length = s["tables"].shape
    s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)

    def pool(cache, form):
        layers = torch.tensor([x.data_ptr() for x in cache], dtype=torch.int64, device=DEV)
        s.setdefault("layers", []).append(layers)
        return kvc.Pool(c["layers"], c["heads"], c["head_dim"], dtype | form, cache.shape[2], c["block"], n_rows, length, ptr(layers),
                        ptr(s["tables"]), ptr(s["lens"]), None, ptr(s["err"]))

    s["pool"], s["kvc"] = pool(s["held"], kvc.KVC_HELD_Q4), kvc
    if c["op"] == "convert":
        s["wide_pool"] = pool(s["wide"], 0)
        return
    one_each = s["most_new"] == 1
    s["batch"] = kvc.Batch(s["rows"].numel(), s["n_new"], s["most_new"], ptr(s["rows"]), None if one_each else ptr(s["starts"]))
    if c["op"] == "attend":
        strides = (c["q_heads"] * c["head_dim"], c["head_dim"])
        s["attention"] = kvc.Attention(c["q_heads"], s["scale"], s["most_tokens"], c["prefix"], 0, strides, strides)
        s["workspace"] = torch.empty(kvc.attention_workspace(s["pool"], s["batch"], s["attention"]), dtype=torch.uint8, device=DEV)


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _own_attend(s):
    w = s["workspace"]
    s["kvc"].kvc_attend_paged(s["pool"], s["batch"], s["attention"], 0, s["q"].data_ptr(), s["out"].data_ptr(), s["lse"].data_ptr(),
                              w.data_ptr(), w.numel(), _stream())
    return {"out": s["out"], "lse": s["lse"]}


def _own_write(s):
    c, x = s["case"], s["qkv"]
    k, v = x[:, c["q_heads"]:], x[:, c["q_heads"] + c["heads"]:]
    s["kvc"].kvc_append_paged(s["pool"], s["batch"], 0, k.data_ptr(), v.data_ptr(), x.stride(0), _stream())
    return _own_read(s)


def _own_read(s):
    s["kvc"].kvc_read_paged(s["pool"], s["batch"], None, 0, s["k"].data_ptr(), s["v"].data_ptr(), s["k"].stride(0), _stream())
    return {"k": s["k"], "v": s["v"]}


def _own_convert(s):
    kvc, n = s["kvc"], s["source"].numel()
    if s["case"]["way"] == "both":
        kvc.kvc_pages_convert(s["wide_pool"], s["pool"], s["source"].data_ptr(), s["in_held"].data_ptr(), n, _stream())
    kvc.kvc_pages_convert(s["pool"], s["wide_pool"], s["in_held"].data_ptr(), s["place"].data_ptr(), n, _stream())
    return {"cache": s["wide"]}


# The plain forms.


def _tokens(s):
    """Of every new token: its request, its place among the request's, and its position."""
    starts = s["starts"].long()
    t = torch.arange(s["n_new"], device=DEV)
    r = torch.searchsorted(starts, t, right=True) - 1
    i = t - starts[r]
    length = s["lens"].long()[s["rows"].long()[r]]
    return r, i, length - (starts[r + 1] - starts[r]) + i


def _slots(s, r, at):
    return s["tables"][s["rows"].long()[r], at // s["block"]].long() * s["block"] + at % s["block"]


def _plain_attend(s):
    c, b = s["case"], s["block"]
    P, H, D, n = c["prefix"], c["heads"], c["head_dim"], s["n_new"]
    G, R, m, S = c["q_heads"] // H, s["rows"].numel(), s["most_new"], s["most_tokens"] - P
    r, i, at = _tokens(s)
    kv = _values(s["held"][0], b, H, D, c["dtype"]).flatten(1, 2)  # [2][slots][H][D]
    q = (s["q"].float() * s["scale"]).view(n, H, G, D)

    def slots(table, positions):
        return table.gather(-1, positions // b).clamp(min=0).long() * b + positions % b

    # the prefix, once for all: [H][n G][P]
    positions = torch.arange(P, device=DEV)
    shared = kv[:, slots(s["tables"][0], positions)].permute(0, 2, 1, 3).contiguous()  # [2][H][P][D]
    near = torch.matmul(q.permute(1, 0, 2, 3).reshape(H, n * G, D), shared[0].transpose(1, 2).contiguous()).view(H, n, G, P)
    near = near.masked_fill((positions > at[:, None])[None, :, None, :], -math.inf)
    # each row's own tokens, all rows as long as the longest: [R][H][m G][S]
    ours = P + torch.arange(S, device=DEV).expand(R, S)
    last = s["tables"].shape[1] * b - 1
    where = slots(s["tables"][s["rows"].long()], ours.clamp(max=last))
    k = kv[0, where].permute(0, 2, 3, 1).contiguous()  # [R][H][D][S]
    padded = torch.zeros((R, m, H, G, D), device=DEV)
    padded[r, i] = q
    far = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(R, H, m * G, D), k)
    del k
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
    v = kv[1, where].permute(0, 2, 1, 3).contiguous()  # [R][H][S][D]
    of_own = torch.matmul(padded.permute(0, 2, 1, 3, 4).reshape(R, H, m * G, S), v)
    of_own = of_own.view(R, H, m, G, D).permute(0, 2, 1, 3, 4)[r, i].permute(1, 0, 2, 3)
    out = (of_prefix + of_own) / torch.where(total == 0, torch.ones_like(total), total)
    lse = (most + torch.log(total)).squeeze(-1)
    return {"out": out.permute(1, 0, 2, 3).reshape(n, H * G, D).to(TORCH_DTYPE[c["dtype"]]), "lse": lse.permute(1, 0, 2).reshape(n, H * G).contiguous()}


def _words_at(c, slot):
    """Of slots [n]: where their words lie in a layer's pages of one kind, codes [n][H][D / 8] and pairs [n][H]."""
    b, H, W = c["block"], c["heads"], c["head_dim"] // 8
    page, at = slot // b * (H * b * (W + 1)), slot % b
    head = torch.arange(H, device=DEV)
    codes = (page + (at // 4) * (W * 4) + at % 4)[:, None, None] + (head * (b * W))[:, None] + torch.arange(W, device=DEV) * 4
    return codes, (page + H * b * W + at)[:, None] + head * b


def _plain_write(s):
    c = s["case"]
    H, D = c["heads"], c["head_dim"]
    r, _, at = _tokens(s)
    codes, pairs = _words_at(c, _slots(s, r, at))
    x = s["qkv"][:, c["q_heads"]:].view(-1, 2, H, D).permute(1, 0, 2, 3).contiguous()
    # a page of four equal tokens holds each of them at its first place
    words = _hold(x[:, :, None].expand(2, s["n_new"], 4, H, D).contiguous())
    W = D // 8
    for kind in range(2):
        flat = s["held"][0, kind].view(-1)
        flat[codes] = words[kind, :, :H * 4 * W].view(-1, H, W, 4)[..., 0]
        flat[pairs] = words[kind, :, H * 4 * W:].view(-1, H, 4)[..., 0]
    return _plain_read(s)


def _plain_read(s):
    c = s["case"]
    r, _, at = _tokens(s)
    codes, pairs = _words_at(c, _slots(s, r, at))
    n, H, W = codes.shape
    got = []
    for kind in range(2):
        flat = s["held"][0, kind].view(-1)
        word = flat[codes][:, :, :, None].expand(n, H, W, 4).reshape(n, -1)
        pair = flat[pairs][:, :, None].expand(n, H, 4).reshape(n, -1)
        got.append(_narrow(_values(torch.cat([word, pair], dim=-1), 4, H, 8 * W, c["dtype"])[:, 0], c["dtype"]))
    return {"k": got[0], "v": got[1]}


def _plain_convert(s):
    c = s["case"]
    b, H, D = c["block"], c["heads"], c["head_dim"]
    source, held, place = s["source"].long(), s["in_held"].long(), s["place"].long()
    if c["way"] == "both":
        s["held"][:, :, held] = _hold(s["wide"][:, :, source])
    s["wide"][:, :, place] = _narrow(_values(s["held"][:, :, held], b, H, D, c["dtype"]), c["dtype"])
    return {"cache": s["wide"]}


_PLAIN = {"attend": _plain_attend, "write": _plain_write, "read": _plain_read, "convert": _plain_convert}
_OWN = {"attend": _own_attend, "write": _own_write, "read": _own_read, "convert": _own_convert}


# ------------------------------------------------------------------ from the definition, in 64 bits


def _stands_for(c, kind_words, pages_of_tokens, slots_of_tokens):
    """What tokens on these pages and slots stand for, element by element: [tokens][H][D] in 64 bits."""
    b, H, D = c["block"], c["heads"], c["head_dim"]
    W = D // 8
    d = torch.arange(D, device=DEV)
    h = torch.arange(H, device=DEV)[:, None]
    slot = slots_of_tokens[:, None, None]
    words = kind_words[pages_of_tokens]
    word = words.gather(1, (((h * (b // 4) + slot // 4) * W + d // 8) * 4 + slot % 4).flatten(1)).view(-1, H, D)
    code = (word.long() & 0xffffffff) >> (4 * (d % 8 // 2) + 16 * (d % 2)) & 15
    pair = words.gather(1, (H * b * W + h * b + slot).flatten(1)).contiguous().view(TORCH_DTYPE[c["dtype"]]).view(-1, H, 2).double()
    return code.double() * pair[..., :1] + pair[..., 1:]


def _rounded_there_and_back(x, dtype):
    """Tokens x [..][D] in 64 bits -> what their codes stand for.  The definition's steps are of 32 bits: each is taken in 64 and rounded."""
    def single(y):
        return y.float().double()

    mn, most = x.amin(dim=-1, keepdim=True), x.amax(dim=-1, keepdim=True)
    step = single(single(most - mn) / 15)
    scale = step.to(TORCH_DTYPE[dtype]).double()
    if dtype == "f16":  # a step of the type at this size: 2^-10 of its power of two, 2^-24 at least
        unit = torch.exp2(torch.floor(torch.log2(scale.clamp(min=2.0 ** -14))) - 10)
    else:
        unit = torch.exp2(torch.floor(torch.log2(scale.clamp(min=2.0 ** -126))) - 7)
    scale = torch.where(scale < step, scale + unit, scale)
    inv = torch.where(scale == 0, torch.zeros_like(scale), single(1 / scale))
    code = torch.round(single(single(x - mn) * inv)).clamp(max=15)
    return code * scale + mn


def exact(case, seed):
    """Attention request by request over the whole of its row, prefix and all, head by head, and codes element by element."""
    c, s = case, prepare(case, seed)
    b, H = c["block"], c["heads"]
    if c["op"] == "convert":
        wide, source, held, place = s["wide"].double(), s["source"].tolist(), s["in_held"].tolist(), s["place"].tolist()
        slots = torch.arange(b, device=DEV)
        for layer in range(c["layers"]):
            for kind in range(2):
                if c["way"] == "both":
                    wide[layer, kind, place] = _rounded_there_and_back(wide[layer, kind, source], c["dtype"])
                else:
                    pages = torch.tensor(held, device=DEV).repeat_interleave(b)
                    values = _stands_for(c, s["held"][layer, kind], pages, slots.repeat(len(held)))
                    wide[layer, kind, place] = values.view(len(held), b, H, -1)
        return {"cache": wide}
    starts, lens, tables = s["starts"].tolist(), s["lens"].tolist(), s["tables"].long()
    if c["op"] == "write":
        x = s["qkv"][:, c["q_heads"]:].double().view(s["n_new"], 2, H, -1)
        return {name: _rounded_there_and_back(x[:, kind], c["dtype"]) for kind, name in enumerate("kv")}

    def row_values(row, first, end):
        at = torch.arange(first, end, device=DEV)
        return [_stands_for(c, s["held"][0, kind], tables[row, at // b], at % b) for kind in range(2)]

    if c["op"] == "read":
        rows = [row_values(row, 0, lens[row]) for row in s["rows"].tolist()]
        return {name: torch.cat([row[kind] for row in rows]) for kind, name in enumerate("kv")}
    G = c["q_heads"] // H
    out = torch.zeros((s["n_new"], c["q_heads"], c["head_dim"]), dtype=torch.float64, device=DEV)
    lse = torch.full((s["n_new"], c["q_heads"]), -math.inf, dtype=torch.float64, device=DEV)
    for request, row in enumerate(s["rows"].tolist()):
        first, end, n = starts[request], starts[request + 1], lens[row]
        k, v = row_values(row, 0, n)
        seen = torch.arange(n, device=DEV)[None] <= n - (end - first) + torch.arange(end - first, device=DEV)[:, None]
        for head in range(H):
            heads = slice(head * G, head * G + G)
            score = (s["q"][first:end, heads].double().reshape(-1, c["head_dim"]) @ k[:, head].T.contiguous()).view(end - first, G, n) * s["scale"]
            score = score.masked_fill(~seen[:, None], -math.inf)
            norm = torch.logsumexp(score, dim=-1)
            share = torch.where(norm[..., None] == -math.inf, torch.zeros_like(score), torch.exp(score - norm[..., None]))
            out[first:end, heads] = (share.view(-1, n) @ v[:, head].contiguous()).view(end - first, G, -1)
            lse[first:end, heads] = norm
    return {"out": out, "lse": lse}
