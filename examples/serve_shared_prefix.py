"""Serving from a restored cache: a prompt's KV cache comes out of packed frames into pages, many requests take it up, and each
goes on with tokens of its own.

  restore   kvc_pages_grow, kvc_restore_paged: the prompt's pages are row 0's (of a pool in 4 bits: restored beside it, a chunk at a time, and moved by kvc_pages_convert)
  admit     kvc_pages_fork: the requests' rows share whole pages of the prompt, and have a copy of its last one
  step      kvc_pages_grow, then in every layer kvc_append_paged and kvc_attend_paged
  finish    kvc_pages_free: pages that no row holds any more are free again
  compact   kvc_pages_compact: what is in use moves to the lowest pages, for an engine that gives the others back

The model is a stand-in (random projections around the attention, no feed-forward part): what is shown is the cache's life.

  python examples/serve_shared_prefix.py [--layers 32] [--prompt 32768] [--requests 64] [--steps 16] [--dtype f16] [--held]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import kv_synth  # noqa: E402
import paper_2602_09725_amd as kvc  # noqa: E402

DTYPES = {"f16": (torch.float16, kvc.KVC_F16), "bf16": (torch.bfloat16, kvc.KVC_BF16)}


def stream():
    return torch.cuda.current_stream().cuda_stream


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Model:
    """Weights of the stand-in: per layer a projection to queries, keys and values, and one back."""

    def __init__(self, layers, q_heads, heads, head_dim, dtype, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.layers, self.q_heads, self.heads, self.head_dim, self.dtype = layers, q_heads, heads, head_dim, dtype
        self.width = q_heads * head_dim

        def weights(rows, columns):
            return (torch.randn((rows, columns), generator=g, device="cuda") / math.sqrt(rows)).to(DTYPES[dtype][0])

        self.qkv = [weights(self.width, (q_heads + 2 * heads) * head_dim) for _ in range(layers)]
        self.back = [weights(self.width, self.width) for _ in range(layers)]


class Server:
    """A pool of pages with rows 1 .. max_rows for requests; row 0 is the prompt's.  held: its pages hold tokens in 4 bits."""

    def __init__(self, model, max_rows, max_tokens, num_blocks, block_size, held=False):
        m, (dtype, code) = model, DTYPES[model.dtype]
        self.model, self.block, self.max_tokens = model, block_size, max_tokens
        self.held = held
        shape = (m.heads * (m.head_dim // 8 + 1) * block_size,) if held else (block_size, m.heads, m.head_dim)
        self.cache = [torch.zeros((2, num_blocks, *shape), dtype=torch.int32 if held else dtype, device="cuda") for _ in range(m.layers)]
        self.pointers = torch.tensor([c.data_ptr() for c in self.cache], dtype=torch.int64, device="cuda")
        self.table_len = -(-max_tokens // block_size)
        self.tables = torch.full((max_rows + 1, self.table_len), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(max_rows + 1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(num_blocks, dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pool = kvc.Pool(m.layers, m.heads, m.head_dim, code | (kvc.KVC_HELD_Q4 if held else 0), num_blocks, block_size, max_rows + 1, self.table_len, self.pointers.data_ptr(),
                             self.tables.data_ptr(), self.lens.data_ptr(), self.refs.data_ptr(), self.err.data_ptr())
        self.books = torch.empty(kvc.pages_workspace(self.pool), dtype=torch.uint8, device="cuda")
        self.where = torch.empty(num_blocks, dtype=torch.int32, device="cuda")
        self.space = torch.empty(0, dtype=torch.uint8, device="cuda")
        self.prompt, self.length = 0, {}  # the host's own knowledge of rows: they need not be read back

    def _room(self):
        return self.books.data_ptr(), self.books.numel(), stream()

    def restore(self, layout, frames, meta, n_tokens):
        """The prompt's cache, from packed frames to pages that row 0 takes."""
        row, count = i32([0]), i32([n_tokens])
        kvc.kvc_pages_grow(self.pool, row.data_ptr(), count.data_ptr(), 1, *self._room())
        if self.held:
            self._restore_held(layout, frames, meta, n_tokens)
        else:
            kvc.kvc_restore_paged(layout, frames.data_ptr(), meta.data_ptr(), 0, n_tokens, self.pointers.data_ptr(), self.pool.num_blocks, self.block,
                                  self.tables.data_ptr(), self.table_len, self.err.data_ptr(), stream())
        self.prompt = n_tokens

    def _restore_held(self, layout, frames, meta, n_tokens):
        """Restores chunk by chunk to a few pages of 16 bits, taken in turn, and moves those that are complete to row 0's."""
        m, (dtype, code), pages = self.model, DTYPES[self.model.dtype], -(-n_tokens // self.block)
        chunk, (frame_bytes, meta_bytes, _) = layout.chunk_tokens, kvc.chunk_sizes(layout)
        ring = min(pages, chunk // self.block + 2)
        wide = torch.zeros((m.layers, 2, ring, self.block, m.heads, m.head_dim), dtype=dtype, device="cuda")
        pointers = torch.tensor([c.data_ptr() for c in wide], dtype=torch.int64, device="cuda")
        turn = torch.arange(pages, dtype=torch.int32, device="cuda") % ring
        pool = kvc.Pool(m.layers, m.heads, m.head_dim, code, ring, self.block, 1, 1, pointers.data_ptr(), self.tables.data_ptr(), self.lens.data_ptr(), None,
                        self.err.data_ptr())
        moved = 0
        for i, begin in enumerate(range(0, n_tokens, chunk)):
            end = min(n_tokens, begin + chunk)
            kvc.kvc_restore_paged(layout, frames.data_ptr() + i * frame_bytes, meta.data_ptr() + i * meta_bytes, begin, end - begin, pointers.data_ptr(), ring, self.block,
                                  turn.data_ptr(), pages, self.err.data_ptr(), stream())
            whole = pages if end == n_tokens else end // self.block  # (a page that the chunk ends in waits for the next one)
            kvc.kvc_pages_convert(pool, self.pool, turn[moved:].data_ptr(), self.tables[0, moved:].data_ptr(), whole - moved, stream())
            moved = whole

    def read_back(self, row, layer):
        """Keys and values of a row, as what its pages hold stands for."""
        m, n = self.model, self.length.get(row, self.prompt)
        rows, starts = i32([row]), i32([0, n])
        k, v = (torch.empty((n, m.heads, m.head_dim), dtype=DTYPES[m.dtype][0], device="cuda") for _ in range(2))
        batch = kvc.Batch(1, n, n, rows.data_ptr(), starts.data_ptr())
        kvc.kvc_read_paged(self.pool, batch, None, layer, k.data_ptr(), v.data_ptr(), m.heads * m.head_dim, stream())
        return k, v

    def admit(self, rows):
        parents, children = i32([0] * len(rows)), i32(rows)
        kvc.kvc_pages_fork(self.pool, parents.data_ptr(), children.data_ptr(), len(rows), *self._room())
        self.length.update({row: self.prompt for row in rows})

    def finish(self, rows):
        gone = i32(rows)
        kvc.kvc_pages_free(self.pool, gone.data_ptr(), len(rows), stream())
        for row in rows:
            del self.length[row]

    def compact(self):
        kvc.kvc_pages_compact(self.pool, self.where.data_ptr(), self.tables.data_ptr(), self.refs.data_ptr(), *self._room())

    def step(self, x, rows, new):
        """x: [tokens][width], new[i] tokens of row rows[i] after one another.  -> the same of the last layer; each layer's attention is kept in
        `seen` as (queries, keys, values, result, logarithms of sums)."""
        m, n = self.model, sum(new)
        starts = [0]
        for count in new:
            starts.append(starts[-1] + count)
        d_rows, d_new, d_starts = i32(rows), i32(new), i32(starts)
        kvc.kvc_pages_grow(self.pool, d_rows.data_ptr(), d_new.data_ptr(), len(rows), *self._room())
        for row, count in zip(rows, new):
            self.length[row] += count
        most = max(self.length[row] for row in rows)
        batch = kvc.Batch(len(rows), n, max(new), d_rows.data_ptr(), None if max(new) == 1 and min(new) == 1 else d_starts.data_ptr())
        wide = (m.q_heads + 2 * m.heads) * m.head_dim
        attention = kvc.Attention(m.q_heads, m.head_dim ** -0.5, most, self.prompt, 0, (wide, m.head_dim), (m.width, m.head_dim))
        need = kvc.attention_workspace(self.pool, batch, attention)
        if need > self.space.numel():
            self.space = torch.empty(need, dtype=torch.uint8, device="cuda")
        self.seen = []
        for layer in range(m.layers):
            qkv = (x @ m.qkv[layer]).view(n, m.q_heads + 2 * m.heads, m.head_dim)
            q, k, v = qkv[:, :m.q_heads], qkv[:, m.q_heads:m.q_heads + m.heads], qkv[:, m.q_heads + m.heads:]
            kvc.kvc_append_paged(self.pool, batch, layer, k.data_ptr(), v.data_ptr(), wide, stream())
            out, lse = torch.empty((n, m.q_heads, m.head_dim), dtype=x.dtype, device="cuda"), torch.empty((n, m.q_heads), device="cuda")
            kvc.kvc_attend_paged(self.pool, batch, attention, layer, q.data_ptr(), out.data_ptr(), lse.data_ptr(), self.space.data_ptr(),
                                 self.space.numel(), stream())
            self.seen.append((q, k, v, out, lse))
            x = x + out.view(n, m.width) @ m.back[layer]
            x = (x.float() / x.float().pow(2).mean(dim=-1, keepdim=True).sqrt()).to(x.dtype)
        return x


def packed_prompt(model, n_tokens, seed=kv_synth.BASE_SEED):
    """A synthetic prompt's cache as an engine would fetch it: layout, frames, scales and minima."""
    m, (dtype, code) = model, DTYPES[model.dtype]
    tokens, width = 2048, m.heads * m.head_dim
    tile_w = min(128, width)
    layout = kvc.Layout(m.layers, m.heads, m.head_dim, code, tokens, width // tile_w, tile_w, 8, 64)
    frame_bytes, meta_bytes, _ = kvc.chunk_sizes(layout)
    chunks = -(-n_tokens // tokens)
    kv = kv_synth.make_kv(m.layers, m.heads, m.head_dim, n_tokens, dtype, seed, device="cuda")
    frames = torch.empty(chunks * frame_bytes, dtype=torch.uint8, device="cuda")
    meta = torch.empty(chunks * meta_bytes, dtype=torch.uint8, device="cuda")
    kvc.kvc_pack(layout, kv.data_ptr(), (2 * n_tokens * width, n_tokens * width, width), n_tokens, frames.data_ptr(), frames.numel(), meta.data_ptr(),
                 meta.numel(), stream())
    return layout, frames, meta


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("layers", 32), ("q-heads", 32), ("heads", 8), ("head-dim", 128), ("prompt", 32768), ("requests", 64), ("question", 30),
                        ("steps", 16), ("block", 16)):
        a.add_argument("--" + name, type=int, default=value)
    a.add_argument("--dtype", choices=sorted(DTYPES), default="f16")
    a.add_argument("--held", action="store_true", help="hold the cache in 4 bits")
    o = a.parse_args()
    model = Model(o.layers, o.q_heads, o.heads, o.head_dim, o.dtype)
    own = o.question + 2 * o.steps
    blocks = -(-o.prompt // o.block) + o.requests * (-(-own // o.block) + 2)
    server = Server(model, o.requests, o.prompt + own, blocks, o.block, o.held)
    server.restore(*packed_prompt(model, o.prompt), o.prompt)
    rows = list(range(1, o.requests + 1))
    server.admit(rows)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)

    def tokens(n):
        return torch.randn((n, model.width), generator=g, device="cuda").to(DTYPES[o.dtype][0])

    def timed(what, call):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        result = call()
        end.record()
        end.synchronize()
        print(f"{what}: {begin.elapsed_time(end):.3f} ms")
        return result

    def decode(rows, x):
        for _ in range(o.steps):
            x = server.step(x, rows, [1] * len(rows))
        return x

    questions = [1 + (i * 7) % o.question for i in range(len(rows))]
    timed(f"questions of up to {o.question} tokens", lambda: server.step(tokens(sum(questions)), rows, questions))
    timed(f"{o.steps} steps of {len(rows)} requests", lambda: decode(rows, tokens(len(rows))))
    gone, rows = rows[::2], rows[1::2]
    server.finish(gone)
    timed("compact", server.compact)
    if rows:
        timed(f"{o.steps} steps of {len(rows)} requests", lambda: decode(rows, tokens(len(rows))))
    used = int((server.refs > 0).sum())
    assert int(server.err.item()) == 0, "the books are at fault"
    print(f"pages in use: {used} of {blocks}; faults: {int(server.err.item())}")


if __name__ == "__main__":
    main()
