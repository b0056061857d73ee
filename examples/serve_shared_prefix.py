"""Serving from a restored cache: a prompt's KV cache comes out of packed frames into pages, many requests take it up, and each
goes on with tokens of its own.

  restore   kvc_pages_grow, kvc_restore_paged: the prompt's pages are row 0's
  admit     kvc_pages_fork: the requests' rows share whole pages of the prompt, and have a copy of its last one
  step      kvc_pages_grow, then in every layer kvc_append_paged and kvc_attend_paged
  finish    kvc_pages_free: pages that no row holds any more are free again
  compact   kvc_pages_compact: what is in use moves to the lowest pages, for an engine that gives the others back

The model is a stand-in (random projections around the attention, no feed-forward part): what is shown is the cache's life.

  python examples/serve_shared_prefix.py [--layers 32] [--prompt 32768] [--requests 64] [--steps 16] [--dtype f16]
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
    """A pool of pages with rows 1 .. max_rows for requests; row 0 is the prompt's."""

    def __init__(self, model, max_rows, max_tokens, num_blocks, block_size):
        m, (dtype, code) = model, DTYPES[model.dtype]
        self.model, self.block, self.max_tokens = model, block_size, max_tokens
        self.cache = [torch.zeros((2, num_blocks, block_size, m.heads, m.head_dim), dtype=dtype, device="cuda") for _ in range(m.layers)]
        self.pointers = torch.tensor([c.data_ptr() for c in self.cache], dtype=torch.int64, device="cuda")
        self.table_len = -(-max_tokens // block_size)
        self.tables = torch.full((max_rows + 1, self.table_len), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(max_rows + 1, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(num_blocks, dtype=torch.int32, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.pool = kvc.Pool(m.layers, m.heads, m.head_dim, code, num_blocks, block_size, max_rows + 1, self.table_len, self.pointers.data_ptr(),
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
        kvc.kvc_restore_paged(layout, frames.data_ptr(), meta.data_ptr(), 0, n_tokens, self.pointers.data_ptr(), self.pool.num_blocks, self.block,
                              self.tables.data_ptr(), self.table_len, self.err.data_ptr(), stream())
        self.prompt = n_tokens

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
    o = a.parse_args()
    model = Model(o.layers, o.q_heads, o.heads, o.head_dim, o.dtype)
    own = o.question + 2 * o.steps
    blocks = -(-o.prompt // o.block) + o.requests * (-(-own // o.block) + 2)
    server = Server(model, o.requests, o.prompt + own, blocks, o.block)
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
