"""Answer a question on a translated cache: handoff, question, decoding, budget.

A source model's cache of some contexts is translated into a paged cache of the
target model; the target model then reads a question of a few tokens in one
chunk and answers token by token.  Each layer stores its new tokens
(``kvx_attn_append``), attends to the cache (``kvx_attn_forward``) and adds up
the weight that every cached token receives (``kvx_attn_mass``).  When the
cache has outgrown its budget, the tokens of least weight are dropped from all
layers in place (``kvx_attn_evict``) and decoding goes on in the same blocks.

The answer's step is captured once into a graph and replayed: lengths and
positions are counted on the device.  The target model is a stand-in of its
attention layers with random weights (there are no checkpoints here); caches,
translators and head layouts are those of the workload.

    python examples/decode.py                        # Qwen2.5-7B -> 1.5B, 1024 tokens
    python examples/decode.py --config 3 --batch 2   # Gemma-2-2B, spans of 1-3 tokens
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_30963_amd import kvx, synth as S  # noqa: E402

BLOCK = 16  # tokens per block of the cache

#: Query heads and the scores' tanh cap of the workloads' target models.
HEADS = {2: (12, 0.0), 3: (8, 50.0), 4: (8, 50.0), 5: (28, 0.0)}


def _dev(a):
    if a.dtype == np.uint16:
        return torch.from_numpy(a.view(np.int16).copy()).view(torch.bfloat16).cuda()
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Layers:
    """The attention layers' weights of a target model, drawn."""

    def __init__(self, shape, n_heads, seed=0):
        g = torch.Generator("cuda").manual_seed(seed)
        self.shape, self.n_heads = shape, n_heads
        self.width = n_heads * shape.head_dim
        rows = (n_heads + 2 * shape.n_kv_heads) * shape.head_dim

        def draw(a, b):
            w = torch.randn(shape.n_layers, a, b, device="cuda", generator=g) * a ** -0.5
            return w.to(torch.bfloat16)

        self.qkv, self.o = draw(self.width, rows), draw(self.width, self.width)

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)


class Decoder:
    """A target model that decodes on one batch of paged caches.

    ``k``, ``v``, ``table``: the cache as kvx_translate wrote it; ``lengths``:
    its tokens per context; ``budget``: cached tokens per context to which an
    eviction goes back, ``slack``: by how many more the cache may grow before."""

    def __init__(self, shape, n_heads, softcap, k, v, table, lengths, budget, slack, seed=0):
        self.model = Layers(shape, n_heads, seed)
        self.att = kvx.Attention(shape, n_heads, kvx.KVX_BF16, softcap=softcap)
        self.cache = kvx.make_cache(k, v, table)
        self.k, self.v, self.table = k, v, table
        self.batch = len(lengths)
        self.budget, self.slack = budget, slack
        self.longest = max(lengths)  # the host's count, for when to evict
        self.tokens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.pos = self.tokens.clone()  # of the next token; evictions do not move it
        room = table.shape[1] * k.shape[3]
        self.mass = torch.zeros(shape.n_layers, self.batch, shape.n_kv_heads, room, device="cuda")
        self.kept = torch.empty(shape.n_layers, self.batch, shape.n_kv_heads, budget,
                                dtype=torch.int32, device="cuda")
        self.left = torch.empty_like(self.tokens)
        self.workspace = self.att.workspace()
        self.one = self._calls(1)
        self.x = torch.zeros(self.batch, self.model.width, dtype=torch.bfloat16, device="cuda")
        self.graph = None

    def _calls(self, new):
        """Buffers and one struct per layer for calls of ``new`` tokens per context."""
        m, d, rows = self.model.shape, self.model.shape.head_dim, self.batch * new
        heads = self.model.n_heads, m.n_kv_heads, m.n_kv_heads
        qkv = torch.empty(rows, sum(heads), d, dtype=torch.bfloat16, device="cuda")
        q, key, value = qkv.split(heads, dim=1)
        out = torch.empty(rows, m.n_layers, self.model.n_heads, d, dtype=torch.bfloat16,
                          device="cuda")
        lse = torch.empty(rows, self.model.n_heads, device="cuda")
        pos = torch.empty(1, rows, dtype=torch.int32, device="cuda")
        start = None if new == 1 else torch.arange(0, rows + 1, new, dtype=torch.int32,
                                                   device="cuda")
        ios = [kvx.make_attn_io(self.cache, self.tokens, q, layer=l, q_start=start, max_new=new,
                                new_q=q, new_k=key, new_v=value, pos=pos, out=out[:, l], lse=lse,
                                mass_in=self.mass[l], mass=self.mass[l])
               for l in range(m.n_layers)]
        return dict(new=new, qkv=qkv, out=out, pos=pos, ios=ios,
                    step=torch.arange(new, dtype=torch.int32, device="cuda"))

    def _run(self, c, x):
        """Hidden states after all layers; counts the new tokens first."""
        self.tokens += c["new"]
        c["pos"].copy_((self.pos[:, None] + c["step"]).view(1, -1))
        self.pos += c["new"]
        flat = c["qkv"].view(x.shape[0], -1)
        for l, io in enumerate(c["ios"]):
            torch.mm(self.model.norm(x), self.model.qkv[l], out=flat)
            self.att.append(io)
            self.att.forward(io, self.workspace)
            self.att.mass(io)
            x = x + torch.mm(c["out"][:, l].reshape(x.shape[0], -1), self.model.o[l])
        return self.model.norm(x)

    def evict(self):
        """Back to the budget: what got the least weight goes, the first four
        tokens and the last eighth of the budget stay."""
        io = kvx.make_evict_io(self.cache, self.tokens, self.mass, self.kept, self.budget,
                               sink=min(4, self.budget // 2), recent=self.budget // 8,
                               mass_out=self.mass, tokens_out=self.left)
        self.att.evict(io)
        self.tokens.copy_(self.left)
        self.longest = min(self.longest, self.budget)

    def _grow(self, new):
        room = self.table.shape[1] * self.k.shape[3]
        if self.longest + new > min(room, self.budget + self.slack):
            self.evict()
        self.longest += new
        if self.longest > room:
            raise ValueError(f"{self.longest} tokens do not fit {room} slots")

    def read(self, x):
        """Reads the question ``x`` [batch][tokens][width] in one chunk."""
        new = x.shape[1]
        self._grow(new)
        y = self._run(self._calls(new), x.reshape(self.batch * new, -1))
        self.x.copy_(y.view(self.batch, new, -1)[:, -1])

    def step(self, eager=False):
        """One token of every context; returns its hidden states (valid until
        the next step)."""
        self._grow(1)
        if eager:
            self.x.copy_(self._run(self.one, self.x))
            return self.x
        if self.graph is None:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph, stream=side):
                self.x.copy_(self._run(self.one, self.x))
        self.graph.replay()
        return self.x

    def close(self):
        torch.cuda.synchronize()
        self.graph = None
        self.att.close()


def handoff(config, src_tokens, batch, room):
    """Translates the workload's source caches; (target shape, k, v, table,
    lengths) of a paged cache with room for `room` more tokens per context."""
    spec = S.config(config, src_tokens=src_tokens, batch=batch)
    prob = S.make_problem(spec)
    tr = kvx.Translator(spec.src, spec.tgt, spec.mix, spec.layer_map, kvx.KVX_BF16,
                        _dev(prob.w_k), _dev(prob.w_v))
    lengths = [int(n) for n in prob.tgt_tokens]
    per = -(-(max(lengths) + room) // BLOCK)
    table = torch.randperm(batch * per, generator=torch.Generator().manual_seed(0))
    table = table.to(torch.int32).view(batch, per).cuda()
    shape = (spec.tgt.n_layers, batch * per, spec.tgt.n_kv_heads, BLOCK, spec.tgt.head_dim)
    k = torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    csr = {}
    if prob.row_ptr is not None:
        csr = dict(tgt_tokens=prob.tgt_tokens, row_ptr=_dev(prob.row_ptr),
                   col_idx=_dev(prob.col_idx), weight=_dev(prob.weight))
    tr(_dev(prob.src_k), _dev(prob.src_v), k, v, None, block_table=table, block_size=BLOCK, **csr)
    torch.cuda.synchronize()
    tr.close()
    return spec.tgt, k, v, table, lengths


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--config", type=int, default=2, choices=sorted(HEADS))
    p.add_argument("--tokens", type=int, default=1024, help="source tokens of a context")
    p.add_argument("--batch", type=int, default=1, help="contexts")
    p.add_argument("--question", type=int, default=48, help="tokens of the question")
    p.add_argument("--answer", type=int, default=256, help="tokens of the answer")
    p.add_argument("--budget", type=int, default=768, help="cached tokens after an eviction")
    p.add_argument("--slack", type=int, default=512, help="tokens over the budget before one")
    a = p.parse_args(argv)
    shape, k, v, table, lengths = handoff(a.config, a.tokens, a.batch, a.question + a.answer)
    heads, cap = HEADS[a.config]
    dec = Decoder(shape, heads, cap, k, v, table, lengths, a.budget, a.slack)
    g = torch.Generator("cuda").manual_seed(1)
    dec.read(torch.randn(a.batch, a.question, dec.model.width, device="cuda",
                         generator=g).to(torch.bfloat16))
    dec.step()
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(a.answer - 1):
        x = dec.step()
    torch.cuda.synchronize()
    spent = time.perf_counter() - began
    if not torch.isfinite(x).all():
        raise RuntimeError("non-finite hidden states")
    print(f"{lengths} translated tokens, {a.question} of question, {a.answer} of answer: "
          f"{dec.tokens.tolist()} cached, position {dec.pos.tolist()}, "
          f"{spent / max(1, a.answer - 1) * 1e3:.3f} ms per token and batch")
    dec.close()


if __name__ == "__main__":
    main()
