"""Draft on a compressed translated cache: handoff, 8 bits, trees, accepted paths.

A source model's cache is translated into a paged cache of the target model and
packed into 8 bits (``kvx_attn_pack``); the target then decodes by trees of
drafted tokens.  A step finds what every node of a tree sees (``kvx_attn_tree``);
each layer stores the nodes' keys and values as codes (``kvx_attn_append_coded``)
and attends to the cache through a window with sinks
(``kvx_attn_forward_view``); the path whose tokens the target itself would have
chosen moves behind the context's other tokens in all layers
(``kvx_attn_accept``), and the rest of the tree is forgotten.

The step is captured once into a graph and replayed: lengths, trees, positions
and paths live on the device.  The target model is a stand-in of its attention
layers with random weights and a small vocabulary; the drafts are guesses of
which some are the target's own choices.

    python examples/draft.py                        # Qwen2.5-7B -> 1.5B, 1024 tokens
    python examples/draft.py --config 3 --batch 2   # Gemma-2-2B, spans of 1-3 tokens
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from examples.decode import HEADS, Layers, handoff  # noqa: E402
from paper_2608_30963_amd import kvx  # noqa: E402

VOCABULARY = 32


def tree_of(nodes, width):
    """Parents of a tree of `nodes` whose nodes have up to `width` children."""
    return [-1] + [(i - 1) // width for i in range(1, nodes)]


def deepest_of(up):
    """Nodes of the path to the last node, the longest in trees of tree_of."""
    node, nodes = len(up) - 1, 1
    while up[node] >= 0:
        node, nodes = up[node], nodes + 1
    return nodes


class Drafter:
    """A target model that decodes by drafted trees on a cache of 8 bits."""

    def __init__(self, shape, n_heads, softcap, k, v, table, lengths, nodes=16, width=2, window=0,
                 sink=0, code=torch.int8, seed=0):
        self.model = Layers(shape, n_heads, seed)
        self.att = kvx.Attention(shape, n_heads, kvx.KVX_BF16, softcap=softcap)
        self.batch, self.nodes, self.room = len(lengths), nodes, table.shape[1] * k.shape[3]
        self.tokens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.most = max(lengths)  # tokens of the longest context, at most: known without the device
        self.k, self.v = torch.zeros_like(k, dtype=code), torch.zeros_like(v, dtype=code)
        self.scale = torch.zeros(k.shape[:-1] + (2,), dtype=torch.bfloat16, device="cuda")
        self.cache = kvx.make_cache8(self.k, self.v, self.scale, table)
        self.att.pack(kvx.make_pack_io(kvx.make_cache(k, v, table), self.cache, self.tokens))
        rows = self.batch * nodes
        heads = n_heads, shape.n_kv_heads, shape.n_kv_heads
        g = torch.Generator("cuda").manual_seed(seed + 1)
        self.embedding = torch.randn(VOCABULARY, self.model.width, device="cuda",
                                     generator=g).to(torch.bfloat16)

        def ints(*size):
            return torch.zeros(size, dtype=torch.int32, device="cuda")

        torch.mm(self.embedding, self.model.qkv[0])  # sets the library up before a capture
        up = tree_of(nodes, width)
        self.parent = torch.tensor(up * self.batch, dtype=torch.int32, device="cuda")
        self.up = torch.tensor(up, device="cuda")
        self.deepest = deepest_of(up)
        starts = torch.arange(0, rows + 1, self.nodes, dtype=torch.int32, device="cuda")
        self.mask, self.depth, self.pos = ints(rows, -(-self.nodes // 32)), ints(rows), ints(1, rows)
        self.path, self.count, self.left = ints(self.batch, self.deepest), ints(self.batch), ints(self.batch)
        self.drafted = torch.zeros(self.batch, self.nodes, dtype=torch.int64, device="cuda")
        self.chosen = torch.zeros_like(self.drafted)
        self.qkv = torch.empty(rows, sum(heads), shape.head_dim, dtype=torch.bfloat16, device="cuda")
        q, key, value = self.qkv.split(heads, dim=1)
        self.out = torch.empty(rows, n_heads, shape.head_dim, dtype=torch.bfloat16, device="cuda")
        self.workspace = self.att.workspace()
        self.tree = kvx.make_tree_io(self.tokens, self.parent, self.mask, depth=self.depth, pos=self.pos,
                                     q_start=starts, window=window, sink=sink)
        self.ios = [kvx.make_attn_io(self.cache, self.tokens, q, layer=l, q_start=starts,
                                     max_new=self.nodes, new_q=q, new_k=key, new_v=value, pos=self.pos,
                                     out=self.out, window=window, sink=sink, tree=self.mask,
                                     depth=self.depth) for l in range(shape.n_layers)]
        self.accepted = kvx.make_accept_io(self.cache, self.tokens, self.path, self.count, q_start=starts,
                                           tokens_out=self.left)
        self.graph = None

    def _read(self):
        """The target's choice after every node."""
        x = self.embedding[self.drafted.view(-1)]
        flat = self.qkv.view(x.shape[0], -1)
        self.att.tree(self.tree)
        for l, io in enumerate(self.ios):
            torch.mm(self.model.norm(x), self.model.qkv[l], out=flat)
            self.att.append(io)
            self.att.forward(io, self.workspace)
            x = x + torch.mm(self.out.view(x.shape[0], -1), self.model.o[l])
        scores = torch.mm(self.model.norm(x), self.embedding.t().contiguous())
        self.chosen.copy_(scores.view(self.batch, self.nodes, -1).argmax(-1))

    def _step(self):
        """One tree of every context: the root is the last chosen token, and a child is
        accepted if it is what the target chose after its accepted parent."""
        self.tokens += self.nodes
        self._read()
        here = torch.zeros(self.batch, dtype=torch.int64, device="cuda")
        alive = torch.ones(self.batch, dtype=torch.bool, device="cuda")
        self.path.fill_(-1)
        self.path[:, 0] = 0
        self.count.fill_(1)
        for depth in range(1, self.deepest):
            wanted = self.chosen.gather(1, here[:, None])
            child = (self.up[None] == here[:, None]) & (self.drafted == wanted)
            alive = alive & child.any(1)
            here = torch.where(alive, child.int().argmax(1), here)
            self.path[:, depth] = torch.where(alive, here, -1).int()
            self.count += alive.int()
        self.last = self.chosen.gather(1, here[:, None])[:, 0]
        self.att.accept(self.accepted)
        self.tokens.copy_(self.left)

    def step(self, drafted, eager=False):
        """Reads the trees `drafted` [batch][nodes] of tokens; the accepted nodes and the
        token that the target chooses after them (both valid until the next step)."""
        if self.most + self.nodes > self.room:
            self.most = int(self.tokens.max())
            if self.most + self.nodes > self.room:
                raise ValueError(f"a tree of {self.nodes} does not fit {self.room} slots")
        self.most += self.deepest
        self.drafted.copy_(drafted)
        if eager:
            self._step()
        else:
            if self.graph is None:
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                self.graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(self.graph, stream=side):
                    self._step()
            self.graph.replay()
        return self.count, self.last

    def close(self):
        torch.cuda.synchronize()
        self.graph = None
        self.att.close()


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--config", type=int, default=2, choices=sorted(HEADS))
    p.add_argument("--tokens", type=int, default=1024, help="source tokens of a context")
    p.add_argument("--batch", type=int, default=1, help="contexts")
    p.add_argument("--steps", type=int, default=32, help="drafted trees")
    p.add_argument("--nodes", type=int, default=16, help="nodes of a tree")
    p.add_argument("--window", type=int, default=0, help="positions that a token sees, 0: all")
    p.add_argument("--sink", type=int, default=4, help="first positions that stay visible")
    a = p.parse_args(argv)
    if a.steps < 1 or a.nodes < 1:
        p.error("at least one tree of one node is wanted")
    room = a.steps * deepest_of(tree_of(a.nodes, 2)) + a.nodes  # if whole paths are accepted
    shape, k, v, table, lengths = handoff(a.config, a.tokens, a.batch, room)
    heads, cap = HEADS[a.config]
    d = Drafter(shape, heads, cap, k, v, table, lengths, a.nodes, window=a.window, sink=a.sink)
    g = torch.Generator("cuda").manual_seed(1)
    root = torch.zeros(a.batch, dtype=torch.int64, device="cuda")
    total, began = torch.zeros((), dtype=torch.int64, device="cuda"), None
    for i in range(a.steps):
        drafted = torch.randint(0, VOCABULARY, (a.batch, a.nodes), device="cuda", generator=g)
        drafted[:, 0] = root
        count, last = d.step(drafted)
        root = last.clone()
        total += count.sum()
        if i == 0:
            torch.cuda.synchronize()
            began = time.perf_counter()
    torch.cuda.synchronize()
    spent = (time.perf_counter() - began) / max(1, a.steps - 1)
    print(f"{lengths} translated tokens, {a.steps} trees of {a.nodes}: {int(total)} tokens accepted, "
          f"{d.tokens.tolist()} cached, {spent * 1e3:.3f} ms a tree and batch")
    d.close()


if __name__ == "__main__":
    main()
