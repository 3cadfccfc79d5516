"""Operators of serving on a translated cache that is held in 8 bits, bounded by
a window with sinks, and decoded by drafted trees, as cases that can be timed.

``listed()`` names the cases, ``draw(rng)`` draws one more of the same ranges,
``prepare(case, seed)`` makes what a serving program holds before the call,
``run(state)`` is one call, ``work(case)`` the bytes and flops it cannot do
without and ``exact(case, seed)`` the same outputs in 64 bits.  With ``own``
false ``run`` computes the operators by elementary torch operations in 32
bits; with ``own`` true it calls the framework's.

A cache of 8 bits holds codes (int8, or e4m3 floating point) and for every
slot and KV head a scale of its key and one of its value: the smallest power of
two, from 2^-100 on, under which the row's largest magnitude is not past the
largest code (127 or 448).  A number is its code times its row's scale.

A case is a dict of plain values:
  op       "store8"  rotate new queries and keys, store keys and values in 8 bits
           "pack"    a cache to one of 8 bits, all layers
           "unpack"  a cache of 8 bits to one of the case's dtype, all layers
           "attend"  attention of new tokens over the cache
           "tree"    what the tokens of drafted trees see, by their parents, and
                     the trees' attention over the cache
           "accept"  the accepted path of every tree moves behind its context's
                     other tokens, all layers
  hq hkv d query heads, KV heads, head_dim; base: RoPE base
  layers   layers of the cache (pack, unpack, accept handle all, others the last)
  batch    contexts; new: new tokens of the longest one (pack, unpack: 0)
  tokens   cached tokens of the longest context, the new ones included
  ragged   contexts of different lengths (else all alike)
  page     tokens per block of a paged cache (0: contiguous)
  cap      tanh cap of the scores (0: none)
  window   visible tokens before a new one (0: all); sink: first tokens that stay
           visible outside of it
  code     "i8", "e4m3" or "" (the cache is of the case's dtype)
  dtype    "bf16" or "f32", of all that is not codes
"""
import math
from types import SimpleNamespace

import torch

own = False


def _case(name, op, **kw):
    c = dict(op=op, hq=12, hkv=2, d=128, base=1e6, layers=2, batch=1, new=1, tokens=256,
             ragged=False, page=16, cap=0.0, window=0, sink=0, code="", dtype="bf16")
    c.update(kw)
    return {"name": name, **c} if name else c


# Head layouts of the target models of the framework's workloads.
_QWEN_SMALL = dict(hq=12, hkv=2, d=128, base=1e6)
_QWEN = dict(hq=28, hkv=4, d=128, base=1e6)
_GEMMA = dict(hq=8, hkv=4, d=256, base=1e4)
_LLAMA = dict(hq=64, hkv=8, d=128, base=5e5)


def listed():
    return [
        # one decoding step of one user: a single token is stored
        _case("store8_token", "store8", **_QWEN_SMALL, tokens=1000, code="e4m3"),
        # prompts of different lengths arrive
        _case("store8_prompts_x4", "store8", **_QWEN, batch=4, new=2049, tokens=4096, ragged=True,
              code="e4m3"),
        # a handoff's cache is compressed
        _case("pack_4k", "pack", **_QWEN_SMALL, layers=28, new=0, tokens=4096, code="i8"),
        # a few compressed caches go to a program that knows only bf16
        _case("unpack_2k_x4", "unpack", **_GEMMA, layers=26, batch=4, new=0, tokens=2048,
              ragged=True, page=32, code="e4m3"),
        # a serving step of many users at different lengths
        _case("decode8_8k_x64", "attend", **_QWEN, layers=1, batch=64, tokens=8192, ragged=True,
              code="i8"),
        # a long question on a compressed context
        _case("chunk8_1k_of_8k", "attend", **_LLAMA, new=1021, tokens=8192, page=64, code="e4m3"),
        # a serving step of a model with a window, sinks and capped scores
        _case("sink_decode_x16", "attend", **_GEMMA, layers=1, batch=16, tokens=8192, ragged=True,
              page=32, cap=50.0, window=1024, sink=4),
        # fp32 check of a few contexts read in chunks through a window
        _case("sink_chunk_f32_x3", "attend", **_QWEN_SMALL, batch=3, new=257, tokens=2900,
              ragged=True, page=0, window=500, sink=4, dtype="f32"),
        # one user's drafted tree after a short handoff
        _case("tree_16_of_1k", "tree", **_QWEN_SMALL, new=16, tokens=1000),
        # drafted trees of several users over compressed contexts
        _case("tree_64_of_8k_x8", "tree", **_QWEN, layers=1, batch=8, new=64, tokens=8192,
              ragged=True, code="i8"),
        # what was accepted of one tree, and of many
        _case("accept_16", "accept", **_QWEN_SMALL, layers=28, new=16, tokens=1000),
        _case("accept_64_x32", "accept", **_GEMMA, layers=26, batch=32, new=64, tokens=1024,
              ragged=True, page=32, code="e4m3"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case, of no more work than the largest listed one of its operator."""
    op = rng.choice(["store8", "pack", "unpack", "attend", "attend", "attend", "tree", "tree",
                     "accept"])
    most = [work(c) for c in listed() if c["op"] == op]
    bound = {k: max(w[k] for w in most) for k in ("bytes", "flops")}
    while True:
        hkv = rng.choice([1, 2, 4, 8])
        c = dict(hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 6, 7, 8]),
                 d=rng.choice([64, 80, 128, 128, 256]), base=rng.choice([1e4, 5e5, 1e6]),
                 batch=_log_int(rng, 1, 64), tokens=_log_int(rng, 16, 65536),
                 ragged=rng.random() < 0.6, page=rng.choice([0, 16, 16, 32, 48, 64]),
                 code=rng.choice(["i8", "e4m3"]))
        if op == "store8":
            c["code"] = "e4m3"
            c["new"] = rng.choice([1, _log_int(rng, 1, c["tokens"])])
        elif op in ("pack", "unpack"):
            c.update(new=0, layers=rng.randint(2, 32), dtype=rng.choice(["bf16", "bf16", "f32"]))
        else:
            c["code"] = rng.choice(["", "", "i8", "e4m3"])
            if not c["code"]:
                c["dtype"] = rng.choice(["bf16", "bf16", "f32"])
        if op == "attend":
            c["new"] = rng.choice([1, _log_int(rng, 1, c["tokens"])])
            c["window"] = rng.choice([0, _log_int(rng, 8, c["tokens"])])
            if c["window"] or not c["code"]:
                c["window"] = c["window"] or _log_int(rng, 8, c["tokens"])
                c["sink"] = rng.choice([1, 4, 4, _log_int(rng, 4, 128)])
        if op == "tree":
            c["new"] = min(c["tokens"], _log_int(rng, 2, 128))
            c["window"] = rng.choice([0, 0, 0, _log_int(rng, 8, c["tokens"])])
            c["sink"] = 4 if c["window"] else 0
        if op in ("attend", "tree"):
            c["cap"] = rng.choice([0.0, 0.0, 30.0, 50.0])
        if op == "accept":
            c.update(new=min(c["tokens"], _log_int(rng, 2, 64)), layers=rng.randint(2, 32))
        c = _case(None, op, **c)
        if c["layers"] * c["batch"] * c["tokens"] * c["hkv"] * c["d"] > 1 << 29:
            continue  # a cache of 4 GB in fp32
        w = work(c)
        slow = 8 if c["dtype"] == "f32" and c["new"] > 1 else 1
        # the plain form holds one score per padded (query head, token) pair
        scores = c["batch"] * c["hq"] * c["new"] * c["tokens"]
        if w["bytes"] <= bound["bytes"] and w["flops"] * slow <= bound["flops"] and \
                scores <= 64 * 1024 * 8192:
            return c


def _lengths(c):
    """(new, cached) tokens of every context."""
    out = []
    for b in range(c["batch"]):
        f = ((b + 1) * 0.6180339887498949) % 1.0 if c["ragged"] and b else 1.0
        n = max(1, int(c["tokens"] * (0.1 + 0.9 * f)))
        out.append((min(n, max(min(1, c["new"]), int(c["new"] * f))), n))
    return out


def _longest_path(c):
    """Nodes of the longest path that is accepted."""
    return max(1, min(c["new"], 12))


def work(c):
    es = 4 if c["dtype"] == "f32" else 2
    lens = _lengths(c)
    rows = sum(m for m, _ in lens)
    cached = sum(n for _, n in lens)
    row = c["d"] * es
    held = c["d"] + 2 if c["code"] else row  # a row of the cache
    if c["op"] == "store8":
        return {"bytes": rows * ((2 * c["hq"] + 2 * c["hkv"]) * row + 2 * c["hkv"] * held + 4),
                "flops": rows * c["d"] * (3 * c["hq"] + 6 * c["hkv"])}
    if c["op"] in ("pack", "unpack"):
        numbers = 2 * c["layers"] * c["hkv"] * cached
        return {"bytes": numbers * (row + held), "flops": 2 * numbers * c["d"]}
    if c["op"] == "accept":
        moved = sum(min(m, _longest_path(c)) for m, _ in lens) / 2
        return {"bytes": 4 * c["layers"] * c["hkv"] * moved * held + 8 * rows, "flops": moved}
    seen = visible = 0
    for m, n in lens:
        w = c["window"] or n
        first = max(0, n - m - w + 1)  # of the first new token's window
        seen += n - first + min(c["sink"], first)
        if c["op"] == "tree":
            lo = max(0, n - m - w + 1)
            visible += m * (n - m - lo + min(c["sink"], lo) + max(1, math.log2(m)))
            continue
        p = torch.arange(n - m, n)
        lo = (p - w + 1).clamp(min=0)
        visible += int((p + 1 - lo + lo.clamp(max=c["sink"])).sum())
    q = rows * c["hq"]
    words = -(-max(m for m, _ in lens) // 32) if c["op"] == "tree" else 0
    return {"bytes": q * (2 * row + 4) + 2 * seen * c["hkv"] * held + 4 * rows * (1 + words),
            "flops": 4 * c["hq"] * c["d"] * visible}


def _randn(g, shape, dt, by=None):
    """N(0, 1), columns scaled by `by`, on the GPU in dtype dt, one leading slice at a time."""
    out = torch.empty(shape, dtype=dt, device="cuda")
    for i in range(shape[0]):
        x = torch.randn(shape[1:], generator=g, device="cuda")
        out[i] = x if by is None else x.mul_(by)
    return out


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


_CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def _bytes(x):
    """A cache's numbers as they are moved: codes as bytes."""
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _inputs(c, seed):
    """Lengths, cache and the new tokens' rows, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed * 2 + 1)
    gc = torch.Generator().manual_seed(seed * 2 + 1)
    s = SimpleNamespace(case=c, dt=torch.float32 if c["dtype"] == "f32" else torch.bfloat16)
    s.lens = _lengths(c)
    s.rows = sum(m for m, _ in s.lens)
    s.starts = [sum(m for m, _ in s.lens[:b]) for b in range(c["batch"] + 1)]
    s.single = all(m == 1 for m, _ in s.lens)
    s.q_start, s.tokens = _int32(s.starts), _int32([n for _, n in s.lens])
    if c["page"]:
        per = -(-c["tokens"] // c["page"])
        s.table = torch.randperm(c["batch"] * per, generator=gc).to(torch.int32)
        s.table = s.table.view(c["batch"], per).cuda()
        shape = (c["layers"], c["batch"] * per, c["hkv"], c["page"], c["d"])
    else:
        s.table = None
        shape = (c["layers"], c["batch"], c["hkv"], c["tokens"], c["d"])
    s.shape = shape
    # channels of keys differ in size
    by = torch.randn((c["hkv"], 1, c["d"]), generator=g, device="cuda").mul_(0.5).exp_()
    if c["op"] == "pack" or not c["code"]:
        s.k, s.v = _randn(g, shape, s.dt, by), _randn(g, shape, s.dt)
    else:
        s.scale = torch.empty(shape[:-1] + (2,), dtype=torch.bfloat16, device="cuda")
        s.k8 = torch.empty(shape, dtype=_CODES[c["code"]], device="cuda")
        s.v8 = torch.empty_like(s.k8)
        for i in range(shape[0]):
            for e, (to, f) in enumerate(((s.k8, by), (s.v8, None))):
                x = torch.randn(shape[1:], generator=g, device="cuda")
                codes, s.scale[i, ..., e] = _quantised(c, x if f is None else x.mul_(f))
                to[i] = codes
    if c["op"] in ("tree", "accept"):
        # every node's parent is one of the few before it; a path of every tree
        s.parents, s.paths = [], []
        for m, _ in s.lens:
            back = torch.randint(1, 9, (m,), generator=gc).tolist()
            up = [-1] + [max(0, i - back[i]) for i in range(1, m)]
            most = min(m, _longest_path(c))
            count = int(torch.randint(1, most + 1, (1,), generator=gc))
            some = torch.randperm(m - 1, generator=gc)[:count - 1] + 1
            s.parents.append(up)
            s.paths.append([0] + sorted(some.tolist()))
        s.parent = _int32([p for up in s.parents for p in up])
        longest = _longest_path(c)
        s.path = _int32([p + [-1] * (longest - len(p)) for p in s.paths])
        s.count = _int32([len(p) for p in s.paths])
    if c["op"] in ("pack", "unpack", "accept"):
        return s
    # rows of a fused projection: the heads of q, k and v side by side
    fused = torch.randn((s.rows, c["hq"] + 2 * c["hkv"], c["d"]), generator=g, device="cuda")
    fused[:, c["hq"]:c["hq"] + c["hkv"]] *= by[:, 0]
    s.new_q, s.new_k, s.new_v = fused.to(s.dt).split([c["hq"], c["hkv"], c["hkv"]], 1)
    if c["op"] == "store8":
        s.pos = torch.cat([torch.arange(n - m, n) for m, n in s.lens]).to(torch.int32)[None].cuda()
    else:
        s.q = s.new_q.contiguous()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    c = case
    if c["op"] == "store8":
        s.q = torch.zeros((s.rows, c["hq"], c["d"]), dtype=s.dt, device="cuda")
    elif c["op"] == "pack":
        s.k8 = torch.zeros(s.shape, dtype=_CODES[c["code"]], device="cuda")
        s.v8 = torch.zeros_like(s.k8)
        s.scale = torch.zeros(s.shape[:-1] + (2,), dtype=torch.bfloat16, device="cuda")
    elif c["op"] == "unpack":
        s.k = torch.zeros(s.shape, dtype=s.dt, device="cuda")
        s.v = torch.zeros_like(s.k)
    if own:
        _prepare_own(c, s)
    return s


def _prepare_own(c, s):
    from paper_2608_30963_amd import kvx
    model = kvx.ModelShape(c["layers"], c["hkv"], c["d"], c["base"])
    s.att = kvx.Attention(model, c["hq"], kvx.KVX_F32 if c["dtype"] == "f32" else kvx.KVX_BF16,
                          softcap=c["cap"])
    if c["op"] in ("pack", "unpack"):
        plain = kvx.make_cache(s.k, s.v, s.table)
        coded = kvx.make_cache8(s.k8, s.v8, s.scale, s.table)
        s.io = kvx.make_pack_io(plain, coded, s.tokens)
        return
    cache = kvx.make_cache8(s.k8, s.v8, s.scale, s.table) if c["code"] else \
        kvx.make_cache(s.k, s.v, s.table)
    if c["op"] == "accept":
        s.tokens_out = torch.empty_like(s.tokens)
        s.io = kvx.make_accept_io(cache, s.tokens, s.path, s.count, q_start=s.q_start,
                                  tokens_out=s.tokens_out)
        return
    kw = dict(layer=c["layers"] - 1, q_start=None if s.single else s.q_start,
              max_new=max(m for m, _ in s.lens))
    if c["op"] == "store8":
        s.io = kvx.make_attn_io(cache, s.tokens, s.q, new_q=s.new_q, new_k=s.new_k, new_v=s.new_v,
                                pos=s.pos, **kw)
        return
    kw.update(window=c["window"], sink=c["sink"])
    if c["op"] == "tree":
        s.mask = torch.empty((s.rows, -(-kw["max_new"] // 32)), dtype=torch.int32, device="cuda")
        s.depth = torch.empty(s.rows, dtype=torch.int32, device="cuda")
        s.pos = torch.empty((1, s.rows), dtype=torch.int32, device="cuda")
        s.tree = kvx.make_tree_io(s.tokens, s.parent, s.mask, depth=s.depth, pos=s.pos,
                                  q_start=s.q_start, window=c["window"], sink=c["sink"])
        kw.update(tree=s.mask, depth=s.depth, q_start=s.q_start)
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty((s.rows, c["hq"]), device="cuda")
    s.io = kvx.make_attn_io(cache, s.tokens, s.q, out=s.out, lse=s.lse, **kw)
    s.workspace = s.att.workspace(s.io)


def run(state):
    s = state
    op = s.case["op"]
    if not own:
        return _PLAIN[op](s.case, s)
    if op == "store8":
        s.att.append(s.io)
        return s.q, s.k8[-1], s.v8[-1], s.scale[-1]
    if op == "pack":
        s.att.pack(s.io)
        return s.k8, s.v8, s.scale
    if op == "unpack":
        s.att.unpack(s.io)
        return s.k, s.v
    if op == "attend":
        s.att.forward(s.io, s.workspace)
        return s.out, s.lse
    if op == "tree":
        s.att.tree(s.tree)
        s.att.forward(s.io, s.workspace)
        return s.out, s.lse, s.mask, s.pos
    s.att.accept(s.io)
    return _moved(s) + (s.tokens_out,)


def _moved(s):
    return (s.k8, s.v8, s.scale) if s.case["code"] else (s.k, s.v)


# The plain forms: elementary operations on all contexts at once, padded to
# the longest.

def _quantised(c, x):
    """Codes of fp32 rows x [..., d] and their scales."""
    most, drop = (127 / 128, 7) if c["code"] == "i8" else (448 / 512, 9)
    m, e = torch.frexp(x.abs().amax(-1))
    e = torch.where(m > 0, e - drop + (m > most), -100).clamp_(min=-100)
    # powers of two by their bits: torch's own may be a rounding off
    up, down = (((127 + y) << 23).view(torch.float32) for y in (e, -e))
    x = x * down[..., None]
    return (x.round() if c["code"] == "i8" else x).to(_CODES[c["code"]]), up


def _slots(s):
    """Context and slot of every new token."""
    row = torch.arange(s.rows, device="cuda")
    ctx = torch.bucketize(row, s.q_start[1:].long(), right=True)
    return ctx, s.tokens[ctx] + row - s.q_start[ctx + 1]


def _at(c, s, ctx, slot):
    """Where slots lie: (block or context, slot)."""
    if s.table is None:
        return ctx, slot
    return s.table[ctx, slot // c["page"]].long(), slot % c["page"]


def _plain_store8(c, s):
    half = c["d"] // 2
    # angles in 64 bits: their error would grow with the position
    f = c["base"] ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    ang = (s.pos[0].double()[:, None] * f)[:, None]
    cs, sn = torch.cos(ang).float(), torch.sin(ang).float()

    def turn(x):
        a, b = x.float().split(half, -1)
        return torch.cat([a * cs - b * sn, b * cs + a * sn], -1)

    s.q.copy_(turn(s.new_q))
    blk, slot = _at(c, s, *_slots(s))
    for e, (to, x) in enumerate(((s.k8, turn(s.new_k)), (s.v8, s.new_v.float()))):
        codes, scale = _quantised(c, x)
        to[-1].view(torch.uint8)[blk, :, slot] = codes.view(torch.uint8)
        s.scale[-1, ..., e][blk, :, slot] = scale.to(torch.bfloat16)
    return s.q, s.k8[-1], s.v8[-1], s.scale[-1]


def _held(c, s):
    """Which slots of the cache hold tokens, [block or context, 1, slot, 1]."""
    j = torch.arange(c["tokens"], device="cuda")
    if s.table is None:
        return (j < s.tokens[:, None])[:, None, :, None]
    j = torch.arange(s.table.shape[1] * c["page"], device="cuda")
    held = torch.empty(s.shape[1], c["page"], dtype=torch.bool, device="cuda")
    held[s.table.long().flatten()] = (j < s.tokens[:, None]).view(-1, c["page"])
    return held[:, None, :, None]


def _plain_pack(c, s):
    held = _held(c, s)
    for e, (to, x) in enumerate(((s.k8, s.k), (s.v8, s.v))):
        codes, scale = _quantised(c, x.float())
        to.view(torch.uint8).copy_(torch.where(held, codes.view(torch.uint8), to.view(torch.uint8)))
        s.scale[..., e] = torch.where(held[..., 0], scale.to(torch.bfloat16), s.scale[..., e])
    return s.k8, s.v8, s.scale


def _plain_unpack(c, s):
    held = _held(c, s)
    for e, (to, x) in enumerate(((s.k, s.k8), (s.v, s.v8))):
        x = x.float() * s.scale[..., e, None].float()
        to.copy_(torch.where(held, x.to(s.dt), to))
    return s.k, s.v


def _rows(c, s, x):
    """The last layer's rows in order, [B, Hkv, tokens, ...]."""
    if s.table is None:
        return x[-1]
    x = x[-1][s.table.long()].transpose(1, 2)
    return x.reshape((c["batch"], c["hkv"], -1) + x.shape[4:])[:, :, :c["tokens"]]


def _values(c, s, e):
    """The last layer's keys (e = 0) or values (1) in 32 bits."""
    if not c["code"]:
        return _rows(c, s, (s.k, s.v)[e]).float()
    codes = _rows(c, s, _bytes((s.k8, s.v8)[e])).contiguous().view(_CODES[c["code"]])
    return codes.float().mul_(_rows(c, s, s.scale)[..., e, None].float())


def _ancestors(c, s, row, i):
    """[B, m, m]: whether new token k of a context is on the path from its root
    to new token i, itself included."""
    m = i.shape[0]
    there = i < (s.q_start[1:] - s.q_start[:-1])[:, None]
    up = (s.parent[row][..., None] == i) & there[..., None]
    reach = (up | torch.eye(m, dtype=torch.bool, device="cuda")).float()
    for _ in range(max(1, (m - 1).bit_length())):  # paths of twice the length each time
        reach = torch.matmul(reach, reach).clamp_(max=1.0)
    return (reach > 0) & there[..., None] & there[:, None]


def _attention(c, s, see, row, n_new):
    """Outputs and log-sum-exp of padded new tokens that see slots `see` [B, m, tokens]."""
    grp, m = c["hq"] // c["hkv"], row.shape[1]
    q = s.q[row].float().view(c["batch"], m, c["hkv"], grp, c["d"]).permute(0, 2, 3, 1, 4)
    q = q.reshape(c["batch"], c["hkv"], grp * m, c["d"])
    x = torch.matmul(q, _values(c, s, 0).transpose(2, 3).contiguous()).mul_(c["d"] ** -0.5)
    if c["cap"]:
        x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
    see = see[:, None, None].expand(-1, -1, grp, -1, -1).reshape(c["batch"], 1, grp * m, -1)
    x.masked_fill_(~see, -math.inf)
    top = x.amax(-1, keepdim=True).clamp_(min=-1e30)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    lse = (total.log() + top)[..., 0]
    out = torch.matmul(x, _values(c, s, 1)).div_(total.clamp(min=1e-30))

    def unpad(y):
        y = y.view((c["batch"], c["hq"], m) + y.shape[3:]).transpose(1, 2)
        return y[torch.arange(m, device="cuda") < n_new[:, None]]

    return unpad(out).to(s.dt), unpad(lse)


def _plain_attend(c, s):
    i = torch.arange(max(m for m, _ in s.lens), device="cuda")
    row = (s.q_start[:-1, None] + i).clamp(max=s.rows - 1).long()
    n_new = s.q_start[1:] - s.q_start[:-1]
    p = ((s.tokens - n_new)[:, None] + i)[:, :, None]
    j = torch.arange(c["tokens"], device="cuda")
    see = (j <= p) & (j < s.tokens[:, None, None])
    if c["window"]:
        see &= (j > p - c["window"]) | (j < c["sink"])
    return _attention(c, s, see, row, n_new)


def _plain_tree(c, s):
    m = max(m for m, _ in s.lens)
    i = torch.arange(m, device="cuda")
    row = (s.q_start[:-1, None] + i).clamp(max=s.rows - 1).long()
    n_new = s.q_start[1:] - s.q_start[:-1]
    first = (s.tokens - n_new)[:, None]
    reach = _ancestors(c, s, row, i)
    depth = (reach.sum(-1) - 1).clamp(min=0)
    pos = first + depth
    if c["window"]:
        near = pos[:, None] > pos[:, :, None] - c["window"]
        reach &= near | (pos[:, None] < c["sink"])
    j = torch.arange(c["tokens"], device="cuda")
    see = (j < first[:, :, None]).expand(-1, m, -1)
    if c["window"]:
        see = see & ((j > pos[:, :, None] - c["window"]) | (j < c["sink"]))
    k = j - first  # new token of a slot
    drafted = ((k >= 0) & (k < n_new[:, None]))[:, None].expand(-1, m, -1)
    k = k.clamp(0, m - 1)[:, None].expand(-1, m, -1)
    see = see | (drafted & reach.gather(2, k))
    out, lse = _attention(c, s, see, row, n_new)
    there = i < n_new[:, None]
    words = torch.nn.functional.pad(reach, (0, -m % 32)).view(c["batch"], m, -1, 32).long()
    words = (words << torch.arange(32, device="cuda")).sum(-1)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return out, lse, words[there], pos[there].to(torch.int32)[None]


def _plain_accept(c, s):
    n_new = s.q_start[1:] - s.q_start[:-1]
    first = (s.tokens - n_new)[:, None]
    i = torch.arange(s.path.shape[1], device="cuda")
    kept = i < s.count[:, None]
    # what is not kept stands for the last slot, which stays
    to = torch.where(kept, first + i, s.tokens[:, None] - 1).flatten()
    of = torch.where(kept, first + s.path, s.tokens[:, None] - 1).flatten()
    ctx = torch.arange(c["batch"], device="cuda").repeat_interleave(i.shape[0])
    of, to = _at(c, s, ctx, of), _at(c, s, ctx, to)
    for x in _moved(s):
        x = _bytes(x)
        x[:, to[0], :, to[1]] = x[:, of[0], :, of[1]]
    return _moved(s) + ((first[:, 0] + s.count).to(torch.int32),)


_PLAIN = {"store8": _plain_store8, "pack": _plain_pack, "unpack": _plain_unpack,
          "attend": _plain_attend, "tree": _plain_tree, "accept": _plain_accept}


# The same in 64 bits, from the definitions, one context (and head) at a time.

def _place(c, s, b, j):
    """Index of cache row j (a tensor) of context b: (block or context, slot)."""
    if s.table is None:
        return torch.full_like(j, b), j
    return s.table[b].long()[j // c["page"]], j % c["page"]


def _coded(c, x):
    """Codes (as numbers) and scales of rows x, by trying the powers of two."""
    most = 127.0 if c["code"] == "i8" else 448.0
    x = x.double()
    powers = torch.tensor([2.0 ** e for e in range(-100, 123)], dtype=torch.float64, device="cuda")
    which = torch.searchsorted(most * powers, x.abs().amax(-1))  # the first that is not less
    scale = powers[which]
    y = x / scale[..., None]
    if c["code"] == "i8":
        return torch.round(y), scale
    # three bits behind the leading one, from 2^-6 down in steps of 2^-9
    step = powers[torch.searchsorted(powers, y.abs(), right=True).clamp(min=95) - 1] / 8
    return torch.round(y / step) * step, scale


def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    return {"store8": _exact_store8, "pack": _exact_pack, "unpack": _exact_unpack,
            "attend": _exact_attend, "tree": _exact_tree, "accept": _exact_accept}[c["op"]](c, s)


def _exact_store8(c, s):
    half = c["d"] // 2
    turn = torch.empty((s.rows, half), dtype=torch.complex128, device="cuda")
    for e in range(half):
        ang = s.pos[0].double() * c["base"] ** (-2.0 * e / c["d"])
        turn[:, e] = torch.polar(torch.ones_like(ang), ang)

    def rotated(x):
        z = torch.complex(x[..., :half].double(), x[..., half:].double()) * turn[:, None]
        return torch.cat([z.real, z.imag], -1)

    k, v, scale = s.k8[-1].double(), s.v8[-1].double(), s.scale[-1].double()
    new = [_coded(c, rotated(s.new_k)), _coded(c, s.new_v)]
    for b, (m, n) in enumerate(s.lens):
        blk, slot = _place(c, s, b, torch.arange(n - m, n, device="cuda"))
        rows = slice(s.starts[b], s.starts[b] + m)
        for e, to in enumerate((k, v)):
            to[blk, :, slot] = new[e][0][rows]
            scale[blk, :, slot, e] = new[e][1][rows]
    return rotated(s.new_q), k, v, scale


def _exact_pack(c, s):
    codes = [torch.zeros(s.shape, dtype=torch.float32, device="cuda") for _ in range(2)]
    scale = torch.zeros(s.shape[:-1] + (2,), dtype=torch.float64, device="cuda")
    for l in range(c["layers"]):
        for b, (_, n) in enumerate(s.lens):
            blk, slot = _place(c, s, b, torch.arange(n, device="cuda"))
            for e, x in enumerate((s.k, s.v)):
                y, f = _coded(c, x[l, blk, :, slot])
                codes[e][l, blk, :, slot] = y.float()  # codes have few bits
                scale[l, blk, :, slot, e] = f
    return (None, None, scale) if c["code"] == "i8" else (codes[0], codes[1], scale)


def _exact_unpack(c, s):
    out = [torch.zeros(s.shape, dtype=torch.float64, device="cuda") for _ in range(2)]
    for l in range(c["layers"]):
        for b, (_, n) in enumerate(s.lens):
            blk, slot = _place(c, s, b, torch.arange(n, device="cuda"))
            for e, x in enumerate((s.k8, s.v8)):
                y = _bytes(x[l])[blk, :, slot].view(_CODES[c["code"]]).float().double()
                out[e][l, blk, :, slot] = y * s.scale[l, blk, :, slot, e].double()[..., None]
    return out


def _exact_rows(c, s, b, n, h, e):
    """Keys or values of one context and KV head in 64 bits."""
    blk, slot = _place(c, s, b, torch.arange(n, device="cuda"))
    if not c["code"]:
        return (s.k, s.v)[e][-1, blk, h, slot].double()
    y = _bytes((s.k8, s.v8)[e])[-1, blk, h, slot].view(_CODES[c["code"]]).float().double()
    return y * s.scale[-1, blk, h, slot, e].double()[:, None]


def _exact_context(c, s, b, see, out, lse):
    """Rows of context b, which see slots `see` [m, n]."""
    m, n = see.shape
    rows = slice(s.starts[b], s.starts[b] + m)
    grp = c["hq"] // c["hkv"]
    for h in range(c["hkv"]):
        k, v = _exact_rows(c, s, b, n, h, 0).t().contiguous(), _exact_rows(c, s, b, n, h, 1)
        for g in range(h * grp, (h + 1) * grp):
            x = torch.mm(s.q[rows, g].double(), k) / math.sqrt(c["d"])
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            x[~see] = -math.inf
            lse[rows, g] = torch.logsumexp(x, 1)
            out[rows, g] = torch.mm(torch.softmax(x, 1), v)


def _exact_attend(c, s):
    out = torch.zeros((s.rows, c["hq"], c["d"]), dtype=torch.float64, device="cuda")
    lse = torch.full((s.rows, c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, (m, n) in enumerate(s.lens):
        p = torch.arange(n - m, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")
        see = j <= p
        if c["window"]:
            see &= (p - j < c["window"]) | (j < c["sink"])
        _exact_context(c, s, b, see, out, lse)
    return out, lse


def _exact_tree(c, s):
    out = torch.zeros((s.rows, c["hq"], c["d"]), dtype=torch.float64, device="cuda")
    lse = torch.full((s.rows, c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, (m, n) in enumerate(s.lens):
        see = torch.zeros((m, n), dtype=torch.bool)
        for i in range(m):
            path, k = [], i
            while k >= 0:
                path.append(k)
                k = s.parents[b][k]
            p = n - m + len(path) - 1
            see[i, :n - m] = True
            if c["window"]:
                see[i, min(c["sink"], n - m):max(0, p - c["window"] + 1)] = False
            for up, k in enumerate(path):  # `up` positions before it
                see[i, n - m + k] = not c["window"] or up < c["window"] or p - up < c["sink"]
        _exact_context(c, s, b, see.cuda(), out, lse)
    return out, lse, None, None


def _exact_accept(c, s):
    out = [x.double() if x.element_size() > 1 else x.float() for x in _moved(s)]
    for b, (m, n) in enumerate(s.lens):
        for i, k in enumerate(s.paths[b]):
            of, to = (_place(c, s, b, torch.tensor([n - m + x], device="cuda")) for x in (k, i))
            for y, x in zip(out, _moved(s)):
                row = _bytes(x)[:, of[0], :, of[1]]
                row = row.view(x.dtype).float() if x.element_size() == 1 else row.double()
                y[:, to[0], :, to[1]] = row
    if c["code"] == "i8":
        out[:2] = [None, None]
    return tuple(out) + (None,)
