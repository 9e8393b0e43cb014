"""Timed cases of the operators for drafted tokens and 8-bit pages: append with norms, page conversion, attention over
pages with a tree's mask, commit of accepted tokens.

The cache of a layer is one K and one V buffer of slots; a sequence names its slots in a row of the block table.
``new`` tokens of each sequence are packed one sequence after the other (``cu_q``), and ``kv_len`` counts a sequence's
cached tokens, the new ones included.  Pages hold 16-bit elements ``[slots][kv_heads][block][head_dim]``, or 8-bit ones:
a slot is then ``[kv_heads][block][head_dim]`` e4m3 elements followed by ``[kv_heads][block][4 * ceil(head_dim / 128)]``
exponents, one to 32 elements: 2^(byte - 127) times the element.

* ``append``: norms the new tokens' queries and keys per head, turns them by positions on one to three axes and writes
  keys and values to pages of either kind.
* ``convert``: pages of cached tokens from 16 bits to 8 or back, into slots of another cache.
* ``attention``: the new tokens over pages of either kind, causally or by a tree's mask among the new ones.
* ``commit``: the accepted ones of the drafted tokens move together in the cache.

Where ``own`` is false ``run`` computes them with elementary torch operations in 32 bits on padded batches.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

LLAMA, GPT_OSS, QWEN3 = (32, 8, 128), (64, 8, 64), (32, 4, 128)   # query heads, KV heads, head_dim
LONGEST = 131072            # tokens of the longest context
MOST_FLOPS = 1.11e12        # of the largest listed case
MOST_BYTES = 1.1e9
MOST_SCORES = 1 << 32       # padded scores of the plain form: 16 GiB in 32 bits
EPS = 1e-6                  # of the norms
LEAST = {"bf16": -117, "f16": -15}   # exponents that keep every element exact and finite in the 16-bit type
MOST = {"bf16": 120, "f16": 8}


def _case(op, shape, n_seq, new, kv, *, pages="e4m3", dtype="bf16", block=16, window=0, sinks=False, tree=False, rot=None,
          interleaved=False, axes=1, norm=True, back=False, lens=0, name=None):
    c = {"op": op, "heads": shape[0], "kv_heads": shape[1], "head_dim": shape[2], "n_seq": n_seq, "new": new, "kv": kv,
         "pages": pages, "dtype": dtype, "block": block, "window": window, "sinks": sinks, "tree": tree,
         "rot": shape[2] if rot is None else rot, "interleaved": interleaved, "axes": axes, "norm": norm, "back": back,
         "lens": lens}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of a batch into 8-bit pages
        _case("append", QWEN3, 32, 1, 4096, lens=1, name="append, decode step of 32"),
        # packed prompts with images: three axes, a quarter of each head unturned, pairs interleaved, 16-bit pages
        _case("append", GPT_OSS, 5, 4096, 4096, pages="16", dtype="f16", rot=48, interleaved=True, axes=3, lens=2,
              name="append, packed prompts, 3 axes"),
        # contexts that came back from the pool in 8 bits, for operators that take 16-bit pages
        _case("convert", LLAMA, 8, 0, 16384, back=True, lens=3, name="read back 8 x 16K"),
        # one context before it is offloaded; odd head size, pages of 8
        _case("convert", (15, 5, 80), 1, 0, 5001, dtype="f16", block=8, name="quantise 5001, odd shape"),
        # one user's decoding step on a short context: latency
        _case("attention", LLAMA, 1, 1, 1000, name="decode 1 x 1000, 8 bits"),
        # a decoding step of a busy server, contexts of all lengths
        _case("attention", LLAMA, 32, 1, 16384, lens=3, name="decode 32 x 16K ragged, 8 bits"),
        # a question about a long document that was retrieved in 8 bits: the largest case
        _case("attention", LLAMA, 1, 512, LONGEST, name="chunk of 512 over 128K, 8 bits"),
        # a small tree of drafted tokens to every sequence of a batch
        _case("attention", LLAMA, 16, 8, 8192, tree=True, pages="16", lens=4, name="tree of 8 x 16 over 8K"),
        # a large tree over one long context in 8 bits
        _case("attention", QWEN3, 1, 64, LONGEST, tree=True, name="tree of 64 over 128K, 8 bits"),
        # a windowed layer with attention sinks, trees of different sizes
        _case("attention", GPT_OSS, 8, 24, 4099, tree=True, dtype="f16", window=128, sinks=True, lens=5,
              name="windowed trees of 24, 8 bits"),
        # after the check of 32 small drafts
        _case("commit", LLAMA, 32, 8, 2048, pages="16", lens=6, name="commit 8 x 32"),
        # after the check of large trees, 8 bits
        _case("commit", QWEN3, 48, 256, 4096, lens=7, name="commit 256 x 48, 8 bits"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(("append", "convert", "attention", "attention", "attention", "attention", "commit"))
        group = rng.choice((1, 2, 3, 4, 7, 8))
        kv_heads = rng.choice((1, 2, 4, 5, 8))
        shape = rng.choice((LLAMA, GPT_OSS, QWEN3, (group * kv_heads, kv_heads, rng.choice((64, 80, 96, 112, 128)))))
        kv = _log(rng, 16, LONGEST)
        n_seq = _log(rng, 1, 64)
        more = {"dtype": rng.choice(("bf16", "bf16", "f16")), "block": rng.choice((16, 16, 8, 32)),
                "lens": rng.randint(0, 1 << 20), "pages": rng.choice(("e4m3", "e4m3", "16"))}
        new = 0
        if op == "append":
            new = rng.choice((1, _log(rng, 2, 2048), kv))
            more.update(rot=rng.choice((shape[2], shape[2] // 2)), interleaved=rng.random() < 0.5,
                        axes=rng.choice((1, 2, 3)), norm=rng.random() < 0.75)
        elif op == "convert":
            more.update(back=rng.random() < 0.5)
        elif op == "commit":
            new = _log(rng, 2, 256)
        else:
            more.update(window=rng.choice((0, 0, 0, 128, _log(rng, 1, 8192))), sinks=rng.random() < 0.25,
                        tree=more["pages"] == "16" or rng.random() < 0.5)
            new = _log(rng, 2, 256) if more["tree"] else rng.choice((1, _log(rng, 2, 2048), kv))
        case = _case(op, shape, n_seq, min(new, kv), kv, **more)
        need = work(case)
        if (need["flops"] <= MOST_FLOPS and 1 << 16 <= need["bytes"] <= MOST_BYTES and n_seq * kv <= 1 << 19
                and (op != "attention" or n_seq * shape[0] * case["new"] * kv <= MOST_SCORES)):
            return case


def _lengths(case):
    """(new tokens, cached ones with them) of every sequence: the first has the most, the others an eighth or more."""
    rng = random.Random(case["lens"])
    out = []
    for i in range(case["n_seq"]):
        share = 1.0 if i == 0 or not case["lens"] else math.exp(rng.uniform(math.log(0.125), 0.0))
        kv = max(1, int(case["kv"] * share))
        new = kv if case["new"] == case["kv"] else min(kv, int(case["new"] * share) or min(1, case["new"]))
        out.append((new, kv))
    return out


def _dtype(case):
    return {"bf16": torch.bfloat16, "f16": torch.float16}[case["dtype"]]


def _exponents(case):
    """Bytes of exponents to a row of 8-bit elements, and the bytes of a slot."""
    s = 4 * -(-case["head_dim"] // 128)
    return s, -(-case["kv_heads"] * case["block"] * (case["head_dim"] + s) // 16) * 16


def _parents(rng, n):
    """A draft tree of n tokens: token 0 is the last accepted one, the others have a parent before them."""
    return [-1] + [rng.randrange(max(0, i - 4), i) for i in range(1, n)]


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    draft = random.Random(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, bs, dev = _lengths(case), case["block"], "cuda"
    h, hk, d, n = case["heads"], case["kv_heads"], case["head_dim"], case["n_seq"]
    dtype = _dtype(case)
    stride = -(-case["kv"] // bs)
    blocks = [-(-kv // bs) for _, kv in lens]
    slots = sum(blocks) + sum(blocks) // 4 + 1       # a fifth of the cache belongs to others

    def tables():
        free, at = rng.permutation(slots), 0
        table = np.full((n, stride), -1, np.int32)
        for i, b in enumerate(blocks):
            table[i, :b] = free[at:at + b]
            at += b
        return torch.from_numpy(table).to(dev)

    cu = np.concatenate([[0], np.cumsum([new for new, _ in lens])]).astype(np.int32)
    total = int(cu[-1])

    def normal(*size, std=1.0, to=dtype):
        return torch.empty(size, dtype=torch.float32, device=dev).normal_(0.0, std, generator=gen).to(to)

    def pages(kind):
        """A cache of one kind: 16-bit elements, or bytes by slot."""
        if kind == "16":
            return normal(slots, hk, bs, d)
        s_bytes, slot_bytes = _exponents(case)
        cache = torch.zeros(slots, slot_bytes, dtype=torch.uint8, device=dev)
        e, x = _pack(case, normal(slots, hk, bs, d))
        _elements(case, cache)[:] = x
        _scales(case, cache)[:] = e
        return cache

    s = dict(case, total=total, slots=slots, stride=stride, scale=d ** -0.5, cu=torch.from_numpy(cu).to(dev),
             kv_len=torch.tensor([kv for _, kv in lens], dtype=torch.int32, device=dev), table=tables())
    kind = case["pages"] if case["op"] != "convert" else "e4m3" if case["back"] else "16"
    s["k_cache"], s["v_cache"] = pages(kind), pages(kind)
    if case["op"] == "append":
        qkv = normal(total, h + 2 * hk, d)           # as one projection writes them
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        s["q_weight"], s["k_weight"] = ((1.0 + normal(d, std=0.2, to=torch.float32)).to(dtype) for _ in range(2))
        turn = torch.arange(case["kv"], dtype=torch.float64)[:, None] * 500000.0 ** (
            -torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])
        s["angles"] = torch.stack([turn.cos(), turn.sin()], -1).float().contiguous().to(dev)
        at = np.concatenate([np.arange(kv - new, kv) for new, kv in lens] + [np.zeros(0, np.int64)]).astype(np.int32)
        rows = [at] + [rng.integers(0, case["kv"], total).astype(np.int32) for _ in range(case["axes"] - 1)]
        s["positions"] = torch.from_numpy(np.stack(rows)).to(dev)
        s["axis_of"] = [j * case["axes"] // (case["rot"] // 2) for j in range(case["rot"] // 2)]   # time, height, width
        s["q_out"] = torch.empty(total, h, d, dtype=dtype, device=dev)
        s["pos"] = torch.full((n, hk, case["kv"]), -1, dtype=torch.int32, device=dev)
    elif case["op"] == "convert":
        s["to_table"] = tables()
        other = "16" if case["back"] else "e4m3"
        s["k_to"], s["v_to"] = pages(other), pages(other)
    elif case["op"] == "attention":
        s["q"] = normal(total, h, d, std=2.0)
        if case["sinks"]:
            s["sinks"] = normal(h, std=2.0, to=torch.float32)
        if case["tree"]:
            words = -(-case["new"] // 64)
            mask = np.zeros((total, words), np.uint64)
            for i, (new, _) in enumerate(lens):
                for j, p in enumerate(_parents(draft, new)):
                    row = mask[cu[i] + j]
                    if p >= 0:
                        row |= mask[cu[i] + p]
                    row[j // 64] |= np.uint64(1 << (j % 64))
            s["tree"] = torch.from_numpy(mask.view(np.int64)).to(dev)
        s["out"] = torch.empty(total, h, d, dtype=dtype, device=dev)
        s["lse"] = torch.empty(h, total, dtype=torch.float32, device=dev)
    else:
        path, taken = np.zeros(total, np.int32), []
        for i, (new, _) in enumerate(lens):
            chosen = [j for j in range(new) if draft.random() < 0.6]
            path[cu[i]:cu[i] + len(chosen)] = chosen
            taken.append(len(chosen))
        s["path"] = torch.from_numpy(path).to(dev)
        s["accepted"] = torch.tensor(taken, dtype=torch.int32, device=dev)
        s["pos"] = torch.arange(case["kv"], dtype=torch.int32, device=dev).repeat(n, hk, 1)
        s["len_out"] = torch.zeros_like(s["kv_len"])
    if own:
        _handles(s)
    return s


# ---- the framework's calls

def _handles(s):
    from paper_2606_14779_amd import kvpool as K
    s["shape"] = K.CacheShape(s["dtype"], s["heads"], s["kv_heads"], s["head_dim"], s["block"], s["slots"])
    s["batch"] = K.Batch(s["n_seq"], s["total"], s["new"], s["kv"], s["cu"].data_ptr(), s["kv_len"].data_ptr(),
                         s["table"].data_ptr(), s["stride"])
    kind = s["pages"] if s["op"] != "convert" else "e4m3" if s["back"] else "16"
    s["cache"] = K.Pages(kind, s["k_cache"].data_ptr(), s["v_cache"].data_ptr())
    if s["op"] == "convert":
        s["to"] = K.Pages("16" if s["back"] else "e4m3", s["k_to"].data_ptr(), s["v_to"].data_ptr())
    if s["op"] == "append":
        s["normed"] = K.HeadNorm(s["q_weight"].data_ptr(), s["k_weight"].data_ptr(), EPS) if s["norm"] else None
        s["turned"] = K.RopeAxes(s["axes"], s["axis_of"]) if s["axes"] > 1 else None
    if s["op"] == "attention":
        need = K.attention_pages_workspace(s["shape"], s["batch"])
        s["work"] = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")


def _run_own(s):
    from paper_2606_14779_amd import kvpool as K
    stream = torch.cuda.current_stream().cuda_stream
    shape, batch, cache = s["shape"], s["batch"], s["cache"]
    if s["op"] == "append":
        K.norm_rope_append(shape, batch, cache, s["angles"].data_ptr(), s["angles"].shape[0], s["rot"],
                           s["positions"].data_ptr(), s["k"].data_ptr(), s["k"].stride(0), s["v"].data_ptr(),
                           s["v"].stride(0), norm=s["normed"], axes=s["turned"], q=s["q"].data_ptr(),
                           q_stride=s["q"].stride(0), q_out=s["q_out"].data_ptr(), q_out_stride=s["q_out"].stride(0),
                           pos=s["pos"].data_ptr(), pos_stride=s["kv"], interleaved=s["interleaved"], stream=stream)
    elif s["op"] == "convert":
        K.convert_pages(shape, batch, cache, s["to"], s["to_table"].data_ptr(), s["stride"], s["slots"], stream=stream)
    elif s["op"] == "attention":
        K.attention_pages(shape, batch, cache, s["q"].data_ptr(), s["q"].stride(0), s["scale"], s["out"].data_ptr(),
                          s["out"].stride(0), tree=s["tree"].data_ptr() if s["tree"] is not False else 0,
                          tree_words=-(-s["new"] // 64) if s["tree"] is not False else 0, window=s["window"],
                          sinks=s["sinks"].data_ptr() if s["sinks"] is not False else 0, lse=s["lse"].data_ptr(),
                          workspace=s["work"].data_ptr(), workspace_bytes=s["work"].numel(), stream=stream)
    else:
        K.tree_commit(shape, batch, cache, s["path"].data_ptr(), s["accepted"].data_ptr(), s["len_out"].data_ptr(),
                      pos=s["pos"].data_ptr(), pos_stride=s["kv"], stream=stream)
    return _outputs(s)


def _outputs(s):
    if s["op"] == "append":
        return s["q_out"], _values(s, s["k_cache"], s["pages"]), _values(s, s["v_cache"], s["pages"]), s["pos"]
    if s["op"] == "convert":
        kind = "16" if s["back"] else "e4m3"
        return _values(s, s["k_to"], kind), _values(s, s["v_to"], kind)
    if s["op"] == "attention":
        return s["out"], s["lse"]
    return _values(s, s["k_cache"], s["pages"]), _values(s, s["v_cache"], s["pages"]), s["pos"], s["len_out"]


def _values(s, cache, kind):
    """A cache as numbers: 16-bit elements, or 8-bit ones and the powers of two they are multiplied by."""
    return cache if kind == "16" else (_elements(s, cache), _scales(s, cache).view(torch.float8_e8m0fnu))


def run(state):
    if own:
        return _run_own(state)
    {"append": _append, "convert": _convert, "attention": _attend, "commit": _commit}[state["op"]](state)
    return _outputs(state)


# ---- the plain forms

def _elements(s, cache):
    n = s["kv_heads"] * s["block"] * s["head_dim"]
    return cache[:, :n].view(-1, s["kv_heads"], s["block"], s["head_dim"]).view(torch.float8_e4m3fn)


def _scales(s, cache):
    rows = s["kv_heads"] * s["block"]
    s_bytes, _ = _exponents(s)
    return cache[:, rows * s["head_dim"]:rows * (s["head_dim"] + s_bytes)].view(-1, s["kv_heads"], s["block"], s_bytes)


def _pack(s, x):
    """(exponents, elements) of 8-bit rows."""
    d = x.shape[-1]
    least, most = LEAST[s["dtype"]], MOST[s["dtype"]]
    part = torch.nn.functional.pad(x.float(), (0, -d % 32)).unflatten(-1, (-1, 32))
    mantissa, e = part.abs().amax(-1).frexp()
    e = torch.where(mantissa == 0, least, torch.where(mantissa <= 0.875, e - 9, e - 8).clamp(least, most))
    part = part * ((127 - e) << 23).view(torch.float32)[..., None]
    limit = torch.where(e == most, 240.0, 448.0)[..., None]
    part = part.clamp(-limit, limit).flatten(-2)[..., :d].to(torch.float8_e4m3fn)
    s_bytes, _ = _exponents(s)
    return torch.nn.functional.pad((e + 127).to(torch.uint8), (0, s_bytes - e.shape[-1])), part


def _unpack(s, elements, scales):
    power = (scales.int() << 23).view(torch.float32).repeat_interleave(32, -1)[..., :s["head_dim"]]
    return elements.float() * power


def _rows(s):
    """Sequence and cache index of every packed new token."""
    row = torch.arange(s["total"], device="cuda")
    seq = torch.bucketize(row, s["cu"][1:].long(), right=True)
    return seq, s["kv_len"][seq].long() - s["cu"][seq + 1] + row


def _put(s, cache, kind, slot, off, x):
    """Rows x to a cache of one kind."""
    if kind == "16":
        cache[slot, :, off] = x.to(_dtype(s))
    else:
        e, x = _pack(s, x)
        _elements(s, cache).view(torch.uint8)[slot, :, off] = x.view(torch.uint8)
        _scales(s, cache)[slot, :, off] = e


def _append(s):
    seq, at = _rows(s)
    rot = s["rot"]
    pair = torch.arange(rot // 2, device="cuda")
    axis = pair * s["axes"] // (rot // 2)
    cos, sin = s["angles"][s["positions"].t()[:, axis].long(), pair].unbind(-1)
    cos, sin = cos[:, None], sin[:, None]

    def turned(x, weight):
        x = x.float()
        if s["norm"]:
            x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.float()
        a, b = (x[..., :rot:2], x[..., 1:rot:2]) if s["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        pair = a * cos - b * sin, b * cos + a * sin
        pair = torch.stack(pair, -1).flatten(-2) if s["interleaved"] else torch.cat(pair, -1)
        return torch.cat([pair, x[..., rot:]], -1)

    slot, off = s["table"][seq, at // s["block"]].long(), at % s["block"]
    s["q_out"].copy_(turned(s["q"], s["q_weight"]))
    _put(s, s["k_cache"], s["pages"], slot, off, turned(s["k"], s["k_weight"]))
    _put(s, s["v_cache"], s["pages"], slot, off, s["v"])
    s["pos"][seq, :, at] = s["positions"][0][:, None].expand(-1, s["kv_heads"])


def _convert(s):
    token = torch.arange(s["kv"], device="cuda").expand(s["n_seq"], -1)
    seq, at = (token < s["kv_len"][:, None]).nonzero().unbind(1)
    off = at % s["block"]
    slot, to = s["table"][seq, at // s["block"]].long(), s["to_table"][seq, at // s["block"]].long()
    for cache, out in ((s["k_cache"], s["k_to"]), (s["v_cache"], s["v_to"])):
        if s["back"]:
            x = _elements(s, cache).view(torch.uint8)[slot, :, off].view(torch.float8_e4m3fn)
            _put(s, out, "16", to, off, _unpack(s, x, _scales(s, cache)[slot, :, off]))
        else:
            _put(s, out, "e4m3", to, off, cache[slot, :, off])


def _tokens(s, cache):
    """A cache's tokens by sequence and KV head, padded, in 32 bits: [n_seq][kv_heads][tokens][head_dim]."""
    slot = s["table"].clamp(min=0).long()
    if s["pages"] == "16":
        pages = cache[slot].float()
    else:
        x = _elements(s, cache).view(torch.uint8)[slot].view(torch.float8_e4m3fn)
        pages = _unpack(s, x, _scales(s, cache)[slot])
    pages = pages.permute(0, 2, 1, 3, 4).reshape(s["n_seq"], s["kv_heads"], -1, s["head_dim"])
    return pages[:, :, :s["kv"]].contiguous()


def _attend(s):
    n, h, hk, new, kv, total = s["n_seq"], s["heads"], s["kv_heads"], s["new"], s["kv"], s["total"]
    row = torch.arange(new, device="cuda")
    n_q = s["cu"][1:] - s["cu"][:-1]
    at = (s["cu"][:-1, None] + row).clamp(max=total - 1).long()
    q = s["q"][at].float().permute(0, 2, 1, 3).reshape(n, hk, -1, s["head_dim"])
    logits = torch.matmul(q, _tokens(s, s["k_cache"]).transpose(2, 3).contiguous()).mul_(s["scale"])
    token = torch.arange(kv, device="cuda")
    first = (s["kv_len"] - n_q)[:, None, None]       # cached tokens before the new ones
    if s["tree"] is False:
        hidden = token > first + row[:, None]
        ahead = row[:, None]                         # place among the new tokens
    else:
        bits = (s["tree"][at][..., None] >> torch.arange(64, device="cuda") & 1).flatten(2)   # [n][new][64 words]
        drafted = (token - first).expand(-1, new, -1)
        shown = bits.gather(2, drafted.clamp(0, bits.shape[2] - 1).long()).bool()
        hidden = (drafted >= 0) & ~(shown & (drafted < n_q[:, None, None]))
        ahead = bits.sum(-1, keepdim=True) - 1       # depth
    hidden = hidden | (row[:, None] >= n_q[:, None, None])
    if s["window"]:
        early = token <= first + ahead - s["window"]
        hidden |= early if s["tree"] is False else early & (token < first)
    logits.view(n, hk, -1, new, kv).masked_fill_(hidden[:, None, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
    if s["sinks"] is not False:
        sink = s["sinks"].view(hk, -1, 1).expand(-1, -1, new).reshape(1, hk, -1, 1)
        top = torch.maximum(top, sink)
    weights = logits.sub_(top).exp_()
    weight = weights.sum(-1, keepdim=True)
    if s["sinks"] is not False:
        weight = weight + (sink - top).exp()
    seq, index = _rows(s)
    place = index - s["kv_len"][seq] + n_q[seq]
    s["lse"].copy_((weight.log() + top).view(n, h, new)[seq, :, place].t())
    out = torch.matmul(weights, _tokens(s, s["v_cache"])).div_(weight).view(n, h, new, -1)
    s["out"].copy_(out[seq, :, place])


def _commit(s):
    seq, _ = _rows(s)
    place = torch.arange(s["total"], device="cuda") - s["cu"][seq]
    seq, place, path = (x[place < s["accepted"][seq]] for x in (seq, place, s["path"].long()))
    first = (s["kv_len"] - s["cu"][1:] + s["cu"][:-1])[seq].long()
    came, to = first + path, first + place

    def slots(at):
        return s["table"][seq, at // s["block"]].long(), at % s["block"]

    (a, i), (b, j) = slots(came), slots(to)
    for cache in (s["k_cache"], s["v_cache"]):
        if s["pages"] == "16":
            cache[b, :, j] = cache[a, :, i]
        else:
            for part in (_elements(s, cache).view(torch.uint8), _scales(s, cache)):
                part[b, :, j] = part[a, :, i]
    s["pos"][seq, :, to] = s["pos"][seq, :, came]
    s["len_out"].copy_(s["kv_len"] - s["cu"][1:] + s["cu"][:-1] + s["accepted"])


# ---- from the definitions, in 64 bits, one sequence and head at a time

def _cache_index(s, i, first, end, table="table"):
    """Slots and offsets of tokens of a sequence, from its block table row."""
    slots = np.repeat(s[table][i].cpu().numpy().astype(np.int64), s["block"])[first:end]
    return torch.from_numpy(slots).cuda(), torch.arange(first, end, device="cuda") % s["block"]


def _exact_pages(s, cache, kind):
    """The numbers of a cache in 64 bits: (elements, powers of two), the powers None in 16 bits."""
    if kind == "16":
        return cache.double(), None
    return _elements(s, cache).double(), torch.pow(2.0, _scales(s, cache).double() - 127.0)


def _exact_rows(s, pages, slot, off):
    """Rows [tokens][kv_heads][head_dim] of such a cache."""
    x, power = pages
    x = x[slot, :, off]
    if power is not None:
        x = x * power[slot, :, off].repeat_interleave(32, -1)[..., :s["head_dim"]]
    return x


def _exact_put(s, pages, slot, off, x):
    """Rows to such a cache; elements of 8 bits as they are before their rounding."""
    elements, power = pages
    if power is None:
        elements[slot, :, off] = x
        return
    for b in range(0, s["head_dim"], 32):
        top = x[..., b:b + 32].abs().amax(-1)
        e = torch.log2(top / 448.0).ceil()
        e = torch.where(top <= 448.0 * torch.pow(2.0, e - 1), e - 1, torch.where(top > 448.0 * torch.pow(2.0, e), e + 1, e))
        e = e.clamp(LEAST[s["dtype"]], MOST[s["dtype"]])
        power[slot, :, off, b // 32] = torch.pow(2.0, e)
        elements[slot, :, off, b:b + 32] = x[..., b:b + 32] / torch.pow(2.0, e)[..., None]
    used = -(-s["head_dim"] // 32)
    power[slot, :, off, used:] = 2.0 ** -127


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"append": _exact_append, "convert": _exact_convert, "attention": _exact_attention, "commit": _exact_commit}[
        s["op"]](s)


def _exact_turned(s, x, weight):
    x = x.double().clone()
    if s["norm"]:
        x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / s["head_dim"] + EPS) * weight.double()
    rot, half = s["rot"], s["rot"] // 2
    first = list(range(0, rot, 2)) if s["interleaved"] else list(range(half))
    second = [i + 1 for i in first] if s["interleaved"] else [i + half for i in first]
    where = s["positions"].long()[torch.tensor(s["axis_of"], device="cuda")]            # [pairs][tokens]
    turn = torch.view_as_complex(s["angles"].double().contiguous())
    turn = torch.stack([turn[where[j], j] for j in range(half)], 1)[:, None]
    z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_append(s):
    q, k = _exact_turned(s, s["q"], s["q_weight"]), _exact_turned(s, s["k"], s["k_weight"])
    pos = s["pos"].clone()
    pages = [_exact_pages(s, s[c], s["pages"]) for c in ("k_cache", "v_cache")]
    for i, (new, kv) in enumerate(_lengths(s)):
        rows = slice(int(s["cu"][i]), int(s["cu"][i]) + new)
        slot, off = _cache_index(s, i, kv - new, kv)
        _exact_put(s, pages[0], slot, off, k[rows])
        _exact_put(s, pages[1], slot, off, s["v"][rows].double())
        pos[i, :, kv - new:kv] = s["positions"][0, rows]
    return q, _laid(pages[0]), _laid(pages[1]), pos


def _laid(pages):
    return pages[0] if pages[1] is None else pages


def _exact_convert(s):
    kinds = ("e4m3", "16") if s["back"] else ("16", "e4m3")
    out = []
    for a, b in (("k_cache", "k_to"), ("v_cache", "v_to")):
        came, to = _exact_pages(s, s[a], kinds[0]), _exact_pages(s, s[b], kinds[1])
        for i, (_, kv) in enumerate(_lengths(s)):
            slot, off = _cache_index(s, i, 0, kv)
            _exact_put(s, to, *_cache_index(s, i, 0, kv, "to_table"), _exact_rows(s, came, slot, off))
        out.append(_laid(to))
    return tuple(out)


def _exact_attention(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["heads"], s["total"], dtype=torch.float64, device="cuda")
    group = s["heads"] // s["kv_heads"]
    tree = s["tree"].cpu().numpy().view(np.uint64) if s["tree"] is not False else None
    for i, (new, kv) in enumerate(_lengths(s)):
        rows, first = slice(int(s["cu"][i]), int(s["cu"][i + 1])), kv - new
        sees = np.ones((new, kv), bool)
        place = np.arange(new)
        if tree is None:
            sees[:, first:] = np.tril(np.ones((new, new), bool))
        else:
            sees[:, first:] = np.unpackbits(tree[rows].view(np.uint8), axis=1, bitorder="little")[:, :new]
            place = sees[:, first:].sum(1) - 1
        if s["window"]:
            near = np.arange(kv)[None] > (first + place)[:, None] - s["window"]
            sees &= near if tree is None else near | (np.arange(kv) >= first)
        hidden = torch.from_numpy(~sees).cuda()
        slot, off = _cache_index(s, i, 0, kv)
        # only this sequence's slots in 64 bits
        own_slots, slot = slot.unique(return_inverse=True)
        k, v = (_exact_rows(s, _exact_pages(s, s[c][own_slots], s["pages"]), slot, off) for c in ("k_cache", "v_cache"))
        for head in range(s["heads"]):
            z = (s["q"][rows, head].double() @ k[:, head // group].t().contiguous()) * s["scale"]
            z[hidden] = -math.inf
            if s["sinks"] is not False:              # one more key, without a value
                z = torch.cat([z, s["sinks"][head].double().expand(new, 1)], 1)
            lse[head, rows] = torch.logsumexp(z, 1)
            out[rows, head] = torch.softmax(z, 1)[:, :kv] @ v[:, head // group].contiguous()
    return out, lse


def _exact_commit(s):
    pos, left = s["pos"].clone(), []
    pages = [_exact_pages(s, s[c], s["pages"]) for c in ("k_cache", "v_cache")]
    for i, (new, kv) in enumerate(_lengths(s)):
        count = int(s["accepted"][i])
        left.append(kv - new + count)
        path = s["path"][int(s["cu"][i]):int(s["cu"][i]) + count].long()
        slot, off = _cache_index(s, i, kv - new, kv)
        for cache in pages:
            for part in cache:
                if part is not None:
                    part[slot[:count], :, off[:count]] = part[slot[path], :, off[path]].clone()
        pos[i, :, kv - new:left[-1]] = pos[i, :, kv - new + path].clone()
    return _laid(pages[0]), _laid(pages[1]), pos, torch.tensor(left, dtype=torch.int32, device="cuda")


def _pairs(case, new, kv):
    """Query-key pairs of one head of one sequence."""
    w, first = case["window"], kv - new
    if case["tree"]:                                 # an ancestor of a token lies about two places before it
        depth = [min(i, i // 2 + 1) + 1 for i in range(new)]
        return sum(d + (min(first, max(0, w - d)) if w else first) for d in depth)
    if not w or w >= kv:
        return (first + 1 + kv) * new // 2
    short = max(0, min(kv, w) - first)               # queries that see less than a window
    return (first + 1 + first + short) * short // 2 + (new - short) * w


def work(case):
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    lens = _lengths(case)
    new, kv = sum(n for n, _ in lens), sum(n for _, n in lens)
    row8 = d + -(-d // 32)                           # bytes of a row of 8-bit elements
    row = row8 if case["pages"] == "e4m3" else 2 * d
    if case["op"] == "append":
        moved = new * (h + 2 * hk) * d * 2 + new * (h * d * 2 + 2 * hk * row)
        return {"bytes": moved + new * (4 * case["rot"] + 4 * case["axes"] + 4 * hk),
                "flops": new * (h + hk) * (3 * case["rot"] + 4 * d * case["norm"])}
    if case["op"] == "convert":
        return {"bytes": 2 * kv * hk * (row8 + 2 * d), "flops": 0}
    if case["op"] == "commit":                       # those of the accepted that are not in place already
        taken = sum(int(0.6 * n) for n, _ in lens)
        return {"bytes": 2 * taken * hk * (2 * row + 4) + 4 * taken, "flops": 0}
    if case["window"]:                               # the tokens that some query sees
        kv = sum(min(m, n - 1 + case["window"]) for n, m in lens)
    pairs = sum(_pairs(case, n, m) for n, m in lens)
    masks = new * 8 * -(-case["new"] // 64) if case["tree"] else 0
    return {"bytes": 2 * new * h * d * 2 + 4 * h * new + 2 * kv * hk * row + masks, "flops": 4 * d * h * pairs}
