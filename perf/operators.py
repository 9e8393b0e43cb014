"""Timed cases of the operators on the engine's paged cache: rotary append, attention, attention mass, eviction.

The cache of a layer is one K and one V buffer ``[slots][kv_heads][block][head_dim]``; a sequence names its slots
in a row of the block table.  ``new`` tokens of each sequence are packed one sequence after the other
(``cu_q``), and ``kv_len`` counts a sequence's cached tokens, the new ones included.

* ``rope``: rotates the new tokens' queries and keys and writes keys, values and positions to their pages.
* ``attention``: the new tokens attend causally over all cached ones: single tokens, chunks, whole prompts.
* ``mass``: the attention weight that each cached token collects from the last queries, added to its score.
* ``evict``: keeps the tokens of largest score and moves them together.

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


def _case(op, shape, n_seq, new, kv, *, dtype="bf16", block=16, window=0, sinks=False, rot=None, interleaved=False,
          last=0, keep=0, recent=0, lens=0, name=None):
    c = {"op": op, "heads": shape[0], "kv_heads": shape[1], "head_dim": shape[2], "n_seq": n_seq, "new": new, "kv": kv,
         "dtype": dtype, "block": block, "window": window, "sinks": sinks, "rot": shape[2] if rot is None else rot,
         "interleaved": interleaved, "last": last, "keep": keep, "recent": recent, "lens": lens}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decoding step of a batch: 32 tokens rotated and written to their pages
        _case("rope", LLAMA, 32, 1, 4096, lens=1, name="rope, decode step of 32"),
        # the same for packed prompts; a quarter of each head unrotated, pairs interleaved
        _case("rope", GPT_OSS, 5, 4096, 4096, rot=48, interleaved=True, dtype="f16", lens=2, name="rope, packed prompts"),
        # one user's decoding step on a short context: latency
        _case("attention", LLAMA, 1, 1, 1000, name="decode 1 x 1000"),
        # a decoding step of a busy server, contexts of all lengths
        _case("attention", LLAMA, 32, 1, 16384, lens=3, name="decode 32 x 16K ragged"),
        # a decoding step on a long context with attention sinks
        _case("attention", GPT_OSS, 1, 1, LONGEST, sinks=True, name="decode 1 x 128K, sinks"),
        # a question about a long document whose cache was just retrieved: the largest case
        _case("attention", LLAMA, 1, 512, LONGEST, name="chunk of 512 over 128K"),
        # prompts of several users, packed
        _case("attention", QWEN3, 6, 4096, 4096, lens=4, name="packed prompts of up to 4096"),
        # chunked prefill of a windowed layer; odd head size, three heads to a KV head, pages of 8
        _case("attention", (15, 5, 80), 3, 777, 9001, window=1024, dtype="f16", block=8, lens=5,
              name="windowed chunks, odd shape"),
        # the weight that a decoding step gives to the cached tokens
        _case("mass", LLAMA, 8, 1, 16384, lens=6, name="mass, decode 8 x 16K"),
        # the weight from the last queries of a prompt over a long context
        _case("mass", QWEN3, 1, 256, LONGEST, last=256, name="mass, 256 over 128K"),
        # a decoding batch goes back to its budget after 64 new tokens
        _case("evict", LLAMA, 16, 64, 2048 + 64, keep=2048, recent=128, name="evict 64 of 2112 x 16"),
        # a long context is cut to a sixteenth after its prompt
        _case("evict", GPT_OSS, 1, 1, LONGEST, keep=8192, recent=1024, name="evict 128K to 8K"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(("rope", "attention", "attention", "attention", "mass", "evict"))
        group = rng.choice((1, 2, 3, 4, 7, 8))
        kv_heads = rng.choice((1, 2, 4, 5, 8))
        shape = rng.choice((LLAMA, GPT_OSS, QWEN3, (group * kv_heads, kv_heads, rng.choice((64, 80, 96, 112, 128)))))
        kind = rng.choice(("decode", "chunk", "prompt"))
        kv = _log(rng, 16, LONGEST)
        n_seq = _log(rng, 1, 64)
        new = {"decode": 1, "chunk": _log(rng, 2, 2048), "prompt": kv}[kind]
        more = {"dtype": rng.choice(("bf16", "bf16", "f16")), "block": rng.choice((16, 16, 8, 32)),
                "lens": rng.randint(0, 1 << 20)}
        if op == "rope":
            more.update(rot=rng.choice((shape[2], shape[2] // 2)), interleaved=rng.random() < 0.5)
        elif op == "evict":
            more.update(keep=_log(rng, 1, kv), recent=rng.choice((0, 16, 128)))
        else:
            more.update(window=rng.choice((0, 0, 0, 128, _log(rng, 1, 8192))))
            if op == "attention":
                more.update(sinks=rng.random() < 0.25)
            else:
                more.update(last=rng.choice((0, 1, 32, 256)))
        case = _case(op, shape, n_seq, min(new, kv), kv, **more)
        need = work(case)
        if (need["flops"] <= MOST_FLOPS and 1 << 16 <= need["bytes"] <= MOST_BYTES and n_seq * kv <= 1 << 19
                and n_seq * shape[0] * case["new"] * kv <= MOST_SCORES):
            return case


def _lengths(case):
    """(new tokens, cached ones with them) of every sequence: the first has the most, the others an eighth or more."""
    rng = random.Random(case["lens"])
    out = []
    for i in range(case["n_seq"]):
        share = 1.0 if i == 0 or not case["lens"] else math.exp(rng.uniform(math.log(0.125), 0.0))
        kv = max(1, int(case["kv"] * share))
        new = kv if case["new"] == case["kv"] else min(kv, max(1, int(case["new"] * share)))
        out.append((new, kv))
    return out


def _pairs(case, new, kv):
    """Query-key pairs of one head of one sequence."""
    first = kv - min(new, case["last"] or new) if case["op"] == "mass" else kv - new
    seen = range(first + 1, kv + 1)                  # what each query sees without a window
    w = case["window"]
    if not w or w >= kv:
        return (seen.start + kv) * len(seen) // 2
    short = max(0, min(kv, w) - first)               # queries that see less than a window
    return (first + 1 + first + short) * short // 2 + (len(seen) - short) * w


def _dtype(case):
    return {"bf16": torch.bfloat16, "f16": torch.float16}[case["dtype"]]


def prepare(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    lens, bs, dev = _lengths(case), case["block"], "cuda"
    h, hk, d, n = case["heads"], case["kv_heads"], case["head_dim"], case["n_seq"]
    dtype = _dtype(case)
    stride = -(-case["kv"] // bs)
    blocks = [-(-kv // bs) for _, kv in lens]
    slots = sum(blocks) + sum(blocks) // 4 + 1       # a fifth of the cache belongs to others
    free = rng.permutation(slots)
    table, at = np.full((n, stride), -1, np.int32), 0
    for i, b in enumerate(blocks):
        table[i, :b] = free[at:at + b]
        at += b
    cu = np.concatenate([[0], np.cumsum([new for new, _ in lens])]).astype(np.int32)
    total = int(cu[-1])

    def normal(*size, std=1.0, to=dtype):
        return torch.empty(size, dtype=torch.float32, device=dev).normal_(0.0, std, generator=gen).to(to)

    s = dict(case, total=total, slots=slots, stride=stride, scale=d ** -0.5,
             cu=torch.from_numpy(cu).to(dev), kv_len=torch.tensor([kv for _, kv in lens], dtype=torch.int32, device=dev),
             table=torch.from_numpy(table).to(dev))
    s["k_cache"] = normal(slots, hk, bs, d)
    s["v_cache"] = normal(slots, hk, bs, d)
    if case["op"] == "rope":
        qkv = normal(total, h + 2 * hk, d)           # as one projection writes them
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h:h + hk], qkv[:, h + hk:]
        turn = torch.arange(case["kv"], dtype=torch.float64)[:, None] * 500000.0 ** (
            -torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])
        s["angles"] = torch.stack([turn.cos(), turn.sin()], -1).float().contiguous().to(dev)
        at = np.concatenate([np.arange(kv - new, kv) for new, kv in lens]).astype(np.int32)
        s["positions"] = torch.from_numpy(at).to(dev)
        s["q_out"] = torch.empty(total, h, d, dtype=dtype, device=dev)
        s["pos"] = torch.full((n, hk, case["kv"]), -1, dtype=torch.int32, device=dev)
    elif case["op"] in ("attention", "mass"):
        s["q"] = normal(total, h, d, std=2.0)
        if case["sinks"]:
            s["sinks"] = normal(h, std=2.0, to=torch.float32)
        if case["op"] == "attention":
            s["out"] = torch.empty(total, h, d, dtype=dtype, device=dev)
            s["lse"] = torch.empty(h, total, dtype=torch.float32, device=dev)
        else:
            s["score_in"] = normal(n, hk, case["kv"], to=torch.float32).abs_()
            s["score"] = torch.zeros_like(s["score_in"])
            s["lse"] = _attend(s, values=False)[1]   # the attention before it left these
    else:
        # a sum over many queries, with equal values among the tokens that none looked at
        s["score_in"] = normal(n, hk, case["kv"], std=3.0, to=torch.float32).exp_().mul_(64.0).floor_().div_(64.0)
        s["pos_in"] = torch.arange(case["kv"], dtype=torch.int32, device=dev).repeat(n, hk, 1)
        s["score"], s["pos"] = torch.zeros_like(s["score_in"]), torch.zeros_like(s["pos_in"])
        s["keeps"] = torch.full((n,), case["keep"], dtype=torch.int32, device=dev)
        s["protect"] = s["kv_len"] - case["recent"]
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
    need = {"attention": K.attention_workspace, "evict": K.evict_workspace}.get(s["op"])
    s["work"] = torch.empty(max(16, need(s["shape"], s["batch"]) if need else 0), dtype=torch.uint8, device="cuda")


def _run_own(s):
    from paper_2606_14779_amd import kvpool as K
    stream = torch.cuda.current_stream().cuda_stream
    shape, batch = s["shape"], s["batch"]
    k_cache, v_cache = s["k_cache"].data_ptr(), s["v_cache"].data_ptr()
    if s["op"] == "rope":
        K.rope_append(shape, batch, s["angles"].data_ptr(), s["angles"].shape[0], s["rot"], s["positions"].data_ptr(),
                      s["k"].data_ptr(), s["k"].stride(0), s["v"].data_ptr(), s["v"].stride(0), k_cache, v_cache,
                      q=s["q"].data_ptr(), q_stride=s["q"].stride(0), q_out=s["q_out"].data_ptr(),
                      q_out_stride=s["q_out"].stride(0), pos=s["pos"].data_ptr(), pos_stride=s["kv"],
                      interleaved=s["interleaved"], stream=stream)
        return s["q_out"], s["k_cache"], s["v_cache"], s["pos"]
    if s["op"] == "attention":
        sinks = s["sinks"].data_ptr() if s["sinks"] is not False else 0
        K.attention(shape, batch, s["q"].data_ptr(), s["q"].stride(0), k_cache, v_cache, s["scale"], s["out"].data_ptr(),
                    s["out"].stride(0), window=s["window"], sinks=sinks, lse=s["lse"].data_ptr(),
                    workspace=s["work"].data_ptr(), workspace_bytes=s["work"].numel(), stream=stream)
        return s["out"], s["lse"]
    if s["op"] == "mass":
        K.attention_mass(shape, batch, s["q"].data_ptr(), s["q"].stride(0), k_cache, s["scale"], s["lse"].data_ptr(),
                         s["score_in"].data_ptr(), s["score"].data_ptr(), s["kv"], window=s["window"], last=s["last"],
                         stream=stream)
        return s["score"]
    K.evict(shape, batch, s["keeps"].data_ptr(), s["score_in"].data_ptr(), s["score"].data_ptr(), s["kv"], k_cache, v_cache,
            s["len_out"].data_ptr(), s["work"].data_ptr(), s["work"].numel(), protect=s["protect"].data_ptr(),
            pos_in=s["pos_in"].data_ptr(), pos_out=s["pos"].data_ptr(), pos_stride=s["kv"], stream=stream)
    return s["k_cache"], s["v_cache"], s["score"], s["pos"], s["len_out"]


# ---- the plain forms

def _rows(s):
    """Sequence and cache index of every packed new token."""
    row = torch.arange(s["total"], device="cuda")
    seq = torch.bucketize(row, s["cu"][1:].long(), right=True)
    return seq, s["kv_len"][seq].long() - s["cu"][seq + 1] + row


def _rope(s):
    seq, at = _rows(s)
    cos, sin = s["angles"][s["positions"].long()].unbind(-1)
    cos, sin, rot = cos[:, None], sin[:, None], s["rot"]

    def turned(x):
        x = x.float()
        a, b = (x[..., :rot:2], x[..., 1:rot:2]) if s["interleaved"] else (x[..., :rot // 2], x[..., rot // 2:rot])
        pair = a * cos - b * sin, b * cos + a * sin
        pair = torch.stack(pair, -1).flatten(-2) if s["interleaved"] else torch.cat(pair, -1)
        return torch.cat([pair, x[..., rot:]], -1).to(_dtype(s))

    slot, off = s["table"][seq, at // s["block"]].long(), at % s["block"]
    s["q_out"].copy_(turned(s["q"]))
    s["k_cache"][slot, :, off] = turned(s["k"])
    s["v_cache"][slot, :, off] = s["v"]
    s["pos"][seq, :, at] = s["positions"][:, None].expand(-1, s["kv_heads"])
    return s["q_out"], s["k_cache"], s["v_cache"], s["pos"]


def _tokens(s, cache):
    """A cache's tokens by sequence and KV head, padded, in 32 bits: [n_seq][kv_heads][tokens][head_dim]."""
    pages = cache[s["table"].clamp(min=0).long()].permute(0, 2, 1, 3, 4)
    return pages.reshape(s["n_seq"], s["kv_heads"], -1, s["head_dim"])[:, :, :s["kv"]].float().contiguous()


def _logits(s):
    """Masked logits [n_seq][kv_heads][group * new][tokens], queries padded to the longest sequence's."""
    n, hk, new = s["n_seq"], s["kv_heads"], s["new"]
    row = torch.arange(new, device="cuda")
    n_q = s["cu"][1:] - s["cu"][:-1]
    at = (s["cu"][:-1, None] + row).clamp(max=s["total"] - 1).long()
    q = s["q"][at].float().permute(0, 2, 1, 3).reshape(n, hk, -1, s["head_dim"])
    logits = torch.matmul(q, _tokens(s, s["k_cache"]).transpose(2, 3).contiguous()).mul_(s["scale"])
    end = (s["kv_len"] - n_q)[:, None, None] + row[:, None]           # cache index of each query
    token = torch.arange(s["kv"], device="cuda")
    hidden = (token > end) | (row[:, None] >= n_q[:, None, None])
    if s["window"]:
        hidden |= token <= end - s["window"]
    view = logits.view(n, hk, -1, new, s["kv"])
    view.masked_fill_(hidden[:, None, None], -math.inf)
    return logits, n_q


def _attend(s, values=True):
    n, h, new, total = s["n_seq"], s["heads"], s["new"], s["total"]
    logits, _ = _logits(s)
    top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
    if s["sinks"] is not False:
        sink = s["sinks"].view(s["kv_heads"], -1, 1).expand(-1, -1, new).reshape(1, s["kv_heads"], -1, 1)
        top = torch.maximum(top, sink)
    weights = logits.sub_(top).exp_()
    weight = weights.sum(-1, keepdim=True)
    if s["sinks"] is not False:
        weight = weight + (sink - top).exp()
    seq, at = _rows(s)
    row = at - s["kv_len"][seq] + s["cu"][seq + 1] - s["cu"][seq]
    lse = (weight.log() + top).view(n, h, new)[seq, :, row].t().contiguous()
    if not values:
        return None, lse
    out = torch.matmul(weights, _tokens(s, s["v_cache"])).div_(weight).view(n, h, new, -1)
    return out[seq, :, row].to(_dtype(s)), lse


def _mass(s):
    n, hk, new = s["n_seq"], s["kv_heads"], s["new"]
    logits, n_q = _logits(s)
    row = torch.arange(new, device="cuda")
    at = (s["cu"][:-1, None] + row).clamp(max=s["total"] - 1).long()
    lse = s["lse"][:, at].permute(1, 0, 2).reshape(n, hk, -1, 1)
    weights = logits.sub_(lse).exp_().view(n, hk, -1, new, s["kv"])
    if s["last"]:
        weights.mul_((row >= n_q[:, None] - s["last"]).view(n, 1, 1, new, 1))
    live = torch.arange(s["kv"], device="cuda") < s["kv_len"][:, None, None]
    s["score"].copy_(torch.where(live, s["score_in"] + weights.sum((2, 3)), s["score"]))
    return s["score"]


def _evict(s):
    token = torch.arange(s["kv"], device="cuda").expand_as(s["score_in"])
    length, keep = s["kv_len"][:, None, None], s["keeps"][:, None, None]
    key = s["score_in"].masked_fill(s["pos_in"] >= s["protect"][:, None, None], math.inf)
    key = key.masked_fill(token >= length, -math.inf)
    order = key.sort(stable=True, dim=-1, descending=True).indices
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(2, order, (token < keep).contiguous()) & (token < length)
    hole = ~kept & (token < torch.minimum(keep, length))
    movers = torch.where(kept & (token >= keep), token, s["kv"]).sort(-1).values
    of = torch.where(hole, movers.gather(2, (hole.cumsum(-1) - 1).clamp(min=0)), token)
    heads = torch.arange(s["kv_heads"], device="cuda")[:, None]
    seq = torch.arange(s["n_seq"], device="cuda")[:, None, None]

    def places(at):
        return s["table"].long()[seq, at // s["block"]], heads.expand_as(at), at % s["block"]

    to = torch.where(token < length, token, 0)[:, :, :min(s["keep"], s["kv"])]   # past the end: token 0 once more
    came = of.gather(2, to)
    for cache in (s["k_cache"], s["v_cache"]):
        cache[places(to)] = cache[places(came)]
    live, left = token < length, token < keep
    s["score"].copy_(torch.where(live, torch.where(left, s["score_in"].gather(2, of), 0.0), s["score"]))
    s["pos"].copy_(torch.where(live & left, s["pos_in"].gather(2, of), s["pos"]))
    s["len_out"].copy_(torch.minimum(s["kv_len"], s["keeps"]))
    return s["k_cache"], s["v_cache"], s["score"], s["pos"], s["len_out"]


def run(state):
    if own:
        return _run_own(state)
    return {"rope": _rope, "attention": _attend, "mass": _mass, "evict": _evict}[state["op"]](state)


# ---- from the definitions, in 64 bits, one sequence and head at a time

def _cache_index(s, i, count):
    """Slot and offset of the first tokens of a sequence, from its block table row."""
    slots = np.repeat(s["table"][i].cpu().numpy().astype(np.int64), s["block"])[:count]
    return torch.from_numpy(slots).cuda(), torch.arange(count, device="cuda") % s["block"]


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"rope": _exact_rope, "attention": _exact_attention, "mass": _exact_mass, "evict": _exact_evict}[s["op"]](s)


def _exact_rope(s):
    rot, half = s["rot"], s["rot"] // 2
    first = list(range(0, rot, 2)) if s["interleaved"] else list(range(half))
    second = [i + 1 for i in first] if s["interleaved"] else [i + half for i in first]
    turn = torch.view_as_complex(s["angles"].double().contiguous())[s["positions"].long()][:, None]

    def turned(x):
        x = x.double().clone()
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    q, k, pos = turned(s["q"]), turned(s["k"]), s["pos"].clone()
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    for i, (new, kv) in enumerate(_lengths(s)):
        rows = slice(int(s["cu"][i]), int(s["cu"][i]) + new)
        slot, off = (x[kv - new:] for x in _cache_index(s, i, kv))
        k_cache[slot, :, off], v_cache[slot, :, off] = k[rows], s["v"][rows].double()
        pos[i, :, kv - new:kv] = s["positions"][rows]
    return q, k_cache, v_cache, pos


def _exact_rows(s, i, head, new, kv):
    """Logits of one head's last `new` queries of a sequence over its `kv` tokens, hidden ones at -inf."""
    slot, off = _cache_index(s, i, kv)
    end = int(s["cu"][i + 1])
    q = s["q"][end - new:end, head].double()
    k = s["k_cache"][slot, head // (s["heads"] // s["kv_heads"]), off].double()
    z = (q @ k.t().contiguous()) * s["scale"]
    ahead = torch.arange(kv, device="cuda")[None] - torch.arange(kv - new, kv, device="cuda")[:, None]
    z[ahead > 0] = -math.inf
    if s["window"]:
        z[ahead <= -s["window"]] = -math.inf
    return z


def _exact_attention(s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["heads"], s["total"], dtype=torch.float64, device="cuda")
    for i, (new, kv) in enumerate(_lengths(s)):
        slot, off = _cache_index(s, i, kv)
        rows = slice(int(s["cu"][i]), int(s["cu"][i + 1]))
        for head in range(s["heads"]):
            z = _exact_rows(s, i, head, new, kv)
            if s["sinks"] is not False:              # one more key, without a value
                z = torch.cat([z, s["sinks"][head].double().expand(new, 1)], 1)
            lse[head, rows] = torch.logsumexp(z, 1)
            v = s["v_cache"][slot, head // (s["heads"] // s["kv_heads"]), off].double()
            out[rows, head] = torch.softmax(z, 1)[:, :kv] @ v
    return out, lse


def _exact_mass(s):
    score = s["score"].double()
    group = s["heads"] // s["kv_heads"]
    for i, (new, kv) in enumerate(_lengths(s)):
        count, end = min(new, s["last"] or new), int(s["cu"][i + 1])
        score[i, :, :kv] = s["score_in"][i, :, :kv].double()
        for head in range(s["heads"]):
            z = _exact_rows(s, i, head, count, kv) - s["lse"][head, end - count:end, None].double()
            score[i, head // group, :kv] += z.exp().sum(0)
    return score


def _exact_evict(s):
    k_cache, v_cache = s["k_cache"].clone(), s["v_cache"].clone()
    score_in, pos_in = s["score_in"].cpu().numpy(), s["pos_in"].cpu().numpy()
    score, pos, keep = s["score"].cpu().numpy().astype(np.float64), s["pos"].cpu().numpy(), s["keep"]
    left = []
    for i, (_, kv) in enumerate(_lengths(s)):
        left.append(min(kv, keep))
        slot, off = _cache_index(s, i, kv)
        for head in range(s["kv_heads"]):
            guarded = pos_in[i, head, :kv] >= int(s["protect"][i])
            best = np.lexsort((np.arange(kv), -score_in[i, head, :kv].astype(np.float64), ~guarded))[:keep]
            stay, come = np.sort(best[best < keep]), np.sort(best[best >= keep])
            holes = np.setdiff1d(np.arange(min(kv, keep)), stay)
            source = np.arange(kv)
            source[holes] = come
            score[i, head, :kv] = np.where(np.arange(kv) < keep, score_in[i, head, source], 0.0)
            pos[i, head, :left[-1]] = pos_in[i, head, source[:left[-1]]]
            a, b = torch.from_numpy(holes).cuda(), torch.from_numpy(come).cuda()
            for cache in (k_cache, v_cache):
                cache[slot[a], head, off[a]] = cache[slot[b], head, off[b]]
    return (k_cache, v_cache, torch.from_numpy(score).cuda(), torch.from_numpy(pos).cuda(),
            torch.tensor(left, dtype=torch.int32, device="cuda"))


def work(case):
    h, hk, d, e = case["heads"], case["kv_heads"], case["head_dim"], 2
    lens = _lengths(case)
    new, kv = sum(n for n, _ in lens), sum(n for _, n in lens)
    pairs = sum(_pairs(case, n, m) for n, m in lens)
    if case["op"] == "rope":
        moved = new * (h + 2 * hk) * d * e
        return {"bytes": 2 * moved + new * (4 * case["rot"] + 4 + 4 * hk), "flops": 3 * new * (h + hk) * case["rot"]}
    if case["window"]:                               # the tokens that some query sees
        kv = sum(min(m, n - 1 + case["window"]) for n, m in lens)
    if case["op"] == "attention":
        return {"bytes": 2 * new * h * d * e + 4 * h * new + 2 * kv * hk * d * e, "flops": 4 * d * h * pairs}
    if case["op"] == "mass":
        asked = sum(min(n, case["last"] or n) for n, _ in lens)
        every = sum(m for _, m in lens)
        return {"bytes": asked * h * (d * e + 4) + kv * hk * d * e + 8 * every * hk, "flops": 2 * d * h * pairs}
    # which tokens move depends on the scores: where these are spread evenly, the share of the kept ones past `keep`
    moved = sum(min(m, case["keep"]) * max(0, m - case["keep"]) // m for _, m in lens)
    return {"bytes": hk * (8 * kv + 4 * kv + 4 * sum(min(m, case["keep"]) for _, m in lens) + 4 * moved * d * e), "flops": 0}
