"""The measured work of a decode step that verifies drafted tokens over a paged
bf16 KV cache, and the same results in plain torch.

Every sequence of a batch holds ``context`` tokens and gets n new ones, its
nodes: rows of a packed array, in the order of their slots in the cache.  Node 0
is the sequence's newest token, the others are drafts, each the child of an
earlier node (a chain, or a tree); a prompt is a chain too.

Four kinds of pass:

  append   the nodes' queries and keys are rotated to their positions and keys
           and values written into the cache (for a tree: its ancestor bits and
           positions first)
  attend   the nodes' queries attend to the context, to their ancestors and to
           themselves
  accept   the drafts are verified against the target's probabilities, and the
           accepted nodes' keys and values move up to the context's end
  step     all of these in a row

Rotation.  Pair i of the first ``rot`` dims of a head (dims i and i + rot/2, or
2i and 2i + 1) turns by position * freqs[i] radians and is multiplied by a
factor.  A node's position is its context plus its depth.

Verification.  From node 0 on, the children of the current node are tried in
order.  With draft probabilities q (the children were drawn from them) a child
of token x is accepted if u q(x) F < p(x) - a q(x), with a = 0 and F = 1 for the
first; after each rejection a grows by F, and F becomes the sum over the
vocabulary of max(p - a q, 0).  Without them (the drafts are what they are) it
is accepted if u R < p(x), R = 1 less what the rejected siblings' tokens have.
The first child accepted becomes the current node.  Where none is, the next
token is drawn from max(p - a q, 0), or from p without the rejected tokens: the
first token where the running sum passes the last random number times the total.

Head shapes, contexts and pages are those of this repository's workloads and
measured calls (32/8, 64/8 and 8/2 heads, up to 64K tokens).
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
MAX_BYTES = 4_500_000_000           # cache bytes that a drawn case attends to
MAX_FLOPS = 2.0e12


def _case(name, **kw):
    case = {
        "kind": "attend", "batch": 1, "kv_heads": 8, "group": 4, "page": 64,
        # tokens that each sequence holds, and its nodes
        "len_lo": 4096, "len_hi": 4096, "new_lo": 1, "new_hi": 1, "len_seed": 0,
        "tree": True,               # False: a chain
        "interleaved": False,       # pairs of dims 2i, 2i + 1; else i, i + rot/2
        "rot": 128,                 # dims that are rotated
        "factor": 1.0,              # positions are divided by it (longer contexts)
        "rows": "bf16",             # type of the new queries, keys and values
        "bf16_out": True,
        "vocab": 0, "probs": "f32",
        "sampled": False,           # the drafts were drawn from given probabilities
    }
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token of one request: the write of a plain decode step, all latency
        _case("append_one", kind="append", kv_heads=2, len_lo=1000, len_hi=1000, tree=False),
        # small trees of a decode batch, pages of 16 tokens
        _case("append_64_trees", kind="append", batch=64, group=8, page=16, len_lo=100, len_hi=30000,
              len_seed=3, new_lo=5, new_hi=16, interleaved=True),
        # a prefill batch: ragged prompts behind short contexts, half of each head
        # rotated, positions scaled for a long context
        _case("append_prompts", kind="append", batch=8, len_lo=0, len_hi=2000, len_seed=8, new_lo=500,
              new_hi=16384, tree=False, rot=64, factor=4.0),
        # a request with two KV heads and a short chain of drafts
        _case("attend_one_4k", kv_heads=2, new_lo=4, new_hi=4, tree=False, bf16_out=False),
        # a chat batch: short ragged contexts, trees of any size, pages of 16 tokens
        _case("attend_chat_ragged_2k", batch=16, page=16, len_lo=0, len_hi=2048, len_seed=5, new_lo=1,
              new_hi=33, bf16_out=False),
        # an 8B-shaped layer at batch 8, trees of 16
        _case("attend_8x32k", batch=8, len_lo=32768, len_hi=32768, new_lo=16, new_hi=16, len_seed=6),
        # the headline batch: 64/8 heads, ragged 8K to 64K, chains of 8
        _case("attend_ragged_64k", batch=32, group=8, len_lo=8192, len_hi=65536, len_seed=4, new_lo=8,
              new_hi=8, tree=False),
        # wide trees: enough rows a head for the matrix cores to be the bound
        _case("attend_wide_trees", batch=8, group=8, page=128, len_lo=8000, len_hi=16384, len_seed=9,
              new_lo=200, new_hi=256),
        # a chunk of two long prompts behind what the cache holds already
        _case("attend_prompt_chunk", batch=2, len_lo=14000, len_hi=16384, len_seed=10, new_lo=3500,
              new_hi=4096, tree=False),
        # sampled chains of 8 against a large vocabulary
        _case("accept_chains", kind="accept", batch=32, new_lo=9, new_hi=9, tree=False, vocab=128000,
              sampled=True, len_lo=100, len_hi=4000, len_seed=11),
        # trees of the likeliest drafts, 16-bit probabilities, an odd vocabulary
        _case("accept_trees", kind="accept", batch=48, kv_heads=4, page=16, new_lo=17, new_hi=64,
              vocab=32001, probs="bf16", len_lo=0, len_hi=3000, len_seed=12),
        # all calls of a step on the 8B-shaped layer
        _case("step_8x32k", kind="step", batch=8, len_lo=30000, len_hi=32700, new_lo=16, new_hi=16,
              vocab=32000, len_seed=13),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["append"] * 2 + ["attend"] * 5 + ["accept"] * 2 + ["step"])
    group = rng.choice([1, 2, 3, 4, 4, 4, 5, 8, 8, 16])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    batch = _log_int(rng, 1, 48)
    tree = rng.random() < 0.6
    case = dict(kind=kind, batch=batch, kv_heads=kv_heads, group=group, tree=tree,
                page=rng.choice([16, 32, 64, 64, 128, 256]), len_seed=rng.randrange(1, 1 << 20),
                interleaved=rng.random() < 0.4, rot=rng.choice([128, 128, 96, 64, 32, 20]),
                factor=rng.choice([1.0, 1.0, 4.0]))
    rows = 256 if tree else 4096
    if kind == "append":
        heads = kv_heads * (group + 2)
        hi = _log_int(rng, 1, max(1, min(rows, 3_000_000 // (batch * heads))))
        case.update(rows=rng.choice(["bf16", "bf16", "f16", "f32"]), new_hi=hi,
                    new_lo=hi if rng.random() < 0.3 else max(1, int(hi * rng.uniform(0, 0.9))),
                    len_lo=0, len_hi=_log_int(rng, 1, 3000))
        return _case(None, **case)
    if kind == "accept":
        vocab = _log_int(rng, 1000, 130000)
        hi = _log_int(rng, 2, max(2, min(64, 40_000_000 // (vocab * batch))))
        case.update(group=1, vocab=vocab, new_lo=max(1, int(hi * rng.uniform(0.3, 1))), new_hi=hi,
                    sampled=rng.random() < 0.5, probs=rng.choice(["f32", "f32", "bf16", "f16"]),
                    len_lo=0, len_hi=_log_int(rng, 1, 3000))
        return _case(None, **case)
    row = kv_heads * D * 4                     # cache bytes of a token
    hi = _log_int(rng, 64, min(131072, MAX_BYTES // (batch * row)))
    lo = hi if rng.random() < 0.4 else int(hi * rng.uniform(0, 0.9))
    per = batch * kv_heads * group * D * 4.0
    new = _log_int(rng, 1, max(1, min(rows if kind == "attend" else 64, int(MAX_FLOPS / (per * (hi + 500))))))
    case.update(len_lo=lo, len_hi=hi, new_hi=new, new_lo=max(1, int(new * rng.uniform(0.2, 1))),
                bf16_out=kind == "step" or rng.random() < 0.7)
    if kind == "step":
        case.update(vocab=_log_int(rng, 1000, max(1001, min(64000, 40_000_000 // (batch * new)))),
                    sampled=rng.random() < 0.3)
    return _case(None, **case)


def _lengths(case):
    """(tokens held, nodes) of every sequence."""
    rng = random.Random(case["len_seed"])
    held = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["batch"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    return held, new


def _parents(case, new):
    """The parent of every node, sequence after sequence (-1 for node 0)."""
    rng = random.Random(case["len_seed"] + 1)
    if not case["tree"]:
        return [i - 1 for n in new for i in range(n)]
    return [rng.randint((i - 1) // 3, i - 1) if i else -1 for n in new for i in range(n)]


# ---- inputs -------------------------------------------------------------------

def prepare(case, seed):
    held, new = _lengths(case)
    batch, heads, group, page = case["batch"], case["kv_heads"], case["group"], case["page"]
    kind, count = case["kind"], sum(new)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pages_of = [-(-(a + b) // page) for a, b in zip(held, new)]
    width, pages = max(pages_of), sum(pages_of)
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.zeros((batch, width), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages_of):
        table[b, :n] = order[at: at + n]
        at += n
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    parents = _parents(case, new)
    state = {"case": case, "table": table, "context": as_int(held), "offsets": as_int(offsets),
             "parents": as_int(parents), "count": count, "most": max(new)}
    q = normal(count, heads * group, D)
    k, v = normal(pages, heads, page, D).bfloat16(), normal(pages, heads, page, D).bfloat16()
    if kind in ("attend", "step"):
        # sinks at the first tokens, needles anywhere: keys along the queries of node 0
        u = q[state["offsets"][:-1].long()].view(batch, heads, group, D).sum(2)
        u = 3.0 * math.sqrt(D) * u / u.norm(dim=-1, keepdim=True)
        rng = random.Random(seed)
        for b, n in enumerate(held):
            if n:
                where = torch.tensor(list(range(min(4, n))) + [rng.randrange(n) for _ in range(8)], device="cuda")
                k[table[b, where // page].long(), :, where % page] += u[b].bfloat16()
    state["k"], state["v"] = k, v
    if kind != "accept":
        state["q"] = q.to(TYPES[case["rows"]])
    if kind in ("append", "step"):
        state["new_k"], state["new_v"] = (normal(count, heads, D).to(TYPES[case["rows"]]) for _ in range(2))
        half = case["rot"] // 2
        state["freqs"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half) / case["factor"]
    if kind == "attend":
        # a program lays a tree out once, and attends to it in every layer
        state["mask"] = _ancestors(state)[0] if case["tree"] else None
    if kind in ("accept", "step"):
        vocab, probs = case["vocab"], TYPES[case["probs"]]
        target = 4.0 * normal(count, vocab)
        guess = target + 0.8 * normal(count, vocab)
        tokens = torch.randint(vocab, (count,), generator=gen, device="cuda")
        row0 = [o for o, n in zip(offsets, new) for _ in range(n)]
        inner = [r for r in range(count) if parents[r] >= 0]
        if inner:
            source = [row0[r] + parents[r] for r in inner]
            if case["sampled"]:
                rows = torch.softmax(guess, -1).to(probs).float()[source]
                drawn = torch.multinomial(rows, 1, generator=gen)[:, 0]
            else:
                # the j-th child of a node has its j-th likeliest guess
                nth, seen = [], {}
                for s in source:
                    nth.append(seen.get(s, 0))
                    seen[s] = nth[-1] + 1
                best = guess.topk(min(vocab, max(nth) + 1), dim=-1).indices
                drawn = best[torch.tensor(source, device="cuda"), torch.tensor(nth, device="cuda")]
            tokens[torch.tensor(inner, device="cuda")] = drawn
        state["target"] = torch.softmax(target, -1).to(probs)
        state["draft"] = torch.softmax(guess, -1).to(probs) if case["sampled"] else None
        state["tokens"] = tokens.int()
        state["uniforms"] = torch.rand(count, generator=gen, device="cuda")
        state["last"] = torch.rand(batch, generator=gen, device="cuda")
    return state


# ---- the passes ----------------------------------------------------------------

def run(state):
    case, result = state["case"], {}
    kind = case["kind"]
    q, mask, positions = state.get("q"), state.get("mask"), None
    if kind in ("append", "step"):
        if case["tree"]:
            result["mask"], result["positions"] = mask, positions = _layout(state)
        result["q"] = q = _append(state, positions)
    if kind in ("attend", "step"):
        result["out"], result["lse"] = _attend(state, q, mask)
    if kind in ("accept", "step"):
        result["accepted"], result["counts"], result["next"] = _verify(state)
        _keep(state, result["accepted"], result["counts"])
    if kind != "attend":
        result["k"], result["v"] = state["k"], state["v"]
    return result


def _owner(state):
    """The sequence of every row, and the row's place in it."""
    r = torch.arange(state["count"], device="cuda")
    b = torch.searchsorted(state["offsets"][1:].contiguous(), r.int(), right=True)
    return b, r - state["offsets"].long()[b]


def _ancestors(state):
    """Bits of every node's ancestors and itself [rows][words], and its depth."""
    b, i = _owner(state)
    first = state["offsets"].long()[b]
    words = -(-state["most"] // 64)
    sees = torch.zeros((state["count"], 64 * words), dtype=torch.bool, device="cuda")
    depth = torch.zeros(state["count"], dtype=torch.int64, device="cuda")
    parents = state["parents"].long()
    at = i
    for _ in range(state["most"]):                 # a step up for every node at once
        live = at >= 0
        sees[torch.nonzero(live)[:, 0], at[live]] = True
        at = torch.where(live, parents[first + at.clamp_min(0)], at)
        depth += at >= 0
    bits = torch.ones(64, dtype=torch.int64, device="cuda") << torch.arange(64, device="cuda")
    return (sees.view(-1, words, 64) * bits).sum(-1), depth


def _layout(state):
    if own:
        from paper_2606_00024_amd import api
        return api.tree_layout(state["parents"], state["context"], token_offsets=state["offsets"],
                               mask_words=-(-state["most"] // 64))
    mask, depth = _ancestors(state)
    return mask, (state["context"].long()[_owner(state)[0]] + depth).int()


def _mscale(case):
    """The factor on rotated values that goes with positions divided by `factor`."""
    return 0.1 * math.log(case["factor"]) + 1.0


def _append(state, positions):
    case = state["case"]
    if own:
        from paper_2606_00024_amd import api
        rope = api.Rope(state["freqs"], "interleaved" if case["interleaved"] else "half", _mscale(case))
        return api.rope_append(state["k"], state["v"], state["new_k"], state["new_v"], state["table"],
                               state["context"], rope=rope, q=state["q"], token_offsets=state["offsets"],
                               row_positions=positions)
    b, i = _owner(state)
    slot = state["context"].long()[b] + i
    angle = (slot if positions is None else positions).double()[:, None] * state["freqs"]
    # cosines and sines in 64 bits (far positions lose them in 32), then rounded
    cos, sin = ((f(angle) * _mscale(case)).float()[:, None] for f in (torch.cos, torch.sin))

    def rotated(x):
        x, rot = x.float(), case["rot"]
        y = x.clone()
        if case["interleaved"]:
            a, c = x[..., 0:rot:2], x[..., 1:rot:2]
            y[..., 0:rot:2], y[..., 1:rot:2] = a * cos - c * sin, c * cos + a * sin
        else:
            a, c = x[..., : rot // 2], x[..., rot // 2: rot]
            y[..., : rot // 2], y[..., rot // 2: rot] = a * cos - c * sin, c * cos + a * sin
        return y.bfloat16()

    pages, slots = state["table"][b, slot // case["page"]].long(), slot % case["page"]
    state["k"][pages, :, slots] = rotated(state["new_k"])
    state["v"][pages, :, slots] = state["new_v"].bfloat16()
    return rotated(state["q"])


def _attend(state, q, mask):
    case = state["case"]
    out_type = torch.bfloat16 if case["bf16_out"] else torch.float32
    if own:
        from paper_2606_00024_amd import api
        return api.tree_attention(q, state["k"], state["v"], state["table"], state["context"], mask=mask,
                                  token_offsets=state["offsets"], out_dtype=out_type)
    batch, heads, group, most = case["batch"], case["kv_heads"], case["group"], state["most"]
    b, i = _owner(state)
    context, new = state["context"].long(), (state["offsets"][1:] - state["offsets"][:-1]).long()
    tokens = state["table"].shape[1] * case["page"]

    def gathered(pool):                                                  # [batch * heads][tokens][128]
        return pool[state["table"].long()].permute(0, 2, 1, 3, 4).reshape(batch * heads, tokens, D).float()

    padded = torch.zeros((batch, most, heads, group, D), device="cuda")
    padded[b, i] = q.float().view(-1, heads, group, D)
    padded = padded.transpose(1, 2).reshape(batch * heads, most * group, D)
    # what node i sees of nodes 0 ..: its bits, or all up to itself
    sees = torch.zeros((batch, most, most), dtype=torch.bool, device="cuda")
    j = torch.arange(most, device="cuda")
    sees[b, i] = (j <= i[:, None]) if mask is None else (mask[:, j // 64] >> (j % 64) & 1).bool()
    t = torch.arange(tokens, device="cuda")
    node = t - context[:, None]                                          # [batch][tokens]
    dead = ((node < 0)[:, None] | sees.gather(2, node.clamp(0, most - 1)[:, None].expand(-1, most, -1))
            & (node < new[:, None])[:, None]).logical_not_()             # [batch][most][tokens]
    s = torch.matmul(padded, gathered(state["k"]).transpose(1, 2).contiguous())
    s = s.mul_(SCALE).view(batch, heads, most, group, tokens)
    s.masked_fill_(dead[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, torch.zeros_like(top))
    p = s.sub_(top).exp_()
    mass = p.sum(-1, dtype=torch.float64)
    vec = torch.matmul(p.view(batch * heads, most * group, tokens), gathered(state["v"]))
    vec = vec.view(batch, heads, most, group, D) / torch.where(mass > 0, mass, torch.ones_like(mass))[..., None]
    lse = top[..., 0].double() + mass.log()
    vec, lse = vec.transpose(1, 2)[b, i], lse.transpose(1, 2)[b, i]      # back to rows
    return vec.reshape(-1, heads * group, D).to(out_type), lse.reshape(-1, heads * group).float()


def _verify(state):
    if own:
        from paper_2606_00024_amd import api
        return api.verify_drafts(state["target"], state["tokens"], state["parents"], state["uniforms"],
                                 state["last"], draft=state["draft"], token_offsets=state["offsets"],
                                 max_path=state["most"])
    batch, most, target, draft = state["case"]["batch"], state["most"], state["target"], state["draft"]
    first = state["offsets"][:-1].long()
    new = (state["offsets"][1:] - state["offsets"][:-1]).long()
    every = torch.arange(batch, device="cuda")
    now = torch.zeros(batch, dtype=torch.int64, device="cuda")
    count = torch.ones_like(now)
    accepted = torch.full((batch, most), -1, dtype=torch.int64, device="cuda")
    accepted[:, 0] = 0
    # sums over the vocabulary in 64 bits: a random number is compared with them
    a, f = (torch.full((batch,), x, dtype=torch.float64, device="cuda") for x in (0.0, 1.0))
    gone = torch.zeros((batch, target.shape[1]), dtype=torch.bool, device="cuda")
    for c in range(1, most):                       # children come after their parents
        row = first + torch.where(c < new, c, torch.zeros_like(new))
        tried = (c < new) & (state["parents"].long()[row] == now)
        token, u = state["tokens"].long()[row], state["uniforms"].double()[row]
        px = target[first + now, token].double()
        if draft is not None:
            qx = draft[first + now, token].double()
            ok = tried & (u * qx * f < (px - a * qx).clamp_min(0))
        else:
            ok = tried & (u * f < torch.where(gone[every, token], torch.zeros_like(px), px))
        lost = tried & ~ok
        if draft is not None:
            a = torch.where(lost, a + f, a)
            rest = (target[first + now].double() - a[:, None] * draft[first + now].double()).clamp_min(0).sum(-1)
            f = torch.where(lost, rest, f)
        else:
            f = torch.where(lost & ~gone[every, token], f - px, f).clamp_min(0)
            gone[every, token] |= lost
        accepted[every, torch.where(ok, count, most - 1)] = torch.where(
            ok, c, accepted[every, torch.where(ok, count, most - 1)])
        count = count + ok
        now = torch.where(ok, c, now)
        a, f = torch.where(ok, torch.zeros_like(a), a), torch.where(ok, torch.ones_like(f), f)
        gone &= ~ok[:, None]
    p = target[first + now].double()
    w = (p - a[:, None] * draft[first + now].double()).clamp_min(0) if draft is not None else p.masked_fill(gone, 0.0)
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, p)
    run_sum = w.cumsum(-1)
    after = run_sum > state["last"].double()[:, None] * run_sum[:, -1:]
    token = torch.where(after.any(-1), after.int().argmax(-1), w.shape[1] - 1 - (w.flip(-1) > 0).int().argmax(-1))
    return accepted.int(), count.int(), token.int()


def _keep(state, accepted, counts):
    if own:
        from paper_2606_00024_amd import api
        api.keep_accepted(state["k"], state["v"], state["table"], state["context"], accepted, counts)
        return
    page, table = state["case"]["page"], state["table"].long()
    j = torch.arange(accepted.shape[1], device="cuda").expand_as(accepted)
    live = j < counts[:, None]
    b = torch.nonzero(live)[:, 0]
    context = state["context"].long()[b]
    old, new = context + accepted[live].long(), context + j[live]
    for pool in (state["k"], state["v"]):
        pool[table[b, new // page], :, new % page] = pool[table[b, old // page], :, old % page]


def work(case):
    held, new = _lengths(case)
    heads, group, kind, count = case["kv_heads"], case["group"], case["kind"], sum(new)
    batch, moved, flops = case["batch"], 8 * case["batch"], 0.0
    words = -(-max(new) // 64)
    if kind in ("append", "step"):
        moved += count * D * (SIZES[case["rows"]] + 2) * heads * (group + 2)
        flops += count * 3.0 * case["rot"] * heads * (group + 1)
        if case["tree"]:
            moved += count * (4 + 4 + 8 * words)
    if kind in ("attend", "step"):
        parents, seen, at = _parents(case, new), 0, 0
        for a, n in zip(held, new):
            depth = []
            for i in range(n):
                up = parents[at + i]
                depth.append(depth[up] + 1 if up >= 0 else 1)
            seen += n * a + sum(depth)
            at += n
        moved += sum(a + n for a, n in zip(held, new)) * heads * 2 * D * 2
        moved += count * heads * group * (D * (2 + (2 if case["bf16_out"] else 4)) + 4)
        moved += count * 8 * words if case["tree"] else 0
        flops += seen * heads * group * D * 4.0
    if kind in ("accept", "step"):
        # one row of the target (and of the draft) for every sequence, and the
        # tokens that move: about half of the longest path, at most 4
        rows = 2 if case["sampled"] else 1
        moved += batch * rows * case["vocab"] * SIZES[case["probs"]] + count * 12 + batch * 4 * (max(new) + 2)
        moved += batch * min(4, max(new) // 2) * heads * D * 2 * 2 * 2
        flops += batch * case["vocab"] * 3.0
    return {"bytes": int(moved), "flops": int(flops)}


# ---- the same from the definitions, in 64 bits ---------------------------------

def _path_up(parents, i):
    path = []
    while i >= 0:
        path.append(i)
        i = parents[i]
    return path


def _turned(x, position, case, freqs):
    """Rows [n][heads][128] turned to `position` [n], as complex numbers."""
    rot = case["rot"]
    x = x.double()
    turn = torch.polar(torch.full_like(freqs, _mscale(case)).expand(len(position), -1).contiguous(),
                       position.double()[:, None] * freqs)[:, None]
    part = x[..., :rot]
    if case["interleaved"]:
        z = torch.view_as_complex(part.reshape(*part.shape[:2], rot // 2, 2).contiguous()) * turn
        part = torch.view_as_real(z).reshape(part.shape)
    else:
        z = torch.complex(part[..., : rot // 2].contiguous(), part[..., rot // 2:].contiguous()) * turn
        part = torch.cat([z.real, z.imag], -1)
    return torch.cat([part, x[..., rot:]], -1)


def _exact_walk(target, draft, tokens, parents, uniforms, last):
    """One sequence: (accepted nodes, next token), straight from the rules."""
    now, path = 0, [0]
    while True:
        p = target[now].double()
        q = draft[now].double() if draft is not None else None
        left, weight, scale = 1.0, p.clone(), 0.0
        chosen = None
        for c in [c for c in range(now + 1, len(parents)) if parents[c] == now]:
            x, u = tokens[c], uniforms[c]
            if q is not None:
                if u * float(q[x]) * left < float(weight[x]):
                    chosen = c
                    break
                scale += left
                weight = (p - scale * q).clamp_min(0)
                left = float(weight.sum())
            else:
                if u * left < float(weight[x]):
                    chosen = c
                    break
                left = max(0.0, left - float(weight[x]))
                weight[x] = 0.0
        if chosen is None:
            if not float(weight.sum()) > 0:
                weight = p
            total = weight.cumsum(0)
            above = torch.nonzero(total > last * total[-1])
            if len(above) == 0:
                above = torch.nonzero(weight > 0)[-1:]
            return path, int(above[0])
        now = chosen
        path.append(now)


def exact(case, seed):
    state, result = prepare(case, seed), {}
    kind, heads, group, page = case["kind"], case["kv_heads"], case["group"], case["page"]
    held, new = _lengths(case)
    parents, offsets, table = _parents(case, new), state["offsets"].tolist(), state["table"].long()
    trees = [parents[offsets[b]: offsets[b + 1]] for b in range(case["batch"])]
    place = lambda b, t: (table[b][t // page], t % page)  # noqa: E731
    k, v, q = state["k"].double(), state["v"].double(), state["q"].double() if "q" in state else None
    if kind in ("append", "step"):
        q = torch.empty_like(q)
        for b, n in enumerate(new):
            span = slice(offsets[b], offsets[b + 1])
            slot = torch.arange(held[b], held[b] + n, device="cuda")
            depth = torch.tensor([len(_path_up(trees[b], i)) - 1 for i in range(n)], device="cuda")
            where = held[b] + depth if case["tree"] else slot
            q[span] = _turned(state["q"][span], where, case, state["freqs"])
            pages, slots = place(b, slot)
            k[pages, :, slots] = _turned(state["new_k"][span], where, case, state["freqs"])
            v[pages, :, slots] = state["new_v"][span].double()
        if case["tree"]:
            result["mask"], result["positions"] = None, None
        result["q"] = q
    if kind in ("attend", "step"):
        if kind == "step":             # attention reads what the append has rounded
            q, k, v = (x.bfloat16().double() for x in (q, k, v))
        out = torch.zeros((state["count"], heads * group, D), dtype=torch.float64, device="cuda")
        lse = torch.full((state["count"], heads * group), -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(new):
            total = held[b] + n
            pages, slots = place(b, torch.arange(total, device="cuda"))
            see = torch.ones((n, total), dtype=torch.bool, device="cuda")
            if case["tree"]:
                see[:, held[b]:] = False
                for i in range(n):
                    see[i, [held[b] + x for x in _path_up(trees[b], i)]] = True
            else:
                see[:, held[b]:] = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
            for h in range(heads):
                keys, values = k[pages, h, slots], v[pages, h, slots]
                for r in range(0, n, 1024):
                    x = q[offsets[b] + r: offsets[b] + min(n, r + 1024), h * group: (h + 1) * group]
                    s = torch.matmul(x.reshape(-1, D), keys.t()) / math.sqrt(D)
                    s = s.view(-1, group, total).masked_fill(~see[r: r + 1024, None], -math.inf)
                    span = slice(offsets[b] + r, offsets[b] + r + len(x))
                    lse[span, h * group: (h + 1) * group] = torch.logsumexp(s, -1)
                    out[span, h * group: (h + 1) * group] = torch.matmul(
                        torch.softmax(s, -1).view(-1, total), values).view(-1, group, D)
        result["out"], result["lse"] = out, lse
    if kind in ("accept", "step"):
        accepted = torch.full((case["batch"], max(new)), -1, dtype=torch.int32)
        counts, following = [], []
        uniforms, last, tokens = state["uniforms"].tolist(), state["last"].tolist(), state["tokens"].tolist()
        for b in range(case["batch"]):
            span = slice(offsets[b], offsets[b + 1])
            draft = state["draft"][span] if case["sampled"] else None
            path, token = _exact_walk(state["target"][span], draft, tokens[span], trees[b], uniforms[span], last[b])
            accepted[b, : len(path)] = torch.tensor(path, dtype=torch.int32)
            counts.append(len(path))
            following.append(token)
            old = torch.tensor([held[b] + i for i in path], device="cuda")
            to = torch.arange(held[b], held[b] + len(path), device="cuda")
            for pool in (k, v):
                (a, c), (d, e) = place(b, to), place(b, old)
                pool[a, :, c] = pool[d, :, e].clone()
        result["accepted"], result["counts"] = accepted, torch.tensor(counts, dtype=torch.int32)
        result["next"] = torch.tensor(following, dtype=torch.int32)
    if kind != "attend":
        result["k"], result["v"] = k, v
    return result
