"""The measured work on a paged KV cache held in 8 bits: the calls that write
it, read it back and attend to it, and the same results in plain torch.

Four kinds of pass:

  decode   one new token of every sequence of a batch attends to its 8-bit
           cache, with or without early stop
  append   new tokens of every sequence are quantised into the cache: one each
           (a decode step), or whole prompts
  read     stored tokens come back as rows of 16 or 32 bits
  step     what a decode step does with the cache: append one token to every
           sequence, then attend

The cache.  Codes are e4m3 (448 the largest, NaN 0x7f) or int8 (-127..127), in
pools [page][kv_head][slot][128].  A run of ``scale_tokens`` slots of a page
and head shares one fp32 scale, the smallest power of two 2^e, e >= -120, that
brings the run's largest finite magnitude within the largest code; a token
stands for code * scale.  A run that already holds tokens never gets a smaller
scale, and where it gets a larger one its old codes are rounded anew, half to
even.

Head shapes, contexts, blocks and pages are those of this repository's
workloads and measured calls (32/8, 64/8 and 8/2 heads, 4K to 512K tokens,
blocks of 64 and 128).  Caches hold Gaussian keys and values with sink and
needle tokens along the queries of their group, pages permuted in one pool.
"""
from __future__ import annotations

import math
import random

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
TOP = {"e4m3": 448.0, "int8": 127.0}
LOWEST = -120                       # exponent of the smallest scale
MAX_BYTES = 2_400_000_000           # code bytes (and row bytes) of a drawn case
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(name, **kw):
    case = {
        "kind": "decode", "batch": 1, "kv_heads": 8, "group": 4,
        # tokens that each sequence holds, and how many it appends or reads
        "len_lo": 4096, "len_hi": 4096, "new_lo": 1, "new_hi": 1, "len_seed": 0,
        "block": 64, "page": 64, "scale_tokens": 64, "format": "e4m3",
        "rows": "bf16",             # type of appended rows and of rows read back
        "tau": 1e-2, "phi": 1e-2, "patience": 5,
        "detector": True,           # False: full attention, no stability test
        "forward": False,           # oldest block first
        "per_head": False,          # every query head stops on its own
        "bf16_out": True,
        "share": 1.0,               # share of the cache in front of the stops
    }
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one short request with two KV heads: all latency
        _case("decode_tiny_4k", kv_heads=2, bf16_out=False, share=0.31),
        # a chat batch: short ragged contexts (an empty one among them), pages
        # of 16 tokens, the finest scales
        _case("decode_chat_ragged_2k", batch=16, len_lo=0, len_hi=2048, len_seed=3, page=16,
              scale_tokens=16, format="int8", share=0.72),
        # an 8B-shaped layer at batch 8 as full attention: the plain case
        _case("decode_8x32k_full", batch=8, len_lo=32768, len_hi=32768, detector=False),
        # the same layer with early stop, int8
        _case("decode_8x32k_stop", batch=8, len_lo=32768, len_hi=32768, format="int8", share=0.125),
        # the headline batch: 64/8 heads, ragged 8K to 64K; the stability test
        # runs at the paper's thresholds, which stop nothing here
        _case("decode_ragged_64k", batch=32, group=8, len_lo=8192, len_hi=65536, len_seed=4,
              tau=1e-5, phi=1e-3),
        # one very long document in blocks and pages of 128 tokens, full attention
        _case("decode_long_512k", len_lo=524288, len_hi=524288, block=128, page=128,
              scale_tokens=32, format="int8", detector=False, bf16_out=False),
        # one token of one sequence: the smallest write
        _case("append_one", kind="append", kv_heads=2, len_lo=1000, len_hi=1000),
        # a decode step's write: one token each of 64 sequences, within a run
        # of slots that holds tokens already
        _case("append_64_tokens", kind="append", batch=64, len_lo=100, len_hi=4000, len_seed=7),
        # a prefill batch: ragged prompts, chunks that begin inside a page
        _case("append_prompts", kind="append", batch=8, len_lo=0, len_hi=2000, new_lo=500,
              new_hi=16384, len_seed=8, format="int8"),
        # shared prefixes brought back for a prefill's attention
        _case("read_prefix_8x16k", kind="read", batch=8, len_lo=0, len_hi=100, new_lo=8192,
              new_hi=16384, len_seed=9),
        # a few short spans of an int8 cache, in 32 bits
        _case("read_short_f32", kind="read", batch=3, kv_heads=4, len_lo=0, len_hi=300, new_lo=50,
              new_hi=400, len_seed=10, format="int8", scale_tokens=16, rows="f32"),
        # a decode step's cache work on the 8B-shaped layer: write, then attend
        _case("step_8x32k", kind="step", batch=8, len_lo=30000, len_hi=32767, len_seed=11,
              share=0.15),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["decode"] * 5 + ["append"] * 2 + ["read"] * 2 + ["step"])
    group = rng.choice([1, 2, 4, 4, 4, 8, 8, 16])
    kv_heads = rng.choice([1, 2, 4, 8, 8])
    block = rng.choice([64, 64, 64, 128, 256])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    scale_tokens = min(page, rng.choice([16, 32, 64, 64, 128, 256]))
    batch = _log_int(rng, 1, 48)
    row = kv_heads * D * 2                     # code bytes of a token
    case = dict(kind=kind, batch=batch, kv_heads=kv_heads, group=group, block=block, page=page,
                scale_tokens=scale_tokens, format=rng.choice(["e4m3", "int8"]),
                len_seed=rng.randrange(1, 1 << 20))
    if kind in ("append", "read"):
        rows = rng.choice(["bf16", "bf16", "f16", "f32"])
        hi = _log_int(rng, 1, min(32768, 300_000_000 // (batch * row)))
        case.update(rows=rows, new_lo=hi if rng.random() < 0.3 else max(0, int(hi * rng.uniform(0, 0.9))),
                    new_hi=hi, len_lo=0, len_hi=_log_int(rng, 1, 3000))
        return _case(None, **case)
    hi = _log_int(rng, 64, min(524288, MAX_BYTES // (batch * row)))
    lo = hi if rng.random() < 0.4 else int(hi * rng.uniform(0, 0.9))
    detector = rng.random() < 0.6
    tau, phi = rng.choice([(1e-2, 1e-2), (1e-5, 1e-3)])
    forward = rng.random() < 0.2
    share = 1.0
    if detector and tau > 1e-5 and hi > 8192:
        share = 0.1 if forward else 0.4
    return _case(None, **case, len_lo=lo, len_hi=hi, tau=tau, phi=phi, patience=rng.choice([2, 5, 5, 10]),
                 detector=detector, forward=forward, per_head=detector and rng.random() < 0.15,
                 bf16_out=rng.random() < 0.7, share=share)


def _lengths(case):
    """(tokens held, tokens appended or read) of every sequence."""
    rng = random.Random(case["len_seed"])
    held = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["batch"])]
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    if case["kind"] in ("append", "read") and sum(new) == 0:
        new[0] = 1
    return held, new if case["kind"] != "decode" else [0] * case["batch"]


# ---- inputs -------------------------------------------------------------------

def _exponent(a, top):
    """Smallest e >= LOWEST with a <= top * 2^e, exactly."""
    m, k = torch.frexp(a)
    tm, tk = math.frexp(top)
    e = k - tk + (m > tm).to(k.dtype)
    return torch.where(a > 0, e, torch.full_like(e, LOWEST)).clamp_min(LOWEST)


def _power(e):
    return ((e.int() + 127) << 23).view(torch.float32)          # from its bits: exact


def _encode(x, form):
    """Bytes of the codes nearest to x (within the largest code)."""
    if form == "e4m3":
        return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return x.clamp(-127.0, 127.0).round().to(torch.int8).view(torch.uint8)


def _typed(bytes_, form):
    return bytes_.view(torch.float8_e4m3fn if form == "e4m3" else torch.int8)


def _quantised(x, case):
    """Pools of bytes and scales of x [pages][heads][page][128]."""
    pages, heads, page, _ = x.shape
    run = case["scale_tokens"]
    runs = x.view(pages, heads, page // run, run * D)
    scale = _power(_exponent(runs.abs().amax(-1), TOP[case["format"]]))
    return _encode(runs / scale[..., None], case["format"]).view(x.shape), scale


def prepare(case, seed):
    held, new = _lengths(case)
    batch, heads, group, page = case["batch"], case["kv_heads"], case["group"], case["page"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    counts = [-(-(a + b) // page) for a, b in zip(held, new)]
    width, pages = max(1, max(counts)), max(1, sum(counts))
    order = torch.randperm(pages, generator=gen, device="cuda").int()
    table = torch.zeros((batch, width), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = order[at: at + n]
        at += n
    q = normal(batch, heads * group, D).bfloat16()
    k, v = normal(pages, heads, page, D), normal(pages, heads, page, D)
    if case["kind"] in ("decode", "step"):
        # sinks at the first tokens, needles anywhere: keys along the group's queries
        u = q.float().view(batch, heads, group, D).sum(2)
        u = 3.0 * math.sqrt(D) * u / u.norm(dim=-1, keepdim=True)
        rng = random.Random(seed)
        for b, n in enumerate(held):
            if n:
                where = torch.tensor(list(range(min(4, n))) + [rng.randrange(n) for _ in range(8)], device="cuda")
                k[table[b, where // page].long(), :, where % page] += u[b]
    state = {"case": case, "q": q, "table": table}
    for name, x in (("k", k), ("v", v)):
        state[name], state[name + "_scale"] = _quantised(x, case)
    del k, v
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    state["lens"] = as_int([a + b for a, b in zip(held, new)] if case["kind"] == "step" else held)
    state["positions"] = as_int(held)
    offsets = [0]
    for n in new:
        offsets.append(offsets[-1] + n)
    state["offsets"], state["count"] = as_int(offsets), offsets[-1]
    if case["kind"] in ("append", "step"):
        for name in ("new_k", "new_v"):
            state[name] = (normal(offsets[-1], heads, D) * 1.5).to(TYPES[case["rows"]])
    if case["kind"] == "append" and case["format"] == "int8":
        # int8 codes come back as the values they stand for: the new tokens and
        # the old ones of the runs that they end
        run = case["scale_tokens"]
        first = [a // run * run for a in held]
        spans = [0]
        for a, b, n in zip(first, held, new):
            spans.append(spans[-1] + b + n - a)
        state["back_from"], state["back_offsets"], state["back_count"] = as_int(first), as_int(spans), spans[-1]
    return state


# ---- the passes ----------------------------------------------------------------

def run(state):
    case, result = state["case"], {}
    kind = case["kind"]
    if kind == "read":
        result["k"], result["v"] = _read(state, state["positions"], state["offsets"], state["count"],
                                         TYPES[case["rows"]])
    if kind in ("append", "step"):
        _append(state)
        result["k_scale"], result["v_scale"] = state["k_scale"], state["v_scale"]
        if "back_from" in state:
            result["k"], result["v"] = _read(state, state["back_from"], state["back_offsets"],
                                             state["back_count"], torch.float32)
        else:
            result["k"], result["v"] = (_typed(state[x], case["format"]) for x in ("k", "v"))
    if kind in ("decode", "step"):
        result["out"], result["lse"], result["stop"] = _decode(state)
    return result


def _cache(state):
    from paper_2606_00024_amd import api
    form = state["case"]["format"]
    return api, api.QuantCache(_typed(state["k"], form), _typed(state["v"], form),
                               state["k_scale"], state["v_scale"])


def _rows(state, positions, offsets, count):
    """Page, slot and page's run of rows of the packed form, and their tokens."""
    page, run = state["case"]["page"], state["case"]["scale_tokens"]
    r = torch.arange(count, device="cuda")
    b = torch.searchsorted(offsets[1:].contiguous(), r.int(), right=True)
    t = positions[b].long() + r - offsets[b]
    pages = state["table"][b, t // page].long()
    return pages, t % page, t % page // run


def _read(state, positions, offsets, count, dtype):
    if own:
        api, cache = _cache(state)
        return api.quant_read(cache, state["table"], positions, token_offsets=offsets, rows=count,
                              dtype=dtype)
    form = state["case"]["format"]
    pages, slots, runs = _rows(state, positions, offsets, count)
    return tuple((_typed(state[x][pages, :, slots], form).float()
                  * state[x + "_scale"][pages, :, runs][..., None]).to(dtype) for x in ("k", "v"))


def _append(state):
    if own:
        api, cache = _cache(state)
        api.quant_append(cache, state["new_k"], state["new_v"], state["table"], state["positions"],
                         token_offsets=state["offsets"])
        return
    case = state["case"]
    form, page, run = case["format"], case["page"], case["scale_tokens"]
    positions, offsets = state["positions"].long(), state["offsets"].long()
    pages, slots, runs = _rows(state, state["positions"], state["offsets"], state["count"])
    per = page // run
    flat = pages * per + runs
    # runs that hold tokens of their sequence already
    half = torch.nonzero((positions % run > 0) & (offsets[1:] > offsets[:-1]))[:, 0]
    kept = positions[half] % run
    old_page = state["table"][half, positions[half] // page].long()
    old_run = positions[half] % page // run
    for name in ("k", "v"):
        x = state["new_" + name].float()
        pool, scale = state[name], state[name + "_scale"]
        heads = scale.shape[1]
        by_run = scale.transpose(1, 2).reshape(-1, heads)                # [run of the pool][heads]
        top = torch.zeros_like(by_run).scatter_reduce_(
            0, flat[:, None].expand(-1, heads), x.abs().amax(-1), "amax")
        need = _power(_exponent(top, TOP[form]))
        touched = torch.zeros(len(by_run), dtype=torch.bool, device="cuda")
        touched[flat] = True
        holds = torch.zeros_like(touched)
        holds[old_page * per + old_run] = True
        fresh = torch.where(holds[:, None], torch.maximum(need, by_run), need)
        fresh = torch.where(touched[:, None], fresh, by_run)
        view = pool.view(len(pool), heads, per, run, D)
        codes = view[old_page, :, old_run]                               # [n][heads][run][128]
        ratio = (by_run / fresh)[old_page * per + old_run]
        anew = _encode(_typed(codes, form).float() * ratio[..., None, None], form)
        mask = torch.arange(run, device="cuda")[None, None, :, None] < kept[:, None, None, None]
        view[old_page, :, old_run] = torch.where(mask, anew, codes)
        scale.copy_(fresh.view(len(pool), per, heads).transpose(1, 2))
        pool[pages, :, slots] = _encode(x / fresh[flat][..., None], form)


def _decode(state):
    case = state["case"]
    if own:
        api, cache = _cache(state)
        return api.decode_attention_quant(
            state["q"], cache, state["table"], state["lens"], block_size=case["block"],
            tau=case["tau"], phi=case["phi"], patience=case["patience"],
            dense_order=1 if case["forward"] else 0,
            out_dtype=torch.bfloat16 if case["bf16_out"] else torch.float32,
            no_detector=not case["detector"], per_head_stop=case["per_head"])
    batch, heads, group, block = case["batch"], case["kv_heads"], case["group"], case["block"]
    lens = state["lens"].long()
    blocks = -(-state["table"].shape[1] * case["page"] // block)
    tokens = blocks * block

    def gathered(name):                                                  # [batch][heads][tokens][128]
        codes = _typed(state[name][state["table"].long()], case["format"]).float()
        scale = state[name + "_scale"][state["table"].long()]
        x = (codes.view(*scale.shape, -1, D) * scale[..., None, None]).view(codes.shape)
        x = x.permute(0, 2, 1, 3, 4).reshape(batch, heads, -1, D)
        return torch.nn.functional.pad(x, (0, 0, 0, tokens - x.shape[2]))

    q = state["q"].float().view(batch, heads, group, D)
    s = torch.matmul(gathered("k"), q.transpose(2, 3).contiguous()).transpose(2, 3) * SCALE
    dead = torch.arange(tokens, device="cuda") >= lens[:, None, None, None]
    s = s.masked_fill(dead, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(top.isfinite(), top, torch.zeros_like(top))
    p = torch.exp(s - top).view(batch, heads, group, blocks, block)
    mass = p.sum(-1).double()                                            # [batch][heads][group][blocks]
    v = gathered("v").view(batch, heads, blocks, block, D)
    vec = torch.matmul(p.transpose(2, 3).contiguous(), v).transpose(2, 3)
    steps = -(-lens // block)                                            # blocks of each sequence
    at = steps[:, None, None].expand(batch, heads, group)
    if not case["detector"]:
        a, o = mass.sum(-1), vec.sum(-2, dtype=torch.float64)
    else:
        t = torch.arange(blocks, device="cuda")
        walk = t.expand(batch, -1) if case["forward"] else steps[:, None] - 1 - t
        walk = walk.clamp_min(0)[:, None, None, :].expand(batch, heads, group, -1)
        a = mass.gather(3, walk).cumsum(-1)
        o = vec.gather(3, walk[..., None].expand(-1, -1, -1, -1, D)).double().cumsum(3) / a[..., None]
        far = (o[..., 1:, :] - o[..., :-1, :]).norm(dim=-1)
        size = o.norm(dim=-1)
        turn = 1.0 - (o[..., 1:, :] * o[..., :-1, :]).sum(-1) / (size[..., 1:] * size[..., :-1])
        tau, phi = (float(torch.tensor(case[x], dtype=torch.float32)) for x in ("tau", "phi"))
        ok = torch.nn.functional.pad((far < tau) & (turn < phi), (1, 0))
        if not case["per_head"]:
            ok = ok.all(2, keepdim=True).expand(batch, heads, group, blocks)
        n = t + 1
        length = n - torch.where(ok, torch.zeros_like(n), n).cummax(-1).values
        done = (length >= case["patience"]) & (n <= steps[:, None, None, None])
        at = torch.where(done.any(-1), done.int().argmax(-1) + 1, at)
        last = (at - 1).clamp_min(0)[..., None]
        a = a.gather(3, last)[..., 0]
        o = o.gather(3, last[..., None].expand(-1, -1, -1, 1, D))[..., 0, :] * a[..., None]
    empty = (lens == 0)[:, None, None]
    out = torch.where(empty[..., None], torch.zeros_like(o), o / a[..., None])
    lse = torch.where(empty, torch.full_like(a, -math.inf), top[..., 0].double() + a.log())
    stop = at.reshape(batch, -1) if case["per_head"] else at[:, :, 0]
    dtype = torch.bfloat16 if case["bf16_out"] else torch.float32
    return out.view(batch, -1, D).to(dtype), lse.view(batch, -1).float(), stop.int()


def work(case):
    held, new = _lengths(case)
    heads, group, run, block = case["kv_heads"], case["group"], case["scale_tokens"], case["block"]
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["rows"]]
    moved, flops = 4 * 2 * case["batch"], 0.0
    if case["kind"] in ("append", "step"):
        n = sum(new)
        runs = sum(-(-(a + b) // run) - a // run for a, b in zip(held, new) if b)
        moved += 2 * heads * (n * D * (size + 1) + 4 * runs) + 4 * runs
        flops += 2 * heads * n * D * 3
        if "append" == case["kind"] and case["format"] == "int8":
            back = sum(a % run + b for a, b in zip(held, new))
            moved += 2 * heads * back * D * 5
            flops += 2 * heads * back * D
    if case["kind"] == "read":
        n = sum(new)
        runs = sum(-(-(a + b) // run) - a // run for a, b in zip(held, new) if b)
        moved += 2 * heads * (n * D * (size + 1) + 4 * runs) + 4 * runs
        flops += 2 * heads * n * D
    if case["kind"] in ("decode", "step"):
        tokens = sum(a + b for a, b in zip(held, new)) * case["share"]
        queries = case["batch"] * heads * group
        moved += tokens * heads * (2 * D + 8 / run) + 4 * tokens / case["page"]
        moved += queries * (D * (2 + (2 if case["bf16_out"] else 4)) + 8)
        flops += tokens * heads * group * D * 4
    return {"bytes": int(moved), "flops": int(flops)}


# ---- the same from the definitions, in 64 bits ---------------------------------

def _values(bytes_, form):
    """What codes stand for, apart from their scale."""
    if form == "int8":
        table = [float(c if c < 128 else c - 256) for c in range(256)]
    else:
        table = []
        for c in range(256):
            e, m = c >> 3 & 15, c & 7
            x = math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10)
            table.append((-x if c >> 7 else x) if c & 127 != 127 else math.nan)
    return torch.tensor(table, dtype=torch.float64, device="cuda")[bytes_.int()]


def _nearest(x, form):
    """x rounded to the nearest code's value, ties to even."""
    if form == "int8":
        return x.round()
    e = torch.frexp(x).exponent.clamp_min(-5).long() - 4
    step = ((e + 1023) << 52).view(torch.float64)
    return (x / step).round() * step


def _spans(state, positions, offsets):
    """(first row, rows, pages and slots of the tokens) of every sequence."""
    page = state["case"]["page"]
    for b, p in enumerate(positions.tolist()):
        first, end = offsets[b].item(), offsets[b + 1].item()
        t = torch.arange(p, p + end - first, device="cuda")
        yield b, p, first, end, state["table"][b][t // page].long(), t % page


def _exact_read(state, pools, scales, positions, offsets, count):
    found = []
    for pool, scale in zip(pools, scales):
        rows = torch.zeros((count, pool.shape[1], D), dtype=torch.float64, device="cuda")
        for _, _, first, end, pages, slots in _spans(state, positions, offsets):
            run = slots // state["case"]["scale_tokens"]
            rows[first:end] = pool[pages, :, slots] * scale[pages, :, run][..., None]
        found.append(rows)
    return found


def _exact_append(state):
    """The pools' values (without scales) and scales after the call."""
    case = state["case"]
    form, run, page = case["format"], case["scale_tokens"], case["page"]
    pools, scales = [], []
    for name in ("k", "v"):
        pool, scale = _values(state[name], form), state[name + "_scale"].double()
        x = state["new_" + name].double()
        for b, p, first, end, pages, slots in _spans(state, state["positions"], state["offsets"]):
            if first == end:
                continue
            old = p % run
            t = torch.arange(p - old, p, device="cuda")
            old_pages, old_slots = state["table"][b][t // page].long(), t % page
            rows = torch.cat([torch.zeros((old, *x.shape[1:]), dtype=x.dtype, device="cuda"), x[first:end]])
            rows = torch.nn.functional.pad(rows, (0, 0, 0, 0, 0, -len(rows) % run))
            top = rows.abs().view(-1, run, *x.shape[1:]).amax((1, 3))     # [runs][heads]
            e = (top / TOP[form]).log2().floor().clamp(LOWEST, 1000).long()
            need = ((e + 1023) << 52).view(torch.float64)
            for _ in range(2):
                need = torch.where(top > TOP[form] * need, 2 * need, need)
            if old:
                was = scale[old_pages[0], :, old_slots[0] // run]
                need[0] = torch.maximum(need[0], was)
                pool[old_pages, :, old_slots] = _nearest(
                    pool[old_pages, :, old_slots] * (was / need[0])[None, :, None], form)
            which = (torch.arange(p, p + end - first, device="cuda") - (p - old)) // run
            scale[pages, :, slots // run] = need[which]
            pool[pages, :, slots] = _nearest(x[first:end] / need[which][..., None], form)
        pools.append(pool)
        scales.append(scale)
    return pools, scales


def _exact_decode(state, pools, scales):
    """Appendix A's recurrence, one block of every sequence after the other."""
    case = state["case"]
    batch, heads, group, block = case["batch"], case["kv_heads"], case["group"], case["block"]
    page, run = case["page"], case["scale_tokens"]
    lens = state["lens"].tolist()
    most = max(1, max(-(-n // block) for n in lens))
    weight = torch.full((batch, most, heads, group), -math.inf, dtype=torch.float64, device="cuda")
    mean = torch.zeros((batch, most, heads, group, D), dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        used, pad, blocks = state["table"][b, : -(-n // page)].long(), -n % block, -(-n // block)
        if not n:
            continue
        k, v = ((x[used].view(len(used), heads, page // run, run, D) * s[used][..., None, None])
                .view(len(used), heads, page, D).transpose(0, 1).reshape(heads, -1, D)[:, :n]
                for x, s in zip(pools, scales))
        q = state["q"][b].double().view(heads, group, D)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)
        s = torch.nn.functional.pad(s, (0, pad), value=-math.inf).view(heads, group, blocks, block)
        v = torch.nn.functional.pad(v, (0, 0, 0, pad)).view(heads, blocks, block, D)
        lse = torch.logsumexp(s, -1)
        u = torch.matmul(torch.exp(s - lse[..., None]).transpose(1, 2).contiguous(), v)
        if not case["forward"]:
            lse, u = lse.flip(2), u.flip(1)
        weight[b, :blocks] = lse.permute(2, 0, 1)
        mean[b, :blocks] = u.transpose(0, 1)
    tau, phi = (float(torch.tensor(case[x], dtype=torch.float32)) for x in ("tau", "phi"))
    total = torch.full((batch, heads, group), -math.inf, dtype=torch.float64, device="cuda")
    o = torch.zeros((batch, heads, group, D), dtype=torch.float64, device="cuda")
    count = torch.zeros((batch, heads, group), dtype=torch.int64, device="cuda")
    stop = torch.zeros_like(count)
    going = torch.ones_like(count, dtype=torch.bool)
    ends = torch.tensor([-(-n // block) for n in lens], device="cuda")[:, None, None]
    for t in range(most):
        w = weight[:, t]
        now = torch.logaddexp(total, w)
        d = (w - now).exp()[..., None] * (mean[:, t] - o)
        d = torch.where((t < ends)[..., None] & (w > -math.inf)[..., None], d, torch.zeros_like(d))
        after = o + d
        going = going & (t < ends)
        if case["detector"]:
            cosine = (o * after).sum(-1) / (o.norm(dim=-1) * after.norm(dim=-1))
            ok = (d.norm(dim=-1) < tau) & (1.0 - cosine < phi) & (t > 0)
            if not case["per_head"]:
                ok = ok.all(-1, keepdim=True).expand_as(ok)
            count = torch.where(ok, count + 1, torch.zeros_like(count))
        total = torch.where(going, now, total)
        o = torch.where(going[..., None], after, o)
        stop = torch.where(going, t + 1, stop)
        if case["detector"]:
            going = going & (count < case["patience"])
    stop = stop.view(batch, -1) if case["per_head"] else stop[..., 0]
    return o.view(batch, -1, D), total.view(batch, -1), stop.int()


def exact(case, seed):
    state = prepare(case, seed)
    kind, form, result = case["kind"], case["format"], {}
    if kind in ("append", "step"):
        pools, scales = _exact_append(state)
        result["k_scale"], result["v_scale"] = scales
        if "back_from" in state:
            result["k"], result["v"] = _exact_read(state, pools, scales, state["back_from"],
                                                   state["back_offsets"], state["back_count"])
        else:
            result["k"], result["v"] = pools
    else:
        pools = [_values(state[x], form) for x in ("k", "v")]
        scales = [state[x + "_scale"].double() for x in ("k", "v")]
    if kind == "read":
        result["k"], result["v"] = _exact_read(state, pools, scales, state["positions"],
                                               state["offsets"], state["count"])
    if kind in ("decode", "step"):
        result["out"], result["lse"], result["stop"] = _exact_decode(state, pools, scales)
    return result
