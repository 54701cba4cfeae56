"""Decode attention over a cache held in 8 bits (needs a gfx950 GPU): against
the oracle on the values that the codes stand for, and against full attention
in 64 bits where scales are arbitrary."""
from __future__ import annotations

import math
import sys

import numpy as np
import pytest
import torch

import quantref as R
from helpers import random_lists, small_workload
from parity import compare_per_head, compare_workload, host_copy
from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
THRESHOLDS = [(1e-3, 1e-4, 5), (0.05, 1e-3, 2), (0.02, math.inf, 1), (0.1, 0.1, 3), (0.0, 1e-4, 5)]


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _draw(i):
    rng = np.random.default_rng(17000 + i)
    g = int(rng.choice([1, 2, 4, 8, 16]))
    hkv = int(rng.integers(1, 3 if g == 16 else 5))
    batch = int(rng.integers(1, 5))
    bk = int(rng.choice([64, 128, 192, 256]))
    ps = int(rng.choice([16, 32, 64] if bk == 192 else [16, 32, 64, 128, 256]))
    lens = []
    for _ in range(batch):
        r = rng.random()
        lens.append(0 if r < 0.08 else 1 if r < 0.14 else int(rng.integers(2, 2600)))
    if max(lens) == 0:
        lens[0] = int(rng.integers(64, 2000))
    return dict(seed=17000 + i, g=g, hkv=hkv, batch=batch, bk=bk, ps=ps, lens=tuple(lens),
                run=int(rng.choice([r for r in (16, 32, 64, 128, 256) if r <= ps])),
                form=R.FORMATS[i % 2], order=int(rng.integers(0, 2)), lists=bool(rng.random() < 0.3),
                fraction=float(rng.uniform(0.2, 0.9)),
                thr=THRESHOLDS[int(rng.integers(0, len(THRESHOLDS)))],
                chunk=int(rng.choice([0, 0, 1, 2, 3, 5, 9])),
                per_head=bool(rng.random() < 0.2), ahead=int(rng.choice([0, 0, 0, 1, 3])),
                probe=int(rng.choice([1, 1, 4])))


def _call(plain, cache, **kw):
    s = plain.spec
    args = dict(block_size=s.block_size, softmax_scale=s.softmax_scale, tau=s.tau, phi=s.phi,
                patience=s.patience, dense_order=s.dense_order, block_list=plain.block_list,
                block_list_len=plain.block_list_len)
    args.update(kw)
    return api.decode_attention_quant(plain.q, cache, plain.page_table, plain.seq_lens, **args)


def _on_gpu(plain):
    host = host_copy(plain)
    for name in ("q", "page_table", "seq_lens", "block_list", "block_list_len"):
        t = getattr(plain, name)
        if t is not None:
            setattr(plain, name, t.to(DEV))
    return host


@pytest.mark.parametrize("i", range(40))
def test_random_shape_against_the_oracle(i):
    c = _draw(i)
    _say(f"  case {i}: {c}")
    wl = small_workload(c["seed"], batch=c["batch"], kv_heads=c["hkv"], group=c["g"],
                        seq_len=c["lens"], block_size=c["bk"], page_size=c["ps"],
                        dense_order=c["order"], needles=2)
    if c["lists"]:
        wl.block_list, wl.block_list_len = random_lists(wl, c["seed"], fraction=c["fraction"])
    cache, plain = R.quantised(wl, c["form"], c["run"])
    host = _on_gpu(plain)
    tau, phi, p = c["thr"]
    gpu = _call(plain, R.to_device(cache, DEV), tau=tau, phi=phi, patience=p,
                chunk_blocks=c["chunk"], per_head_stop=c["per_head"], max_ahead_chunks=c["ahead"],
                probe_stride=c["probe"])
    torch.cuda.synchronize()
    compare = compare_per_head if c["per_head"] else compare_workload
    rep = compare(plain, gpu, tau=tau, phi=phi, patience=p, host=host, name="quant_random",
                  probe_stride=c["probe"])
    assert rep.ok(), f"case {i} {c}: {rep}"


@pytest.mark.parametrize("i", range(40))
def test_full_attention_random_shape(i):
    """no_detector: the same shapes and lists, against the oracle that never
    stops."""
    c = _draw(i)
    _say(f"  full {i}: {c}")
    wl = small_workload(c["seed"], batch=c["batch"], kv_heads=c["hkv"], group=c["g"],
                        seq_len=c["lens"], block_size=c["bk"], page_size=c["ps"],
                        dense_order=c["order"], needles=2)
    if i % 3 == 0:
        wl.block_list, wl.block_list_len = random_lists(wl, c["seed"], fraction=c["fraction"])
    cache, plain = R.quantised(wl, c["form"], c["run"])
    host = _on_gpu(plain)
    gpu = _call(plain, R.to_device(cache, DEV), tau=1.0, phi=1.0, patience=1, no_detector=True,
                per_head_stop=i % 2 == 0)
    torch.cuda.synchronize()
    rep = compare_workload(plain, gpu, tau=0.0, phi=0.0, patience=1, host=host, name="quant_full")
    assert rep.ok(), f"case {i} {c}: {rep}"


@pytest.mark.parametrize("g,lens", [
    (4, [1 + 37 * (i % 9) for i in range(700)]),        # more sequences than threads
    (8, [0, 0, 5, 0, 40000, 0, 1, 0, 0, 64, 129, 0]),   # empty ones between, one in many parts
    (1, [90000]), (16, [30000, 17]), (2, [0] * 300 + [4000] + [0] * 300),
    (4, [(7 * i) % 130 for i in range(3000)]),          # a wavefront to every group
    (1, [i % 3 for i in range(5000)]),
])
def test_full_attention_ragged(g, lens):
    rng = np.random.default_rng(len(lens))
    H, Ps, run = 1, 64, 32
    width = -(-max(lens) // Ps)
    P = sum(-(-n // Ps) for n in lens)
    cache = _random_cache(rng, R.FORMATS[g % 2], P, H, Ps, run, spread=2.0)
    order = rng.permutation(P).astype(np.int32)
    table = np.full((len(lens), width), -5, dtype=np.int32)
    at = 0
    for b, n in enumerate(lens):
        m = -(-n // Ps)
        table[b, :m] = order[at: at + m]
        at += m
    q = torch.from_numpy(rng.standard_normal((len(lens), H * g, 128)).astype(np.float32)).to(DEV).bfloat16()
    got = api.decode_attention_quant(
        q, cache, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
        block_size=64, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1, no_detector=True)
    _check_full(cache, q, table, lens, got, float(np.float32(0.1)))
    assert got[2][:, 0].cpu().tolist() == [-(-n // 64) for n in lens]


def test_full_attention_scores_that_rise_and_fall():
    """Scores from -2000 to 2000 over the sequence: the running maximum moves
    by more than any factor of fp32 holds, up and down."""
    rng = np.random.default_rng(8)
    Ps, n = 64, 6400
    P = n // Ps
    for rising in (True, False):
        cache = _random_cache(rng, "e4m3", P, 1, Ps, 64)
        k = cache.k.view(torch.uint8)
        k.fill_(0x38)                                              # 1.0
        ramp = torch.linspace(-20, 20, P, device=DEV)
        cache.k_scale.copy_((ramp if rising else -ramp).view(P, 1, 1))
        table = np.arange(P, dtype=np.int32).reshape(1, P)
        q = torch.ones((1, 8, 128), dtype=torch.bfloat16, device=DEV)
        got = api.decode_attention_quant(
            q, cache, torch.from_numpy(table).to(DEV), torch.tensor([n], dtype=torch.int32, device=DEV),
            block_size=64, tau=0.0, phi=0.0, patience=1, softmax_scale=1.0, no_detector=True)
        _check_full(cache, q, table, [n], got, 1.0)


def _bytes_on_gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("g", [1, 2, 4, 8, 16])
def test_every_code(form, g):
    """256 sequences of one token: the probability is 1, so the output is the
    token's V, exactly, and with a one-hot query lse is one value of its K (a
    product of the code, two powers of two and fp32 scales: a few roundings)."""
    _say("  every code", form, g)
    codes = np.arange(256, dtype=np.uint8)
    if form == "e4m3":
        codes = np.where((codes & 127) == 127, 0, codes).astype(np.uint8)
    pool = np.zeros((256, 1, 16, 128), dtype=np.uint8)
    pool[:, 0, 0, :] = codes[:, None]
    pool[:, 0, 1:, :] = 0x7F
    k = _bytes_on_gpu(pool).view(R.DTYPE[form])
    v = _bytes_on_gpu(np.roll(pool, 1, axis=0)).view(R.DTYPE[form])
    rng = np.random.default_rng(3)
    ks = rng.uniform(0.1, 1.0, (256, 1, 1)).astype(np.float32)
    vs = rng.uniform(0.1, 1.0, (256, 1, 1)).astype(np.float32)
    q = torch.zeros((256, g, 128), dtype=torch.bfloat16, device=DEV)
    q[torch.arange(256), :, torch.arange(256) % 128] = 0.5
    out, lse, stop = api.decode_attention_quant(
        q, api.QuantCache(k, v, torch.from_numpy(ks).to(DEV), torch.from_numpy(vs).to(DEV)),
        torch.arange(256, dtype=torch.int32, device=DEV).view(256, 1),
        torch.ones(256, dtype=torch.int32, device=DEV), block_size=64, tau=0.0, phi=0.0, patience=1,
        softmax_scale=0.25, no_detector=True)
    vals = R.table(form)
    want_k = 0.125 * vals[codes] * ks[:, 0, 0]
    want_v = vals[np.roll(codes, 1)] * vs[:, 0, 0].astype(np.float64)
    got = out.double().cpu().numpy()
    # P carries the V scale in three bf16 parts (24 bits): one rounding, half an ulp,
    # then the sum of three parts and the division by a mass of 1: 3 more
    assert np.all(np.abs(got - want_v[:, None, None]) <= 4 * 2.0 ** -24 * np.abs(want_v)[:, None, None])
    assert np.all(np.abs(lse.double().cpu().numpy() - want_k[:, None]) <= 6 * 2.0 ** -24 * np.abs(want_k)[:, None] + 2.0 ** -24)
    assert torch.all(stop == 1)


def _host(cache):
    """The cache's arrays in numpy."""
    return [t.view(torch.uint8).cpu().numpy() for t in cache[:2]] + [t.cpu().numpy().astype(np.float64) for t in cache[2:]]


def _dequantised(cache, table, length, h, host=None):
    """fp64 K and V [length][D] of one sequence and head."""
    out = []
    form = "e4m3" if cache.k.dtype == torch.float8_e4m3fn else "int8"
    k, v, ks, vs = host or _host(cache)
    for codes, scale in ((k, ks), (v, vs)):
        Ps = codes.shape[2]
        run = Ps // scale.shape[2]
        t = np.arange(length)
        pages, slots = table[t // Ps], t % Ps
        out.append(R.table(form)[codes[pages, h, slots]] * scale[pages, h, slots // run][:, None])
    return out


def _check_full(cache, q, table, lens, got, softmax_scale, out_eps=0.0):
    out, lse, _ = (x.float().cpu().numpy().astype(np.float64) for x in got)
    H = cache.k.shape[1]
    g = q.shape[1] // H
    qd, host = q.double().cpu().numpy(), _host(cache)
    for b, n in enumerate(lens):
        for h in range(H):
            rows = slice(h * g, (h + 1) * g)
            if n == 0:
                assert not out[b, rows].any() and np.all(np.isneginf(lse[b, rows]))
                continue
            k, v = _dequantised(cache, table[b], n, h, host)
            o, l, ds = R.full_attention(qd[b, rows], k, v, softmax_scale)
            # a score off by ds moves a weight by at most a factor e^ds either way,
            # an output by 2 ds of the largest |v|; exp2, the sums over n tokens
            # (in a tree of tiles) and the parts of P add a few roundings more
            most = np.abs(v).max()
            tol = (2 * ds + 64 * 2.0 ** -24) * most + out_eps * np.abs(o).max()
            assert np.all(np.abs(out[b, rows] - o) <= tol[:, None]), (b, h, np.abs(out[b, rows] - o).max(), tol)
            assert np.all(np.abs(lse[b, rows] - l) <= ds + 64 * 2.0 ** -24 * np.maximum(1, np.abs(l))), (b, h)


def _random_cache(rng, form, P, H, Ps, run, spread=6.0):
    """Random codes under scales that are no powers of two, some negative."""
    codes = [rng.integers(0, 256, (P, H, Ps, 128), dtype=np.uint8) for _ in range(2)]
    if form == "e4m3":
        codes = [np.where((c & 127) == 127, c & 0x80, c) for c in codes]
    size = 300.0 if form == "e4m3" else 80.0
    scales = [(np.exp2(rng.uniform(-spread, 0, (P, H, Ps // run))) * rng.choice([-1.0, 1.0], (P, H, Ps // run))
               / size).astype(np.float32) for _ in range(2)]
    return api.QuantCache(*(_bytes_on_gpu(c).view(R.DTYPE[form]) for c in codes),
                          *(torch.from_numpy(s).to(DEV) for s in scales))


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("g,Ps,run", [(1, 16, 16), (2, 64, 32), (4, 256, 16), (8, 128, 128), (16, 64, 64)])
def test_arbitrary_scales(form, g, Ps, run):
    _say("  arbitrary scales", form, g, Ps, run)
    rng = np.random.default_rng(g * 100 + Ps)
    lens, H = [1, 0, 63, 64, 65, 777], 2
    width = -(-max(lens) // Ps)
    P = width * len(lens)
    cache = _random_cache(rng, form, P, H, Ps, run)
    table = rng.permutation(P).reshape(len(lens), width).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((len(lens), H * g, 128)).astype(np.float32)).to(DEV).bfloat16()
    for no_detector, dtype in ((True, torch.float32), (False, torch.bfloat16)):
        got = api.decode_attention_quant(
            q, cache, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
            block_size=64, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1, no_detector=no_detector,
            out_dtype=dtype)
        assert got[0].dtype == dtype
        _check_full(cache, q, table, lens, got, float(np.float32(0.1)),
                    2.0 ** -8 if dtype == torch.bfloat16 else 0.0)
        assert got[2].cpu().tolist() == [[-(-n // 64)] * H for n in lens]


def test_scales_far_apart():
    """Runs whose scales differ by 2^60 and more, the small ones with all the
    weight: their values keep their own precision."""
    rng = np.random.default_rng(5)
    cache = _random_cache(rng, "int8", 4, 1, 64, 16)
    small = torch.zeros_like(cache.v_scale, dtype=torch.bool)
    small[:, :, 1] = True
    cache.v_scale.copy_(torch.where(small, cache.v_scale.new_tensor(2.0 ** -40), cache.v_scale.new_tensor(2.0 ** 20)))
    k = cache.k.view(torch.uint8)
    k.fill_(0x81)                      # -127 everywhere, with q = 1: scores far below
    k[:, :, 16:32] = 0                 # but in the runs with small values
    cache.k_scale.fill_(1.0)
    q = torch.ones((1, 4, 128), dtype=torch.bfloat16, device=DEV)
    table = np.arange(4, dtype=np.int32).reshape(1, 4)
    out, _, _ = api.decode_attention_quant(
        q, cache, torch.from_numpy(table).to(DEV), torch.tensor([256], dtype=torch.int32, device=DEV),
        block_size=64, tau=0.0, phi=0.0, patience=1, no_detector=True)
    v = _dequantised(cache, table[0], 256, 0)[1].reshape(4, 64, 128)[:, 16:32].reshape(-1, 128)
    # weights of exp(-127 * 128 / 11.3) vanish beside 2^60: the plain mean of the small rows
    assert np.all(np.abs(out.double().cpu().numpy()[0] - v.mean(0)) <= 16 * 2.0 ** -24 * np.abs(v).max())


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("g", [4, 8])
def test_strides(form, g):
    """Pools laid out [page][slot][head][dim] and with gaps, scales of another
    order: the same bits as of contiguous ones."""
    rng = np.random.default_rng(11)
    lens, H, Ps, run = [500, 129], 3, 32, 16
    width = 16
    P = width * 2
    cache = _random_cache(rng, form, P, H, Ps, run)
    table = torch.from_numpy(rng.permutation(P).reshape(2, width).astype(np.int32)).to(DEV)
    q = torch.from_numpy(rng.standard_normal((2, H * g, 128)).astype(np.float32)).to(DEV).bfloat16()
    kw = dict(block_size=64, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1)
    sl = torch.tensor(lens, dtype=torch.int32, device=DEV)

    def swapped(t):
        return t.view(torch.uint8).transpose(1, 2).contiguous().transpose(1, 2).view(t.dtype)

    def gaps(t):
        big = torch.full((P, H, Ps + 3, 144), 0x55, dtype=torch.uint8, device=DEV)
        view = big[:, :, 1:Ps + 1, :128]
        view.copy_(t.view(torch.uint8))
        return view.view(t.dtype)

    want = api.decode_attention_quant(q, cache, table, sl, **kw)
    ks = cache.k_scale.transpose(0, 1).contiguous().transpose(0, 1)
    for k, v in ((swapped(cache.k), gaps(cache.v)), (gaps(cache.k), swapped(cache.v))):
        got = api.decode_attention_quant(q, api.QuantCache(k, v, ks, cache.v_scale), table, sl, **kw)
        for a, b in zip(want, got):
            assert torch.equal(a, b)


def test_offsets_past_32_bits():
    """Pages 2.5 GB apart: byte offsets past 2^32."""
    rng = np.random.default_rng(12)
    far = 2_500_000_000 // 16 * 16
    buf = torch.empty(2 * far + 64 * 128, dtype=torch.uint8, device=DEV)
    small = _random_cache(rng, "e4m3", 3, 1, 64, 64)
    pool = buf.as_strided((3, 1, 64, 128), (far, 64 * 128, 128, 1))
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=DEV)
    sl = torch.tensor([170], dtype=torch.int32, device=DEV)
    q = torch.from_numpy(rng.standard_normal((1, 4, 128)).astype(np.float32)).to(DEV).bfloat16()
    kw = dict(block_size=64, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1)
    want = api.decode_attention_quant(q, small, table, sl, **kw)
    for which in ("k", "v"):
        pool.copy_(getattr(small, which).view(torch.uint8))
        got = api.decode_attention_quant(q, small._replace(**{which: pool.view(torch.float8_e4m3fn)}), table, sl, **kw)
        for a, b in zip(want, got):
            assert torch.equal(a, b)


def test_same_bits_again_and_on_another_stream():
    wl = small_workload(77, batch=3, kv_heads=2, group=4, seq_len=(3000, 1, 1700), needles=2)
    cache, plain = R.quantised(wl, "e4m3", 32)
    _on_gpu(plain)
    cache = R.to_device(cache, DEV)
    want = _call(plain, cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [_call(plain, cache) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(side)
    for got in again:
        for a, b in zip(want, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("per_head", [True, False])
def test_full_attention_lists_of_many_groups(per_head):
    """Lists (one per KV head or shared) over many sequences: a wavefront to
    every group, empty lists among them."""
    rng = np.random.default_rng(31)
    B, H, g, Ps, bk = 1500, 2, 4, 64, 64
    lens = rng.integers(0, 400, B).tolist()
    width = 7
    cache = _random_cache(rng, "int8", 512, H, Ps, 64, spread=2.0)
    table = rng.integers(0, 512, (B, width)).astype(np.int32)
    rows = (B, H) if per_head else (B,)
    lists = np.full((*rows, width), -1, dtype=np.int32)
    counts = np.zeros(rows, dtype=np.int32)
    for i in np.ndindex(*rows):
        n = -(-lens[i[0]] // bk)
        counts[i] = rng.integers(0, n + 1)
        lists[i][: counts[i]] = rng.permutation(n)[: counts[i]]
    q = torch.from_numpy(rng.standard_normal((B, H * g, 128)).astype(np.float32)).to(DEV).bfloat16()
    out, lse, stop = api.decode_attention_quant(
        q, cache, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
        block_size=bk, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1, no_detector=True,
        block_list=torch.from_numpy(lists).to(DEV), block_list_len=torch.from_numpy(counts).to(DEV),
        list_per_head=per_head)
    out, lse, stop = (x.double().cpu().numpy() for x in (out, lse, stop))
    qd, host = q.double().cpu().numpy(), _host(cache)
    for b in range(0, B, 7):
        for h in range(H):
            i = (b, h) if per_head else (b,)
            n = int(counts[i])
            assert stop[b, h] == n
            at = np.concatenate([np.arange(j * bk, min((j + 1) * bk, lens[b])) for j in lists[i][:n]]) if n else []
            qs = slice(h * g, (h + 1) * g)
            if n == 0:
                assert not out[b, qs].any() and np.all(np.isneginf(lse[b, qs]))
                continue
            k, v = _dequantised(cache, table[b], lens[b], h, host)
            o, l, ds = R.full_attention(qd[b, qs], k[at], v[at], float(np.float32(0.1)))
            tol = (2 * ds + 64 * 2.0 ** -24) * np.abs(v[at]).max()
            assert np.all(np.abs(out[b, qs] - o) <= tol[:, None]), (b, h)
            assert np.all(np.abs(lse[b, qs] - l) <= ds + 64 * 2.0 ** -24 * np.maximum(1, np.abs(l)))


@pytest.mark.parametrize("B,H,g,lo,hi", [
    (60, 8, 4, 100, 3000),      # equal ranges of the line, some of many short groups
    (45, 8, 8, 376, 1056),      # a workgroup to every group
    (64, 8, 16, 1, 200),
    (40, 8, 1, 0, 5000),        # ranges again, sequences of no token among them
    (24, 8, 2, 2000, 6000),     # groups in parts
    (300, 4, 4, 1, 1500),
    (9, 8, 8, 1000, 1000),
])
def test_full_attention_cuts(B, H, g, lo, hi):
    rng = np.random.default_rng(B)
    Ps, pages = 64, 700
    lens = rng.integers(lo, hi + 1, B).tolist()
    lens[B // 2] = lo
    width = -(-hi // Ps)
    cache = _random_cache(rng, R.FORMATS[B % 2], pages, H, Ps, 16, spread=2.0)
    table = rng.integers(0, pages, (B, width)).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((B, H * g, 128)).astype(np.float32)).to(DEV).bfloat16()
    out, lse, stop = (x.double().cpu().numpy() for x in api.decode_attention_quant(
        q, cache, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
        block_size=64, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1, no_detector=True))
    assert np.array_equal(stop, np.repeat([[-(-n // 64)] for n in lens], H, axis=1))
    assert np.isfinite(out).all()
    qd, host = q.double().cpu().numpy(), _host(cache)
    for b, h in [divmod(i, H) for i in range(0, B * H, 7)]:
        qs = slice(h * g, (h + 1) * g)
        if lens[b] == 0:
            assert not out[b, qs].any() and np.all(np.isneginf(lse[b, qs]))
            continue
        k, v = _dequantised(cache, table[b], lens[b], h, host)
        o, l, ds = R.full_attention(qd[b, qs], k, v, float(np.float32(0.1)))
        tol = (2 * ds + 64 * 2.0 ** -24) * np.abs(v).max()
        assert np.all(np.abs(out[b, qs] - o) <= tol[:, None]), (b, h)
        assert np.all(np.abs(lse[b, qs] - l) <= ds + 64 * 2.0 ** -24 * np.maximum(1, np.abs(l)))


def test_calls_of_every_kind_share_a_workspace():
    """Full attention, the stability test and the bf16 call in turn over one
    workspace, each with the bits that it has over one of its own."""
    wl = small_workload(78, batch=5, kv_heads=2, group=4, seq_len=(9000, 1, 64, 5000, 333), needles=2)
    cache, plain = R.quantised(wl, "int8", 64)
    _on_gpu(plain)
    cache = R.to_device(cache, DEV)
    kw = dict(block_size=plain.spec.block_size, tau=1e-2, phi=1e-2, patience=2)
    rest = (plain.page_table, plain.seq_lens)
    pools = [t.to(DEV) for t in (plain.k_cache, plain.v_cache)]
    kinds = {
        "full": lambda **w: api.decode_attention_quant(plain.q, cache, *rest, no_detector=True, **kw, **w),
        "test": lambda **w: api.decode_attention_quant(plain.q, cache, *rest, **kw, **w),
        "bf16": lambda **w: api.decode_attention(plain.q, *pools, *rest, **kw, **w),
        "bf16 full": lambda **w: api.decode_attention(plain.q, *pools, *rest, no_detector=True, **kw, **w),
    }
    size = 1 << 24
    want = {n: call(workspace=api.new_workspace(size, DEV)) for n, call in kinds.items()}
    shared = api.new_workspace(size, DEV)
    for n in ["full", "test", "full", "bf16", "full", "full", "bf16 full", "test", "test", "full"]:
        for a, b in zip(want[n], kinds[n](workspace=shared)):
            assert torch.equal(a, b), n
