"""Every way in which full attention over an 8-bit cache cuts its tiles, dense
and over lists (needs a gfx950 GPU): against full attention in 64 bits.  Each
case names the cut that it takes, which planref derives from the sizes."""
from __future__ import annotations

import sys

import numpy as np
import pytest
import torch

import planref
import quantref as R
from paper_2606_00024_amd import _lib, api

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PAGES = 120


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    _lib.load()
    yield


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def _cache(rng, form, H, page, run):
    """Random codes under scales of either sign that are no powers of two."""
    codes = [rng.integers(0, 256, (PAGES, H, page, 128), dtype=np.uint8) for _ in range(2)]
    if form == "e4m3":
        codes = [np.where((c & 127) == 127, c & 0x80, c).astype(np.uint8) for c in codes]
    size = 300.0 if form == "e4m3" else 80.0
    shape = (PAGES, H, page // run)
    scales = [(np.exp2(rng.uniform(-2, 0, shape)) * rng.choice([-1.0, 1.0], shape) / size).astype(np.float32)
              for _ in range(2)]
    host = [R.table(form)[c] for c in codes], [np.repeat(s.astype(np.float64), run, axis=2) for s in scales]
    return api.QuantCache(*(torch.from_numpy(c).to(DEV).view(R.DTYPE[form]) for c in codes),
                          *(torch.from_numpy(s).to(DEV) for s in scales)), host


def _rows(host, side, pages, h, page, tokens):
    at, slot = pages[tokens // page], tokens % page
    return host[0][side][at, h, slot] * host[1][side][at, h, slot][:, None]


def _check(form, cut, H, g, lens, *, block=64, page=64, run=32, lists=None, per_head=True, every=1, seed=0):
    """lists: numpy [B][H][n] or [B][n] of block ids, -1 behind a list's end."""
    rng = np.random.default_rng(seed)
    B, width = len(lens), -(-max(lens) // page)
    count = None if lists is None else (lists >= 0).sum(-1).astype(np.int32)
    t_cap = max(-(-width * page // block), 0 if lists is None else lists.shape[-1])
    if lists is None:
        tiles, heads = [-(-n // 64) for n in lens], H
    else:
        tiles, heads = (count.reshape(-1) * (block // 64)).tolist(), 1 if per_head else H
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert planref.cut(tiles, heads, g, t_cap, block, cus) == cut
    _say("  cut", cut, form, f"H={H} g={g} B={B} block={block} lists={lists is not None} per_head={per_head}")
    cache, host = _cache(rng, form, H, page, run)
    table = rng.integers(0, PAGES, (B, width)).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((B, H * g, 128)).astype(np.float32)).to(DEV).bfloat16()
    kw = {}
    if lists is not None:
        kw = dict(block_list=torch.from_numpy(lists).to(DEV), block_list_len=torch.from_numpy(count).to(DEV),
                  list_per_head=per_head)
    call = lambda: api.decode_attention_quant(  # noqa: E731
        q, cache, torch.from_numpy(table).to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
        block_size=block, tau=0.0, phi=0.0, patience=1, softmax_scale=0.1, no_detector=True, **kw)
    got, again = call(), call()
    for a, b in zip(got, again):
        assert torch.equal(a, b)
    out, lse, stop = (x.double().cpu().numpy() for x in got)
    assert np.isfinite(out).all()
    qd = q.double().cpu().numpy()
    for i in range(0, B * H, every):
        b, h = divmod(i, H)
        rows, n = slice(h * g, (h + 1) * g), lens[b]
        if lists is None:
            tokens, blocks = np.arange(n), -(-n // block)
        else:
            mine = lists[b, h] if per_head else lists[b]
            mine = mine[mine >= 0]
            blocks = len(mine)
            tokens = np.concatenate([np.arange(j * block, min((j + 1) * block, n)) for j in mine] + [np.empty(0, int)])
            tokens = tokens.astype(np.int64)
        assert stop[b, h] == blocks, (b, h)
        if blocks == 0:
            assert not out[b, rows].any() and np.all(np.isneginf(lse[b, rows]))
            continue
        k, v = (_rows(host, side, table[b], h, page, tokens) for side in (0, 1))
        o, l, ds = R.full_attention(qd[b, rows], k, v, float(np.float32(0.1)))
        # (as in test_gpu_quant_decode: a score off by ds, twice, and the roundings
        # of exp2, the parts of P and sums in a tree of tiles)
        tol = (2 * ds + 64 * 2.0 ** -24) * np.abs(v).max()
        assert np.all(np.abs(out[b, rows] - o) <= tol[:, None]), (b, h, np.abs(out[b, rows] - o).max(), tol)
        assert np.all(np.abs(lse[b, rows] - l) <= ds + 64 * 2.0 ** -24 * np.maximum(1, np.abs(l))), (b, h)


def _lens(seed, B, lo, hi):
    lens = np.random.default_rng(seed).integers(lo, hi + 1, B)
    lens[0], lens[-1] = hi, lo
    return lens.tolist()


def _lists(seed, lens, rows, block, lo, hi):
    """Lists of lo to hi blocks (fewer where the sequence has fewer), `rows` of
    [B] or [B][H], some empty where lo is 0."""
    rng = np.random.default_rng(seed)
    lists = np.full((*rows, hi), -1, dtype=np.int32)
    for i in np.ndindex(*rows):
        n = -(-lens[i[0]] // block)
        m = min(n, int(rng.integers(lo, hi + 1)))
        lists[i][:m] = rng.permutation(n)[:m]
    return lists


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("cut,B,H,g,lo,hi,every", [
    ("each", 4096, 8, 4, 65, 128, 463),
    ("each", 4096, 8, 8, 65, 128, 463),
    ("each", 2048, 8, 16, 65, 128, 231),
    ("each", 600, 8, 2, 257, 320, 61),         # groups of five tiles
    ("each", 680, 3, 1, 700, 768, 41),         # of twelve, heads no power of two
    ("each", 5000, 1, 4, 0, 2, 91),
    ("wave line", 300, 4, 4, 1, 1500, 29),
    ("wave line", 130, 8, 16, 0, 900, 23),
    ("wave line", 3000, 1, 8, 0, 130, 71),
    ("line", 3, 8, 4, 20000, 60000, 5),
    ("line", 60, 8, 2, 100, 3000, 17),
    ("line", 40, 8, 16, 0, 2500, 13),
    ("parts", 4, 8, 8, 2000, 6000, 3),
    ("parts", 9, 5, 1, 0, 700, 2),
    ("whole", 45, 8, 4, 376, 640, 13),
    ("whole", 64, 8, 16, 1, 200, 19),
])
def test_dense(form, cut, B, H, g, lo, hi, every):
    _check(form, cut, H, g, _lens(B, B, lo, hi), every=every, seed=B + g)


@pytest.mark.parametrize("form", R.FORMATS)
@pytest.mark.parametrize("per_head", [True, False])
@pytest.mark.parametrize("cut,B,H,g,n,lo,hi,block,every", [
    ("each", 1000, 8, 4, 640, 3, 4, 64, 97),
    ("each", 1500, 4, 8, 500, 1, 2, 64, 71),
    ("each", 700, 8, 16, 640, 2, 3, 128, 61),
    ("wave line", 400, 8, 4, 900, 0, 14, 64, 37),
    ("wave line", 1500, 2, 1, 400, 0, 7, 64, 31),
    ("line", 2, 2, 4, 150000, 2200, 2300, 64, 1),
    ("line", 2, 4, 2, 200000, 600, 800, 128, 3),
    ("parts", 6, 4, 8, 5000, 0, 60, 64, 3),
    ("parts", 3, 2, 16, 4000, 5, 20, 128, 1),
    ("whole", 45, 8, 4, 640, 6, 9, 64, 17),
])
def test_lists(form, per_head, cut, B, H, g, n, lo, hi, block, every):
    lens = _lens(B, B, max(1, n - 200), n)
    rows = (B, H) if per_head else (B,)
    _check(form, cut, H, g, lens, block=block, lists=_lists(B + g, lens, rows, block, lo, hi), per_head=per_head,
           every=every, seed=B + g, run=16)
