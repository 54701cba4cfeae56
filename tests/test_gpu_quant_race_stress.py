"""The cross-workgroup protocol over codes under injected delays (needs a gfx950
GPU): the decode kernels of the 8-bit caches, three workgroups a CU and chunks
of their own, in the build that test_gpu_race_stress runs over bf16."""
from __future__ import annotations

import math
import sys

import pytest
import torch

import planref
import quantref as R
from helpers import random_lists, small_workload
from parity import compare_per_head, compare_workload, host_copy
from paper_2606_00024_amd import _lib, api, build

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
THRESHOLDS = [(1e-3, 1e-4, 5), (0.05, 1e-3, 2), (0.0, 1e-4, 5), (0.02, math.inf, 3)]


def _say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def stress_lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return _lib.load_variant(build.STRESS_LIB)


def _prepared(wl, form, blocks=0):
    cache, plain = R.quantised(wl, form, 32)
    if blocks:
        table = torch.full((wl.spec.batch, blocks), -1, dtype=torch.int32)    # (pages of a block)
        table[:, : plain.page_table.shape[1]] = plain.page_table
        plain.page_table = table
    host = host_copy(plain)
    for name in ("q", "page_table", "seq_lens", "block_list", "block_list_len"):
        t = getattr(plain, name)
        if t is not None:
            setattr(plain, name, t.to(DEV))
    return plain, host, R.to_device(cache, DEV)


def _call(plain, cache, ws, **kw):
    s = plain.spec
    got = api.decode_attention_quant(
        plain.q, cache, plain.page_table, plain.seq_lens, block_size=s.block_size, softmax_scale=s.softmax_scale,
        dense_order=s.dense_order, block_list=plain.block_list, block_list_len=plain.block_list_len, workspace=ws, **kw)
    assert api.workspace_status(ws) == _lib.OK
    return got


CASES = [
    # seed, B, Hkv, g, seq_len(s), lists, format, blocks of the table (0: as needed)
    (191, 2, 2, 4, (9000, 6000), False, "e4m3", 0),
    (192, 1, 2, 8, (12000,), False, "int8", 0),
    (193, 2, 1, 4, (8000, 7000), True, "int8", 0),
    (194, 1, 4, 1, (10000,), False, "e4m3", 0),
    (195, 1, 2, 16, (9000,), False, "e4m3", 0),       # chunks of 9
    (196, 2, 2, 2, (11000, 4000), False, "int8", 768),  # of 15
]


@pytest.mark.parametrize("case", CASES, ids=[f"s{c[0]}" for c in CASES])
def test_delayed_handovers_keep_the_sequential_result(stress_lib, case):
    seed, B, hkv, g, L, lists, form, blocks = case
    if seed == 195:
        assert planref.chunks(g, B * hkv, -(-L[0] // 64), 64)[0] == 9
    if blocks:
        assert planref.chunks(g, B * hkv, blocks, 64)[0] == 15
    wl = small_workload(seed, batch=B, kv_heads=hkv, group=g, seq_len=L, needles=4)
    if lists:
        wl.block_list, wl.block_list_len = random_lists(wl, seed, fraction=0.7)
    plain, host, cache = _prepared(wl, form, blocks)
    ws = api.new_workspace(64 << 20, DEV)
    with _lib.using(stress_lib):
        for tau, phi, p in THRESHOLDS:
            kw = dict(tau=tau, phi=phi, patience=p)
            for chunk in (1, 2, 0):
                _say(f"  stress call s{seed} {kw} chunk={chunk}")
                rep = compare_workload(plain, _call(plain, cache, ws, chunk_blocks=chunk, **kw), host=host,
                                       name="quant_race_stress", **kw)
                assert rep.ok(), f"{kw} chunk {chunk}: {rep}"
            rep = compare_per_head(plain, _call(plain, cache, ws, chunk_blocks=1, per_head_stop=True, **kw), host=host,
                                   name="quant_race_stress_per_head", **kw)
            assert rep.ok(), f"per head {kw}: {rep}"


@pytest.mark.parametrize("form", R.FORMATS)
def test_look_first_under_delays(stress_lib, form):
    """128 groups of a few chunks each: a chunk looks back once before it
    publishes its aggregate."""
    plain, host, cache = _prepared(small_workload(197, batch=32, kv_heads=4, group=4, seq_len=1500, needles=2), form)
    ws = api.new_workspace(64 << 20, DEV)
    with _lib.using(stress_lib):
        for tau, phi, p in THRESHOLDS:
            kw = dict(tau=tau, phi=phi, patience=p)
            for chunk in (0, 1):
                _say(f"  stress call s197 {form} {kw} chunk={chunk}")
                rep = compare_workload(plain, _call(plain, cache, ws, chunk_blocks=chunk, **kw), host=host,
                                       name="quant_race_stress", **kw)
                assert rep.ok(), f"{kw} chunk {chunk}: {rep}"


def test_the_stress_build_delays_calls_over_codes(stress_lib):
    """The delays are there: a call in chunks of one block takes clearly longer."""
    plain, _, cache = _prepared(small_workload(198, batch=2, kv_heads=2, group=4, seq_len=(9000, 6000), needles=4),
                                "int8")
    ws = api.new_workspace(64 << 20, DEV)

    def timed():
        ms = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            a.record()
            _call(plain, cache, ws, tau=0.0, phi=1e-4, patience=5, chunk_blocks=1)
            b.record()
            torch.cuda.synchronize()
            ms.append(a.elapsed_time(b))
        return sorted(ms)[2]
    own = timed()
    with _lib.using(stress_lib):
        stressed = timed()
    _say(f"  one call: library {own * 1e3:.0f} us, stress build {stressed * 1e3:.0f} us")
    assert stressed > 2 * own
