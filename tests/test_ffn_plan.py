"""Plans of the feed-forward block's products, on the host: parts of K cover it and stay inside the workspace, counters inside theirs, rows
are taken once, launches stay as small as they have to be."""
import ctypes as C
import math
import os
import random

import pytest

import ffn_plan as fp
from paper_2104_01981_amd import binding, build

F32, BF16, F16 = 0, 1, 2


def sizes(count, seed):
    """Rows, columns, hidden columns over the range that a block may have, those that memory holds."""
    rng = random.Random(seed)

    def some(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))

    found = []
    while len(found) < count:
        n, D, F = some(1, 1 << 26), 4 * some(1, 1 << 14), 4 * some(1, 1 << 14)
        if n * (D + F) < 1 << 36 and D * F < 1 << 31:
            found.append((n, D, F))
    return found


def launches(n, D, F, type, p):
    """Of each launch that is planned by tiles: name, plan, its products as (rows, columns, K tiles, how many, parts)."""
    elements = fp.constants()["row_bytes"] // (4 if type == F32 else 2)

    def k_tiles(K):
        return -(-K // elements)

    for name in fp.NAMES:
        rows, main, rest = p[name]
        whole = F if name == "weights" else n
        assert 0 < rows <= whole and (name != "weights" or rows == whole)
        for plan, m, first in ((main, rows, True), (rest, whole - rows, False)):
            if m == 0:
                continue
            assert plan.planned
            if name in ("gate", "out") and fp.is_skinny(m, type):
                continue
            products = []
            if name == "weights" or (name == "both" and first):
                products.append((F, D, k_tiles(n), 3, plan.splits[0]))
            if name == "gate":
                products.append((m, F, k_tiles(D), 1, plan.splits[0]))
            if name == "back":
                products.append((m, F, k_tiles(D), 1, plan.splits[0]))
            if name == "out":
                products.append((m, D, k_tiles(F), 1, plan.splits[0]))
            if name in ("input", "both"):
                products.append((m, D, 2 * k_tiles(F), 1, plan.splits[1 if products else 0]))
            yield name, plan, products


@pytest.mark.parametrize("cus", [256, 304, 80])
@pytest.mark.parametrize("type", [F32, BF16, F16])
def test_plans_hold_over_the_range(type, cus):
    c = fp.constants()
    for n, D, F in sizes(1000, cus + type):
        p = fp.plans(n, D, F, type, cus)
        for name, plan, products in launches(n, D, F, type, p):
            what = (n, D, F, name, plan)
            side = fp.side(plan.tiling)
            assert side != (256 if type == F32 else 32), what
            parts = counters = workgroups = 0
            for M, N, K, count, (splits, each) in products:
                assert splits >= 1 and splits * each >= K > (splits - 1) * each, what          # all of K, and no part without any
                tiles = -(-M // side) * -(-N // fp.columns(side, name == "gate")) * count
                workgroups += tiles * splits
                if splits > 1:
                    assert name not in ("gate", "back"), what
                    parts += tiles * splits * side * side * 4
                    counters += tiles
            assert parts <= c["part_most"] and counters == plan.counters <= c["counters"], what
            assert workgroups * 512 < 1 << 32, what
        # few rows' parts: a place for each of 64 lanes' four sums, of up to two blocks of rows
        parts, blocks = fp.skinny_parts(D, F, type, cus), -(-D // 16)
        assert 1 <= parts <= c["skinny_parts"] and (parts == 1 or (parts * blocks <= cus and parts * blocks * 2 * 1024 <= c["part_most"]))


@pytest.mark.parametrize("cus", [256, 304])
@pytest.mark.parametrize("type", [F32, BF16])
def test_the_workspace_has_room_for_the_same_plans(type, cus):
    """With what a block's workspace has for parts, calls of fewer rows, too, are planned as with all there may be."""
    rng = random.Random(cus)
    for n, D, F in sizes(600, 3 * cus + type) + [(m, D, F) for m in (1, 16, 17, 32, 33, 64, 100) for D, F in ((4, 4), (64, 132), (1024, 4096))]:
        for training in (False, True):
            room = fp.room(D, F, n, type, training)
            assert room <= fp.constants()["part_most"]
            for rows in {n, rng.randint(1, n), min(n, 32)}:
                free, held = fp.plans(rows, D, F, type, cus), fp.plans(rows, D, F, type, cus, room)
                for name in fp.NAMES if training else ("gate", "out"):
                    assert free[name] == held[name], (n, D, F, rows, name)
                blocks, parts = -(-D // 16), fp.skinny_parts(D, F, type, cus)
                if parts > 1 and fp.is_skinny(min(rows, 16), type):
                    assert blocks * (2 if type != F32 else 1) * parts * 1024 <= room, (n, D, F)


def workspace_size(**kw):
    if not os.path.exists(binding.library_path()):
        build.build()
    lib, ffn = binding.load_library(), C.c_void_p(0)
    assert lib.ecrm_ffn_create(C.byref(binding.EcrmFfnConfig(**kw)), C.byref(ffn)) == 0
    held = lib.ecrm_ffn_bytes(ffn)
    lib.ecrm_ffn_destroy(ffn)
    return held


def test_a_larger_block_has_a_workspace_for_a_smaller_one():
    rng = random.Random(7)
    for n, D, F in sizes(2000, 11):
        D, F = min(D, 65536), min(F, 65536)
        t, training = rng.randint(0, 2), rng.randint(0, 1)
        smaller = dict(dim=4 * rng.randint(1, D // 4), hidden=4 * rng.randint(1, F // 4), max_rows=rng.randint(1, n), training=rng.randint(0, training))
        larger = dict(dim=D, hidden=F, max_rows=n, training=training)
        for key in rng.sample(list(smaller), rng.randint(0, 3)):                   # as large in some
            smaller[key] = larger[key]
        assert workspace_size(type=t, activation=0, **smaller) <= workspace_size(type=t, activation=1, **larger), (t, smaller, larger)


def test_small_blocks_have_small_workspaces():
    """Parts of products take memory only where there can be any: bytes of the whole workspace, of blocks that need no more of it."""
    size = workspace_size
    counters, h = 4 * fp.constants()["counters"], 1024
    assert size(dim=4, hidden=4, type=BF16, activation=0, max_rows=1, training=0) <= h + counters
    # a decoding step's rows: a long K of few rows in 16 parts at most, 2 KB for 16 columns
    assert size(dim=1024, hidden=4096, type=BF16, activation=0, max_rows=32, training=0) <= 32 * (8192 + 512) + counters + 64 * 16 * 2048
    assert size(dim=128, hidden=512, type=F32, activation=0, max_rows=16, training=0) <= 16 * (2048 + 512) + counters + 8 * 16 * 2048
    # 256 x 256 tiles of one product with two K tiles are the most a tiny block's gradients can have
    assert size(dim=4, hidden=4, type=BF16, activation=0, max_rows=1, training=1) <= 4 * h + counters + 2 * 256 * 256 * 4
    assert size(dim=4096, hidden=16384, type=BF16, activation=0, max_rows=8192, training=1) >= fp.constants()["part_most"]


def test_the_sizes_of_the_gpu_tests_take_every_kind_of_launch():
    """Whatever kind of launch a block of some size has -- product, tile, rows up to the last whole tiles or those behind, parts of K -- the
    exact tests have a size that has it, too, in 16 and in 32 bits.  (Of a million sizes none had another kind.)"""
    import test_gpu_feed_forward as ff
    import test_gpu_feed_forward_plans as more
    taken, rng, asked = {k for size in ff.SIZES + ff.LARGE + more.PLANNED for t in (F32, BF16) for k in fp.kinds(*size, t)}, random.Random(4), 0
    while asked < 15000:
        n, D, F = (int(math.exp(rng.uniform(0, math.log(m)))) * (1 if i == 0 else 4) for i, m in enumerate((1 << 17, 1 << 11, 1 << 12)))
        if n * (D + F) > 3 << 26 or n * D * F > 1 << 38:
            continue
        asked += 1
        for t in (F32, BF16):
            assert not fp.kinds(n, D, F, t) - taken, (n, D, F)


def test_types_of_16_bits_have_the_same_plans():
    for size in sizes(300, 9):
        assert fp.plans(*size, BF16) == fp.plans(*size, F16)
