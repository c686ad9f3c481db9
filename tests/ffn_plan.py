"""The library's own plans of the feed-forward block's products: csrc/ffn_plan.hip compiled for the host, so that no test has to repeat its
formulas."""
from __future__ import annotations

import ctypes as C
import os
import subprocess
import tempfile
from collections import namedtuple

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2104_01981_amd", "csrc")
SOURCE = """
#include "ffn_plan.hip"
using namespace ecrm;
static void write(const Plan &p, uint32_t *to)
{
    const uint32_t words[] = {p.tiling, p.split[0].splits, p.split[0].each, p.split[1].splits, p.split[1].each, p.counters, p.cost > 0};
    for (uint32_t w : words) *to++ = w;
}
extern "C" {
uint32_t plan_constants(int i)
{
    const uint32_t values[] = {(uint32_t)kPartMost, kCounters, kRowBytes, kSkinnyParts};
    return values[i];
}
uint32_t plan_side(uint32_t tiling) { return kCosts[tiling].side; }
uint32_t plan_columns(uint32_t side, uint32_t dual) { return columns_of(side, dual != 0); }
uint32_t plan_is_skinny(uint32_t rows, uint32_t type) { return is_skinny(rows, type); }
uint32_t plan_skinny_parts(uint32_t N, uint32_t K, uint32_t type, uint32_t cus) { return skinny_parts(N, K, type, cus); }
uint64_t plan_room(uint32_t dim, uint32_t hidden, uint64_t max_rows, uint32_t type, uint32_t training)
{
    return parts_room(dim, hidden, max_rows, type, training != 0);
}
// gate, out, back, weights, input, both: of each the rows of the first part, its plan, and the others' plan
void plan_all(uint32_t rows, uint32_t dim, uint32_t hidden, uint32_t type, uint32_t cus, uint64_t room, uint32_t *to)
{
    BlockPlans p;
    for (int what = 0; what < kPlans; ++what) plan_block(p, what, rows, dim, hidden, type, cus, room);
    for (const RowPlan *r : {&p.gate, &p.out, &p.back, &p.weights, &p.input, &p.both}) {
        *to++ = r->rows;
        write(r->main, to);
        write(r->rest, to + 7);
        to += 14;
    }
}
}
"""
NAMES = "gate", "out", "back", "weights", "input", "both"
Plan = namedtuple("Plan", "tiling splits counters planned")              # splits: (parts, K tiles of each), of two sizes where there are two
RowPlan = namedtuple("RowPlan", "rows main rest")
CUS = 256
_lib = None


def lib():
    global _lib
    if _lib is None:
        with tempfile.TemporaryDirectory() as tmp:
            src, out = os.path.join(tmp, "plan.cpp"), os.path.join(tmp, "plan.so")
            with open(src, "w") as f:
                f.write(SOURCE)
            subprocess.check_call(["g++", "-O2", "-std=c++17", "-fPIC", "-shared", "-I", CSRC, "-I", os.path.join(ROOT, "include"), src, "-o", out])
            _lib = C.CDLL(out)
            _lib.plan_all.argtypes = [C.c_uint32] * 5 + [C.c_uint64, C.POINTER(C.c_uint32)]
            _lib.plan_room.argtypes, _lib.plan_room.restype = [C.c_uint32, C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32], C.c_uint64
    return _lib


def constants():
    return dict(zip(("part_most", "counters", "row_bytes", "skinny_parts"), (int(lib().plan_constants(i)) for i in range(4))))


def side(tiling):
    return int(lib().plan_side(tiling))


def columns(tile, dual):
    return int(lib().plan_columns(tile, dual))


def is_skinny(rows, type):
    return bool(lib().plan_is_skinny(rows, type))


def skinny_parts(N, K, type, cus=CUS):
    return int(lib().plan_skinny_parts(N, K, type, cus))


def room(dim, hidden, max_rows, type, training):
    return int(lib().plan_room(dim, hidden, max_rows, type, 1 if training else 0))


def plans(n, dim, hidden, type, cus=CUS, room=None):
    """All plans of a block's launches: {name: RowPlan}."""
    to = (C.c_uint32 * (15 * len(NAMES)))()
    lib().plan_all(n, dim, hidden, type, cus, room if room is not None else constants()["part_most"], to)
    out = {}
    for i, name in enumerate(NAMES):
        w = list(to[15 * i:15 * i + 15])
        main, rest = (Plan(x[0], ((x[1], x[2]), (x[3], x[4])), x[5], bool(x[6])) for x in (w[1:8], w[8:15]))
        out[name] = RowPlan(w[0], main, rest)
    return out


def kinds(n, dim, hidden, type):
    """What kinds of launches a block of such sizes has: (bits of an element, launch, which rows, tile, which of its products are cut along K)."""
    out, bits = set(), 32 if type == 0 else 16
    for name, p in plans(n, dim, hidden, type).items():
        whole = p.rows == (hidden if name == "weights" else n)
        for which, plan, rows in (("first", p.main, p.rows),) if whole else (("first", p.main, p.rows), ("last", p.rest, n - p.rows)):
            if name in ("gate", "out") and is_skinny(rows, type):
                parts = skinny_parts(dim, hidden, type) if name == "out" else 1
                out.add((bits, name, which, f"skinny {(rows + 15) // 16}", (parts > 1,)))
            else:
                cut = tuple(s > 1 for s, _ in plan.splits[:2 if name == "both" and which == "first" else 1])
                out.add((bits, name, which, side(plan.tiling), cut))
    return out
