"""Outputs of the cache's reading and writing, of rotary positions and of attention whose rows and heads lie in each other are refused, on a device that need not be there."""
import pytest
import torch

import kv_plain
from paper_2602_17698_amd import binding as sb
from recording_runtime import record

SCRIPT = r"""
import ctypes as C
device(256, 1)
ctx = sb.Context(0, 0)
A = fake(1)
turns = sb.Rotary(A, 16, 0, 1.0)
seqs = sb.Sequences(A, A, A, 4, 3, 4, 0, 0)
def call(name, *args):
    return getattr(sb.load(), "sbits_" + name)(ctx.h, *[C.addressof(a) if isinstance(a, C.Structure) else a for a in args])
def rotate(tokens, heads, ld, hd):
    return call("rotate", turns, A, tokens, heads, 32, A, 0, 0, 0, 0, A + 8192, ld, hd)
def every(tokens, heads, ld, hd):
    of = lambda n: sb.KvCache(A, A, A, A, 8, n * 16 * 16, n * 16 * 4, 16, n, 32)
    out = [rotate(tokens, heads, ld, hd),
           call("kv_load", of(heads), seqs, tokens, A, ld, hd, None, 0, 0, 1), call("kv_load", of(heads), seqs, tokens, A, heads * 32, 32, A, ld, hd, 1),
           call("kv_attention", of(1), seqs, tokens, heads, A, heads * 32, 32, 0.1, 1, 0, A, ld, hd, None, A, 1 << 30),
           call("kv_store", of(1), seqs, tokens, A, 32, 32, A, 0, 0, 1, turns, None, A, 0, 0, heads, A + 8192, ld, hd)]
    launches = sum(line.startswith("launch") for line in log())
    return out, launches
"""
LAYOUTS = [(tokens, heads, ld, hd) for tokens in (1, 2, 3, 5) for heads in (1, 2, 4) for ld in (32, 40, 64, 96, 128, 160, 256) for hd in (32, 40, 64, 96, 136, 160, 320)]


def overlaps(tokens, heads, ld, hd, dim):
    """From the definition: every element's owner."""
    taken = set()
    for t in range(tokens):
        for h in range(heads):
            mine = set(range(t * ld + h * hd, t * ld + h * hd + dim))
            if taken & mine:
                return True
            taken |= mine
    return False


def test_outputs_that_lie_in_each_other_are_refused(tmp_path):
    got = record(tmp_path, SCRIPT + "answer([every(*a) for a in %r])" % LAYOUTS)
    refused = 0
    for layout, (codes, launches) in zip(LAYOUTS, got):
        bad = overlaps(*layout, 32)
        refused += bad
        assert codes == [sb.ERR_INVALID_ARG if bad else sb.OK] * 5, layout
        assert (launches == 0) if bad else (launches >= 5)
    assert 0 < refused < len(LAYOUTS)


# a row further on by one pitch, a head by another: equal for 60000 of the one and 60001 of the other
LARGE = [(1 << 30, 2, 32, 1 << 35, True), (1 << 30, 2, 32, (1 << 35) - 32, False), ((1 << 31) - 1, 65535, 65535 * 32, 32, True), ((1 << 31) - 1, 65535, 65535 * 32 - 8, 32, False),
         (1 << 20, 65535, (1 << 40) - 8, 32, True), (70000, 65535, 32 * 70001, 32 * 70000, True), (70000, 65535, 32 * 60001, 32 * 60000, False),
         (70000, 65535, 32, 32 * 70000, True)]


def test_large_outputs(tmp_path):
    got = record(tmp_path, SCRIPT + "answer([rotate(*a[:4]) for a in %r])" % (LARGE,))
    assert got == [sb.OK if a[4] else sb.ERR_INVALID_ARG for a in LARGE]


def test_attention_of_more_sequences_than_its_numbers_hold_is_refused(tmp_path):
    """Items to be joined are counted in 31 bits: four tiles of rows a sequence, and those of many rows beside them."""
    got = record(tmp_path, SCRIPT + """
out = []
for count in (1 << 24, (1 << 24) + 1, 1 << 30, (1 << 31) - 2):
    seqs = sb.Sequences(A, A, A, 32, count, 32, 0, 0)
    cache = sb.KvCache(A, A, A, A, 8, 64 * 16, 64 * 4, 64, 1, 32)
    need = call("kv_attention_ws_bytes", cache, seqs, 100000, 8)
    log()
    rc = call("kv_attention", cache, seqs, 100000, 8, A, 256, 32, 0.1, 1, 0, A, 256, 32, None, A, 1 << 40)
    lines = [line.split() for line in log()]
    out.append((need > 0, rc, sum(int(line[3].split(",")[2]) for line in lines if "join" in line[1]), sum(int(line[3].split(",")[2]) for line in lines if "many_kernel" in line[1])))
answer(out)
""")
    tiles = 100000 * 8 // 128 + (1 << 24)
    assert got == [[True, sb.OK, 4 << 24, tiles]] + [[False, sb.ERR_BAD_SHAPE, 0, 0]] * 3


def test_queries_and_what_they_become_go_together():
    ctx = sb.Context(device=-1)
    cache, seqs, _ = kv_plain.Batch([(2, 3), (1, 0)], 8, 2, 64).on(sb, dev="cpu")
    k, turn = torch.zeros(3, 2, 64), sb.rotary(torch.zeros(32, dtype=torch.float64))
    for other in (dict(q=k), dict(q_out=k)):
        with pytest.raises(ValueError):
            ctx.kv_store(cache, seqs, k, k, rotary=turn, **other)
    ctx.close()
