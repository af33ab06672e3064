"""Rows turned in place: which layouts have distinct rows, against all pairs of rows, and what dig_rope refuses before a launch."""
import ctypes
import itertools
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2405_18428_b200", "csrc")

CODE = """
#include "row_sets.h"
using namespace dig;
extern "C" int one(int B, int L, long long sb, long long st, long long w) { return distinct({B, L, sb, st, w}); }
extern "C" int two(int B, int L, long long qb, long long qt, long long qw, long long kb, long long kt, long long kw, long long off)
{
    return apart({B, L, qb, qt, qw}, {B, L, kb, kt, kw}, off);
}
extern "C" int block(int B, int L, long long sb, long long st, long long w, long long off, long long width) { return rows_meet_block({B, L, sb, st, w}, off, width); }
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rows")
    (d / "rules.cpp").write_text(CODE)
    so = str(d / "rules.so")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, str(d / "rules.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    ll = ctypes.c_longlong
    lib.one.argtypes = [ctypes.c_int] * 2 + [ll] * 3
    lib.block.argtypes = [ctypes.c_int] * 2 + [ll] * 5
    lib.two.argtypes = [ctypes.c_int] * 2 + [ll] * 7
    return lib


def elements(B, L, sb, st, w, off=0):
    return [range(off + b * sb + l * st, off + b * sb + l * st + w) for b in range(B) for l in range(L)]


def overlap(rows, others=None):
    pairs = itertools.combinations(rows, 2) if others is None else itertools.product(rows, others)
    return any(a.start < b.stop and b.start < a.stop for a, b in pairs)


def test_rows_of_one_tensor(rules):
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(4000):
        B, L, w = rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 4)
        sb, st = (rng.choice([0, w, w - 1, w * L, rng.randint(0, 30)]) for _ in range(2))
        want = not overlap(elements(B, L, sb, st, w))
        assert bool(rules.one(B, L, sb, st, w)) == want, (B, L, sb, st, w)
        seen[want] += 1
    assert min(seen) > 500


def test_rows_of_two_tensors(rules):
    rng = random.Random(2)
    seen = [0, 0]
    for _ in range(8000):
        B, L, qw, kw = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 4)
        pitch = qw + kw + rng.randint(0, 3)
        qt, kt = rng.choice([(pitch, pitch), (pitch, pitch), (qw, kw), (pitch + 1, pitch)])
        qb = kb = rng.choice([L * pitch, L * pitch, L * (qt + kt), pitch])
        if rng.random() < 0.2:
            kb += rng.randint(1, 3)
        off = rng.choice([qw, -kw, L * qt, pitch * B * L, rng.randint(-60, 60)])
        if not (rules.one(B, L, qb, qt, qw) and rules.one(B, L, kb, kt, kw)):
            continue
        want = not overlap(elements(B, L, qb, qt, qw), elements(B, L, kb, kt, kw, off))
        got = bool(rules.two(B, L, qb, qt, qw, kb, kt, kw, off))
        assert want or not got                       # never accepted where they meet
        alike = (B == 1 or qb == kb) and (L == 1 or qt == kt)
        if alike:
            assert got == want, (B, L, qb, qt, qw, kb, kt, kw, off)
        seen[got] += 1
    assert min(seen) > 500
    # queries and keys of a sequence behind one another, sequence by sequence and token by token
    assert rules.two(3, 5, 5 * 12, 8, 8, 5 * 12, 4, 4, 5 * 8)
    assert rules.two(3, 5, 8, 3 * 12, 8, 4, 3 * 12, 4, 3 * 8)


def test_a_block_between_rows(rules):
    rng = random.Random(3)
    seen = [0, 0]
    for _ in range(6000):
        B, L, w = rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 4)
        sb, st = (rng.choice([0, w, w + 3, (w + 3) * L + 9, rng.randint(0, 30)]) for _ in range(2))
        off, width = rng.randint(-20, 90), rng.randint(1, 6)
        want = overlap(elements(B, L, sb, st, w), [range(off, off + width)])
        assert bool(rules.block(B, L, sb, st, w, off, width)) == want, (B, L, sb, st, w, off, width)
        seen[want] += 1
    assert min(seen) > 500


def test_long_strides_and_many_rows(rules):
    far = 1 << 60
    assert rules.one(4, 2, far, 1 << 30, 64) and not rules.one(2, 3, far, 0, 64) and not rules.one(1 << 30, 1, 0, 64, 64)
    assert rules.one(46000, 46000, 64, 46000 * 64, 64) and not rules.one(46000, 46000, 64, 45999 * 64, 64)
    assert rules.two(2, 2, far, 128, 64, far, 128, 64, 64) and not rules.two(2, 2, far, 128, 64, far, 128, 64, far + 32)


BASE = 0x100000          # never dereferenced: validation fails first


def test_rope_refuses_rows_that_coincide_in_place():
    from paper_2405_18428_b200 import build, dig
    build.build()
    lib = dig.lib()

    def rope(q=BASE, k=None, q_out=BASE, k_out=None, strides=None, B=2, L=6, H=4, Hk=0, d=64, dtype=1):
        s = None if strides is None else (ctypes.c_longlong * len(strides))(*strides)
        return lib.dig_rope(q, k, s, BASE, 1, 1, (ctypes.c_double * 4)(1, 1, 1, 1), (ctypes.c_int * 4)(0, 0, 0, 0), 4, q_out, k_out, B, L, H, Hk, d, 0, 0, dtype, None)

    # one sequence for the whole batch, tokens dense or not; sequences or tokens that overlap by a part; one token
    for strides in ((0, 256), (0, 1024), (128, 1024), (1024, 128), (6 * 256 - 8, 256), (0, 0), (256, 256)):
        assert rope(strides=(*strides, 0, 0)) == dig.DIG_ERR_INVALID_ARG, strides
    assert rope(strides=(0, 256, 0, 0), L=1) == rope(strides=(128, 256, 0, 0), L=1) == rope(strides=(0, 128, 0, 0), B=1) == dig.DIG_ERR_INVALID_ARG
    other = BASE + (1 << 20)
    # keys alone
    assert rope(k=other, k_out=other, q_out=other + (1 << 20), Hk=4, strides=(6 * 256, 256, 0, 256)) == dig.DIG_ERR_INVALID_ARG
    # keys that are some of the queries' heads, tokens, or sequences; in place or only read
    for off, strides in ((128, (6 * 256, 256) * 2), (6 * 256 * 2, (6 * 512, 512) * 2), (256 * 2, (6 * 256, 256) * 2), (6 * 256 * 2, (6 * 256, 256) * 2)):
        for k_out in (BASE + off, other):
            assert rope(k=BASE + off, k_out=k_out, Hk=2, strides=strides) == dig.DIG_ERR_INVALID_ARG, (off, strides)
    assert rope(k=BASE + 128, k_out=BASE + 128, Hk=2) == dig.DIG_ERR_INVALID_ARG
