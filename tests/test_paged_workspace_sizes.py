"""A workspace for the largest attention of a program does for its smaller ones: fewer rows and groups, shorter contexts, windows and prompts (no GPU needed)."""
import random

import pytest

import paper_2509_19128_amd as pl

HEADS = [(8, 2, 32), (28, 4, 128), (12, 2, 128), (40, 8, 128), (16, 1, 64), (1, 1, 32), (64, 32, 64)]
LENGTHS = [1, 31, 32, 33, 64, 200, 512, 513, 1000, 1024, 1500, 2048, 2049, 3000, 4096, 5000, 8192, 9000, 16384, 17584, 20000, 32768, 40000, 65536, 131071, 131072, 1 << 20, 1 << 30]
ROWS = [*range(1, 140), *range(140, 420, 3), 500, 511, 512, 513, 700, 1000, 1023, 1024]


def _growing(sizes):
    sizes = list(sizes)
    for a, b in zip(sizes, sizes[1:]):
        assert a <= b, sizes


@pytest.mark.parametrize("Hq,Hkv,hd", HEADS)
def test_decode(Hq, Hkv, hd):
    size = pl.pl_attention_workspace_bytes
    for n in (1, 3, 15, 16, 17, 31, 32, 89, 256, 1024):
        _growing(size(n, Hq, Hkv, hd, c) for c in LENGTHS)
    for most in LENGTHS:
        _growing(size(n, Hq, Hkv, hd, most) for n in ROWS)


@pytest.mark.parametrize("Hq,Hkv,hd", HEADS)
def test_window(Hq, Hkv, hd):
    size = pl.pl_attention_window_workspace_bytes
    for n in (1, 3, 16, 31, 32, 65, 70, 89, 256, 300, 1024):
        for window, sinks in ((1, 0), (200, 4), (4096, 4), (20000, 1), ((1 << 31) - 1, 0)):
            _growing(size(n, Hq, Hkv, hd, c, window, sinks) for c in LENGTHS)
        for most in (500, 8192, 131072):
            _growing(size(n, Hq, Hkv, hd, most, w, 4) for w in LENGTHS)
            _growing(size(n, Hq, Hkv, hd, most, 1000, s) for s in [0, *LENGTHS])
    for most in (500, 4096, 8192, 131072):
        for window in (64, 1000, 4096, 131071, 131072):
            _growing(size(n, Hq, Hkv, hd, most, window, 4) for n in ROWS)


@pytest.mark.parametrize("Hq,Hkv,hd", HEADS)
def test_shared(Hq, Hkv, hd):
    size = pl.pl_attention_shared_workspace_bytes
    for groups in (1, 4, 16):
        for most, shared in ((2000, 300), (8192, 2048), (17584, 16384), (131072, 16384), (131072, 131072)):
            _growing(size(n, groups, Hq, Hkv, hd, most, shared) for n in ROWS if n >= groups)
    for n in (1, 6, 32, 64, 100, 256, 1024):
        for most in (2000, 17584, 131072):
            _growing(size(n, g, Hq, Hkv, hd, most, most // 2) for g in range(1, n + 1))
            _growing(size(n, min(n, 4), Hq, Hkv, hd, most, s) for s in [0, *LENGTHS] if s <= most)
        _growing(size(n, min(n, 4), Hq, Hkv, hd, c, 1) for c in LENGTHS[:-1])
        _growing(size(n, min(n, 4), Hq, Hkv, hd, c, c) for c in LENGTHS[:-1])


def test_whatever_becomes_smaller():
    rng = random.Random(3)
    for _ in range(20000):
        Hq, Hkv, hd = rng.choice(HEADS)
        n, most = rng.choice(ROWS), rng.choice(LENGTHS[:-1])
        groups, shared, window, sinks = rng.randint(1, n), rng.randint(0, most), rng.choice(LENGTHS), rng.choice([0, *LENGTHS])
        n2, most2 = rng.randint(1, n), rng.randint(1, most)
        groups2, shared2 = rng.randint(1, min(n2, groups)), rng.randint(0, min(most2, shared))
        assert (pl.pl_attention_shared_workspace_bytes(n2, groups2, Hq, Hkv, hd, most2, shared2) <= pl.pl_attention_shared_workspace_bytes(n, groups, Hq, Hkv, hd, most, shared))
        assert (pl.pl_attention_window_workspace_bytes(n2, Hq, Hkv, hd, most2, rng.randint(1, window), rng.randint(0, sinks))
                <= pl.pl_attention_window_workspace_bytes(n, Hq, Hkv, hd, most, window, sinks))
