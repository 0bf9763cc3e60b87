"""The paged cache's device rules on the CPU: a small program over the library's own header
answers one query per line."""

import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("kv_rules") / "kv_rules_check")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2605_28053_amd", "csrc"),
                    os.path.join(ROOT, "tests", "c", "kv_rules_check.cpp"), "-o", exe], check=True)

    def query(lines):
        out = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, check=True)
        answers = out.stdout.splitlines()
        assert len(answers) == len(lines)
        return [[int(x) for x in a.split()] for a in answers]
    return query


@pytest.mark.parametrize("spread", [1, 2, 3, 5, 40, 4095, 4096, 4097, 10 ** 6, 2 ** 31, 2 ** 32 - 1])
@pytest.mark.parametrize("close", [0, 6, 512])
def test_the_ranking_keeps_the_largest_scores(ask, spread, close):
    """Every number kept, of scores that tie, are neighbours, or span all 32 bits."""
    rng = random.Random(spread + close)
    cases = []
    for n in (2, 3, 17, 65, 200):
        for _ in range(6):
            base = -(spread // 2)
            score = [base + rng.choice([0, 1, 2, rng.randint(0, spread), spread]) % (spread + 1) for _ in range(n)]
            cases += [(want, score) for want in sorted({1, 2, n // 2, n - 2, n - 1} & set(range(1, n)))]
    got = ask([f"rank {want} {close} {len(s)} {' '.join(map(str, s))}" for want, s in cases])
    for (want, s), kept in zip(cases, got):
        assert kept == sorted(sorted(range(len(s)), key=lambda j: (-s[j], j))[:want]), (want, s)


@pytest.mark.parametrize("tile", [16, 32])
@pytest.mark.parametrize("longest", [16, 32, 48, 64, 256, 4096])
def test_every_tile_is_held_by_one_block_that_is_launched(ask, tile, longest):
    """The smallest caches, one 16-row page an owner, to those whose rows are split: all
    owners as long as they may be, of one row, and ragged with empty ones."""
    rng = random.Random(tile + longest)
    lines = []
    for n in (1, 2, 3, 7, 8, 64, 65, 480, 700):
        for vh in (1, 2, 8, 24):
            if n * vh > 2000:
                continue
            for lens in ([longest] * n, [1] * n, [rng.choice([0, 1, 15, 16, 17, rng.randint(0, longest)]) % (longest + 1)
                                                  for _ in range(n)]):
                for blocks in (256, 512):
                    lines.append(f"cut {blocks} {vh} {tile} {longest} {n} {' '.join(map(str, lens))}")
    for line, (grid, parts, lost, wrong, joins) in zip(lines, ask(lines)):
        assert (lost, wrong, joins) == (0, 0, 0) and 1 <= grid <= 512, line[:80]


def test_the_queries_unit_is_a_number(ask):
    """(1 / a) 127, or 0 where that overflows: the smallest magnitudes."""
    with np.errstate(over="ignore", divide="ignore"):
        values = [np.float32(x) for x in (0, 1e-45, 2.8e-39, 3e-39, 1e-38, 1e-37, 3.7e-37, 3.74e-37, 4e-37, 1e-30, 1, 127, 3e38)]
        for a, (bits,) in zip(values, ask([f"unit {float(a)!r}" for a in values])):
            to = np.float32(1) / a * np.float32(127) if a > 0 else np.float32(0)
            want = to if np.isfinite(to) else np.float32(0)
            assert np.uint32(bits).view(np.float32) == want, a


def test_queries_whose_unit_overflows_count_as_zero(ask):
    (bits,), (some,) = ask(["unit 1e-37", "unit 4e-37"])
    assert bits == 0 and some != 0


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_select_asks_for_lds_beyond_64_kb(ask, dim):
    """A block's fixed LDS counts too, and the widest table fits the CU's 160 KB."""
    sizes = list(range(1, 32768, 97)) + list(range(10900, 12300, 7)) + [11500, 12288, 12289, 32768]
    for pages, (bytes_, asked) in zip(sizes, ask([f"lds {dim} {n}" for n in sizes])):
        assert asked == (bytes_ > 64 * 1024) and bytes_ <= 160 * 1024, pages


def test_extend_never_writes_the_ring_where_it_reads(ask):
    """Every small ring, and a step that takes and returns pages: it is refused where the
    returned ones would lie on those that are taken, and only there."""
    steps = [(front, count, pages, taken, given) for pages in (1, 2, 5, 9) for front in range(pages)
             for count in range(pages + 1) for taken in range(count + 2) for given in range(pages + 2)]
    lines = [f"extend {f} {c} {p} {t} {g} 3 3" for f, c, p, t, g in steps]
    for (front, count, pages, taken, given), (verdict, meet) in zip(steps, ask(lines)):
        assert meet == 0, (front, count, pages, taken, given)
        assert verdict == (2 if taken > count else 1 if count + given > pages else 0)
    assert ask(["extend 0 4 5 1 1 4 3", "extend 5 0 5 0 0 0 0", "extend 0 6 5 0 0 0 0", "extend -1 0 5 0 0 0 0"]) == \
        [[2, 0], [1, 0], [1, 0], [1, 0]]


def test_the_hint_goes_by_the_most_a_call_can_read(ask):
    """64 KB a page of 16 rows: 1024 pages are 64 MB."""
    page = 64 << 10

    def hint(n_pages=100000, owners=8, max_pages=1000, keep=0, window=0, rows=16, layers=1):
        return ask([f"stream {n_pages} {owners} {max_pages} {keep} {window} {rows} {page} {layers}"]) == [[1]]
    assert hint() and not hint(n_pages=1024) and hint(n_pages=1025)            # the pool
    assert not hint(max_pages=128) and hint(max_pages=129)                     # what the listed owners can hold
    assert not hint(owners=1) and hint(owners=2) and hint(owners=1, layers=2)
    assert not hint(keep=128) and hint(keep=129) and not hint(keep=2000, max_pages=100)
    # a window of 16 * 127 + 1 rows touches 128 pages where it begins in a page's last row, of 16 * 127 + 2 one more
    assert not hint(window=16 * 127 + 1) and hint(window=16 * 127 + 2) and hint(window=1 << 23)


@pytest.mark.parametrize("blocks", [256, 512, 768])
@pytest.mark.parametrize("tile", [16, 32, 64])
@pytest.mark.parametrize("longest", [16, 48, 64, 256, 4096, 65536])
def test_every_tile_is_held_for_any_number_of_blocks(ask, blocks, tile, longest):
    """The same for three blocks a CU and tiles of 64 rows, and no more blocks launched than a call may have."""
    rng = random.Random(blocks + tile + longest)
    lines = []
    for n in (1, 2, 5, 8, 65, 480, 800):
        for vh in (1, 3, 8, 24):
            if n * vh > 2000 or n * vh * longest > 1 << 22:
                continue
            for lens in ([longest] * n, [1] * n, [rng.choice([0, 1, 15, 16, 17, 63, 64, 65, rng.randint(0, longest)]) % (longest + 1)
                                                  for _ in range(n)]):
                lines.append(f"cut {blocks} {vh} {tile} {longest} {n} {' '.join(map(str, lens))}")
    assert len(lines) > 8
    for line, (grid, parts, lost, wrong, joins) in zip(lines, ask(lines)):
        assert (lost, wrong, joins) == (0, 0, 0) and 1 <= grid <= blocks and parts <= grid, line[:80]
