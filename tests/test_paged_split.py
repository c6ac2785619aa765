"""How attention over pages cuts tokens into pieces: the kernels' arithmetic, compiled by itself, up to the longest sequences and largest batches that
the calls admit (table_pages * page_tokens < 2^31 - 4096, 2^35 over the batch)."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2501_19392_amd", "csrc")
PROGRAM = """
#include <cstdio>
#include "paged_split.h"
using namespace aquakv::paged;
int main() {
  char what;
  int a, b, c, d;
  while (std::scanf(" %c %d %d %d %d", &what, &a, &b, &c, &d) == 5) {
    if (what == 'r') { const TokenRange r = piece_range(a, b, c, d); std::printf("%d %d\\n", r.begin, r.end); }
    else if (what == 'p') std::printf("%d %d\\n", piece_tiles(a, b, c), short_piece(a, b));
    else std::printf("%d 0\\n", tiles_of_tokens(a, b));
  }
}
"""
LONGEST = 2 ** 31 - 4104                                                    # a multiple of 8


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("split")
    (d / "t.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, "-o", str(d / "t"), str(d / "t.cpp")], check=True)

    def ask(calls):
        text = "\n".join(" ".join(map(str, c)) for c in calls)
        out = subprocess.run([str(d / "t")], input=text, check=True, capture_output=True, text=True).stdout.split()
        return list(zip(map(int, out[::2]), map(int, out[1::2])))
    return ask


def covered(ranges, tokens, tile, each):
    """Pieces follow each other, each begins on a tile and holds `each` of them but for the last, and the last ends with the tokens."""
    at = 0
    for begin, end in ranges:
        if begin == end:
            continue
        assert begin == at and begin % tile == 0 and 0 < end - begin <= each * tile
        at = end
    assert at == max(tokens, 0)


@pytest.mark.parametrize("tokens", [-5, 0, 1, 31, 32, 33, 63, 64, 65, 700, 131072, 2 ** 26 + 1, 2 ** 30 + 77, LONGEST - 64, LONGEST - 1, LONGEST])
@pytest.mark.parametrize("slots", [1, 2, 3, 128, 170, 255, 256, 512, 1365, 2048, 4096])
def test_the_pieces_of_one_sequence(ask, slots, tokens):
    for tile in (32, 64):
        tiles = -(-max(tokens, 0) // tile)
        assert ask([("t", tokens, tile, 0, 0)]) == [(tiles, 0)]
        each = -(-tiles // slots)
        covered(ask([("r", i, each, tile, tokens) for i in range(slots)]), tokens, tile, each)


@pytest.mark.parametrize("slots,lengths", [
    (1, [2 ** 30] * 32), (2, [LONGEST] * 16), (1, [LONGEST] * 4 + [0, 5]), (64, [LONGEST, 1, 0, 33] * 4), (512, [LONGEST] * 16), (512, [3000] * 24),
    (128, [700] * 300), (4096, [LONGEST, 64]), (4096, [2 ** 19] * 65535), (1, [8] * 65535)])
def test_the_pieces_of_a_batch(ask, slots, lengths):
    """No more pieces than the workspace and the launch have room for, and every sequence whole."""
    assert sum(lengths) <= 2 ** 35
    tiles = [max(-(-n // 32), 1) for n in lengths]
    (each, short), = ask([("p", sum(tiles), slots, len(lengths), 0)])
    assert sum(-(-n // each) for n in tiles) <= max(slots, max(slots // 2, 1) + len(lengths))
    assert 1 <= short <= 4
    for each in (each, max(each, short)):
        for n in sorted(set(lengths)):
            pieces = -(-max(-(-n // 32), 1) // each)
            covered(ask([("r", i, each, 32, n) for i in range(pieces)]), n, 32, each)


RESULTS = """
#include <cstdio>
#include "paged_split.h"
using namespace aquakv::paged;
int main() {
  int a, b, c;
  while (std::scanf("%d %d %d", &a, &b, &c) == 3) std::printf("%d %d\\n", piece_tiles(a, b, c), piece_results(b, c));
}
"""


def test_the_results_of_sequences_in_several_pieces(tmp_path):
    """Whatever the lengths, there is room for the pieces of all sequences that have more than one (also where pieces are longer than they have to be, or as
    short as makes no more of them than `slots`)."""
    import random
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    (tmp_path / "t.cpp").write_text(RESULTS)
    subprocess.run(["g++", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", CSRC, "-o", str(tmp_path / "t"), str(tmp_path / "t.cpp")], check=True)
    rng, calls = random.Random(4), []
    for _ in range(4000):
        slots, batch = rng.choice([1, 2, 3, 4, 5, 8, 16, 31, 32, 64, 170]), rng.choice([2, 3, 5, 16, 31, 64, 65, 128, 200])
        top = rng.choice([2, 5, 40, 2000, 10 ** 6])
        tiles = [rng.randint(1, top) if rng.random() < rng.choice([0.02, 0.5, 1.0]) else 1 for _ in range(batch)]
        calls.append((slots, tiles))
    text = "\n".join(f"{sum(t)} {s} {len(t)}" for s, t in calls)
    out = subprocess.run([str(tmp_path / "t")], input=text, check=True, capture_output=True, text=True).stdout.split()
    for (slots, tiles), each, room in zip(calls, map(int, out[::2]), map(int, out[1::2])):
        def kept(n):
            return sum(-(-t // n) for t in tiles if t > n)
        assert kept(each) <= room and kept(each + 1) <= room and kept(4 * each) <= room
        if 2 * len(tiles) <= slots:                                         # the fewest tiles that do
            fewest = next(n for n in range(max(-(-sum(tiles) // slots), 1), each + 1) if sum(-(-t // n) for t in tiles) <= slots or n == each)
            assert kept(fewest) <= room
