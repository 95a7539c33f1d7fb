"""How the choice of continuations is split (csrc/beam_split.h) and its workspace, asked on
the host: it holds what every smaller call writes, and not much more."""
import random
import shutil
import subprocess

import pytest

from paper_2609_39056_amd import _build
from test_abi import L  # noqa: F401

SRC = """
#include "beam_split.h"
#include <stdio.h>
using namespace sq;
int main() {
  int R, V, W;
  while (scanf("%d %d %d", &R, &V, &W) == 3) {
    const int each = beam_each(R, V, W), chunks = beam_chunks(V, each);
    printf("%d %d %zu\\n", each, chunks, (size_t)R * chunks * beam_chunk_bytes(W));
  }
}
"""
EDGES = [1, 2047, 2048, 2049, 4096, 4097, 8191, 8192, 8193, 32000, 50257, 65536, 131071, 1 << 18, (1 << 18) + 1, 1 << 20]
ROWS = [1, 2, 3, 7, 8, 9, 16, 31, 64, 100, 128, 129, 255, 256, 511, 512, 513, 1000, 1024, 1025, 4096, 8191, 8192, 8193, 65535]


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("beams")
    (d / "split.cpp").write_text(SRC)
    subprocess.run([cxx, "-std=c++17", "-O1", f"-I{_build.CSRC}", str(d / "split.cpp"), "-o", str(d / "split")], check=True)

    def ask(rows):
        text = "\n".join(" ".join(map(str, r)) for r in rows) + "\n"
        out = subprocess.run([str(d / "split")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]

    return ask


def nbytes(L, R, V, W):  # noqa: F811
    return L.sq_beam_workspace_bytes(R, 1, V, W)


def test_chunks_cover_a_row(split):
    asked = [(R, V, W) for R in ROWS for V in EDGES for W in (1, 4, 8, 16, 33, 64)]
    for (R, V, W), (each, chunks, _) in zip(asked, split(asked)):
        assert each in (8, 16, 32) and chunks * 256 * each >= V > (chunks - 1) * 256 * each
        assert chunks <= 128  # two of a lane


def test_workspace_holds_every_smaller_call(L, split):  # noqa: F811
    rng = random.Random(1)
    pairs = [((R, V, W), (R, V, W)) for R in ROWS for V in EDGES for W in (1, 8, 64)]
    for _ in range(30000):
        big = rng.choice(ROWS + [int(2 ** rng.uniform(0, 16))]), rng.choice(EDGES + [int(2 ** rng.uniform(0, 20))]), rng.randint(1, 64)
        big = min(big[0], 65535), big[1], big[2]
        small = tuple(rng.choice([b, max(1, b - 1), rng.randint(1, b), max(1, int(b * 2 ** -rng.uniform(0, 8)))]) for b in big)
        pairs.append((big, small))
    for (big, small), (_, _, used) in zip(pairs, split([s for _, s in pairs])):
        assert used <= nbytes(L, *big), (big, small)


def test_workspace_is_what_some_call_needs(L, split):  # noqa: F811
    """Where chunks of 2048 or 4096 tokens are taken, with fewer rows and tokens where the lengths of chunks change."""
    for R in ROWS[:18]:
        for V in EDGES:
            if V > 1 << 18 or R * -(-V // 2048) > 8192:
                continue
            smaller = [(r, v, 1) for v in {min(V, e) for e in EDGES} for r in range(1, R + 1)]
            most = max(used for _, _, used in split(smaller))
            assert nbytes(L, R, V, 1) <= max(256, 1.25 * most + 256), (R, V)
