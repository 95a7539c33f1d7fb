"""The paged attention's workspace, asked on the host: one that is sized for the
largest batch serves every smaller and shorter one."""
import ctypes
import shutil
import subprocess

import pytest

from paper_2609_39056_amd import _build
from paper_2609_39056_amd import binding as B
from test_abi import L  # noqa: F401

SRC = """
#include "attn_split.h"
#include <stdio.h>
using namespace sq;
int main() {
  int R, Hq, Hk, D, longest, window;
  while (scanf("%d %d %d %d %d %d", &R, &Hq, &Hk, &D, &longest, &window) == 6)
    printf("%zu\\n", attn_part_bytes(R, Hq, D, attn_split(attn_heads(R, Hq, Hk), attn_span(longest, window)).count));
}
"""
HEADS = [(40, 8, 128), (16, 16, 128), (8, 1, 256), (32, 1, 128), (20, 20, 96), (14, 2, 64), (512, 256, 64), (1, 1, 64)]
LONGEST = [1, 384, 385, 500, 640, 641, 900, 1000, 1280, 1281, 1500, 2000, 4096, 4097, 8192, 40000, 65536, 65537, 131072]
REQUESTS = [*range(1, 70), 95, 96, 97, 127, 128, 129, 191, 192, 193, 255, 256, 257, 511, 512, 513, 700, 2047, 2048, 2049, 9000, 65535]


def nbytes(L, R, Hq, Hk, D, longest):  # noqa: F811
    kv = B.sq_kv_cache(k=4096, v=4096, num_pages=10, num_heads=Hk, page_size=16, head_dim=D, dtype=B.SQ_OUT_BF16)
    return L.sq_attn_workspace_bytes(R, Hq, ctypes.byref(kv), longest)


@pytest.mark.parametrize("Hq,Hk,D", HEADS)
def test_workspace_grows_with_requests_and_length(L, Hq, Hk, D):  # noqa: F811
    last = [0] * len(REQUESTS)
    for longest in LONGEST:
        row = [nbytes(L, R, Hq, Hk, D, longest) for R in REQUESTS]
        assert row == sorted(row), longest
        assert all(a <= b for a, b in zip(last, row)), longest
        last = row


def test_workspace_holds_what_every_call_writes(L, tmp_path):  # noqa: F811
    cxx = shutil.which("g++") or shutil.which("clang++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "need.cpp").write_text(SRC)
    subprocess.run([cxx, "-std=c++17", "-O1", f"-I{_build.CSRC}", str(tmp_path / "need.cpp"), "-o", str(tmp_path / "need")],
                   check=True)
    asked = [(R, Hq, Hk, D, n, w) for Hq, Hk, D in HEADS for n in LONGEST for R in REQUESTS
             for w in (0, 354, 610, 700, 1250, 5000)]
    text = "\n".join(" ".join(map(str, a)) for a in asked) + "\n"
    out = subprocess.run([str(tmp_path / "need")], input=text, capture_output=True, text=True, check=True).stdout
    size = {}
    for (R, Hq, Hk, D, n, w), need in zip(asked, map(int, out.split())):
        key = (R, Hq, Hk, D, n)
        if key not in size:
            size[key] = nbytes(L, *key)
        assert need <= size[key], (key, w)
