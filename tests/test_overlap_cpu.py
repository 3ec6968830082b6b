"""Whether rows in memory overlap (csrc/overlap.h, compiled on its own) against every byte of them."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MAIN = r"""
#include "overlap.h"
#include <cstdio>
// {address rows width stride} twice a line
int main() {
    long long x[8];
    while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld", x, x + 1, x + 2, x + 3, x + 4, x + 5, x + 6, x + 7) == 8) {
        const a2t::Rows a{(const void*)x[0], x[1], x[2], x[3]}, b{(const void*)x[4], x[5], x[6], x[7]};
        std::printf("%d %d\n", a2t::overlap(a, b), a2t::overlap(b, a));
    }
}
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    tmp = tmp_path_factory.mktemp("overlap")
    (tmp / "main.cpp").write_text(MAIN)
    exe = str(tmp / "main")
    subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined",
                    f"-I{os.path.join(ROOT, 'paper_2609_31224_amd', 'csrc')}", str(tmp / "main.cpp"), "-o", exe], check=True)

    def run(pairs):
        text = "\n".join(" ".join(map(str, a + b)) for a, b in pairs) + "\n"
        got = [l.split() for l in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()]
        assert len(got) == len(pairs) and all(x == y for x, y in got)
        return [x == "1" for x, _ in got]
    return run


def _bytes(r):
    at, rows, width, stride = r
    return {at + i * stride + j for i in range(rows) for j in range(width)}


def test_against_every_byte(overlap):
    rng = random.Random(7)

    def rows():
        width = rng.randint(1, 9)
        return (rng.randint(1, 120), rng.randint(1, 7), width, width + rng.choice([0, 0, 1, 3, 8, 17, 30]))
    pairs = [(rows(), rows()) for _ in range(6000)]
    pairs += [(a, (b[0], b[1], min(b[2], a[3]), a[3])) for a, b in ((rows(), rows()) for _ in range(6000))]      # equal strides
    assert overlap(pairs) == [bool(_bytes(a) & _bytes(b)) for a, b in pairs]


def test_parts_of_one_tensor_and_far_rows(overlap):
    """Queries, keys and values side by side; rows at the ends of a large memory; nothing at address 0 (no tensor)."""
    far = 2 ** 40
    q, k, v = (4096, 1000, 512, 768), (4096 + 512, 1000, 128, 768), (4096 + 640, 1000, 128, 768)
    cases = [(q, k, False), (k, v, False), (q, (4096 + 504, 1000, 128, 768), True), (k, (4096 + 512 + 768 * 999, 1, 128, 128), True),
             (k, (4096 + 640 + 768 * 998, 1, 128 + 512, 640), False), (k, (4096 + 640 + 768 * 998, 1, 128 + 513, 641), True),
             ((4096, 2 ** 20, 64, far), (4096 + 64, 2 ** 20, 64, far), False), ((4096, 2 ** 20, 64, far), (4096 + far * (2 ** 20 - 1) + 63, 1, 1, 1), True),
             ((0, 10, 64, 64), (0, 10, 64, 64), False)]
    assert overlap([c[:2] for c in cases]) == [c[2] for c in cases]
