"""How the key weights are laid out (csrc/sb_plan_key_weight.h), compiled for the host: whatever the sizes, every query row and key is some workgroup's, and launches and
the workspace stay within their bounds."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_17980_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

MAIN = r"""
#include <stdio.h>
#include "sb_plan_key_weight.h"
int main()
{
    int B, H, Hkv, Tq, T;
    while (scanf("%d %d %d %d %d", &B, &H, &Hkv, &Tq, &T) == 5) {
        const sb::key_weight::Plan p = sb::key_weight::plan_of(B, H, Hkv, Tq, T);
        printf("%d %d %d %d %d %d %d %zu %zu\n", p.small, p.pairs, p.groups, p.chunks, p.C, p.Tpad, p.at_once(B * Hkv), p.left_of(), p.floats(B * Hkv));
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if not shutil.which(HIPCC):
        pytest.skip("no hipcc")
    tmp = tmp_path_factory.mktemp("routes_key_weight")
    (tmp / "main.hip").write_text(MAIN)
    subprocess.run([HIPCC, "-std=c++17", "-O1", "--offload-host-only", f"-I{CSRC}", "main.hip", "-o", "main"],
                   cwd=tmp, check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)

    def run(rows):
        text = "".join(" ".join(str(int(x)) for x in r) + "\n" for r in rows)
        out = subprocess.run([str(tmp / "main")], input=text, text=True, check=True, stdout=subprocess.PIPE).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def accepted(B, H, Hkv, Tq, T):
    return B * Hkv <= 65535 and 1 <= Tq <= T <= 524_288 and B * H <= 16_777_215 and (Tq + 31) // 32 * (H // Hkv) * B * Hkv < 2 ** 31


def sizes():
    rng = random.Random(2)
    rows = [(1, 1, 1, 1, 1), (1, 32, 8, 524_288, 524_288), (400, 1, 1, 1, 524_288), (65535, 1, 1, 1, 524_288), (1, 1, 1, 524_288, 524_288), (1, 16_000_000, 1, 1, 31), (1, 100_000, 1, 4096, 4096),
            (16, 64, 64, 33, 65), (1, 4, 4, 1, 524_288), (255, 257, 257, 64, 64), (1, 1024, 1, 32, 524_288)]
    while len(rows) < 30_000:
        Hkv, G = int(2 ** rng.uniform(0, 8)), int(2 ** rng.uniform(0, rng.choice((0, 4, 10))))
        T = int(2 ** rng.uniform(0, 19))
        Tq = rng.choice((T, min(T, int(2 ** rng.uniform(0, 9))), rng.randint(1, T)))
        rows.append((int(2 ** rng.uniform(0, 16)) // Hkv + 1, G * Hkv, Hkv, Tq, T))
    return [r for r in rows if accepted(*r)]


def test_every_plan_covers_its_rows_and_keys(ask):
    seen = set()
    rows = sizes()
    for row, (small, pairs, groups, chunks, C, Tpad, at_once, left, floats) in zip(rows, ask(rows)):
        B, H, Hkv, Tq, T = row
        units, each = (Tq + 31) // 32 * (H // Hkv), 1 if small else 8 if pairs else 4
        assert Tpad == (T + 63) // 64 * 64 and (groups - 1) * each < units <= groups * each, row
        assert C % 64 == 0 and (chunks - 1) * C < T <= chunks * C and (chunks > 1 or C == Tpad), row
        assert not (small and (pairs or chunks > 1)) and not (pairs and chunks > 1), row
        assert 1 <= at_once <= groups and (chunks == 1 or at_once == groups), row
        # threads along x, chunks and heads along y
        assert chunks <= 65535 and (chunks == 1 or B * Hkv * groups * 256 < 2 ** 32) and (not small or groups * 512 < 2 ** 32), row
        assert left == (groups * 4 * chunks * 32 if chunks > 1 else 0), row
        assert floats == B * Hkv * (at_once * (Tpad + 2 * chunks) + 2 * left), row
        assert 4 * floats <= max(2 ** 31, 4 * Tpad * B * Hkv) + 8 * B * Hkv * at_once * chunks + 2 ** 26, row
        seen.add((small, pairs, chunks > 1, at_once < groups))
    assert len(seen) >= 6, seen
