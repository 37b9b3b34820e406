"""How decode on a 4-bit cache splits its keys (csrc/sb_split_kv4.h), compiled for the host: whatever the sizes, some launch writes every output."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_17980_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
NEAR, ROUND, MOST_SLOTS, MOST_T = 256, 256, 128, 524_288

MAIN = r"""
#include <stdio.h>
#include "sb_split_kv4.h"
int main()
{
    int B, H, Hkv, T, d, m;
    while (scanf("%d %d %d %d %d %d", &B, &H, &Hkv, &T, &d, &m) == 6) {
        const sb::kv4::Split s = sb::kv4::split_for(B, H, Hkv, T, d, m);
        printf("%d %d %d\n", s.near, s.C, s.slots);
    }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    if not shutil.which(HIPCC):
        pytest.skip("no hipcc")
    tmp = tmp_path_factory.mktemp("routes_kv4")
    (tmp / "main.hip").write_text(MAIN)
    subprocess.run([HIPCC, "-std=c++17", "-O1", "--offload-host-only", f"-I{CSRC}", "main.hip", "-o", "main"],
                   cwd=tmp, check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)

    def run(rows):
        text = "".join(" ".join(str(int(x)) for x in r) + "\n" for r in rows)
        out = subprocess.run([str(tmp / "main")], input=text, text=True, check=True, stdout=subprocess.PIPE).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def sizes():
    lengths = sorted({max(1, n + e) for n in (1, 32, 256, 1024, 2048, 3328, 4096, 65536, MOST_T - 1) for e in (-1, 0, 1)} | {1300, 2800, 4000})
    heads = [(1, 1, 1), (1, 32, 8), (32, 16, 16), (33, 32, 32), (64, 32, 32), (128, 8, 8), (129, 32, 8), (128, 16, 16), (255, 8, 8), (256, 256, 255), (65535, 1, 1), (1, 1024, 1), (2, 17, 1),
             (140, 128, 1), (128, 144, 1), (129, 128, 1), (341, 48, 1), (1024, 1, 1), (1025, 1, 1), (2047, 1, 1), (2048, 1, 1), (2049, 1, 1), (1, 8_388_000, 8192)]
    rng = random.Random(1)
    for _ in range(4000):
        Hkv = int(2 ** rng.uniform(0, 8))
        G = rng.choice((1, 1, 2, 4, 8, 16, 17, 40, 130, 1000))
        heads.append((min(65535 // Hkv, int(2 ** rng.uniform(0, 16))), G * Hkv, Hkv))
        lengths.append(int(2 ** rng.uniform(0, 19)))
    rows = [(*h, T, d, m) for h in heads[:23] for T in lengths[:40] for d in (32, 64, 128) for m in (0, 1)]
    return rows + [(*h, T, rng.choice((32, 64, 128)), rng.randrange(2)) for h, T in zip(heads[23:], lengths[-4000:])]


def test_every_split_has_launches_for_its_outputs(ask):
    """One chunk is the near launch's alone, which then writes the outputs; without a near launch the chunks' shares go through the last one, which takes two at least.
    Together they cover the keys and little more, and a chunk is whole rounds."""
    rows = sizes()
    for row, (near, C, slots) in zip(rows, ask(rows)):
        T = row[3]
        end = (T + 31) // 32 * 32
        assert 1 <= slots <= MOST_SLOTS, row
        if slots == 1:
            assert near == end, row
        else:
            assert near in (0, NEAR) and C % ROUND == 0 and C > 0, row
            assert slots - (near > 0) >= (2 if near == 0 else 1), row
            covered = near + (slots - (near > 0)) * C
            assert covered >= end and covered - C < T + 31, row
        assert end <= MOST_T


def test_many_workgroups_are_not_spread(ask):
    """Where the chip is full of them, a workgroup a head takes all keys that have to be read."""
    assert ask([(64, 32, 32, 4096, 128, 1), (33, 32, 32, 2049, 32, 1), (129, 32, 8, 4096, 128, 1)]) == [(4096, 128, 1), (2080, 128, 1), (4096, 128, 1)]
    assert [s for _, _, s in ask([(140, 128, 1, 2800, 32, 0), (129, 128, 1, 3500, 32, 0)])] == [1, 1]
    assert all(s > 1 for _, _, s in ask([(32, 32, 32, 4097, 128, 1), (1, 32, 8, 65000, 128, 0)]))
