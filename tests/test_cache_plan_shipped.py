"""The cached attention's division of a batch into shares (csrc/cache_plan.h) with the
constants that its kernels run with, read from the header: the keys of every row block are
read exactly once and every cut unit is joined from all its pieces."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2301_08658_amd", "csrc", "cache_plan.h")
NAMES = ("kGroups", "kLeast", "kFewTile", "kFewExtra", "kWideTile", "kWideExtra")


def _compile(source, exe, *flags):
    r = subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", *flags, source, "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def _constants(tmp_path):
    source = tmp_path / "constants.cpp"
    prints = "".join(f'printf("%d ", atp::plan::{n});' for n in NAMES)
    source.write_text(f'#include <stdio.h>\n#include "{HEADER}"\nint main() {{ {prints} }}\n')
    _compile(str(source), str(tmp_path / "constants"))
    r = subprocess.run([str(tmp_path / "constants")], capture_output=True, text=True)
    return dict(zip(NAMES, map(int, r.stdout.split())))


def _batch(rng, c):
    wide = rng.random() < 0.5
    tile, extra = (c["kWideTile"], c["kWideExtra"]) if wide else (c["kFewTile"], c["kFewExtra"])
    group = rng.choice((1, 1, 2, 3, 5, 8, 16, 64))
    rows = 128 // group if wide else max(1, rng.choice((16, 32)) // group)
    n_seqs, kv = rng.choice((1, 1, 2, 5, 24, 64, 90)), rng.choice((1, 2, 4, 8))
    new = [rng.choice((0, 1, 1, rng.randint(0, 40), rng.randint(0, 1100))) for _ in range(n_seqs)]
    ctx = [rng.choice((0, 1, 319, 320, 321, rng.randint(0, 300), rng.randint(0, 40000)))
           for _ in range(n_seqs)]
    cu = [0]
    for m in new:
        cu.append(cu[-1] + m)
    return (n_seqs, kv, rows, rng.randint(0, 1), c["kGroups"], c["kLeast"], tile, extra,
            cu[-1] + rng.choice((0, 7)), rng.choice((1 << 20, 1 << 20, 4096)), *ctx, *cu)


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_key_is_read_once_with_the_kernels_constants(tmp_path):
    c = _constants(tmp_path)
    exe = str(tmp_path / "plan")
    _compile(os.path.join(ROOT, "tests", "plan", "driver.cpp"), exe, "-g", "-fsanitize=undefined",
             "-fno-sanitize-recover=all")
    rng = random.Random(6)
    lines = [" ".join(map(str, _batch(rng, c))) for _ in range(2000)]
    r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.strip() == "2000 batches"
