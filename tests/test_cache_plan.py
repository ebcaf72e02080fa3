"""The cached attention's division of a batch into shares (csrc/cache_plan.h), on
the host: the keys of every row block are read exactly once and every cut unit is
joined from all its pieces, for random batches (empty sequences, no context,
contexts beyond the table, padding, lists that do not ascend)."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GROUPS = 512


def _batches(rng, n):
    for i in range(n):
        n_seqs = rng.choice((1, 1, 2, 3, 7, 40))
        kv = rng.choice((1, 2, 3, 8))
        group = rng.choice((1, 1, 2, 3, 5, 8, 16, 64))
        rows = rng.choice([t // group for t in (16, 32, 128) if t // group])
        new = [rng.choice((0, 1, 1, rng.randint(0, 40), rng.randint(0, 700))) for _ in range(n_seqs)]
        ctx = [rng.choice((0, 1, 127, 128, rng.randint(0, 300), rng.randint(0, 40000)))
               for _ in range(n_seqs)]
        cu = [0]
        for m in new:
            cu.append(cu[-1] + m)
        tokens = cu[-1] + rng.choice((0, 5))
        cap = rng.choice((1 << 20, 1 << 20, 4096, 16))
        if i % 10 == 0:                    # what a caller must not write
            cu[rng.randrange(n_seqs + 1)] = rng.randint(-5, tokens + 5)
            ctx[rng.randrange(n_seqs)] = rng.choice((-3, (1 << 31) - 1))
        yield (n_seqs, kv, rows, rng.randint(0, 1), rng.choice((GROUPS, GROUPS, 8, 1)),
               rng.choice((128, 128, 512)), rng.choice((64, 128)), rng.choice((0, 128, 192)), tokens, cap, *ctx, *cu)


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_every_key_is_read_once(tmp_path):
    exe = str(tmp_path / "plan")
    r = subprocess.run(["g++", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                        "-std=c++17", "-Wall", os.path.join(ROOT, "tests", "plan", "driver.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    rng = random.Random(5)
    lines = [" ".join(map(str, b)) for b in _batches(rng, 1500)]
    r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.strip() == "1500 batches"
