"""Where tokens' rows lie, by the kernels' own arithmetic on the CPU: as the oracle says for lists that are
sound, and inside the cache for lists of any numbers (address checks on every read)."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import attn8

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def replay(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx or not os.path.exists(os.path.join(ROCM, "include", "hip")):
        pytest.skip("needs g++ and the ROCm headers")
    out = str(tmp_path_factory.mktemp("replay") / "cache8_places")
    subprocess.run([gxx, "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover", "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2406_20037_amd", "csrc"),
                    os.path.join(HERE, "replay", "cache8_places.cpp"), "-o", out], check=True)

    def run(starts, lengths, table, page, pages, tokens):
        table = np.asarray(table).reshape(len(lengths), -1)
        text = f"{len(lengths)} {tokens} {pages} {page} {table.shape[1]}\n" + " ".join(
            str(int(x)) for a in (starts, lengths, table.ravel()) for x in a)
        r = subprocess.run([out], input=text, capture_output=True, text=True,
                           env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0"})
        assert r.returncode == 0, r.stdout[-200:] + r.stderr[-2000:]
        return [tuple(map(int, l.split())) for l in r.stdout.splitlines()]
    return run


@pytest.mark.parametrize("seed", range(12))
def test_places(replay, seed):
    rng = np.random.default_rng(seed)
    seqs, page = int(rng.integers(1, 200 if seed % 3 else 3)), int(rng.choice([16, 48, 64]))
    new = rng.integers(0, 6, seqs)
    starts = int(rng.integers(0, 4)) + np.concatenate([[0], np.cumsum(new)])
    lengths = np.maximum(0, new + rng.integers(-2, 150, seqs))      # some shorter than what is new
    table = rng.integers(0, 40, (seqs, -(-int(lengths.max() + 1) // page)))
    tokens = int(starts[-1]) + 3
    want = attn8.places(starts, lengths, table, page, 40, tokens)
    got = replay(starts, lengths, table, page, 40, tokens)
    for t in range(tokens):
        if want[t] is None:
            assert got[t][0] == -2, t
        elif want[t][2] is None:
            assert got[t][0] == -1, t
        else:
            assert got[t] == want[t][2:], t


@pytest.mark.parametrize("seed", range(12))
def test_any_numbers(replay, seed):
    rng = np.random.default_rng(100 + seed)
    ends = np.array([-2 ** 31, -2 ** 31 + 1, -1, 0, 1, 15, 16, 2 ** 31 - 1, 2 ** 31 - 2])

    def wild(n):
        return np.where(rng.random(n) < 0.6, rng.choice(ends, n), rng.integers(-100, 300, n))
    seqs = int(rng.integers(1, 90))
    for pages in (1, 7, 2 ** 31 - 1):
        replay(wild(seqs + 1), wild(seqs), wild(seqs * 5), 32, pages, 200)


def test_a_short_table(replay):
    """Positions past the table have no place."""
    got = replay([0, 40], [40], [[3, 4]], 16, 9, 40)
    assert got[:16] == [(3, i) for i in range(16)] and got[31] == (4, 15) and got[32:] == [(-1, 0)] * 8
    assert replay([0, 2], [2], np.zeros((1, 0)), 16, 9, 2) == [(-1, 0)] * 2
