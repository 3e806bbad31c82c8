"""Which keys each split of attention over the KV cache takes, compiled for the host: every key that a row sees
belongs to one split."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
MOST = 2 ** 31 - 2 ** 16    # positions of a page table, at most


@pytest.fixture(scope="module")
def splits(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("host") / "kv_split")
    r = subprocess.run([cxx, "-O2", "-std=c++17", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                        os.path.join(ROOT, "paper_2406_06385_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host", "kv_split_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(cases):
        text = "\n".join(" ".join(str(v) for v in c) for c in cases)
        r = subprocess.run([exe], input=text, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        out = [[int(v) for v in line.split()] for line in r.stdout.splitlines()]
        assert len(out) == len(cases)
        return [(v[0], v[1], v[2], list(zip(v[3::2], v[4::2]))) for v in out]

    return run


def _whole(count, spans, seen):
    """The spans that hold keys follow each other from key 0 to the last one seen, and are those that are joined."""
    at = 0
    for i, (k0, k1) in enumerate(spans):
        assert (k1 > k0) == (i < count or i == 0 < seen)
        if k1 > k0:
            assert k0 == at
            at = k1
    assert at == seen, (spans[-3:], seen)


def test_every_key_has_its_split(splits):
    rng = random.Random(11)
    cases = []
    for _ in range(4000):
        heads, group = rng.choice((1, 2, 8, 32)), rng.choice((1, 4, 8))
        new, cached = rng.choice((1, 1, 17, 333, 2000)), int(2 ** rng.uniform(0, 20))
        cases.append((heads, rng.choice((64, 128, 256)), heads * group, 1, new, cached, new, 1 << 30, rng.randint(1, new + cached)))
    for (_, nsplit, count, spans), case in zip(splits(cases), cases):
        _whole(count, spans, case[-1])
    assert len({n for _, n, _, _ in splits(cases)}) > 20


@pytest.mark.parametrize("back", [0, 1, 63, 64, 65536, 2 ** 22, 2 ** 23])
def test_the_last_positions_of_a_full_table(splits, back):
    """Whole splits would end at 2^31 and past it."""
    cases = [(h, 16, h, 1, 1, MOST - back - 1, 1, MOST, seen) for h in (1, 2, 4) for seen in (MOST - back, 1, MOST // 2)]
    for (chunk, nsplit, count, spans), case in zip(splits(cases), cases):
        assert nsplit > 1
        _whole(count, spans, case[-1])


def test_sequences_longer_than_planned(splits):
    """max_cached is the caller's word, the lengths are device memory: past it the last split has the rest, and a plan
    without splits, whose workspace holds no partial results, still has none."""
    rng = random.Random(12)
    cases = [(8, 128, 32, 1, 1, 511, 1, 4096, 513), (8, 128, 32, 1, 1, 300, 1, 4096, 4096), (8, 128, 32, 1, 1, 0, 1, MOST, MOST)]
    for _ in range(4000):
        heads, group = rng.choice((1, 2, 8, 32)), rng.choice((1, 4, 8))
        new, cached = rng.choice((1, 1, 17, 333, 2000)), int(2 ** rng.uniform(0, 16))
        cases.append((heads, rng.choice((64, 128, 256)), heads * group, 1, new, cached, new, MOST,
                      min(MOST, new + cached + int(2 ** rng.uniform(0, 31)))))
    one = 0
    for (chunk, nsplit, count, spans), case in zip(splits(cases), cases):
        assert 1 <= count <= nsplit
        _whole(count, spans, case[-1])
        one += nsplit == 1 and case[-1] > chunk
    assert one > 100
