"""The GPU tests of attention's tiles of 128 and 256 rows run the tiles that they are listed under."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path_factory.mktemp("host") / "kv_plan")
    r = subprocess.run([cxx, "-O2", "-std=c++17", "-I", os.path.join(ROOT, "paper_2406_06385_amd", "csrc"),
                        os.path.join(ROOT, "tests", "host", "kv_plan_host.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

    def run(hq, hkv, d, page, new, cached, extra=1):
        """As test_gpu_kv_attention.Setup makes its batch."""
        width = max(-(-(a + b) // page) for a, b in zip(new, cached)) + extra
        line = f"{hkv} {d} {hq} {len(new)} {max(new)} {max(cached)} {sum(new)} {width * page}"
        out = subprocess.run([exe], input=line, capture_output=True, text=True, check=True).stdout
        return dict(zip(("rows", "waves", "tiles", "chunk", "nsplit", "blocks"), map(int, out.split())))

    return run


def test_the_shapes_reach_their_tiles(plan):
    tests = pytest.importorskip("test_gpu_kv_attention_rows")
    for (rows, width, scales, split), (hq, hkv, d, page, block, new, cached) in tests.SHAPES.items():
        p = plan(hq, hkv, d, page, new, cached)
        assert (p["rows"], p["waves"], p["nsplit"] > 1) == (rows, rows // 32, split), (hq, hkv, d, new, cached, p)
        assert width == (64 if d <= 64 else 128 if d <= 128 else 256) and scales == ("token" if block == 1 else "block")


def test_every_instance_is_reached():
    tests = pytest.importorskip("test_gpu_kv_attention_rows")
    reached = {k[:3] for k in tests.SHAPES}
    assert reached == {(r, w, s) for r in (128, 256) for w in (64, 128, 256) for s in ("token", "block")
                       if not (r == 256 and w == 256)}                          # (no such kernel)
    assert {k[:2] for k in tests.SHAPES if k[3]} == {k[:2] for k in tests.SHAPES if not k[3]}
