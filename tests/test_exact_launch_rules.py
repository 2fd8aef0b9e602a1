"""Which kernels the calls of the GPU tests take (host code of the launch rules, for 256 CUs): that a change of a rule
does not leave a kernel without its tests."""
import os
import shutil
import subprocess

import pytest

pytest.importorskip("torch")

import test_gpu_exact as exact  # noqa: E402
import test_gpu_exact_precision as precision  # noqa: E402
import test_gpu_exact_ranges as ranges  # noqa: E402
import test_gpu_exact_wide as wide  # noqa: E402
from paper_2201_12854_amd import build_lib  # noqa: E402

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    tmp = tmp_path_factory.mktemp("rules")

    def run(*cmd):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]

    objs = []
    for src in build_lib.SOURCES:
        built = os.path.join(build_lib.BUILD, src + ".o")
        if not os.path.exists(built):
            built = str(tmp / (src + ".o"))
            run(hipcc, *build_lib.CXXFLAGS, "-x", "hip", "-c", os.path.join(build_lib.CSRC, src), "-o", built)
        objs.append(built)
    drv, exe = str(tmp / "rules.o"), str(tmp / "rules")
    run(hipcc, *build_lib.CXXFLAGS, "-I", build_lib.CSRC, "-x", "hip", "-c", os.path.join(HERE, "sanitize", "exact_rules.cpp"), "-o", drv)
    run(hipcc, f"--offload-arch={build_lib.ARCH}", drv, *objs, "-o", exe)

    def kernels(shapes, dtype="bf16"):
        """(forward, dQ, dK and dV, parts of the bias gradient) of each call."""
        text = "".join("%d %d %d %d %d %d %d %d %d\n" % (dtype == "bf16", *s[:5], s[5].get("causal", False), s[5].get("window", 0),
                                                       s[5].get("max_distance", 128) if s[5].get("buckets") else 0) for s in shapes)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60, env=dict(os.environ, HIP_VISIBLE_DEVICES=""))
        got = [tuple(l.split()) for l in r.stdout.splitlines()]
        assert r.returncode == 0 and len(got) == len(shapes), r.stderr
        return got

    return kernels


def test_blocks_of_256(rules):
    assert {k[0] for k in rules(wide.WIDE + wide.SHARP)} == {"256"}


def test_every_kernel_is_tested(rules):
    plain, bias = rules(exact.SHAPES), rules(exact.BIAS)
    assert {k[0] for k in plain} >= {"32", "short", "128", "256"} and {k[0] for k in bias} == {"32", "128"}
    for at in (1, 2):
        assert {k[at] for k in plain} == {"32", "short", "128"} and {k[at] for k in bias} == {"32", "128"}
    for masks in (dict(causal=True), dict(window=True), dict(window=True, causal=True)):
        some = [s for s in exact.SHAPES if all(bool(s[5].get(m)) == bool(masks.get(m)) for m in ("causal", "window"))]
        for at in range(3):
            assert {k[at] for k in rules(some)} >= {"32", "128"}, (masks, at)
    assert {k[:3] for k in rules(exact.SHAPES + exact.BIAS, "f32")} == {("32",) * 3}


def test_large_biases_in_blocks_of_128(rules):
    shapes = [s[:5] + (dict(s[5], buckets=8, max_distance=20),) for s in ranges.LARGE]
    # query counts that leave part of a half tile to rows past the last one
    assert sum(k[2] == "128" and s[1] % 32 > 0 for s, k in zip(shapes, rules(shapes))) >= 4


def test_few_keys_or_queries(rules):
    for at in range(3):
        assert {k[at] for k in rules(precision.FEW)} == {"32", "short", "128"}
        assert "128" in {k[at] for k in rules([s for s in precision.FEW if s[5].get("buckets")])}


def test_bound_of_the_bias_gradient(rules):
    """The number of roundings that exact_testutil allows a value of the bias gradient covers what the kernels do. A dS
    of a near tile passes 7 additions along its diagonal, 5 that put the tile's four rows of entries together and 1
    with the next tile's; of a far one 15 in its tile, 1 per query tile of its head (at most), 1 over the wave's
    halves and 1 into the entries. Then those of a bucket's D + 65 entries at most that one of four lanes adds and 2 over
    the lanes, and the parts by 64 lanes and 6 over those."""
    shapes = [s for s in exact.BIAS + precision.FEW if s[5].get("buckets")]
    shapes += [s[:5] + (dict(s[5], buckets=8, max_distance=20),) for s in ranges.LARGE]
    for dtype in ("f32", "bf16"):
        for (B, nq, nk, _, _, kw), k in zip(shapes, rules(shapes, dtype)):
            top = kw.get("max_distance", 128)
            adds = max(7 + 5 + 1, 15 + -(-nq // 32) + 2) + -(-(top + 65) // 4) + 2 + -(-int(k[3]) // 64) + 6
            assert adds <= nq + nk + 8 + 2 * top + 129 + B * nq / 64 + 8, (dtype, B, nq, nk, kw, adds)
