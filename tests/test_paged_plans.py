"""What attention calls over pages plan and launch, on a device of 256 compute units that is made up (tests/sanitize/plan_driver.cpp):
the plan is one that the launched kernel carries out, and long keys of few heads are shared among many workgroups.  CPU only; the
host layer is built under the sanitizers."""
import os
import random
import subprocess
from collections import namedtuple

import pytest

import test_sanitizers as S

Call = namedtuple("Call", "e4m3 prompt batch hq hkv dim rows page width bound splits window sinks")
Plan = namedtuple("Plan", "status launches workgroups rows_per_wg units row_groups splits spread half_ring key_groups bytes")
CUS, COUNTERS = 256, 65536


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    from paper_2606_00535_amd import build as B
    if not os.path.isdir(B.BUILD_DIR) or not all(
            os.path.exists(os.path.join(B.BUILD_DIR, os.path.basename(s) + ".o")) for s in B.sources()):
        B.build()
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc is not installed")
    tmp = tmp_path_factory.mktemp("plans")
    host = [x for flag in S.SAN for x in ("-Xarch_host", flag)]     # host code only: the device code is built as usual
    api, driver, exe = (str(tmp / x) for x in ("api_san.o", "plan_driver.o", "plan_driver"))
    subprocess.run([B.HIPCC] + [f for f in B.CFLAGS if f != "-O3"] + ["-O1", "-g"] + host +
                   ["-c", os.path.join(B.CSRC, "dreams_api.hip"), "-o", api], check=True, capture_output=True)
    subprocess.run([B.HIPCC, "-O1", "-g", "-std=c++17"] + host +
                   ["-I" + B.INCLUDE, "-I" + B.CSRC, "-I/opt/rocm/include", "-D__HIP_PLATFORM_AMD__", "-c",
                    os.path.join(S.HERE, "plan_driver.cpp"), "-o", driver], check=True, capture_output=True)
    objs = [os.path.join(B.BUILD_DIR, os.path.basename(s) + ".o") for s in B.sources()
            if os.path.basename(s) != "dreams_api.hip"]
    subprocess.run([B.HIPCC, "--offload-arch=" + B.ARCH] + host + ["-o", exe, driver, api] + objs,
                   check=True, capture_output=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")

    def run(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        r = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=300, env=env)
        assert r.returncode == 0 and "plan driver: ok (%d calls)" % len(calls) in r.stderr, r.stderr[-2000:]
        return [Plan(*map(int, line.split())) for line in r.stdout.splitlines()]

    return run


def call(e4m3, kind, batch, heads, dim, rows, longest, page=64, splits=0, window=0, sinks=0):
    return Call(int(e4m3), int(kind == "prompt"), batch, *heads, dim, rows, page, -(-(longest + rows) // page), longest, splits,
                window, sinks)


# one group of 128 rows a KV head behind long keys: batch, heads, D, rows, longest prefix, pieces
MANY_ROWS = [(1, (28, 4), 128, 16, 32768, 32), (1, (8, 2), 128, 30, 32768, 32), (3, (28, 4), 128, 18, 30000, 16),
             (4, (32, 8), 128, 30, 32768, 8), (8, (32, 8), 128, 30, 16384, 4), (2, (32, 32), 64, 60, 20000, 4),
             (3, (7, 1), 128, 15, 29358, 32), (7, (16, 16), 64, 38, 6789, 2), (1, (5, 5), 64, 33, 20000, 32),
             (2, (8, 1), 64, 16, 30000, 32)]


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("batch,heads,dim,rows,longest,pieces", MANY_ROWS)
def test_keys_of_128_rows_come_in_pieces(plans, batch, heads, dim, rows, longest, pieces, kind):
    """The kernel of 128 rows does not spread keys: it takes the pieces that merge within the launch."""
    p, = plans([call(True, kind, batch, heads, dim, rows, longest)])
    assert p.status == 0 and p.rows_per_wg == 128 and p.row_groups == 1 and p.spread == 0
    assert p.splits == pieces and p.launches == 1
    assert p.workgroups >= p.units * pieces


# batch, heads, D, rows, longest prefix, window: more (sequence, KV head)s than twice the compute units
FULL = [(14, (37, 37), 128, 5, 16598, 260), (16, (40, 40), 128, 1, 500, 0), (16, (40, 40), 64, 5, 1000, 0), (27, (40, 40), 128, 1, 2000, 0),
        (27, (40, 40), 128, 20, 2000, 0), (27, (40, 40), 128, 60, 2000, 0), (40, (40, 40), 128, 60, 3000, 0), (14, (74, 37), 128, 8, 1000, 0)]


@pytest.mark.parametrize("kind", ["verify", "prompt"])
@pytest.mark.parametrize("batch,heads,dim,rows,longest,window", FULL)
def test_units_that_fill_the_chip_stay_whole(plans, batch, heads, dim, rows, longest, window, kind):
    """Pieces would cost their starts and merges and gain nothing."""
    p, = plans([call(True, kind, batch, heads, dim, rows, longest, window=window, sinks=4)])
    assert p.status == 0 and p.units > 2 * CUS and p.rows_per_wg <= 64
    assert p.splits == 1 and p.bytes == 0


@pytest.mark.parametrize("batch,heads,rows,longest", [(1, (20, 4), 11, 22364), (4, (3, 1), 12, 22285), (3, (2, 1), 22, 17733), (1, (2, 2), 36, 15776)])
def test_spread_rather_than_as_many_pieces_as_there_can_be(plans, batch, heads, rows, longest):
    """64 rows of few heads: 32 pieces leave each compute unit one workgroup, spread keys two."""
    p, = plans([call(True, "verify", batch, heads, 128, rows, longest)])
    assert p.rows_per_wg == 64 and p.spread == 2 * CUS
    forced, = plans([call(True, "verify", batch, heads, 128, rows, longest, splits=60)])
    assert forced.spread == 0 and forced.splits == 32


def test_plans_are_carried_out(plans):
    """Spread keys: two launches, of as many workgroups as planned, up to 64 rows a KV head.  Else one launch of every unit's
    pieces.  The workspace is the launch's."""
    rng = random.Random(5)
    log = lambda lo, hi: round(lo * (hi / lo) ** rng.random())
    calls = []
    for _ in range(8000):
        kind, hkv = rng.choice(("verify", "prompt")), log(1, 40)
        window = rng.choice((0, 0, log(1, 8000)))
        calls.append(call(rng.random() < 0.8, kind, log(1, 80), (hkv * rng.choice((1, 1, 2, 3, 4, 5, 7, 8)), hkv),
                          rng.choice((64, 128)), log(1, 128 if kind == "verify" else 2000), log(1, 40000),
                          rng.choice((16, 32, 64)), rng.choice((0, 0, 0, log(1, 40))), window, rng.choice((0, 4, 70))))
    seen = {"spread": 0, "pieces": 0, "whole": 0, "many": 0}
    for c, p in zip(calls, plans(calls)):
        assert p.status == 0, c
        assert 1 <= p.splits <= 32, (c, p)
        if p.spread:
            assert c.e4m3 and c.splits == 0 and p.splits == 1 and p.rows_per_wg <= 64 and p.row_groups == 1, (c, p)
            assert p.launches == 2 and p.workgroups == p.spread >= 2 * p.units, (c, p)
            partial = p.spread * p.rows_per_wg
        else:
            assert p.launches == 1 and p.workgroups >= p.units * p.row_groups * p.splits, (c, p)
            partial = p.units * p.row_groups * p.splits * p.rows_per_wg if p.splits > 1 else 0
        if partial:
            assert 0 <= p.bytes - COUNTERS - partial * (c.dim + 2) * 4 <= partial * 4 + 3 * 256, (c, p)
        else:
            assert p.bytes == 0, (c, p)
        seen["spread" if p.spread else "pieces" if p.splits > 1 else "whole"] += 1
        seen["many"] += c.e4m3 and p.rows_per_wg == 128
    assert min(seen.values()) >= 50, seen
