"""The launch plan of an attention of drafts (csrc/plan.hpp, host code), compiled here on its own."""
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_03458_amd", "csrc")
FIELDS = ("row_blocks", "n_chunk", "n_wg", "share", "waves", "order")
MAIN = """
#include <cstdio>
#include "plan.hpp"
int main() {
    int a[8];
    while (scanf("%d %d %d %d %d %d %d %d", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7) == 8) {
        const kvarn::TreePlan p = kvarn::plan_tree(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7] != 0);
        printf("%d %d %d %d %d %d\\n", p.row_blocks, p.n_chunk, p.n_wg, p.share, p.waves, p.order);
    }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans([(batch, n_kv, n_q, n_draft, max_len, n_sink, max_blocks, two_pieces), ...]) -> list of plan dicts."""
    d = tmp_path_factory.mktemp("plan")
    (d / "main.cpp").write_text(MAIN)
    cxx = shutil.which("g++") or shutil.which("clang++") or "/opt/rocm/bin/amdclang++"
    subprocess.check_call([cxx, "-O1", "-std=c++17", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "plan")])

    def run(calls):
        text = "\n".join(" ".join(map(str, c)) for c in calls)
        out = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True, check=True).stdout
        return [dict(zip(FIELDS, map(int, line.split()))) for line in out.splitlines()]
    return run


def test_plans_cover_the_rows_and_bound_the_parts(plans):
    rng = random.Random(7)
    calls = []
    for _ in range(4000):
        n_kv, batch, tokens = rng.choice([1, 2, 3, 8, 16]), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(0, 31)) - 1
        sink = rng.choice([0, 0, 5, 128, 1024])
        calls.append((batch, n_kv, n_kv * rng.randint(1, 16), rng.randint(1, 64), tokens, sink,
                      rng.choice([tokens // 128 + 1, tokens // 300]), rng.randint(0, 1)))
    for (batch, n_kv, n_q, drafts, tokens, sink, blocks, two), p in zip(calls, plans(calls)):
        rows = drafts * (n_q // n_kv)
        size = 16 * p["row_blocks"]
        assert p["row_blocks"] in (1, 2) and not (two and p["row_blocks"] == 2)
        assert size * (p["n_chunk"] - 1) < rows <= size * p["n_chunk"]
        assert 1 <= p["n_wg"] <= 32
        units = min(max(tokens - sink, 0) // 128, blocks) + -(-min(sink, tokens) // 32) + 4 + -(-drafts // 32)
        assert p["share"] * p["n_wg"] >= units > p["share"] * p["n_wg"] - p["n_wg"]
        # the kernel forms unit * wave in 32 bits, and a merge reads a part per lane
        assert units * p["waves"] * p["n_wg"] < 2 ** 32 and p["n_wg"] <= 64
        assert p["waves"] * p["n_wg"] <= 128 and (p["waves"] == 4 or (p["waves"] == 8 and p["row_blocks"] == 1))
        # a wave ranks 128 sequences, and a sequence in parts is not ranked
        assert p["order"] == 0 or (p["order"] == 1 and batch <= 128 and p["n_wg"] == 1)
        # several parts only where their partials are few
        assert p["n_wg"] == 1 or batch * n_kv * p["n_chunk"] < 1536


def test_rules(plans):
    half, = plans([(8, 8, 32, 16, 4096, 0, 32, 0)])
    assert half == dict(row_blocks=1, n_chunk=4, n_wg=1, share=37, waves=8, order=0)  # one workgroup on each CU
    one, small, long, many, fp32 = plans([(1, 8, 32, 16, 8192, 0, 64, 0), (1, 8, 32, 1, 100, 0, 1, 0), (66, 8, 32, 16, 32768, 0, 256, 0),
                                          (256, 8, 32, 64, 32768, 0, 256, 0), (256, 8, 32, 64, 32768, 0, 256, 1)])
    assert one == dict(row_blocks=1, n_chunk=4, n_wg=8, share=9, waves=4, order=0)  # few rows: 16 at a time, parts of two units a wave
    assert small["n_wg"] == 1
    assert long["row_blocks"] == 2 and long["n_wg"] == 1 and long["order"] == 1  # two rounds of long sequences
    assert many == dict(row_blocks=2, n_chunk=8, n_wg=1, share=262, waves=4, order=0)
    assert fp32["row_blocks"] == 1 and fp32["n_chunk"] == 16
    round_and_some, = plans([(40, 8, 32, 16, 32768, 0, 256, 0)])
    assert round_and_some["n_wg"] == 4 and round_and_some["order"] == 0
    ranked, short, batch129 = plans([(128, 8, 32, 16, 8192, 0, 64, 0), (128, 8, 32, 4, 1024, 0, 8, 0), (129, 8, 32, 16, 8192, 0, 64, 0)])
    assert ranked["order"] == 1 and ranked["n_wg"] == 1
    assert short["order"] == 0 and batch129["order"] == 0
