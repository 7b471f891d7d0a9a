"""Host only: the planner of requests of few rows (csrc/few_plan.h), compiled on its own: requests that share pages take no more slots for their sums than there
are, whoever's wavefronts share tiles, and calls in which all of them may do so still do."""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SLOTS = 4096   # of 16 rows each

HARNESS = r"""
#include <cstdio>
#include "few_plan.h"
int main() {
    int hq, hkv, n;
    long from;
    while (scanf("%d %d %ld %d", &hq, &hkv, &from, &n) == 4) {
        const int g = hq / hkv;
        std::vector<FewRequest> reqs, members;
        for (int i = 0, row = 0; i < n; ++i) {   // n prompts: requests, rows of each, tiles shared, tiles of its own
            int beams, T, shared, own;
            if (scanf("%d %d %d %d", &beams, &T, &shared, &own) != 4) return 1;
            const auto request = [&](int rows, int tiles) {
                const int all = rows * g;
                return FewRequest{0, row, rows, (all + FEW_GROUP - 1) / FEW_GROUP * hkv, tiles, few_row_blocks(std::min(all, FEW_GROUP)), 1};
            };
            FewRequest several = request(beams * T, shared);
            several.with = SEVERAL;
            reqs.push_back(several);
            for (int b = 0; b < beams; ++b, row += T) {
                FewRequest r = request(T, own);
                r.with = i;
                members.push_back(r);
            }
        }
        reqs.insert(reqs.end(), members.begin(), members.end());
        const size_t apart = fewest_slots(reqs);
        const int together = share_tiles(reqs, g, hkv, from, 4096);
        for (FewRequest& r : reqs) r.weight = r.together ? 1.0 : r.row_blocks;
        const bool fits = plan_few(reqs, 512, 4096);
        size_t used = 0;
        int most = 0, sharers = 0;
        for (const FewRequest& r : reqs) {
            if (r.in_slots()) used += (size_t)r.units * r.parts * r.row_blocks;
            most = std::max(most, r.parts);
            sharers += r.together != 0;
            if (r.together && (r.together != together || r.with != SEVERAL)) return 2;
        }
        printf("%zu %d %d %d %zu %d\n", apart, together, sharers, (int)fits, used, most);
    }
}
"""


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    d = tmp_path_factory.mktemp("few")
    src, exe = d / "harness.cpp", d / "harness"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-Wall",
                    "-I", os.path.join(ROOT, "paper_2509_24381_amd", "csrc"), str(src), "-o", str(exe)], check=True)

    def run(hq, hkv, prompts, from_=3000):
        text = f"{hq} {hkv} {from_} {len(prompts)} " + " ".join(str(v) for p in prompts for v in p)
        env = dict(os.environ, LD_PRELOAD="", ASAN_OPTIONS="detect_leaks=0")
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, env=env).stdout
        return dict(zip(("apart", "together", "sharers", "fits", "used", "parts"), map(int, out.split())))
    return run


@pytest.mark.parametrize("hq, hkv, prompts, beams, rows", [(64, 8, 47, 3, 1), (64, 8, 51, 3, 1), (64, 8, 64, 2, 2), (28, 4, 94, 3, 1), (28, 4, 102, 3, 1)])
def test_sums_fit_where_two_blocks_of_rows_would_become_eight(planner, hq, hkv, prompts, beams, rows):
    """17 to 32 stacked rows a prompt: two slots apart, eight together, which all of them have no room for."""
    got = planner(hq, hkv, [(beams, rows, 16, 1)] * prompts)
    assert 2 * got["apart"] <= SLOTS   # (such calls share pages)
    assert got["fits"] and got["used"] <= SLOTS and got["parts"] > 1
    assert got["together"] == 0


def test_wavefronts_share_tiles_where_there_is_room(planner):
    for hq, hkv, prompts, want in ((64, 8, [(3, 1, 60, 1)] * 20, 1), (64, 8, [(3, 1, 30, 1)] * 5, 0), (64, 8, [(16, 1, 500, 1)] * 4, 2), (28, 4, [(9, 1, 5, 1)], 1),
                                   (28, 4, [(4, 1, 120, 1)] * 16, 1)):
        got = planner(hq, hkv, prompts)
        assert got["together"] == want and got["sharers"] == (len(prompts) if want else 0), (hq, hkv, got)
        assert got["fits"] and got["used"] <= SLOTS
    got = planner(64, 8, [(3, 1, 30, 1)] * 40 + [(5, 1, 30, 1)] * 8)   # (those of more than 32 rows share theirs whatever the others do)
    assert got["together"] == 1 and got["sharers"] == 8 and got["fits"] and got["used"] <= SLOTS


def test_no_mix_of_prompts_goes_beyond_the_slots(planner):
    rng = random.Random(1)
    shared = 0
    for _ in range(400):
        hkv = rng.choice([1, 2, 4, 8])
        hq = hkv * rng.choice([1, 2, 5, 7, 8, 16])
        kinds = [(rng.randint(2, 20), rng.choice([1, 1, 1, 2, 5]), int(2 ** rng.uniform(0, 9)), rng.randint(1, 4)) for _ in range(rng.randint(1, 3))]
        prompts = [rng.choice(kinds) for _ in range(int(2 ** rng.uniform(0, 7)))]
        got = planner(hq, hkv, prompts, rng.choice([0, 3000]))
        if 2 * got["apart"] <= SLOTS:
            shared += 1
            assert got["fits"] and got["used"] <= SLOTS, (hq, hkv, prompts, got)
        elif got["fits"]:
            assert got["used"] <= SLOTS, (hq, hkv, prompts, got)
    assert shared > 200
