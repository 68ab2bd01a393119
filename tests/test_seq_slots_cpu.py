"""How a scan's segments put a state together from what the others published
(csrc/seq_slots.h), on the host: the state is that of one step after the other,
whichever slots are states already, and a wait that ran out gives NaN."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "seq_slots.h"
#include <cmath>
#include <cstdio>
#include <vector>
using namespace tq;
// the state after the slots [0, n), looking back over at most `reach` of them,
// the oldest of which has to be a state
static float walk(const std::vector<Slot> &slots, float first, int reach)
{
    const int n = (int)slots.size(), k = n < reach ? n : reach;
    float h = first;
    for (int i = n - k; i < n; i++) h = slot_step(slot_value(slots[i], n > reach && i == n - reach), h);
    return h;
}
#define CHECK(x) if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; }
int main()
{
    const int n = 50, reach = 32;
    std::vector<Slot> pairs(n), slots(n);
    std::vector<float> states(n);
    float h = 0.75f;
    for (int i = 0; i < n; i++) {
        const float a = 1.f / (1.f + 0.1f * (i % 7)), b = std::sin(0.3f * i);
        pairs[i] = pair_slot(a, b);
        h = std::fma(a, h, b);
        states[i] = h;
    }
    for (int state = 0; state < n; state++) {
        slots = pairs;
        slots[0] = state_slot(states[0]);  // the first of a row is always one
        slots[state] = state_slot(states[state]);
        slots[n - reach] = state_slot(states[n - reach]);
        CHECK(walk(slots, 0.75f, reach) == h)
        CHECK(walk(slots, 0.75f, n) == h)
    }
    // not published, or not a state where one has to be: not known, however far on
    for (int bad = n - reach; bad < n; bad++) {
        slots = pairs;
        slots[n - reach] = state_slot(states[n - reach]);
        slots[bad] = kEmpty;
        CHECK(std::isnan(walk(slots, 0.75f, reach)))
    }
    slots = pairs;
    CHECK(std::isnan(walk(slots, 0.75f, reach)))
    // words of every kind of number differ from a slot that is not published
    const float nan = slot_float(~0u), inf = INFINITY;
    for (float a : {0.f, 1.f, 1e-45f, inf, nan})
        for (float b : {0.f, -0.f, 1.f, -inf, inf, nan}) {
            CHECK(pair_slot(a, b) != kEmpty && slot_ready(pair_slot(a, b), false) && !slot_ready(pair_slot(a, b), true))
            CHECK(state_slot(b) != kEmpty && slot_ready(state_slot(b), true))
        }
    CHECK(!slot_ready(kEmpty, false) && !slot_ready(kEmpty, true))
    printf("ok\n");
    return 0;
}
"""


def test_states_from_published_slots(tmp_path):
    src, exe = tmp_path / "slots.cpp", str(tmp_path / "slots")
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "paper_2003_02989_amd", "csrc"), str(src), "-o",
                    exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout
