"""The ring that the step over a packed prompt streams its tiles through, driven on the host with copies that land late: whatever
a program sets the limit of the waits to, and wherever one of them gives up, no copy is under way when the warp's part ends, and
none is asked for into a place that another is still on its way to."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_01941_b200", "csrc")

DRIVER = r"""
#include "ring.cuh"

template <int STAGES>
struct Copies {
    int in_flight = 0, tile[STAGES], phase[STAGES] = {}, faults = 0, asked = 0, taken = 0, gave_up = 0;
    int late_from;
    long long late_by;
    Copies(int from, long long by) : late_from(from), late_by(by) {
        for (int& t : tile) t = -1;
    }
    void fetch(int t, int stage) {
        if (tile[stage] >= 0) ++faults;                          // into the place of a copy under way
        tile[stage] = t, ++in_flight, ++asked;
    }
    bool landed(int stage, uint32_t parity, long long limit) {
        if (tile[stage] < 0 || (phase[stage] & 1) != (int)parity) {  // nothing to wait for: the wait would never end, or at once
            ++faults;
            return false;
        }
        if (tile[stage] >= late_from && limit < late_by) {
            ++gave_up;
            return false;
        }
        tile[stage] = -1, ++phase[stage], --in_flight, ++taken;
        return true;
    }
};

// a warp's part of a step; the copies of tiles from `late_from` on take `late_by` cycles, the others none
template <int STAGES>
int part(int first, int step, int tiles, int all, long long limit, int late_from, long long late_by) {
    Copies<STAGES> c(late_from, late_by);
    const auto fetch = [&](int t, int s) { c.fetch(t, s); };
    const auto landed = [&](int s, uint32_t p, long long l) { return c.landed(s, p, l); };
    shotkv::TileRing<STAGES> ahead(first, step);
    ahead.ask(all, fetch);
    int used = 0;
    while (ahead.tile < tiles) {
        if (!landed(ahead.stage, ahead.parity, limit)) break;
        if (ahead.tile != first + used * step) return 1;
        ++used;
        ahead.next(tiles, fetch);
    }
    const int wanted = first < tiles ? (tiles - first + step - 1) / step : 0;
    if (c.gave_up > 1 || (c.gave_up == 0 && used != wanted)) return 2;
    if (c.gave_up && first + used * step < late_from) return 3;
    ahead.land(all, tiles, landed);
    if (c.faults) return 4;
    if (c.in_flight) return 5;
    return c.taken == c.asked ? 0 : 6;
}

extern "C" int parts(long long limit, long long late_by, int* ran) {
    for (int step = 1; step <= 9; step += 4)
        for (int first = 0; first < 3 * step; ++first)
            for (int all = 0; all <= 6 * step + 1; ++all)
                for (int tiles = 0; tiles <= all; ++tiles)
                    for (int late = 0; late <= all + 1; ++late) {
                        ++*ran;
                        int rc = part<2>(first, step, tiles, all, limit, late, late_by);
                        if (!rc) rc = part<3>(first, step, tiles, all, limit, late, late_by);
                        if (rc) return rc;
                    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    at = tmp_path_factory.mktemp("ring")
    (at / "driver.cpp").write_text(DRIVER)
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-shared", "-fPIC", "-x", "c++", "-I", CSRC, str(at / "driver.cpp"),
                    "-o", str(at / "driver.so")], check=True)
    lib = C.CDLL(str(at / "driver.so"))
    lib.parts.argtypes = [C.c_longlong, C.c_longlong, C.POINTER(C.c_int)]
    return lib


@pytest.mark.parametrize("limit,late_by", [(1, 0), (1, 2), (1, 10 ** 6), (10 ** 5, 10 ** 6), (4 * 10 ** 9, 10 ** 6), (4 * 10 ** 9, 4 * 10 ** 9)])
def test_every_copy_lands(driver, limit, late_by):
    ran = C.c_int(0)
    assert driver.parts(limit, late_by, C.byref(ran)) == 0, "5: copies still under way at the end; 4: a place used twice, or a wait for nothing"
    assert ran.value > 10000


def test_what_is_in_flight_is_waited_for_whatever_the_limit():
    """In the kernels that copy by descriptor and in those that send messages: the waits at a CTA's end, for what will still be
    written into its memory, do not have the limit that a program sets, and the copies are waited for when another role gave up too."""
    def body(f, name):
        text = open(os.path.join(CSRC, f)).read()
        start = text.index("{", text.index(name + "("))
        depth, end = 1, start + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        return text[start:end]

    message = body("common.cuh", "void outlive_messages")
    assert message.count("kLandCycles") == 2 and "limit)" not in message
    producer = body("score_tc.cuh", "void producer_role")
    last = producer[producer.rindex("tma_load_3d"):]
    assert "kLandCycles" in last and "p.wait_cycles" not in last
    assert "if (!ok)" not in last and "land(pp.qfull()" in last and "land(pp.full(s)" in last


def test_the_step_goes_through_it():
    """The kernel has no ring of its own beside the one tested here."""
    text = open(os.path.join(CSRC, "decode_kv4.cuh")).read()
    assert "ahead.ask(all_tiles, fetch);" in text and "ahead.next(tiles, fetch);" in text and "ahead.land(all_tiles, tiles, landed);" in text
    assert text.count("fetch(") == 0 and text.count("bulk_load(") == 3       # the lambda is handed on; one definition, keys, values
