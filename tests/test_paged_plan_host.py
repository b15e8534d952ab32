"""The arithmetic of paged attention's shares and workspace (csrc/paged_plan.h), compiled for the
host with the undefined-behaviour sanitizer and tried over every workgroup of many launches."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2301_06813_amd",
                    "csrc")

PROGRAM = r"""
#include <limits.h>
#include <stdio.h>
#include <stdlib.h>
#include <initializer_list>
#include "paged_plan.h"
using namespace sbpi;
static uint64_t state = 88172645463325252ull;
static uint32_t draw() {
    state ^= state << 13; state ^= state >> 7; state ^= state << 17;
    return (uint32_t)(state >> 16);
}
#define NEED(x) do { if (!(x)) { printf("line %%d: %%s\n", __LINE__, #x); return 1; } } while (0)
int main() {
%s
    return 0;
}
"""

# Units up to what the launch counts on, more than that, past 31 bits (which the sums wrap): a
# workgroup with a share has room for its partial outputs, and the shares make up the line.
SHARES = r"""
    for (int groups : {2, 256, 512})
        for (int k = 0; k < 4000; ++k) {
            const bool parts = k % 8 == 7;
            const int slots = groups + (int)(draw() % (groups + 1)), holders = parts ? groups : slots / 2;
            int total = k % 3 == 0 ? (int)draw() : (int)(draw() >> (draw() % 32)) & INT_MAX;
            if (k < 4) total = k == 0 ? INT_MAX : k == 1 ? INT_MIN : k == 2 ? 0 : -1;
            if (parts) total = total > 0 ? total % (groups + 1) : total;
            // as the kernel has it: a unit a workgroup where the units are parts
            const int share = parts ? 1 : (total > 0 ? total - 1 : 0) / holders + 1;
            int64_t next = 0;
            for (int wg = 0; wg < groups; ++wg) {
                if (!has_share(total, share, wg, parts, holders)) continue;
                const int at = share * wg, left = total - at < share ? total - at : share;
                NEED(at == next && left > 0);
                next = (int64_t)at + left;
                for (bool began : {false, true}) NEED(slot_of(wg, began, parts) < slots);
            }
            NEED(next == (total > 0 ? total : 0));
        }
"""


def run(tmp_path, body):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(PROGRAM % body)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-fsanitize=undefined",
                    "-fno-sanitize-recover=all", "-I", CSRC, str(src), "-o", exe], check=True, timeout=120)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr


def test_shares_have_room(tmp_path):
    run(tmp_path, SHARES)


# Every size of a workspace about the least that holds a partial output a workgroup, and larger
# ones; odd numbers of rows and slots among them.
ROOM = r"""
    for (int groups : {256, 512})
        for (int rows : {1, 3, 7, 31, 32, 77, 128, 255, 256})
            for (int cols : {4, 40, 64, 128})
                for (int k = 0; k < 300; ++k) {
                    const int64_t slot = rows * (int64_t)(2 + cols), least = stats_at(groups) + groups * slot;
                    const int64_t floats = k < 100 ? least - 50 + k : least + draw() % (2 * groups * slot);
                    const int64_t fit = slots_in(floats, groups, rows, cols);
                    const int slots = (int)(fit < 2 * groups ? fit : 2 * groups);
                    NEED((fit >= groups) == (floats >= least));
                    if (slots == 0) continue;
                    NEED(fit + 2 > (floats - stats_at(groups)) / slot);
                    const int64_t at = parts_at(groups, slots, rows);
                    NEED(at % 4 == 0 && at >= stats_at(groups) + 2 * (int64_t)slots * rows);
                    NEED(at + (int64_t)slots * rows * cols <= floats);
                }
    NEED(slots_in(0, 256, 32, 64) == 0 && slots_in(2000, 256, 32, 64) == 0);
"""


def test_partial_outputs_lie_on_16_bytes(tmp_path):
    run(tmp_path, ROOM)
