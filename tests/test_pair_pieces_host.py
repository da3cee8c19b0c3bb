"""Pieces of a result leave the pair kernel through two places in shared memory.  A piece written to a place that a store still reads spoils the store before, which depends on how far the
stores are behind and cannot be provoked on purpose, so the waits are followed on the CPU, for every run of tiles: as many stores as a wait allows are still reading."""
import os
import re
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2409_16626_b200", "csrc")
PROGRAM = r"""
#include <cstdio>
#include <deque>
#include <vector>
#include "hif8_pair_pieces.h"

// tiles: pieces that are stored; one more (`staged`) may be put in its place and not stored
static int first_clash(const std::vector<int>& tiles, bool staged, bool always_one)
{
    hif8::PiecePlaces places;
    std::deque<int> reading;
    auto wait = [&](int may_read) { while ((int)reading.size() > may_read) reading.pop_front(); };
    for (size_t t = 0; t < tiles.size(); t++) {
        const bool last = t + 1 == tiles.size();
        wait(always_one ? 1 << 30 : places.may_still_read(hif8::PiecePlaces::place_of(0, last)) == 0 ? 0 : 1 << 30);
        for (int i = 0; i < tiles[t] + (staged ? 1 : 0); i++) {
            const int place = hif8::PiecePlaces::place_of(i, last);
            if (place < 2) wait(1);
            for (int p : reading)
                if (p == place) return (int)t + 1;
            if (i < tiles[t]) reading.push_back(place);
        }
        if (tiles[t] > 0) places.stored(hif8::PiecePlaces::place_of(tiles[t] - 1, last));
    }
    return 0;
}

int main()
{
    int clashes = 0, found = 0, tightest = 9;
    for (int a = 0; a <= 8; a++)
        for (int b = 0; b <= 8; b++)
            for (int c = 0; c <= 8; c++)
                for (int d = 0; d <= 8; d++)
                    for (int staged = 0; staged < 2; staged++) {
                        if (staged && (a > 7 || b > 7 || c > 7 || d > 7)) continue;
                        clashes += first_clash({a, b, c, d}, staged, false) != 0;
                        found += first_clash({a, b, c, d}, staged, true) != 0;
                    }
    hif8::PiecePlaces even;
    even.stored(0); even.stored(1);
    tightest = even.may_still_read(0);  // behind an even number the newest store may go on
    std::printf("%d %d %d\n", clashes, found > 0, tightest);
}
"""


@pytest.fixture(scope="module")
def followed(tmp_path_factory):
    where = tmp_path_factory.mktemp("pieces")
    (where / "follow.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I" + CSRC, str(where / "follow.cpp"), "-o", str(where / "follow")], check=True)
    return [int(v) for v in subprocess.run([str(where / "follow")], check=True, capture_output=True, text=True).stdout.split()]


def test_no_piece_is_written_to_a_place_that_a_store_reads(followed):
    assert followed[0] == 0


def test_one_store_too_many_under_way_would_be_found(followed):
    assert followed[1] == 1


def test_the_newest_store_is_not_waited_for_without_need(followed):
    assert followed[2] == 1


def test_the_kernel_waits_so():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hif8_gemm.cu")).read())
    start = re.search(r"\nbf16_gemm_pair_kernel\(const __grid_constant__", text).end()
    body = text[start:text.find("\n}\n", start)]
    first, each, write, store, told = (body.find(t) for t in ('places.may_still_read(place_of(0)) == 0) asm volatile("cp.async.bulk.wait_group.read 0;"', "wait_group.read 1", "sts_v4(at", "tma_store_2d(",
                                                              "if (mapped > 0) places.stored(place_of(mapped - 1));"))
    assert 0 < first < each < write < store < told and body.count("wait_group.read 1") == 1
