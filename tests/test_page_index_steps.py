"""The way of a wave over the keys of a sequence, as the attention takes it: from group to group and from tile to tile in steps without a division (csrc/fwa_page_index.h), each of
which has to be where a division says, over pages of all sizes and tables that end anywhere."""
import subprocess

from paper_2501_06480_amd import build

DRIVER = r'''
#include "fwa_page_index.h"
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
using namespace fwa;
static void need(bool ok, const char* what) { if (!ok) { std::printf("FAILED %s\n", what); std::exit(1); } }
int main() {
    std::mt19937 g(5);
    auto pick = [&](int lo, int hi) { return (int)(lo + (long long)(g() % (uint64_t)((long long)hi - lo + 1))); };
    long long looked = 0, behind = 0;
    for (int round = 0; round < 20000; ++round) {
        const int size = pick(0, 9) ? 16 * pick(1, 20) : 16 * pick(1, 4096), width = pick(1, pick(0, 1) ? 4 : 200), room = width * size, keys = pick(1, room);
        // the keys of a tile, the waves that share its rows or take the tiles in turn, and the rows of a wave that go to one page together
        const int tile = pick(0, 1) ? 64 : 32, waves = 1 << pick(0, 2), turns = pick(0, 1), rows = turns ? tile : tile / waves;
        const int group = rows < kPageRows ? rows : kPageRows, groups = rows / group, stride = turns ? waves * tile : tile;
        const int tiles = (keys + tile - 1) / tile, wave = pick(0, waves - 1), first = turns ? 0 : wave * rows, from = pick(0, tiles - 1) + (turns ? wave : 0);
        auto spot = [&](int key) { return PageSpot{key / size, key % size}; };
        const PageSpot step = spot(stride);
        PageSpot ahead = spot(from * tile + first);
        // every tile of the part, and the two that are looked up behind its last
        for (int t = from, more = 0; more < 2; t += turns ? waves : 1) {
            more += t >= tiles;
            PageSpot p = ahead;
            for (int i = 0; i < groups; ++i) {
                const int key = t * tile + first + i * group, entry = page_entry(p.index, width);
                need(p.index == key / size && p.slot == key % size, "where a division says");
                need(entry >= 0 && entry < width, "an entry of the table");
                need(p.slot + group <= size, "a group in one page");
                if (key < keys) need(entry == p.index, "the entry of a key that there is");
                else need(page_group(key, keys, group, true) == 0, "no rows behind the last key");
                behind += entry != p.index;
                ++looked;
                if (i + 1 < groups) page_advance(p, 0, group, size);
            }
            page_advance(ahead, step.index, step.slot, size);
        }
    }
    // one entry, and the largest table: 2^29 keys
    PageSpot p{(1 << 25) - 1, 0};
    page_advance(p, 16, 0, 16);
    need(p.index == (1 << 25) + 15 && page_entry(p.index, 1 << 25) == (1 << 25) - 1 && page_entry(0, 1) == 0, "the ends");
    std::printf("%lld looked up, %lld behind the table\n", looked, behind);
    return looked > 100000 && behind > 1000 ? 0 : 1;
}
'''


def test_steps_are_where_divisions_say(tmp_path):
    src, exe = tmp_path / "steps.cpp", tmp_path / "steps"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
