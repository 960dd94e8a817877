"""Offsets that fall, where blocks are cut into parts of about one length: no part that the join reads lies behind those that the launch has (the functions of
csrc/fwa_page_index.h, walked on the CPU the way the kernels walk them)."""
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
constexpr int kRows = 128, kTile = 64;
struct Call {
    std::vector<int> offsets, lengths;
    int rows, most, group, room, target, least, alone;
    bool causal;
};
// every job of the launch: blocks of sequences of one block first, then those of the others, from the last block on; returns how many jobs end at the launch's last
static int walk(const Call& c) {
    const int N = (int)c.lengths.size(), jobs = (int)((long long)c.rows * c.group / kRows) + N + c.target;
    std::vector<int> count(N), blocks(N), tiles(N), parts(N);
    int work = 0;
    for (int n = 0; n < N; ++n) {
        count[n] = page_count(page_offset(c.offsets[n], c.rows), page_offset(c.offsets[n + 1], c.rows), c.most);
        blocks[n] = (count[n] * c.group + kRows - 1) / kRows;
        tiles[n] = (page_keys(page_length(c.lengths[n]), count[n], c.room / 16, 16) + kTile - 1) / kTile;
        work += blocks[n] * tiles[n];
    }
    int length = page_length_first(work, c.target, c.least);
    for (int turn = 0;; ++turn) {
        int all = 0;
        for (int n = 0; n < N; ++n) all += blocks[n] * (parts[n] = page_parts(tiles[n], length, c.alone));
        if (turn == 16 || all <= c.target) break;
        length = page_length_next(length);
    }
    struct Job { int n, block, split; };
    std::vector<Job> order;
    for (int many = 0; many < 2; ++many)
        for (int n = 0; n < N; ++n)
            for (int b = blocks[n] - 1; (blocks[n] > 1) == many && b >= 0; --b)
                for (int s = 0; s < parts[n]; ++s) order.push_back({n, b, s});
    int shortened = 0;
    for (int job = 0; job < jobs && job < (int)order.size(); ++job) {
        const Job& j = order[job];
        const int last_row = j.block * kRows + kRows <= count[j.n] * c.group ? j.block * kRows + kRows - 1 : count[j.n] * c.group - 1;
        const int klen = page_keys(page_length(c.lengths[j.n]), count[j.n], c.room / 16, 16), last = page_length(c.lengths[j.n]) + last_row / c.group;
        const int kend = c.causal && last + 1 < klen ? last + 1 : klen, mine = (kend + kTile - 1) / kTile;
        const int most = page_parts_room(parts[j.n], job, j.split, jobs);
        need(most >= 1 && most <= parts[j.n], "room");
        if (j.split >= most) continue;
        const PageCut cut = page_cut(mine, length, c.alone, most, j.split);
        if (j.split >= cut.parts) continue;
        need(job - j.split + cut.parts <= jobs, "parts behind the last workgroup");
        // all parts of a block, each by its own job, make up its tiles
        if (j.split > 0) continue;
        int at = 0;
        for (int s = 0; s < cut.parts; ++s) {
            const PageCut other = page_cut(mine, length, c.alone, page_parts_room(parts[j.n], job + s, s, jobs), s);
            need(other.parts == cut.parts && other.from == at, "parts of a block agree");
            at = other.to;
        }
        need(at == mine, "all tiles");
        shortened += most < parts[j.n];
    }
    return shortened;
}
int main() {
    // 64 sequences whose offsets rise and fall between none and all of 2560 rows, one of which has 256 new tokens on a million
    Call c{{}, {}, 2560, 2560, 1, 1 << 20, 512, 2, 4, true};
    int shortened = 0;
    for (int at = 0; at < 64; ++at) {
        c.offsets.clear();
        c.lengths.assign(64, 0);
        for (int n = 0; n <= 64; ++n) c.offsets.push_back(n % 2 ? 2560 : 0);
        c.offsets[at] = 0;
        c.offsets[at + 1] = 256;
        c.lengths[at] = 1000000;
        shortened += walk(c);
    }
    need(shortened > 0, "a block at the launch's end");
    std::mt19937 g(4);
    auto pick = [&](int lo, int hi) { return (int)(lo + (long long)(g() % (uint64_t)((long long)hi - lo + 1))); };
    for (int round = 0; round < 20000; ++round) {
        const int N = pick(1, 64), rows = pick(1, 3000);
        Call d{{}, {}, rows, pick(0, 2) ? rows : pick(1, rows), pick(1, 4), 16 * pick(0, 4000), pick(1, 512), pick(1, 2), pick(1, 4), pick(0, 1) == 0};
        for (int n = 0; n <= N; ++n) d.offsets.push_back(pick(0, 3) ? pick(-5, rows + 5) : pick(0, 1) ? 0 : rows);
        for (int n = 0; n < N; ++n) d.lengths.push_back(pick(0, 3) ? pick(0, 300) : pick(0, 70000));
        shortened += walk(d);
    }
    std::printf("%d blocks cut shorter\n", shortened);
    return shortened > 100 ? 0 : 1;
}
'''


def test_no_part_behind_the_last_workgroup(tmp_path):
    src, exe = tmp_path / "falling.cpp", tmp_path / "falling"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
