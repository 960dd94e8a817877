"""Where the operators on a paged cache read and write, on the CPU: the functions that the kernels take their addresses from (csrc/fwa_page_index.h), walked the way the
kernels walk them, over tables that hold anything: no access outside the page that was allotted, none of a page that is not there."""
import os
import subprocess

from paper_2501_06480_amd import build

DRIVER = r'''
#include "fwa_page_index.h"
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <random>
using namespace fwa;
static void need(bool ok, const char* what) { if (!ok) { std::printf("FAILED %s\n", what); std::exit(1); } }
int main() {
    std::mt19937 g(1);
    auto pick = [&](int lo, int hi) { return (int)(lo + (long long)(g() % (uint64_t)((long long)hi - lo + 1))); };
    const int odd[] = {INT_MIN, -1, 0, 1, INT_MAX, 1 << 29, (1 << 29) + 1, 17};
    long long loads = 0;
    for (int round = 0; round < 4000; ++round) {
        const int size = 16 * pick(1, 8), width = pick(0, 6), pages = pick(0, 7), rows = pick(1, 200), most = pick(0, 220), heads = pick(1, 3);
        const uint32_t row_bytes = 64u << pick(0, 3), token_bytes = row_bytes * (uint32_t)heads, group = pick(0, 1) ? 16 : 8;
        const uint32_t page_bytes = token_bytes * size + (pick(0, 1) ? 0 : 16u * pick(0, 5));
        int table[8], offsets[2], length;
        for (int& e : table) e = pick(0, 3) ? pick(-1, pages) : odd[pick(0, 7)];
        for (int& e : offsets) e = pick(0, 3) ? pick(-5, rows + 5) : odd[pick(0, 7)];
        length = pick(0, 3) ? pick(-5, width * size + 20) : odd[pick(0, 7)];
        const int begin = page_offset(offsets[0], rows), count = page_count(begin, page_offset(offsets[1], rows), most), start = page_length(length);
        need(begin >= 0 && count >= 0 && begin + count <= rows && count <= most, "new tokens");
        const int keys = page_keys(start, count, width, size);
        need(keys >= 0 && keys <= width * size, "keys");
        // attention: groups of 16 (or 8) keys from the first to one behind the last
        for (int key = 0; key < keys + 64 && keys > 0; key += (int)group) {
            const int last = (keys - 1) / kPageRows, at = key / kPageRows, sub = at < last ? at : last, index = sub / (size / kPageRows);
            need(index >= 0 && index < width, "entry of the table");
            const int page = table[index], n = page_group(key, keys, (int)group, page_exists(page, pages));
            need(n >= 0 && n <= (int)group && (n == 0 || key + n <= keys), "rows of a group");
            if (n == 0) { need(page_bytes_of(n, token_bytes, row_bytes) == 0, "no bytes"); continue; }
            const uint32_t of = (uint32_t)key / kPageRows / (uint32_t)(size / kPageRows), slot = (uint32_t)key - of * (uint32_t)size;
            need(of == (uint32_t)index, "one page");
            const uint64_t from = page_place((uint32_t)page, slot, page_bytes, token_bytes), bytes = page_bytes_of(n, token_bytes, row_bytes);
            need(page >= 0 && page < pages && slot + (uint32_t)n <= (uint32_t)size, "rows of the page");
            need(from >= (uint64_t)page * page_bytes && from + bytes + (uint64_t)(heads - 1) * row_bytes <= (uint64_t)page * page_bytes + (uint64_t)token_bytes * size, "bytes");
            ++loads;
        }
        // append: the places of the new tokens
        for (int i = 0; i < count; ++i) {
            const uint32_t place = (uint32_t)(start + i), index = place / (uint32_t)size;
            if (index >= (uint32_t)width || !page_exists(table[index], pages)) continue;
            const uint64_t to = page_place((uint32_t)table[index], place - index * (uint32_t)size, page_bytes, token_bytes);
            need(to + token_bytes <= (uint64_t)table[index] * page_bytes + (uint64_t)token_bytes * size, "stores");
            ++loads;
        }
    }
    // far into a large cache
    need(page_place(70000u, 255u, 1u << 31, 1u << 22) == 70000ull * (1ull << 31) + 255ull * (1u << 22), "64 bits");
    std::printf("%lld accesses\n", loads);
    return loads > 10000 ? 0 : 1;
}
'''


def test_no_table_leads_outside(tmp_path):
    src, exe = tmp_path / "driver.cpp", tmp_path / "driver"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, env={**os.environ, "UBSAN_OPTIONS": "print_stacktrace=1"})
    assert r.returncode == 0, r.stdout + r.stderr


SHARE = r'''
#include "fwa_page_index.h"
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <vector>
using namespace fwa;
static void need(bool ok, const char* what) { if (!ok) { std::printf("FAILED %s\n", what); std::exit(1); } }
int main() {
    std::mt19937 g(2);
    auto pick = [&](int lo, int hi) { return (int)(lo + (long long)(g() % (uint64_t)((long long)hi - lo + 1))); };
    long long parts_seen = 0;
    for (int round = 0; round < 20000; ++round) {
        const int N = pick(1, 20), workers = pick(1, 300), least = pick(1, 16), turn = 1 << pick(0, 2), most = pick(0, 1) ? 20 : 2000;
        std::vector<int> units, starts;
        int total = 0;
        for (int n = 0; n < N; ++n) {
            const int rows = pick(0, 3), tiles = pick(0, 5) ? pick(0, most) : 0;
            units.push_back(page_units(rows, tiles));
            need(units[n] == (rows == 0 ? 0 : tiles == 0 ? 1 : tiles), "units");
            starts.push_back(total);
            total += units[n];
        }
        if (total == 0) continue;
        const int per = page_share(total, workers, least, turn);
        need(per >= least && per % turn == 0 && (long long)per * workers >= total, "share");
        struct Part { int worker, place, from, to; };
        std::vector<std::vector<Part>> got(N);
        std::map<std::pair<int, int>, int> places;
        std::vector<std::vector<int>> joins(N);  // worker, place, parts
        for (int w = 0; w < workers && (long long)w * per < total; ++w) {
            int begins = 0;
            for (int n = 0; n < N; ++n) {
                if (units[n] == 0 || starts[n] + units[n] <= w * per || starts[n] >= w * per + per) continue;
                const PagePart p = page_part(starts[n], units[n], w * per, per);
                need(p.from >= 0 && p.from < p.to && p.to <= units[n], "units of a part");
                if (p.place < 0) need(p.from == 0 && p.to == units[n] && p.parts == 0, "all of it");
                else need(++places[{w, p.place}] == 1, "a place has one part");
                if (p.parts) {
                    need(p.place >= 0 && p.from == 0 && ++begins == 1, "one block of several is begun");
                    need(n == N - 1 || starts[n] + units[n] >= w * per + per, "the last of the range");
                    joins[n] = {w, p.place, p.parts};
                }
                got[n].push_back({w, p.place, p.from, p.to});
            }
        }
        for (int n = 0; n < N; ++n) {
            int at = 0;
            for (size_t k = 0; k < got[n].size(); ++k) {
                need(got[n][k].from == at, "parts one behind the other");
                at = got[n][k].to;
                if (!joins[n].empty()) need(got[n][k].worker == joins[n][0] + (int)k && got[n][k].place == (k == 0 ? joins[n][1] : 0), "a part where the join looks for it");
            }
            need(at == units[n], "all units");
            need(joins[n].empty() ? got[n].size() <= 1 : (int)got[n].size() == joins[n][2], "as many parts as the join reads");
            parts_seen += got[n].size();
        }
    }
    std::printf("%lld parts\n", parts_seen);
    return parts_seen > 10000 ? 0 : 1;
}
'''


def test_shares_cover_every_unit_once(tmp_path):
    """The ranges of all workers over sequences of all kinds: every unit in one part, every part where the join looks for it, no place used twice."""
    src, exe = tmp_path / "share.cpp", tmp_path / "share"
    src.write_text(SHARE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


CUTS = r'''
#include "fwa_page_index.h"
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
using namespace fwa;
static void need(bool ok, const char* what) { if (!ok) { std::printf("FAILED %s\n", what); std::exit(1); } }
int main() {
    std::mt19937 g(3);
    auto pick = [&](int lo, int hi) { return (int)(lo + (long long)(g() % (uint64_t)((long long)hi - lo + 1))); };
    long long cuts = 0;
    for (int round = 0; round < 20000; ++round) {
        const int N = pick(1, 64), target = pick(1, 600), least = pick(1, 4), alone = pick(1, 8), turns = pick(0, 20), most = pick(0, 1) ? 30 : 4000;
        std::vector<int> blocks, tiles;
        int total = 0, all = 0;
        for (int n = 0; n < N; ++n) {
            blocks.push_back(pick(0, 2) ? pick(0, 2) : pick(0, 60));
            tiles.push_back(pick(0, 5) ? pick(0, most) : 0);
            total += blocks[n] * tiles[n];
            all += blocks[n];
        }
        int length = page_length_first(total, target, least), jobs = 0;
        need(length >= least && (long long)length * target >= total, "first length");
        for (int turn = 0;; ++turn) {
            jobs = 0;
            for (int n = 0; n < N; ++n) jobs += blocks[n] * page_parts(tiles[n], length, alone);
            need(jobs <= target + all, "parts that the grid has");
            if (turn >= turns || jobs <= target) break;
            need(page_length_next(length) > length, "a longer one");
            length = page_length_next(length);
        }
        for (int n = 0; n < N; ++n) {
            const int parts = page_parts(tiles[n], length, alone);
            for (int block = 0; block < blocks[n]; ++block) {
                const int mine = block + 1 == blocks[n] ? tiles[n] : pick(0, tiles[n]);  // causal blocks see fewer
                int at = 0;
                const int count = page_cut(mine, length, alone, parts, 0).parts;
                need(count >= 1 && count <= parts, "places of the sequence's blocks");
                for (int split = 0; split < count; ++split) {
                    const PageCut c = page_cut(mine, length, alone, parts, split);
                    need(c.parts == count && c.from == at && (c.to > c.from || mine == 0), "parts one behind the other");
                    at = c.to;
                    ++cuts;
                }
                need(at == mine, "all tiles");
            }
        }
    }
    std::printf("%lld cuts\n", cuts);
    return cuts > 10000 ? 0 : 1;
}
'''


def test_cuts_cover_every_tile_once(tmp_path):
    """Parts of about one length of blocks of all kinds: no more than the grid has workgroups, every tile in one part, as many as the join reads."""
    src, exe = tmp_path / "cuts.cpp", tmp_path / "cuts"
    src.write_text(CUTS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
