"""Lists that are cut into many parts (csrc/tns_parts.h), built for the host: every one of them is joined, once, wherever it begins.  No GPU."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2311_17410_amd", "csrc")

SOURCE = r"""
#include <cstdio>
#include <random>
#include <vector>

#include "tns_parts.h"

struct Lists {
    std::vector<int64_t> rowptr;
    int64_t total() const { return rowptr.back(); }
    int64_t edge(int64_t s) const { return rowptr[s]; }
    int64_t find(int64_t row) const {                     // the last list that begins at or before the row
        int64_t s = (int64_t)rowptr.size() - 2;
        while (rowptr[s] > row) --s;
        return s;
    }
};

static int wrong = 0, lists_of_many = 0;

static void check(const std::vector<int64_t>& lens, int part, int64_t beyond) {
    Lists l;
    l.rowptr.push_back(0);
    for (int64_t n : lens) l.rowptr.push_back(l.rowptr.back() + n);
    const int64_t size = (int64_t)1 << part, blocks = (l.total() + beyond + size - 1) >> part;
    std::vector<int> joined(lens.size(), 0);
    for (int64_t place = 0; place < tns::many_places(blocks); ++place) {
        int64_t first = -1, end = -1;
        const int64_t list = tns::many_at(place, part, blocks, l, first, end);
        if (list < 0) continue;
        ++joined[list];
        if (first != l.edge(list) / size || end != (l.edge(list + 1) + size - 1) / size) ++wrong;
    }
    for (size_t s = 0; s < lens.size(); ++s) {
        // parts by counting the blocks that hold a row of the list; one that a block holds, or no longer than one, is not cut
        const int64_t b = l.rowptr[s], e = l.rowptr[s + 1], parts = e > b ? (e - 1) / size - b / size + 1 : 0;
        const int want = e - b > size && parts > tns::kMany;
        lists_of_many += want;
        if (joined[s] != want) {
            if (wrong < 5) std::printf("blocks of %lld rows: list [%lld, %lld) of %lld parts is joined %d times\n", (long long)size, (long long)b, (long long)e, (long long)parts, joined[s]);
            ++wrong;
        }
    }
}

int main() {
    check({5, 100000}, 4, 0);
    check({1, 5000}, 4, 0);
    check({5, 4097}, 4, 0);
    for (int part = 4; part <= 9; part += 5) {
        // one list in front and one of 255 to 259 blocks, give or take a row: every begin around the multiples of kMany
        const int64_t size = (int64_t)1 << part;
        for (int64_t block : {0, 1, 2, 254, 255, 256, 257, 511, 512, 513})
            for (int64_t off : {int64_t(0), int64_t(1), int64_t(2), size / 2, size - 1})
                for (int64_t n = 255; n <= 259; ++n)
                    for (int64_t more : {int64_t(-1), int64_t(0), int64_t(1), size / 2})
                        for (int64_t behind : {0, 1, 300})
                            for (int64_t beyond : {int64_t(0), int64_t(1), 600 * size}) check({block * size + off, n * size + more, behind}, part, beyond);
    }
    std::mt19937 rng(1);
    for (int i = 0; i < 3000; ++i) {
        std::vector<int64_t> lens;
        for (int k = rng() % 4; k > 0; --k) lens.push_back(rng() % 300);
        for (int k = rng() % 5; k > 0; --k) lens.push_back(rng() % 3 ? rng() % 20000 : rng() % 40);
        lens.push_back(rng() % 40000);
        check(lens, 4 + rng() % 3, rng() % 2 ? rng() % 10000 : 0);
    }
    std::printf("%d lists of many parts\n", lists_of_many);
    return wrong || lists_of_many < 3000;
}
"""


def test_every_list_of_many_parts_is_joined_once(tmp_path):
    src, exe = tmp_path / "parts.cpp", str(tmp_path / "parts")
    src.write_text(SOURCE)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", exe])
    done = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stdout + done.stderr
