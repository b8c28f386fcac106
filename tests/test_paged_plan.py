"""How the attention over pages cuts its work into shares (csrc/tree_plan.h, compiled for the host): every tile once, partial results where the
merge looks for them, nothing outside the arrays whatever they hold."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2510_15312_b200", "csrc")

PROGRAM = r"""
#include "tree_plan.h"
#include <cstdio>
#include <map>
#include <random>
#include <tuple>
#include <vector>
using namespace sdv;
static std::mt19937 rng(7);
static int pick(int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); }

static int check(const TreeLists& P, int blocks) {
    std::vector<long long> before{0};
    for (int b = 0; b < P.n_seqs; ++b) {
        const TreeSeq s = tree_seq(P, b);
        if (s.first < 0 || s.rows < 0 || s.first + s.rows > P.n_rows || s.rows > SDV_TREE_ROWS) return 1;
        if (s.length < 0 || s.keys < s.length || (long long)s.keys > (long long)P.table_width * P.page_size) return 2;
        if (s.keys - s.length > s.rows || (s.tiles > 0 && (s.tiles - 1) * kTreeKeys >= s.keys)) return 3;
        before.push_back(before.back() + (long long)(P.whole ? s.tiles > 0 : s.tiles) * s.chunks * P.n_kv);
    }
    if (before.back() > 0x3fffffffll) return 0;   // refused by the host
    const int total = (int)before.back();
    if (total == 0) return 0;
    const TreeCut cut(total, blocks);
    int next = 0;
    std::map<std::tuple<int, int, int>, std::vector<std::pair<int, int>>> parts;   // item -> (block, which of its partial results)
    for (int k = 0; k < blocks; ++k) {
        const int t0 = cut.begin(k), t1 = cut.begin(k + 1);
        if (t0 != next || t1 < t0 || t1 - t0 > total / blocks + 1 || t1 - t0 < total / blocks) return 4;
        if (t0 == t1) continue;
        int b = 0;
        while (before[b + 1] <= t0) ++b;
        TreeCursor c;
        c.start(P, b, tree_seq(P, b), (int)(t0 - before[b]), t1 - t0);
        int item = 0;
        while (c.left > 0) {
            if (c.s.tiles == 0 || c.b >= P.n_seqs || c.h >= P.n_kv || c.c >= c.s.chunks || c.tile >= c.s.tiles) return 6;
            const int n = c.run(P), counted = P.whole ? 1 : n;
            const long long at = before[c.b] + ((long long)c.h * c.s.chunks + c.c) * (P.whole ? 1 : c.s.tiles) + (P.whole ? 0 : c.tile);
            if (at != next || (P.whole && (c.tile || n != c.s.tiles))) return 7;
            for (int i = 0; i < counted; ++i)
                if (cut.owner((int)at + i) != k) return 8;
            if (n != c.s.tiles) parts[{c.b, c.h, c.c}].push_back({k, item ? 1 : 0});
            if (n != c.s.tiles && item && c.left != n) return 9;   // a partial item that is not the block's first is its last
            next += counted;
            c.skip(P, n);
            ++item;
        }
        if (next != t1) return 10;
    }
    if (next != total) return 11;
    for (auto& it : parts) {
        const TreeSeq s = tree_seq(P, std::get<0>(it.first));
        const long long tile0 = before[std::get<0>(it.first)] + ((long long)std::get<1>(it.first) * s.chunks + std::get<2>(it.first)) * s.tiles;
        const int k0 = cut.owner((int)tile0), k1 = cut.owner((int)tile0 + s.tiles - 1);
        const bool late = cut.begin(k0) < tile0;
        if ((int)it.second.size() != k1 - k0 + 1) return 12;
        for (int i = 0; i < (int)it.second.size(); ++i)
            if (it.second[i].first != k0 + i || it.second[i].second != (i == 0 && late ? 1 : 0)) return 13;
    }
    return 0;
}

int main() {
    for (int round = 0; round < 3000; ++round) {
        TreeLists P;
        P.n_seqs = pick(1, round % 7 ? 12 : 200);
        P.n_kv = pick(1, 8);
        P.g = pick(0, 9) ? pick(1, 9) : pick(1, 128);
        P.chunk = kTreeTileRows / P.g;
        P.whole = round % 4 == 3;
        P.page_size = 8 << pick(0, 4);
        P.table_width = pick(1, 40);
        std::vector<int> len, cu{0};
        for (int b = 0; b < P.n_seqs; ++b) {
            len.push_back(pick(0, 3) ? pick(0, P.table_width * P.page_size) : pick(0, 3));
            cu.push_back(cu.back() + (pick(0, 4) ? pick(0, 70) : 0));
        }
        P.n_rows = cu.back() + pick(0, 5);
        if (round % 3 == 0) {   // arrays that hold anything
            for (int& x : len) if (pick(0, 2) == 0) x = (int)rng();
            for (int& x : cu) if (pick(0, 2) == 0) x = (int)rng();
        }
        P.kv_len = len.data();
        P.cu_rows = cu.data();
        const int blocks = pick(0, 2) ? 296 : pick(1, 300), rc = check(P, blocks);
        if (rc) {
            std::printf("round %d: %d\n", round, rc);
            return 1;
        }
    }
    // lengths and tables at the ends of their types
    for (int len : {0x7fffffff, -1, 0x7fffffff - 63, 0}) {
        int cu[2] = {0, 9};
        TreeLists P{&len, cu, 1, 9, 1, 1, 0x7fffffff, 1 << 20, kTreeTileRows, 0};
        const TreeSeq s = tree_seq(P, 0);
        if (s.keys < s.length || s.keys < 0 || s.tiles < 1 || (long long)s.tiles * kTreeKeys < s.keys) return 2;
    }
    return 0;
}
"""


def test_every_tile_has_one_block_and_every_part_its_place(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=address,undefined", "-fno-sanitize-recover", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], timeout=300, capture_output=True, text=True)
    assert out.returncode == 0, out.stdout + out.stderr[-2000:]
