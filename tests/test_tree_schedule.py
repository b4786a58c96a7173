"""The schedule of ssd_tree_attention (csrc/tree_sched.cuh) on the CPU: its host
functions are compiled with nvcc into a small program that draws batches and walks
every CTA's range.

Checked for each batch: every unit of every item is in exactly one CTA's range; the
ranges differ by at most one unit, counted with what items count more; a CTA leaves
at most two parts, that of its first segment in slot 0; and for an item that range ends cut,
the CTAs that `holders` names are those that hold its parts, in order, with the slots they use.
Tiles cover the rows, and a chain's tile stops at its last row's position.
"""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "tree_sched.cuh"
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>
using namespace ssd::tree;
static int bad(const char* what, int it) { printf("%s in batch %d\n", what, it); return 1; }
int main(int argc, char** argv) {
    srand(atoi(argv[1]));
    for (int it = 0; it < atoi(argv[2]); ++it) {
        const int B = 1 + rand() % (rand() % 3 ? 6 : 60), tile = rand() % 4 ? rand() % 2 ? 32 : 128 : 1 + rand() % 2, grid = rand() % 4 ? 304 : 1 + rand() % 40;
        Shape s{};
        s.n_requests = B;
        s.page_size = 16 * (1 + rand() % 6);
        s.n_kv_heads = 1 + rand() % 9;
        s.group = 1 + rand() % 9;
        s.chain = rand() % 2;
        std::vector<int32_t> start(B + 1, 0), lens(B);
        int longest = 1;
        for (int b = 0; b < B; ++b) {
            const int n = rand() % 4 ? rand() % 10 : rand() % 300;
            start[b + 1] = start[b] + n;
            lens[b] = rand() % 8 ? rand() % (rand() % 3 ? 300 : 6000) : -1;
            if (lens[b] + n > longest) longest = lens[b] + n;
        }
        s.n_rows = start[B];
        s.max_blocks = rand() % 5 ? (longest + s.page_size - 1) / s.page_size : 1 + rand() % 4;  // sometimes too narrow
        s.row_start = start.data();
        s.lens = lens.data();
        // a prefix sum over the requests, as the kernel forms it
        std::vector<long long> before(B + 1, 0);
        for (int b = 0; b < B; ++b) {
            const Req q = req_of(s, b);
            if (q.n != (lens[b] < 0 ? 0 : start[b + 1] - start[b])) return bad("rows", it);
            if (q.n && (q.total < 1 || q.total > (long long)s.max_blocks * s.page_size || q.total > lens[b] + q.n)) return bad("total", it);
            if (tiles_of(s, q, tile) * tile < q.n * s.group) return bad("tiles", it);
            for (int mt = 0; mt < tiles_of(s, q, tile); ++mt) {
                const int last = std::min(q.n - 1, ((mt + 1) * tile - 1) / s.group);
                const int keys = s.chain ? std::min(q.total, lens[b] + last + 1) : q.total;
                if (units_of(s, q, tile, mt) != (keys + 127) / 128) return bad("units", it);
            }
            before[b + 1] = before[b] + head_units(s, q, tile) * s.n_kv_heads;
        }
        const long long U = before[B];
        const int ctas = ctas_of(U, grid);
        if (ctas < 1 || ctas > grid || (U > 0 && ctas > U)) return bad("ctas", it);
        std::map<std::tuple<int, int, int>, std::vector<int>> seen;                       // item -> units
        std::map<std::tuple<int, int, int>, std::vector<std::pair<int, int>>> parts;      // item -> (CTA, slot)
        std::map<std::tuple<int, int, int>, std::vector<std::tuple<int, int, int>>> cuts;  // item -> (first, last, slot) of each cut
        long long most = 0, least = 1ll << 60;
        for (int c = 0; c < ctas && U; ++c) {
            const long long lo = range_start(U, ctas, c), hi = range_start(U, ctas, c + 1);
            most = std::max(most, hi - lo);
            least = std::min(least, hi - lo);
            int b = 0;
            while (!(before[b] <= lo && lo < before[b + 1])) ++b;
            Walk w;
            walk_init(w, s, tile, b, req_of(s, b), lo - before[b], lo, hi - lo);
            Seg g;
            int n_parts = 0;
            for (bool first = true; walk_next(w, s, tile, g); first = false) {
                const auto item = std::make_tuple(g.b, g.kvh, g.mt);
                if (g.u0 >= g.u1 || g.u1 > g.n || g.kvh >= s.n_kv_heads || g.b >= B || g.q.n < 1) return bad("segment", it);
                for (int u = g.u0; u < g.u1; ++u) {
                    const long long at = g.item + kItemCost + u;
                    if (cta_of(U, ctas, at) != c || at < lo || at >= hi) return bad("cta_of", it);
                    seen[item].push_back(u);
                }
                if (g.u0 > 0 || g.u1 < g.n) {
                    parts[item].push_back({c, first ? 0 : 1});
                    if (++n_parts > 2) return bad("three parts", it);
                    if (g.u1 < g.n) {
                        int f, l, later;
                        holders(g, U, ctas, f, l, later);
                        cuts[item].push_back(std::make_tuple(f, l, later));
                    }
                }
            }
        }
        if (U && most - least > 1) return bad("balance", it);
        for (int b = 0; b < B; ++b) {
            const Req q = req_of(s, b);
            for (int h = 0; h < s.n_kv_heads; ++h)
                for (int mt = 0; mt < tiles_of(s, q, tile); ++mt) {
                    const auto item = std::make_tuple(b, h, mt);
                    const int n = units_of(s, q, tile, mt);
                    if ((int)seen[item].size() != n) return bad("units missing", it);
                    for (int u = 0; u < n; ++u)
                        if (seen[item][u] != u) return bad("order", it);
                    const auto& p = parts[item];
                    if (p.empty() != cuts[item].empty() || (!p.empty() && p.size() != cuts[item].size() + 1)) return bad("cuts", it);
                    for (const auto& c : cuts[item]) {
                        if (std::get<0>(c) != p.front().first || std::get<1>(c) != p.back().first) return bad("holders", it);
                        for (size_t i = 0; i < p.size(); ++i)
                            if (p[i].first != p[0].first + (int)i || p[i].second != (i ? 0 : std::get<2>(c))) return bad("slots", it);
                    }
                }
        }
    }
    printf("ok\n");
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("sched")
    (d / "s.cu").write_text(SOURCE)
    subprocess.check_call(["nvcc", "-O2", "-std=c++17", "-gencode", "arch=compute_103a,code=sm_103a", "-I", os.path.join(ROOT, "paper_2309_08168_gb300", "csrc"),
                           str(d / "s.cu"), "-o", str(d / "s")])
    return str(d / "s")


@pytest.mark.parametrize("seed", range(4))
def test_every_unit_once_and_parts_where_the_join_looks(program, seed):
    r = subprocess.run([program, str(seed), "400"], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout


# Batches of 2^32 units and more (too long to run): the CTA of a unit against one division in 64 bits, the ranges'
# starts around it, and the holders of the items that the range ends cut.
LARGE = r"""
#include "tree_sched.cuh"
#include <cstdio>
using namespace ssd::tree;
int main() {
    const int grids[] = {1, 40, 152, 304};
    const long long around[] = {1ll << 31, 1ll << 32, 3ll << 32, 1ll << 40};
    for (int ctas : grids)
        for (long long top : around)
            for (long long U = top - 2; U <= top + 8200; U += U < top + 2 ? 1 : 911)
                for (int c = 0; c < ctas; ++c) {
                    const long long lo = range_start(U, ctas, c);
                    if (lo != U * c / ctas) return printf("start %lld %d\n", U, c), 1;
                    for (long long u : {lo - 1, lo, lo + 1, (long long)c, 1000ll * c})
                        if (u >= 0 && u < U && cta_of(U, ctas, u) != (int)(((u + 1) * ctas - 1) / U)) return printf("cta_of %lld %d %lld\n", U, ctas, u), 1;
                }
    // one prompt over eight KV heads of eight heads
    for (int rows = 1482451; rows < 1482481; rows += 3) {
        int32_t start[2] = {0, rows}, lens[1] = {0};
        Shape s{};
        s.n_requests = 1;
        s.n_rows = rows;
        s.page_size = 64;
        s.max_blocks = (rows + 63) / 64;
        s.n_kv_heads = s.group = 8;
        s.chain = 1;
        s.row_start = start;
        s.lens = lens;
        const Req q = req_of(s, 0);
        const long long per = head_units(s, q, 128), U = per * 8;
        if (U < 1ll << 32) return printf("units %lld\n", U), 1;
        const int ctas = ctas_of(U, 152);
        for (int c = 0; c < ctas; c += 1 + c % 3 * 37) {
            const long long lo = range_start(U, ctas, c), hi = range_start(U, ctas, c + 1);
            Walk w;
            walk_init(w, s, 128, 0, q, lo, lo, hi - lo, per);
            Seg g;
            while (walk_next(w, s, 128, g))
                if (g.u1 < g.n) {
                    int first, last, later;
                    holders(g, U, ctas, first, last, later);
                    if (first > c || last < c || last >= ctas || range_start(U, ctas, first) > g.item + kItemCost || range_start(U, ctas, first + 1) <= g.item + kItemCost ||
                        range_start(U, ctas, last) > g.item + kItemCost + g.n - 1)
                        return printf("holders of %d rows, CTA %d: %d .. %d\n", rows, c, first, last), 1;
                }
        }
    }
    printf("ok\n");
    return 0;
}
"""


def test_more_units_than_32_bits(tmp_path):
    (tmp_path / "l.cu").write_text(LARGE)
    subprocess.check_call(["nvcc", "-O2", "-std=c++17", "-gencode", "arch=compute_103a,code=sm_103a", "-I", os.path.join(ROOT, "paper_2309_08168_gb300", "csrc"),
                           str(tmp_path / "l.cu"), "-o", str(tmp_path / "l")])
    r = subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout
