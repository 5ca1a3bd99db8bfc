"""Where the kernels that attend over a paged cache read keys and values (csrc/attend_common.h), compiled for the host and enumerated:
every byte that any lane asks for lies in the page that it asks of, the pool's last page and head among them, whatever the capacity, the
page size and the step (those behind the last one too, which waves without a step ask for), and slots in use are read where they lie."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_21513_amd", "csrc")

MAIN = r"""
#include <stdio.h>
#include <string.h>
#include <vector>
#include "attend_common.h"
using namespace intattn;

static long long asked = 0;

// The bytes [at, at + n) of a plane of pages are asked for; 0 if they belong to one page of the last head
static bool outside(const CacheParams &c, const int64_t *stride, int64_t at, int64_t n, int D, int page)
{
    const int64_t first = page * stride[0] + (c.Hkv - 1) * stride[1];
    ++asked;
    return at < first || at + n > first + (c.page_size - 1) * stride[2] + D;
}

template <int D, bool WHOLE> int check(int page_size, int max_pages, int max_len, bool absent)
{
    using K = Keys<D, WHOLE>;
    CacheParams c;
    memset(&c, 0, sizeof(c));
    c.B = 1; c.Hkv = 2; c.n_pages = max_pages; c.page_size = page_size;
    c.capacity = max_pages * page_size;
    if (max_len > 0 && max_len < c.capacity) c.capacity = max_len;
    c.by_page = fast_div((uint32_t)page_size);
    for (int64_t *s : {c.ks, c.vs}) { // whole pages: rows follow each other, and nothing lies between the pages
        s[2] = WHOLE ? D : D + 16;
        s[1] = page_size * s[2];
        s[0] = c.Hkv * s[1];
    }
    if (WHOLE != whole_pages(c, D)) return 1;
    std::vector<int32_t> table(max_pages);
    const int used = (c.capacity - 1) / page_size; // of the last slot
    for (int i = 0; i < max_pages; ++i) table[i] = i < used ? used - 1 - i : i; // the last slot's page has the greatest number of those in use
    for (int i = used; i < max_pages; ++i) table[i] = max_pages - 1 - (i - used); // and is the pool's last
    if (absent)
        for (int i = 1; i < max_pages; i += 3) table[i] = i % 2 ? -1 : c.n_pages;
    const int head = c.Hkv - 1, steps = (c.capacity + 63) / 64;
    const K keys{c, table.data(), head * c.ks[1], head * c.vs[1]};
    for (int step = 0; step < steps + 2 * 16; ++step) {
        for (int lane = 0; lane < 64; ++lane) {
            const auto k = keys.find_k(step, lane);
            for (int i = 0; i < 4; ++i) {
                const typename K::Place &p = k.p[WHOLE ? 0 : i];
                const int page = keys.there(p) ? p.entry : 0, slot = step * 64 + 4 * (lane & 15) + i;
                const int64_t at = keys.k_offset(k, i, lane);
                for (int j = 0; j < D / 64; ++j)
                    if (outside(c, c.ks, at + 64 * j, 16, D, page)) return 2;
                if (slot < c.capacity) {
                    if (p.entry != table[slot / page_size]) return 3;
                    if (keys.there(p) && at != page * c.ks[0] + head * c.ks[1] + slot % page_size * c.ks[2] + 16 * (lane >> 4)) return 4;
                }
            }
            const typename K::Place own = keys.find_v(step, lane);
            for (int i = 0; i < 16; ++i) {
                const typename K::Place p = WHOLE ? own : keys.find_v(step, (lane & 48) + i);
                const bool is = keys.there(p);
                const int page = is ? p.entry : 0, slot = step * 64 + 16 * (lane >> 4) + i;
                const int64_t at = keys.v_offset(page, is ? p.at : 0, lane) + (WHOLE ? i * D : 0);
                if (outside(c, c.vs, at, D / 16, D, page)) return 5;
                if (slot < c.capacity) {
                    if (p.entry != table[slot / page_size]) return 6;
                    if (is && at != page * c.vs[0] + head * c.vs[1] + slot % page_size * c.vs[2] + (lane & 15) * (D / 16)) return 7;
                }
            }
        }
    }
    return 0;
}

int main()
{
    auto run = [](int page, int pages, int len) {
        for (bool absent : {false, true}) {
            const bool whole = page % 16 == 0;
            const int bad = whole ? check<64, true>(page, pages, len, absent) + 10 * check<128, true>(page, pages, len, absent) : 0;
            const int apart = check<64, false>(page, pages, len, absent) + 10 * check<128, false>(page, pages, len, absent);
            if (bad || apart) return printf("check %d, %d: pages of %d, %d of them, max_len %d, absent %d\n", bad, apart, page, pages, len, absent), 1;
        }
        return 0;
    };
    for (int page : {1, 7, 8, 16, 24, 32, 48, 64, 80, 100, 128, 256}) {
        for (int pages : {1, 2, 3, 4, 5, 7, 9, 28}) // capacities that are whole pages
            if (run(page, pages, 0)) return 1;
        for (int len = 1; len <= 2 * 64; ++len) // and every residue by 64
            if (run(page, (len + page - 1) / page + len % 3, len)) return 1;
        for (int len : {190, 192, 193, 257, 320, 447, 448, 449, 1000, 1023, 1025})
            if (run(page, (len + page - 1) / page, len)) return 1;
    }
    printf("%lld reads\n", asked);
    return 0;
}
"""


def test_every_read_of_keys_and_values_stays_in_its_page(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.run([hipcc, "-O2", "-std=c++17", "-x", "hip", "--offload-host-only", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout.split()[0]) > 10 ** 7
