"""Which tiles and pieces the cross entropy over a vocabulary is worked out in (gd_vocab_plan.h), compiled on the host
by itself: no tile of a launch reaches behind its piece while more words follow, whatever the sizes."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2605_17879_amd", "csrc")

MAIN = r"""
#include "gd_vocab_plan.h"
#include <stdio.h>
#include <initializer_list>
using namespace vocab_plan;
static uint64_t seed = 1;
static uint64_t below(uint64_t n) { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return (seed >> 20) % n; }
static uint64_t about(uint64_t most) { uint64_t v = most; for (uint64_t h = below(25); h > 0 && v > 1; --h) v /= 2; return 1 + below(v); }
static int launches = 0, cut = 0;
// One loss: the words of every launch, its tiles, and the parts that its rows' sums take.
static bool sound(uint64_t n, uint64_t V, uint64_t width, uint64_t want, uint64_t most) {
    const bool few = few_tiles(n, V);
    const uint64_t room = few ? up_to(V, 32) / 32 : up_to(V, 128) / 128;
    const uint64_t piece = words_at_once(n, V, want, most);
    if (piece == 0 || piece > V || piece > want || (piece < V && piece % 256)) return false;
    uint64_t parts = 0;
    for (uint64_t v0 = 0; v0 < V; v0 += piece) {
        const uint64_t words = V - v0 < piece ? V - v0 : piece, large = few ? 0 : large_part(words, n, width);
        const bool last = v0 + words == V;
        if (large > words || (large < words && large % 256)) return false;
        // large tiles end where the small ones begin, or where the vocabulary ends
        if (!few && !(large == words && last) && up_to(large, 256) != large) return false;
        if (!few && !last && large < words && up_to(words - large, 128) != words - large) return false;
        const uint64_t a = up_to(large, 256) / 256 * (up_to(n, 256) / 256), b = up_to(words - large, 128) / 128 * (up_to(n, 128) / 128);
        if (!few && (a > MOST_TILES || b > MOST_TILES)) return false;
        parts += parts_of_words(words, n, width, few);
        ++launches;
        cut += !last;
    }
    return parts <= room;
}
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
    // pieces whose number of tiles of 128 words would be odd
    for (uint64_t V : {131072ull, 151936ull, 2000000ull, 16777216ull})
        for (uint64_t t = 1; t <= 131072; t += t < 9000 ? 1 : 997)
            for (uint64_t width : {8ull, 1024ull}) CHECK(sound(t * 128 - 50, V, width, V, MOST_TILES));
    CHECK(cut > 1000);
    for (int i = 0; i < 200000; ++i) {
        const uint64_t n = about(1 << 24), V = about(1 << 24), width = about(65536);
        const uint64_t packed = up_to(1 + below(V), 256);
        const bool whole = few_tiles(n, V) || i % 2;
        // (small limits too, so that many pieces come up: at least the 256 words of one launch)
        const uint64_t most = whole && few_tiles(n, V) ? MOST_TILES : i % 3 ? MOST_TILES : 1 + below(1 << 20);
        const uint64_t want = whole ? V : packed < up_to(V, 256) ? packed : up_to(V, 256);
        if (V / words_at_once(n, V, want, most) > 4096) continue;
        if (!sound(n, V, width, want, most)) { printf("n %lu V %lu width %lu want %lu most %lu\n", n, V, width, want, most); return 1; }
    }
    CHECK(launches > 100000);
    printf("ok\n");
    return 0;
}
"""


def test_no_tile_reaches_behind_its_piece(tmp_path):
    (tmp_path / "main.cpp").write_text(MAIN)
    exe = tmp_path / "plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", f"-I{CSRC}", str(tmp_path / "main.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr

