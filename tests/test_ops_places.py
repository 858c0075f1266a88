"""Places of operand chunks (csrc/km_places.h), on the CPU: the arithmetic that the
kernels load by is compiled for the host, and every chunk that a tile of a transposed
weight loads has to lie within its row, and so within the weight."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1902_09527_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include "km_places.h"
using namespace km;

// Every chunk of every stage of every tile of a K x P matrix: 0, or what is wrong.
template <class T, int TN, int NT>
const char* check(int K, int P) {
    using S = TrStage<T, TN, NT>;
    if (P % S::E != 0) return nullptr;   // rows that are not of whole chunks take another form
    const int64_t es = sizeof(T), row_bytes = P * es, bytes = K * row_bytes;
    int covered = 0;   // columns from the left that some tile holds
    for (int at = 0; at < P; at += TN) {
        const int bn = S::first(at, P);
        if (bn < 0 || bn % S::E || bn > covered) return "a tile's first column";
        covered = bn + TN;
        for (int k = 0; k * S::BK < K + 2 * S::BK; ++k)   // two stages past the end are loaded too
            for (int tid = 0; tid < NT; ++tid)
                for (int i = 0; i < S::N; ++i) {
                    const bool in = S::in(i, tid, k, bn, K, P);
                    if (k >= S::whole(K, P) && !in) continue;   // loads zeros in its place
                    const int64_t from = bn * es + (int64_t)k * S::BK * row_bytes + (int64_t)S::above(i, row_bytes)
                                         + S::behind(i % 2, tid, row_bytes);
                    const int64_t row = (int64_t)k * S::BK + S::row(i, tid), col = bn + S::column(i, tid);
                    if (from != row * row_bytes + col * es) return "a chunk's place";
                    if (from % 16 != 0) return "a chunk's alignment";
                    if (from + 16 > bytes) return "a chunk past the matrix";
                    if (col * es + 16 > row_bytes || row >= K) return "a chunk past its row";
                    if (!in) return "a chunk loaded that has no place";
                }
    }
    return covered >= P ? nullptr : "columns that no tile holds";
}

int main(int argc, char** argv) {
    const int K = atoi(argv[1]);
    for (int i = 2; i < argc; ++i) {
        const int P = atoi(argv[i]);
        const char* e[] = {check<uint16_t, 256, 512>(K, P), check<uint16_t, 128, 256>(K, P),
                           check<uint16_t, 64, 256>(K, P), check<float, 256, 512>(K, P), check<float, 128, 256>(K, P),
                           check<float, 64, 256>(K, P)};
        for (int j = 0; j < 6; ++j)
            if (e[j]) {
                printf("K %d, P %d, %s, tile %d: %s\n", K, P, j < 3 ? "16 bits" : "32 bits", 256 >> j % 3, e[j]);
                return 1;
            }
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("places")
    (at / "places.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I" + CSRC, "-o", str(at / "places"), str(at / "places.cpp")], check=True)
    return str(at / "places")


@pytest.mark.parametrize("K", [32, 64, 96, 128, 1024, 2048, 4096, 1, 40, 100, 1000])
def test_chunks_of_a_transposed_weight(program, K):
    """Widths that the tiles divide, that leave a whole chunk or all but one, and that are
    narrower than a tile."""
    widths = [320, 576, 1408, 2040, 4064, 8, 16, 56, 64, 72, 120, 128, 136, 192, 248, 256, 264, 384, 504, 512, 520, 1000, 4, 12, 60, 68, 132,
              252, 260, 1404]
    r = subprocess.run([program, str(K)] + [str(p) for p in widths], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
