// The plan builder of the 4-bit layers on ragged shapes and refused arguments, for a build with sanitizers (host code only).
#include <cstdio>
#include <cstdlib>
#include <numeric>

#include "pivot_quant.h"

namespace pivot { void set_error(const char*, ...) {} }

using namespace pivot;

static int failures = 0;
#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); ++failures; } } while (0)

int main() {
    for (int M : {1, 15, 16, 100, 257})
        for (int K : {1, 31, 128, 300, 1025})
            for (int bh : {16, 32, 64})
                for (int bw : {32, 64, 128})
                    for (int kept = 0; kept < 3; ++kept)
                        for (int chunk : {0, 1, 2}) {
                            pivot_qfc_desc d{M, K, bh, bw, 64, 0, chunk, -1, 0};
                            const int nbr = (M + bh - 1) / bh, nbc = (K + bw - 1) / bw, ng = (K + 63) / 64;
                            std::vector<uint8_t> mask((size_t)nbr * nbc), zeros((size_t)M * ng, 15);
                            for (size_t i = 0; i < mask.size(); ++i) mask[i] = kept == 2 || (kept == 1 && (i * 7) % 3 == 0);
                            std::vector<int32_t> prow(M), pcol(K);
                            for (int i = 0; i < M; ++i) prow[i] = M - 1 - i;
                            for (int i = 0; i < K; ++i) pcol[i] = (i + 1) % K;
                            std::vector<float> bias(M, 1.f);
                            QfcHost h;
                            CHECK(build_qfc_host(d, zeros.data(), (int64_t)M * ng, mask.data(), prow.data(), pcol.data(), bias.data(), h) == PIVOT_OK);
                            CHECK(h.nchunks >= nbr && h.kb_ptr[nbr] == h.KB && (int)h.pieces.size() == h.KB * (kQBlk / bw));
                            CHECK(h.whole == (h.T == nbr * nbc));
                            int blocks = 0;
                            for (int c = 0; c < h.nchunks; ++c) blocks += h.chunks[8 * c + 2] - h.chunks[8 * c + 1];
                            CHECK(blocks == h.KB);
                            if (K > 1) { pcol[0] = pcol[1]; QfcHost bad; CHECK(build_qfc_host(d, nullptr, 0, mask.data(), prow.data(), pcol.data(), nullptr, bad) == PIVOT_E_NOT_PERMUTATION); }
                            prow[M - 1] = M;
                            QfcHost bad;
                            CHECK(build_qfc_host(d, nullptr, 0, nullptr, prow.data(), nullptr, nullptr, bad) == PIVOT_E_NOT_PERMUTATION);
                        }
    int seen[128] = {};
    for (int c = 0; c < kQBlk; ++c) ++seen[q_byte_pos(c)];
    for (int n : seen) CHECK(n == 1);
    int cols = 0;
    for (int i = 0; i < 8; ++i) cols |= 1 << q_nibble_col(i);
    CHECK(cols == 255);
    std::printf(failures ? "%d failures\n" : "all checks passed\n", failures);
    return failures != 0;
}
