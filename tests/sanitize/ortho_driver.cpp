// Host-only check of how orthogonalised updates are split, built with
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_muon_tiles.py.
// Each input line is a call: a type, then rows, cols and batch of every entry.
// Its output line: "small", or for each table the tile size of each product,
// the splits of the Gram one and its parts' bytes, then the call's workspace.
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

#include "norm.hpp"
#include "ortho_plan.hpp"

using namespace qlayer;

int main() {
    for (std::string line; std::getline(std::cin, line);) {
        std::istringstream in(line);
        int type;
        in >> type;
        std::vector<ql_matrix> mats;
        for (ql_matrix q{}; in >> q.rows >> q.cols >> q.batch;) mats.push_back(q);
        const int count = (int)mats.size(), format = type == E_F64 ? DOUBLE : TWO;
        if (!ortho_launchable(type, mats.data(), count)) {
            std::puts("refused");
            continue;
        }
        if (all_small(type, mats.data(), count)) std::printf("small");
        else
            for (int at = 0; at < count;) {
                Chunk c;
                at = next_chunk(mats.data(), count, at, c, nullptr);
                if (!c.count) break;
                const Choice g = choose(format, GRAM, c), p = choose(format, POLY, c), a = choose(format, APPLY, c);
                std::printf("gram %d splits %d bytes %lld poly %d apply %d ", TILES[g.which], g.splits, (long long)g.bytes,
                            TILES[p.which], TILES[a.which]);
            }
        std::printf(" workspace %zu\n", ortho_workspace(type, mats.data(), count));
    }
}
