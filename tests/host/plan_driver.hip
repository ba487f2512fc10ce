// The choices that the dense operators make on the host, and the order of a tile product's stages, for the tests: questions on
// the standard input, a line each, answers on the standard output.  No GPU is needed.
#include <cstdio>
#include <cstring>

#include "sidco_product.h"

using namespace sidco;

// A block's fetches, `depth` stages ahead of what it multiplies: the tiles' and terms' stages in order, then `depth` more behind
// the last.  Returns the largest stage number among those, or -1 if one before is out of order.
static int sequence(uint32_t stages, int terms, uint32_t tiles, uint32_t blocks, uint32_t block, int depth)
{
    Sequence s = {block, 0, 0};
    for (uint32_t tile = block; tile < tiles; tile += blocks)
        for (int term = 0; term < terms; ++term)
            for (uint32_t u = 0; u < stages; ++u) {
                if (s.tile != tile || s.term != term || s.u != u) return -1;
                const bool other = s.next(stages, terms, tiles, blocks);
                if (other != (u + 1 == stages)) return -1;
            }
    int most = 0;
    for (int k = 0; k < depth; ++k) {
        if (s.tile < tiles) return -1;
        if ((int)s.u > most) most = (int)s.u;
        if (s.next(stages, terms, tiles, blocks)) return -1;
    }
    return most;
}

int main()
{
    char what[32];
    while (std::scanf("%31s", what) == 1) {
        if (!std::strcmp(what, "sequence")) {
            uint32_t stages, tiles, blocks, block;
            int terms, depth;
            if (std::scanf("%u %d %u %u %u %d", &stages, &terms, &tiles, &blocks, &block, &depth) != 6) return 1;
            std::printf("%d\n", sequence(stages, terms, tiles, blocks, block, depth));
        } else {
            return 1;
        }
    }
    return 0;
}
