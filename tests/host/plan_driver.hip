// The choices that the dense operators make on the host, and the order of a tile product's stages, for the tests: questions on
// the standard input, a line each, answers on the standard output.  No GPU is needed.
#include <cstdio>
#include <cstring>

#include "sidco_ortho_plan.h"
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
        } else if (!std::strcmp(what, "plan")) {  // tile, columns and second tile of a batch of products
            long m, n, batch, lines;
            if (std::scanf("%ld %ld %ld %ld", &m, &n, &batch, &lines) != 4) return 1;
            const TilePlan p = plan_tiles(m, n, batch, lines);
            std::printf("%d %ld %d\n", p.pick, (long)p.columns, p.rest_pick);
        } else if (!std::strcmp(what, "triangle")) {  // tile of `count` symmetric products
            long m, count, lines;
            if (std::scanf("%ld %ld %ld", &m, &count, &lines) != 3) return 1;
            std::printf("%d\n", best_triangle(m, count, lines));
        } else if (!std::strcmp(what, "steps")) {  // one block?, steps in pairs, steps in a group of either kind
            long rows, cols;
            int batch, steps, paired;
            float a, b, c;
            if (std::scanf("%d %ld %ld %d %d %f %f %f", &batch, &rows, &cols, &steps, &paired, &a, &b, &c) != 8) return 1;
            if (paired < 0) paired = ortho_paired(steps, a, b, c, paired == -16);  // by the type: -16 bf16, -32 another
            const OrthoGroups g = ortho_groups(batch, rows < cols ? rows : cols, rows < cols ? cols : rows, steps, paired);
            std::printf("%d %d %d %d\n", ortho_one_block(rows, cols, cols, paired > 0), paired, g.paired, g.halves);
        } else {
            return 1;
        }
    }
    return 0;
}
