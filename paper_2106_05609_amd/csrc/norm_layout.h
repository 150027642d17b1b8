// How the rows of the norms' kernels lie in lanes, and how many rows a workgroup takes: what the kernels index by, free of the GPU so that
// norm_check.cpp can try it on the CPU.
#pragma once
#include <stdint.h>

#include <algorithm>

namespace gas {

// A lane's piece of a row, E elements (16 bytes): the first of them, how many of them another piece has already, and whether there is one; a lane
// behind the row's end has the row's first piece and neither counts nor stores it.  MASK: F is no multiple of E; the last piece is the row's last E elements
// then.  A lane has P pieces, as many as its row needs, so only the last may be cut or missing.  Said of three pieces it saves every seventh instruction
// (backward, 1,433 bf16: 101 us, so 92); of two the registers come out worse (100,000 x 400 floats 254 and 269).
struct Piece {
    int c, skip;
    bool on;
};
template <int E, bool MASK, int P>
constexpr Piece piece_of(int index, int i, int F) {
    const bool whole = P > 2 && i < P - 1;
    Piece p = {index * E, 0, whole || index * E < F};
    if (MASK && !whole && p.c + E > F) {
        p.skip = p.c + E - F;
        p.c = F - E;
    }
    if (!p.on) p.c = 0;
    return p;
}
// Bytes from the wavefront's first row to element c of its row `team`.  Rows narrower than a piece: c may lie before the row.
template <int EB>
constexpr uint32_t piece_offset(int team, int64_t ld, int c) { return ((uint32_t)team * (uint32_t)ld + (uint32_t)c) * EB; }
template <int EB>
constexpr int64_t tiny_offset(int team, int64_t ld, int c) { return (team * ld + c) * EB; }

// How rows of F elements lie in lanes, and the workgroups' turns; w = 0: too wide for registers, element by element.  Figures are us.
struct Layout {
    int g, w, p, turns;                  // lanes of a team, wavefronts of a row, pieces of a lane; turns of a workgroup
    int64_t blocks, most_blocks;         // workgroups, and of any fewer rows: never less where there are more rows
};

// At most kMostSums workgroups leave sums, so these take at most 1 MB for every column however many rows there are (without that a third of a float
// matrix).  Without a bound, with 65,536, 32,768 and 16,384: 600,000 x 256 floats 882, 884, 908, 927; 3,125,002 x 256 floats 4,976, 4,894, 4,858, 4,905; x 64 floats
// 1,117, 1,120, 1,155, 1,195; x 256 bf16 2,352, 2,344, 2,368, 2,447; 1 M x 400 floats 2,500, 2,501, 2,366, 2,512.
constexpr int64_t kMostSums = 49152;

inline Layout layout_of(int64_t n, int F, bool bf, bool bwd, int64_t longest_ld) {
    const int e = bf ? 8 : 4, pieces = (F + e - 1) / e;
    Layout l = {64, 1, 1, 1, 0, 0};
    // Beyond 1,024 pieces a lane's share no longer fits: 8,000 x 8,200 bf16 backward 3,400 with its registers spilt, element by element 1,800 (forward 600 and
    // 900).  The widest bf16 rows below spill too, backward: some 10 registers by twelve wavefronts, 100 by sixteen (8,000 x 8,192: 552).
    if (pieces > 1024) return {0, 0, 0, 0, 0, 0};
    // Up to 64 pieces a team with a lane for each, rounded up to a power of two: 3 M x 8 bf16 forward 42, in teams of eight 214, backward 84 and 294; 3 M x 16 floats
    // 149 and 188, 305 and 318.  Up to 192 one wavefront, several pieces a lane, so nothing waits at a barrier: backward, against a wavefront for every 64 pieces,
    // 66,667 x 600 bf16 161 and 168, 40,000 x 1,000 143 and 152, 19,997 x 1,433 108 (92 since) and 115; but 20,000 x 2,000 bf16 262 and 147, where four pieces no longer
    // fit.  Beyond, several wavefronts: 20,000 x 2,000 floats by eight 258, element by element 890.
    if (pieces <= 64)
        while (l.g / 2 >= pieces) l.g /= 2;
    else if (pieces <= 192)
        l.p = (pieces + 63) / 64;
    else
        for (int w : {16, 12, 8, 6, 4})
            if (pieces <= w * 64) l.w = w;
    const int64_t rows = l.w == 1 ? 4 * (64 / l.g) : 1, all = (n + rows - 1) / rows;
    const auto turns_of = [&](int64_t groups) { return (all + groups - 1) / groups; };
    // Backward, every workgroup leaves partial sums: of few turns in all there are no more workgroups than keep memory busy.  512: 50,000 x 256 bf16 46, 1,024 50, 2,048 57.
    // 256 where a lane has several pieces, 19,997 x 1,433 bf16 108, 512 123, or a row many wavefronts, 13,333 x 3,000 bf16, six, 167 and 175; but four,
    // 20,000 x 2,000 bf16, 183 and 148.
    const int64_t fewest = !bwd || (l.p == 1 && l.w <= (bf ? 4 : 6)) ? 512 : 256;
    // Of many turns, what workgroups of few turns save outweighs the sums.  512 workgroups, and 16, 8, 4, 2 turns: 1 M x 256 bf16 813, 763, 727, 779, 999; 600,000 x 256 floats 956,
    // 921, 906, 875, 909; 1 M x 47 floats 352, 333, 300, 282, 315; 100,000 x 256 floats 166, 166, 156, 159, 154, but 25,000 45, -, 48, 48.  Not bf16 rows in which a quarter of
    // the lanes or more have no piece, where the sums weigh more: three quarters filled, 512 workgroups and 8 turns, 1 M x 192 626 and 647, 500,000 x 384 651 and
    // 699, 2 M x 96 623 and 637; 17 of 32 lanes, 1 M x 136, 487 and 567; but 28 of 32, 1 M x 224, 724 and 670.  Nor bf16 in two pieces, 200,000 x 600 456 and 565.
    const bool many = bwd && l.w == 1 && (bf ? l.p == 1 && 4 * pieces > 3 * l.g && all >= 32768 : all >= 16384);
    const int64_t few = bf || all < 32768 ? 8 : 4;
    if (!bwd) {
        // Forward, few rows to a workgroup, next to each other, so that the rows in flight are one stretch of memory that moves along: 3.1 M x 256 bf16, two turns 1,267,
        // four 1,318, eight 1,374, a grid that goes round once and again 1,785; 600,000 x 64 floats, one 121, two 129.
        l.turns = (int)std::min(turns_of(fewest), (int64_t)(l.w > 1 ? (bf ? 4 : 2) : bf || l.p > 1 ? 2 : 1));
    } else if (many) {
        l.turns = (int)std::max(few, turns_of(kMostSums));
    } else {
        // Up to four turns by one workgroup, whose sums need no second launch: 16 x 256 floats 7.6, else 9.7.
        l.turns = (int)(all <= 4 ? all : turns_of(fewest));
    }
    // A launch has less than 2^32 threads: what is more goes by more turns (67,108,869 x 129 floats and up).
    l.turns = (int)std::max((int64_t)l.turns, turns_of(0xFFFFFFFFLL / (l.w == 1 ? 256 : l.w * 64)));
    l.blocks = turns_of(l.turns);
    l.most_blocks = many ? std::min(turns_of(few), kMostSums) : std::min(all, fewest);
    // A wavefront's last byte lies within 32 bits of its first row, or the wavefront has one row.  Rows narrower than a piece have offsets of 64 bits, and one
    // lane: they cannot be loaded whole.
    if (F >= e && ((64 / l.g - 1) * longest_ld + F) * (bf ? 2 : 4) > 0xFFFFFFFFLL) {
        l.turns *= 64 / l.g;
        l.g = 64;
    }
    return l;
}

}  // namespace gas
