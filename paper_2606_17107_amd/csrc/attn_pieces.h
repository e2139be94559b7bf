// Pieces of the many-row kernels: where every row leaves partials anyway (trees of
// drafted tokens), a sequence is cut into as many pieces as its length asks for, so
// that ragged caches keep all workgroups equally long.  The lengths live on the
// device, so each workgroup works the cut out for itself: lane s of a wave holds
// sequence s.
#pragma once

#include "attn_columns.h"

namespace pkv {

constexpr int kPieceTiles = 2;   // shortest run of a piece, in tiles

struct PieceOf {
    int seq, index, count;   // piece `index` of the `count` of sequence `seq`; count 0: none
    SeqInfo si;
};

// Piece `piece` of p.pieces.  Sequence s has ceil(tiles_s / run) pieces, with `run` about the
// smallest for which they are no more than p.pieces, and none more than p.splits (the
// records of a row): ceil(total / pieces), a few larger ones, or
// ceil(total / (pieces - sequences)), for which sum ceil(tiles_s / run) <= pieces always.
__device__ inline PieceOf piece_of(const AttnArgs& a, const Plan& p, int piece) {
    ColPlan cp{};
    cp.streams = 1;
    cp.columns = 1;
    ColSeqs c = col_seqs(a, cp);
    const int top = wave_max_u((int)c.tiles), total = (int)c.total;
    int run = max(max((total + p.pieces - 1) / p.pieces, (top + p.splits - 1) / p.splits), kPieceTiles);
    int n = 0, end = 0, sum = 0;
    for (int k = 0;; ++k) {
        n = ((int)c.tiles + run - 1) / run;
        end = wave_prefix_sum_i(n);
        sum = __builtin_amdgcn_readlane(end, 63);
        if (sum <= p.pieces) break;
        const int sure = p.pieces > a.n_seqs ? (total + p.pieces - a.n_seqs - 1) / (p.pieces - a.n_seqs) : top;
        run = k < 3 ? min(run + (run + 15) / 16, max(sure, run + 1)) : max(sure, run + 1);
        run = __builtin_amdgcn_readfirstlane(run);
    }
    PieceOf r;
    r.count = 0;
    if (piece >= sum) return r;
    r.seq = __builtin_popcountll(__builtin_amdgcn_ballot_w64(end <= piece));
    r.count = __builtin_amdgcn_readlane(n, r.seq);
    r.index = piece - (__builtin_amdgcn_readlane(end, r.seq) - r.count);
    r.si = col_seq_info(c, r.seq);
    return r;
}

}  // namespace pkv
