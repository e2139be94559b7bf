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

// Piece `piece` of p.pieces.  Sequence s has ceil(tiles_s / run) pieces, with `run` the
// smallest for which they are no more than p.pieces, and none more than p.splits (the
// records of a row).  It lies between ceil(total / pieces) and
// ceil(total / (pieces - sequences)), for which sum ceil(tiles_s / run) <= pieces always,
// and is halved in on (16 sequences of 2017..8950 keys in 64 pieces: 43 tiles; a step of 1/16
// at a time ended at 45, 72.2 us a call against 70.3).
__device__ inline PieceOf piece_of(const AttnArgs& a, const Plan& p, int piece) {
    ColPlan cp{};
    cp.streams = 1;
    cp.columns = 1;
    const ColSeqs c = col_seqs(a, cp);
    const int tiles = (int)c.tiles, top = wave_max_u(tiles), total = (int)c.total;
    auto pieces_of = [&](int run) __attribute__((always_inline)) { return (tiles + run - 1) / run; };
    auto fits = [&](int run) __attribute__((always_inline)) {
        return wave_reduce_i(pieces_of(run), [](int x, int y) { return x + y; }) <= p.pieces;
    };
    int run = max(max((total + p.pieces - 1) / p.pieces, (top + p.splits - 1) / p.splits), kPieceTiles);
    if (!fits(run)) {
        int low = run;   // does not fit; `run` does
        run = p.pieces > a.n_seqs ? (total + p.pieces - a.n_seqs - 1) / (p.pieces - a.n_seqs) : top;
        run = max(run, low + 1);
        while (run - low > 1) {
            const int mid = low + (run - low) / 2;
            if (fits(mid)) run = mid;
            else low = mid;
        }
    }
    const int n = pieces_of(run), end = wave_prefix_sum_i(n), sum = __builtin_amdgcn_readlane(end, 63);
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
