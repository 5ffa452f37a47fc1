// The line of tiles of the tcgen05 attention: how new tokens are cut into row pieces, and a batch's pieces into equal shares.
// Plain arithmetic, for the kernel and for tests on the host.
#pragma once

#include "aj_kv.cuh"

#ifdef __CUDACC__

namespace aj {
namespace kv {

// SHARED: of a call whose sequences share their first slots.  (Asked at run time, what only those need cost prompts with a window of heads
// of 64 5 %: 176 us and 185.)
#define AJ_HD __host__ __device__ inline

constexpr int TILE = 128;
// What an item costs beside its tiles (its queries, the pipeline's start, its results), in tiles.
constexpr int CHARGE = 2;

// The tokens of a row piece and the tiles of slots that they see.
struct Piece {
    int ta, n_tok, tok0;          // first token, tokens, tokens of stream 0 (== n_tok: both streams share the rows)
    int first, n_sink, first_tile, units;
    int places;                   // on the line: its tiles, or the same number for every piece (View::align)
};

struct Seqs {                     // a sequence and how its new tokens are cut into pieces
    Seq s;
    int n, each, more;            // pieces, spread evenly
};

struct Line {                     // position in the line
    int b, h, qt, unit;           // sequence, key head, row piece, tile within the item (below 0: its charge)
    Seqs q;
    Piece p;
};

// A CTA's part of an item: `line` places of the line, of which the tiles first .. first + n - 1.
struct Part {
    int line, first, n;
};
template <bool SHARED> AJ_HD Part part_of(const Line &c, int left) {
    Part p;
    p.line = min((SHARED ? c.p.places : c.p.units) - c.unit, left);
    p.first = max(c.unit, 0);
    p.n = max(0, (SHARED ? min(c.unit + p.line, c.p.units) : c.unit + p.line) - p.first);
    return p;
}

// tpt: tokens of a row tile
AJ_HD Seqs pieces_of(const Seq &s, int tpt) {
    Seqs q;
    q.s = s;
    q.n = (s.nq + 2 * tpt - 1) / (2 * tpt);
    q.each = q.n ? s.nq / q.n : 0;
    q.more = s.nq - q.each * q.n;
    return q;
}

template <bool SHARED = true> AJ_HD Piece piece_of(const View &v, const Seqs &q, int qt, int tpt) {
    Piece p;
    p.ta = qt * q.each + min(qt, q.more);
    p.n_tok = q.each + (qt < q.more);
    p.tok0 = p.n_tok <= tpt ? p.n_tok : (p.n_tok + 1) >> 1;
    const int p_lo = q.s.L - q.s.nq + (SHARED ? q.s.ahead : 0) + p.ta, reach = max(0, p_lo + p.n_tok), end = SHARED ? min(q.s.L, reach) : reach;
    p.first = v.window ? min(max(0, p_lo - v.window + 1), end) : SHARED ? q.s.first : 0;
    p.first_tile = p.first / TILE;
    p.n_sink = min((min(v.sinks, p.first) + TILE - 1) / TILE, p.first_tile);
    p.units = max(1, p.n_sink + (end + TILE - 1) / TILE - p.first_tile);
    p.places = SHARED && v.align ? max(p.units, v.align - CHARGE) : p.units;
    return p;
}

// Places on the line of the row pieces at, at + step, ... of a sequence, for one key head.
// How large it gets: a handle allows B * n_q * Hq = 2^30 rows in pieces of more than 128 rows (and a last one per sequence and key
// head, at most 65,535 of them) that see at most 2^20 slots, so a line has less than 2^36 places and needs 64 bits; a
// CTA's share of it, an item and the pieces' numbers stay below 2^31.
template <bool SHARED = true> AJ_HD long long units_of(const View &v, const Seqs &q, int tpt, int at, int step) {
    long long u = 0;
    for (int i = at; i < q.n; i += step) u += CHARGE + piece_of<SHARED>(v, q, i, tpt).places;
    return u;
}

// a / b rounded down, b > 0
AJ_HD int floor_div(int a, int b) { return a >= 0 ? a / b : -((b - 1 - a) / b); }

// Does stream x have a tile in a segment of n tiles of this piece?
AJ_HD bool has_tile(const Piece &p, int x, int n) { return x == 0 || p.tok0 < p.n_tok || n > 1; }

AJ_HD int tile_of(const Piece &p, int unit) { return unit < p.n_sink ? unit : unit - p.n_sink + p.first_tile; }

}  // namespace kv
}  // namespace aj

#endif
