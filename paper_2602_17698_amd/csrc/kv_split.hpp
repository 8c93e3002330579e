// Which keys of a sequence a row sees, and how keys are shared out among workgroups: arithmetic of the attention's kernels that tests run on the host, too.
#pragma once

#include <stdint.h>

namespace sbits {

struct KeyRange { int first, last; };         // first .. last - 1

// The keys that a row at a position sees, of a sequence of `length` tokens whose table of pages reaches `there` of them.  Empty ranges, too, lie within 0 .. there: what walks
// over the keys of several rows goes from the first row's begin to the last one's end, and reads the table's entries up to there.
constexpr KeyRange seen_keys(bool causal, int window, int there, int length, int position)
{
    int last = causal && position < length ? position + 1 : length;
    last = last < there ? last : there;
    last = last > 0 ? last : 0;
    const int first = window && position >= window ? position + 1 - window : 0;
    return {first < last ? first : last, last};
}

// ---- sharing out the keys of few rows ----------------------------------------------------
// An item is a tile of 16 rows of a sequence with a key's head; its work the tiles of keys that the sequence's rows see.  All items, sequence after sequence, a sequence's by tiles of rows,
// then heads, make a line of W tiles of keys, of which workgroup w of G has those from cut(w) to cut(w + 1):  w (W / G), moved to the item's begin or end where that is less than FEW_EDGE tiles
// away, and to the begin of an item of up to FEW_WHOLE tiles.  So workgroups have the same to do, whatever the lengths.  A part of an item goes to slot 2 w + 1 of its workgroup if it is the item's
// first, else to 2 w: a workgroup's last part is an item's first, and of others it has no more than one.
constexpr int FEW_EDGE = 4, FEW_WHOLE = 16, FEW_LEAST = 8;       // FEW_LEAST: tiles of keys a workgroup, at least, where items may be cut
// (Where none may be, a workgroup for each of them costs nothing: 87 sequences of up to 29 tokens, 16 heads of 128: 48 us with eight items in a row a workgroup, 27 with up to three; 8 tokens of one sequence, 16 heads of 256 on 2: 79 and 13.)
constexpr int few_workgroups(int most, bool space, int64_t total)
{
    const int64_t all = space ? total / FEW_LEAST : total;
    return all >= most ? most : all < 1 ? 1 : (int)all;
}
// Where cut w of G falls ahead of its move (w < G): a product in 64 bits, rounded down, which is the same wherever it is asked for.
constexpr int64_t few_cut(int w, int workgroups, int64_t total) { return (int64_t)((double)w * ((double)total / (double)workgroups)); }
// Whether a sequence's items may be cut: not where there is no space for parts (no sequence was announced to be long enough), nor short ones, nor those of more
// rows than were announced (which the parts' join would not reach).
constexpr bool few_cuttable(bool space, int most_rows, int rows, int keys) { return space && keys > FEW_WHOLE && rows <= most_rows; }
// what a cut at `off` tiles of an item becomes
constexpr int few_snap(bool cuttable, int keys, int off) { return off < FEW_EDGE || !cuttable ? 0 : keys - off < FEW_EDGE ? keys : off; }
// The cuts inside an item that begins at `begin`: from the first that is behind its begin, and stays there, on.  Its parts are one more, and the first is workgroup first - 1's.
struct FewCuts { int first, past; };
constexpr FewCuts few_cuts(int64_t begin, int keys, int workgroups, int64_t total)
{
    const double each = (double)total / (double)workgroups;
    int first = (int)((double)begin / each) - 1, past = (int)((double)(begin + keys - FEW_EDGE) / each) + 2;
    if (first < 0) first = 0;
    if (past > workgroups) past = workgroups;
    while (first < workgroups && few_cut(first, workgroups, total) - begin < FEW_EDGE) ++first;
    while (past > first && few_cut(past - 1, workgroups, total) - begin > keys - FEW_EDGE) --past;
    return {first, past};
}

}  // namespace sbits
