// Which keys of a sequence a row sees: arithmetic of the attention's kernels that tests run on the host, too.
#pragma once

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

}  // namespace sbits
