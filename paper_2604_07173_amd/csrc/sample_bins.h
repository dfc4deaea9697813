// Which tokens of a row of logits a lane looks at, and which of them are in a bin: what decides whether a token is listed, and so
// whose logits are read again.  Plain C++.
#pragma once
#include <math.h>

#ifndef LORA_HD
#define LORA_HD __host__ __device__ inline
#endif

namespace lora {

// A row as pieces of VEC logits; it begins `skew` logits into the first one.
template <int VEC>
struct Pieces {
    int skew, vocab;

    LORA_HD int pieces() const { return (skew + vocab + VEC - 1) / VEC; }

    // The number of a piece's logit e: below 0 or from `vocab` on in front of the row and behind it, where -inf stands for the logits.
    LORA_HD int number(int i, int e) const { return i * VEC - skew + e; }
};

// A number of bins over powers of two of weights.
struct Bins {
    float each;                           // to half a difference of logits
    int most;
};

LORA_HD Bins bins_over(float powers, int most, float T) { return Bins{(float)most / powers * (1.44269504f / T) * 2.f, most}; }

// Half of what l is below the largest logit, with one rounding, as the whole: that may be beyond a float where T is as large.
LORA_HD float half_below(float top, float l) { return fmaf(l, -0.5f, top * 0.5f); }

// Rises as l falls; `most` behind the last bin, and for what is no number.
LORA_HD int bin_of(float top, float l, Bins b) { return (int)fminf(half_below(top, l) * b.each, (float)b.most); }

// One bin, as the differences that it has; behind the last one, whatever is not below its end.
struct Bin {
    float each, begin, end;
};

LORA_HD Bin only_bin(Bins b, int which) { return Bin{b.each, (float)which, which == b.most ? NAN : (float)(which + 1)}; }

// A token above `from` that is in the bin.  The first comparison is never left out: the others hold for -inf as well where a
// temperature makes `each` zero or infinite, and -inf is what stands in front of a row and behind it.  (no branches: & in place of &&)
LORA_HD bool is_in(float top, float l, float from, Bin b)
{
    const float x = half_below(top, l) * b.each;
    return (l > from) & !(x < b.begin) & !(x >= b.end);
}

}  // namespace lora
