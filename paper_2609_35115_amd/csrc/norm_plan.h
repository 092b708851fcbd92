// A rule of the norms' stores.  Host code only, so that it can be compiled and
// checked by itself.
#pragma once

namespace dcb {

// Whether neither result (null: not stored) lies in an input's place (h null: none).
// Only then do all threads read the inputs, in whatever order they load and store: with
// one result in place, what a thread reads of another thread's elements may be that
// result already, and must enter neither of the two.
inline bool results_apart(const void* x, const void* h, const void* r, const void* y)
{
    auto apart = [&](const void* o) { return !o || (o != x && o != h); };
    return apart(r) && apart(y);
}

}  // namespace dcb
