// Streams on which something is due: a page call has been enqueued and no paged decode behind it yet.  Host only.
#pragma once

namespace flux {

struct StreamSet {
    static constexpr int kMost = 16;
    void *at[kMost];
    int n;                           // beyond kMost: too many to tell, so all streams are meant from then on
    // 0 and 1 are the same stream: the default one, by its two names
    static void *name(void *stream) { return stream == (void *)1 ? nullptr : stream; }
    void add(void *stream)
    {
        stream = name(stream);
        for (int i = 0; i < n && n <= kMost; ++i)
            if (at[i] == stream) return;
        if (n < kMost) at[n] = stream;
        if (n <= kMost) ++n;
    }
    // true once for a stream that was added
    bool take(void *stream)
    {
        if (n > kMost) return true;
        stream = name(stream);
        for (int i = 0; i < n; ++i)
            if (at[i] == stream) {
                at[i] = at[--n];
                return true;
            }
        return false;
    }
};

}  // namespace flux
