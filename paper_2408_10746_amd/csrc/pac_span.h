// Host side: do two operands of a call share memory?  Results that lie over what other workgroups still read would race.
#pragma once
#include <stdint.h>
#include <initializer_list>
#include <utility>

namespace pac {

// rows of `width` bytes, `pitch` apart (pitch >= width where there are several)
struct Span {
    uintptr_t at;
    int64_t rows, pitch, width;
    Span(const void *p, int64_t rows_, int64_t pitch_, int64_t width_) : at(reinterpret_cast<uintptr_t>(p)), rows(p ? rows_ : 0), pitch(pitch_), width(width_) {}
    Span(const void *p, int64_t bytes) : Span(p, 1, bytes, bytes) {}
    bool empty() const { return rows < 1 || width < 1; }
    uintptr_t end() const { return at + (uintptr_t)((rows - 1) * pitch + width); }
};

// Exact, for matrices side by side in one buffer too.  Rows of one pitch: where b's first row falls among a's decides for all of them.
// Else row by row of the shorter one (operands that interleave at different pitches; nobody has been seen to do it).
static inline bool share(Span a, Span b)
{
    if (a.empty() || b.empty() || a.end() <= b.at || b.end() <= a.at) return false;
    for (Span *s : {&a, &b})
        if (s->rows == 1 || s->pitch == s->width) s->width = (int64_t)(s->end() - s->at), s->rows = 1;
    if (a.rows == 1 && b.rows == 1) return true;
    if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {
        if (b.at < a.at) std::swap(a, b);
        const int64_t by = (int64_t)(b.at - a.at), row = by / a.pitch, in = by % a.pitch;
        return in < a.width || (row + 1 < a.rows && in + b.width > a.pitch);
    }
    if (b.rows < a.rows) std::swap(a, b);
    for (int64_t r = 0; r < a.rows; ++r) {
        // the last row of b that begins before this one of a ends: earlier ones end earlier
        const int64_t from = (int64_t)(a.at - b.at) + r * a.pitch, to = from + a.width - 1;
        if (to < 0) continue;
        const int64_t j = to / b.pitch < b.rows - 1 ? to / b.pitch : b.rows - 1;
        if (j * b.pitch + b.width > from) return true;
    }
    return false;
}

// does `out` share memory with any of those?
static inline bool shares(const Span &out, std::initializer_list<Span> others)
{
    for (const Span &s : others)
        if (share(out, s)) return true;
    return false;
}

} // namespace pac
