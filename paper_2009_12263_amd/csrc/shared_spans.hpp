// Whether some of many arrays share memory with one that is written.  Plain host code without HIP: a CPU test compiles this header.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <vector>

namespace fg {

// The bytes from begin on, to end; `written`, or only read; `of` is the caller's.
struct Span {
    uintptr_t begin, end;
    int64_t of;
    bool written;
};

// Two spans that share bytes, one of them written: `first` begins no later.  False: there are none.  get(list, i) is span i (of `count`) of one of `lists` lists; spans without
// bytes count as none.  Lists are cut where they neither rise nor fall on; of a model's tensors, allocated one after the other, that gives few pieces, and those that lie apart from
// all others need no closer look.
template <class Get> bool shared_spans(int lists, int64_t count, const Get &get, Span &first, Span &second) {
    struct Piece { uintptr_t begin, end; int list; bool falls; int64_t from, to; };
    std::vector<Piece> pieces;
    pieces.reserve(32);
    for (int list = 0; list < lists; ++list) {
        Piece p = {0, 0, list, false, 0, 0};
        int64_t n = 0;                          // spans of p
        for (int64_t i = 0; i < count; ++i) {
            const Span s = get(list, i);
            if (s.begin >= s.end) continue;
            if (n > 0 && s.begin >= p.end && (n == 1 || !p.falls)) {
                p.end = s.end;
                p.falls = false;
            } else if (n > 0 && s.end <= p.begin && (n == 1 || p.falls)) {
                p.begin = s.begin;
                p.falls = true;
            } else {
                if (n > 0) pieces.push_back(p);
                p = {s.begin, s.end, list, false, i, i};
                n = 0;
            }
            ++n;
            p.to = i + 1;
        }
        if (n > 0) pieces.push_back(p);
    }
    std::sort(pieces.begin(), pieces.end(), [](const Piece &a, const Piece &b) { return a.begin < b.begin; });
    auto before = [](const Span &a, const Span &b) { return a.begin != b.begin ? a.begin < b.begin : a.of < b.of; };
    std::vector<Span> spans, other;
    std::vector<size_t> ends;
    for (size_t i = 0, next; i < pieces.size(); i = next) {
        next = i + 1;
        for (uintptr_t end = pieces[i].end; next < pieces.size() && pieces[next].begin < end; ++next) end = std::max(end, pieces[next].end);
        if (next == i + 1) continue;
        // pieces i .. next - 1 in one list, by merging neighbours
        spans.clear();
        ends.assign(1, 0);
        for (size_t k = i; k < next; ++k) {
            for (int64_t j = pieces[k].from; j < pieces[k].to; ++j) {
                const Span s = get(pieces[k].list, j);
                if (s.begin < s.end) spans.push_back(s);
            }
            if (pieces[k].falls) std::reverse(spans.begin() + (std::ptrdiff_t)ends.back(), spans.end());
            ends.push_back(spans.size());
        }
        other.resize(spans.size());
        while (ends.size() > 2) {
            size_t kept = 1;
            for (size_t k = 0; k + 1 < ends.size(); k += 2) {
                const size_t last = ends[std::min(k + 2, ends.size() - 1)];
                const Span *at = spans.data();
                std::merge(at + ends[k], at + ends[k + 1], at + ends[k + 1], at + last, other.data() + ends[k], before);
                ends[kept++] = last;
            }
            ends.resize(kept);
            spans.swap(other);
        }
        Span written = {0, 0, 0, true}, read = {0, 0, 0, false};            // those that reach furthest so far
        for (const Span &s : spans) {
            const Span *with = s.begin < written.end ? &written : s.written && s.begin < read.end ? &read : nullptr;
            if (with) {
                first = *with;
                second = s;
                return true;
            }
            Span &furthest = s.written ? written : read;
            if (s.end > furthest.end) furthest = s;
        }
    }
    return false;
}

}  // namespace fg
