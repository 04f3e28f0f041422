// ace_overlap.h — whether rows of two tensors share memory.
#pragma once

#include <cstdint>
#include <initializer_list>

namespace ace {

using Wide = __int128;                  // strides are whatever a caller says

// Row (t, h) is `row` bytes from at + t * token + h * head on, t < tokens, h < heads; strides in bytes, >= 0.
struct RowSet {
    uintptr_t at;
    Wide token, head;
    long long tokens, heads;
    Wide row;
};

inline Wide floor_div(Wide a, Wide b) { return a >= 0 ? a / b : -((b - 1 - a) / b); }

// Rows of a_row bytes at x * sa (x < na) and of b_row bytes at d + y * sb (y < nb): do any two meet?
inline bool runs_meet(Wide d, Wide sa, long long na, Wide sb, long long nb, Wide a_row, Wide b_row) {
    if (na > 1 && nb > 1 && sa != sb) {
        if (na > nb) return runs_meet(-d, sb, nb, sa, na, b_row, a_row);
        for (long long x = 0; x < na; ++x)
            if (runs_meet(d - x * sa, 0, 1, sb, nb, a_row, b_row)) return true;
        return false;
    }
    // places d + m * s, m from `least` to `most`; the first that ends behind 0
    const Wide s = nb > 1 ? sb : na > 1 ? sa : 1, least = -(Wide)(na - 1), most = nb - 1, m = floor_div(-b_row - d, s) + 1;
    const Wide at = d + (m < least ? least : m) * s;
    return m <= most && at < a_row;
}

// Exact. Tensors apart, and rows that alternate within one projection, are told by a comparison and a division or two; what is left
// goes head by head.
inline bool rows_meet(RowSet a, RowSet b) {
    if (!a.at || !b.at || a.tokens < 1 || a.heads < 1 || b.tokens < 1 || b.heads < 1 || a.row < 1 || b.row < 1) return false;
    for (RowSet* r : {&a, &b}) {
        if (r->token == 0) r->tokens = 1;
        if (r->head == 0) r->heads = 1;
    }
    const Wide tokens_a = (a.tokens - 1) * a.token, heads_a = (a.heads - 1) * a.head;
    const Wide tokens_b = (b.tokens - 1) * b.token, heads_b = (b.heads - 1) * b.head;
    const Wide d = (Wide)b.at - (Wide)a.at;
    if (d >= tokens_a + heads_a + a.row || -d >= tokens_b + heads_b + b.row) return false;
    // both repeat with the same stride, and lie in distinct parts of it
    auto alternate = [&](long long na, Wide sa, long long nb, Wide sb, Wide span_a, Wide span_b) {
        if (na > 1 && nb > 1 && sa != sb) return false;
        const Wide s = na > 1 ? sa : nb > 1 ? sb : 0;
        if (s == 0) return false;
        const Wide from = d - floor_div(d, s) * s;
        return from >= span_a && from + span_b <= s;
    };
    if (alternate(a.tokens, a.token, b.tokens, b.token, heads_a + a.row, heads_b + b.row)) return false;
    if (alternate(a.heads, a.head, b.heads, b.head, tokens_a + a.row, tokens_b + b.row)) return false;
    for (long long i = 0; i < a.heads; ++i)
        for (long long j = 0; j < b.heads; ++j)
            if (runs_meet(d + j * b.head - i * a.head, a.token, a.tokens, b.token, b.tokens, a.row, b.row)) return true;
    return false;
}

}  // namespace ace
