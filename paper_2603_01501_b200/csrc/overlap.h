// Whether two strided blocks of rows share memory: what the argument checks refuse for outputs.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <utility>

namespace {

// Rows of `width` bytes at p + i token + j head, i < nt, j < nh.
struct Rows {
    uint64_t p;
    uint64_t token, head;   // bytes
    uint64_t nt, nh, width;
    uint64_t end() const { return p + (nt - 1) * token + (nh - 1) * head + width; }
};

// Exact where the token strides agree (views of one fused tensor: heads between each other's) or a block has one token;
// otherwise blocks whose spans cross count as sharing.
inline bool share(Rows a, Rows b) {
    if (a.p >= b.end() || b.p >= a.end()) return false;
    for (Rows *r : {&a, &b}) {
        if (r->nt == 1 || r->token == 0) r->nt = 1, r->token = 0;
        if (r->nh == 1 || r->head == 0) r->nh = 1, r->head = 0;
    }
    if (a.nt > 1 && b.nt > 1 && a.token != b.token) return true;
    const int64_t token = int64_t(std::max(a.token, b.token));
    // rows whose first bytes lie d + m token apart (b's behind a's) for m from 1 - a.nt to b.nt - 1
    auto rows_share = [&](int64_t d) {
        const int64_t least = -int64_t(b.width) - d + 1, most = int64_t(a.width) - d - 1;   // m token must be in between
        if (token == 0) return least <= 0 && 0 <= most;
        const int64_t up = least >= 0 ? (least + token - 1) / token : -(-least / token);   // rounded up
        const int64_t m = std::max(up, 1 - int64_t(a.nt));
        return m <= int64_t(b.nt) - 1 && m * token <= most;
    };
    const int64_t d0 = int64_t(b.p) - int64_t(a.p);
    if (a.head == b.head || a.nh == 1 || b.nh == 1) {
        const int64_t head = int64_t(std::max(a.head, b.head));
        for (int64_t c = 1 - int64_t(a.nh); c < int64_t(b.nh); ++c)
            if (rows_share(d0 + c * head)) return true;
        return false;
    }
    if (a.nh * b.nh > (1u << 16)) return true;
    for (uint64_t i = 0; i < a.nh; ++i)
        for (uint64_t j = 0; j < b.nh; ++j)
            if (rows_share(d0 + int64_t(j * b.head) - int64_t(i * a.head))) return true;
    return false;
}

}  // namespace
