// What the entry points of the token and expert layers check of their arguments, and how they launch.  Not part of the public ABI.
#pragma once

#include "token_internal.h"

namespace kfac {

constexpr int kMaxPositions = 1 << 30, kMaxDim = 1 << 20, kMaxExperts = 1 << 16;

inline bool type_ok(kfac_dtype t) { return t == KFAC_F32 || t == KFAC_BF16; }
inline size_t esize(kfac_dtype t) { return t == KFAC_BF16 ? 2 : 4; }

// Bytes that a call touches: one piece of `row` bytes every `ld` bytes from p to p + size; ld = 0: one piece.  Empty: touches nothing.
struct Range {
    const char *p;
    size_t size, row, ld;
    Range(const void *p_ = nullptr, size_t size_ = 0, size_t row_ = 0, size_t ld_ = 0) : p((const char *)p_), size(size_), row(ld_ ? row_ : size_), ld(ld_) {}
};
inline Range matrix(const void *p, long long rows, long long cols, long long ld, size_t es)
{
    if (!p || rows <= 0) return Range();
    return Range(p, (size_t)((rows - 1) * ld + cols) * es, (size_t)cols * es, rows > 1 && ld > cols ? (size_t)ld * es : 0);
}
// Columns beside each other in one wider tensor are apart though their ranges meet: with the same distance of rows (or one piece on
// one side) the two sets of pieces are compared inside one distance.
inline bool overlap(const Range &a, const Range &b)
{
    if (!a.size || !b.size || a.p >= b.p + b.size || b.p >= a.p + a.size) return false;
    if (a.ld != b.ld && a.ld && b.ld) return true;
    const size_t ld = a.ld ? a.ld : b.ld;
    if (!ld) return true;
    const size_t at = a.p <= b.p ? (size_t)(b.p - a.p) % ld : (ld - (size_t)(a.p - b.p) % ld) % ld;   // of b's pieces behind a's
    return at < a.row || at + b.row > ld;
}
// rows that lie ld elements apart: offsets, in bytes too, stay far inside 64 bits
inline bool spread_ok(long long rows, long long ld)
{
    constexpr long long most = 1LL << 40;
    return ld <= most && (rows <= 1 || ld <= most / rows);
}
inline bool aligned(const void *p, size_t es) { return (uintptr_t)p % es == 0; }

// One launch between the profiler's events
template <typename F>
inline bool timed(kfac_ctx *ctx, int kernel, int variant, double flops, double bytes, F launch)
{
    return profile_begin(ctx, kernel, variant, flops, bytes) && launch() == hipSuccess && profile_end(ctx);
}

}  // namespace kfac
