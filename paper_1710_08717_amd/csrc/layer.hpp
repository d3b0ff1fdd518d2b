// What the entry points of the sequence-layer operators share: types, argument checks, a fill kernel (layer_util.hip).
#pragma once
#include "common.hpp"

#include <initializer_list>

namespace la {

inline bool unknown_dtype(la_dtype dt) { return dt != LA_F32 && dt != LA_F64 && dt != LA_BF16 && dt != LA_F16; }
inline bool small_dtype(la_dtype dt) { return dt == LA_BF16 || dt == LA_F16; }
inline size_t bytes_of(la_dtype dt) { return dt == LA_F64 ? 8 : dt == LA_F32 ? 4 : 2; }
// the most blocks of `threads` that one launch takes: its threads are counted in 32 bits
inline int64_t most_blocks(int threads) { return (int64_t)(0xffffffffu / (unsigned)threads); }
inline size_t align_up(size_t n) { return (n + 255) & ~(size_t)255; }
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const char *pa = (const char *)a, *pb = (const char *)b;
    return pa && pb && na && nb && pa < pb + nb && pb < pa + na;
}
struct Span {
    const void *p;
    size_t n;
};
// whether any of `out` overlaps one of `in` or another of `out`
inline bool any_overlap(std::initializer_list<Span> in, std::initializer_list<Span> out)
{
    for (auto o = out.begin(); o != out.end(); ++o) {
        for (const Span &i : in)
            if (overlaps(o->p, o->n, i.p, i.n))
                return true;
        for (auto other = out.begin(); other != o; ++other)
            if (overlaps(o->p, o->n, other->p, other->n))
                return true;
    }
    return false;
}
// LA_ERR_WORKSPACE (and the text) where less than `need` was given, LA_ERR_INVALID_ARG where it is not 256-byte aligned
la_status check_workspace(const void *ws, size_t given, size_t need, const char *asked);
// a kernel that writes zeros (a null pointer: nothing); `bytes` in whole 2-byte elements
la_status zero_bytes(void *p, size_t bytes, hipStream_t st);

}  // namespace la
