// What the entry points of the sequence-layer operators share: types, argument checks, a fill kernel (layer_util.hip).
#pragma once
#include "common.hpp"

namespace la {

inline bool unknown_dtype(la_dtype dt) { return dt != LA_F32 && dt != LA_F64 && dt != LA_BF16 && dt != LA_F16; }
inline bool small_dtype(la_dtype dt) { return dt == LA_BF16 || dt == LA_F16; }
inline size_t bytes_of(la_dtype dt) { return dt == LA_F64 ? 8 : dt == LA_F32 ? 4 : 2; }
inline size_t align_up(size_t n) { return (n + 255) & ~(size_t)255; }
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    const char *pa = (const char *)a, *pb = (const char *)b;
    return pa && pb && na && nb && pa < pb + nb && pb < pa + na;
}
// LA_ERR_WORKSPACE (and the text) where less than `need` was given, LA_ERR_INVALID_ARG where it is not 256-byte aligned
la_status check_workspace(const void *ws, size_t given, size_t need, const char *asked);
// a kernel that writes zeros (a null pointer: nothing); `bytes` in whole 2-byte elements
la_status zero_bytes(void *p, size_t bytes, hipStream_t st);

}  // namespace la
