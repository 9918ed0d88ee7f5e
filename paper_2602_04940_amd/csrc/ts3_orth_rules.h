// The matrices of a list of orthogonalised updates, and which tiles their products take: by their sizes and the compute
// units `cus` alone, on the host.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace ts3 {

// A tensor of the list: nb matrices, wide form r x c, padded to rp x cp (multiples of 64).
struct OrthEntry {
    const void *src;
    void *dst;
    int64_t x, a;             // half floats before its X and its A in their buffers
    int32_t r, c, nb, flags;  // ORTH_TURNED, ORTH_BF16
    int32_t piece, load, gram, update;  // first workgroups of the launches
};
enum { ORTH_TURNED = 1, ORTH_BF16 = 2 };
__host__ __device__ __forceinline__ int orth_pad(int n) { return (n + 63) & ~63; }

constexpr int ORTH_SMALL = 64;  // the longer side of a matrix that one workgroup does

// Tiles of ts x ts of an entry's products: of the update, or of a symmetric one, on and below the diagonal.  A small
// matrix has none.
inline int64_t orth_tiles(const OrthEntry &e, int ts, bool update) {
    const int64_t nr = (orth_pad(e.r) + ts - 1) / ts, nc = (orth_pad(e.c) + ts - 1) / ts;
    return e.c <= ORTH_SMALL ? 0 : e.nb * (update ? nr * nc : nr * (nr + 1) / 2);
}

// Tiles of a product and how many groups of waves share one, from the tiles of 128 and of 64 that there are.
struct OrthShape {
    int side, groups;
};
// A compute unit does one tile of 128 at a time: with one to four rounds of them, the last costs more than
// smaller tiles do, and with fewer than half a round, idle units do.  On the GPU (256 units), 128 against 64: 1,536
// tiles of 256 K 63 against 70 us, 432 of 256 to 1,024 K 44 against 39 and of 256 K 26 against 22, 144 of
// 4,096 K 87 against 99, 1,024 of 1,024 K 136 against 174.  Few tiles of 64 have four groups of waves each
// (18 of 512 K 7.4 against 9 us).
inline OrthShape orth_shape(int64_t large, int64_t half, int64_t cus) {
    if (large >= cus / 2 && (large <= cus || large >= 4 * cus)) return OrthShape{128, 1};
    return OrthShape{64, half <= cus ? 4 : 1};
}
// That of the `count` entries' updates, or of their symmetric products.
inline OrthShape orth_shape(const OrthEntry *e, size_t count, bool update, int64_t cus) {
    int64_t large = 0, half = 0;
    for (size_t i = 0; i < count; ++i) {
        large += orth_tiles(e[i], 128, update);
        half += orth_tiles(e[i], 64, update);
    }
    return orth_shape(large, half, cus);
}

}  // namespace ts3
