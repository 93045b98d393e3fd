// dropout.cuh -- the mask of fiona_adapter.h's dropout: 16 bits per element from
// a counter, so that any kernel can form it again wherever it meets the element.
#pragma once
#include <stdint.h>

#if defined(__CUDACC__)
#define DROP_HD __host__ __device__ __forceinline__
#else
#define DROP_HD inline
#endif

namespace dropout {

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;
constexpr uint64_t kStream = 4;  // stream under the user's seed (1 to 3, 9: synthetic layers)

// SplitMix64's output function (Steele, Lea, Flood, OOPSLA 2014)
DROP_HD uint64_t mix64(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// A mask, ready for a kernel: element (t, i) of a matrix with `groups` =
// ceil(cols / 4) is kept iff field i % 4 of mix64(base + (t groups + i / 4) golden)
// is at least `level`.  level = 0: no dropout.
struct Mask {
    uint64_t base = 0;
    uint64_t groups = 0;
    uint32_t level = 0;
    float factor = 1.f;

    // the four fields of columns 4 g .. 4 g + 3 of row t
    DROP_HD uint64_t draw(uint64_t t, uint64_t g) const { return mix64(base + (t * groups + g) * kGolden); }
    DROP_HD static uint32_t field(uint64_t v, uint32_t k) { return (uint32_t)(v >> (16 * k)) & 0xFFFFu; }
    DROP_HD bool keep(uint64_t t, uint64_t i) const { return field(draw(t, i >> 2), i & 3) >= level; }
};

}  // namespace dropout
