// Where the lines of an operand lie that start off a 16-byte boundary, or an odd number of elements apart, and which of their 16-byte units a lane reads
// (skew_product.cu). Plain arithmetic, which the host compiles too. Not part of the public ABI.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define SKEW_BOTH __host__ __device__ __forceinline__
#else
#define SKEW_BOTH inline
#endif

namespace skew {

constexpr int kOperandLines = 128;             // of an operand, in a CTA's stage
constexpr int kRawLine = 144;                  // a line of 64 elements that starts anywhere, by 16-byte units

SKEW_BOTH constexpr int64_t within(int64_t low, int64_t x, int64_t high) { return x < low ? low : x > high ? high : x; }

// A warp's `N` of an operand's 128 lines of a tile's stages, from line `from` on, eight lanes to a line. MAJOR: lines along the summed index, numbered l0 on, of which
// those before l_end are there; a stage is 64 elements, from s0 on, before s_end. Else two blocks of 64 lines, one for each step of the summed index (s0 on, before
// s_end), of elements from l0 (and l0 + 64), before l_end; a stage is 64 lines.
template <bool MAJOR, int N>
struct Lines {
    const char *at;         // the lane's first line, in this stage
    int64_t four, stage;    // bytes from a line to the lane's next, and to the next stage
    int lines, n;           // that are there from the lane's first line on (negative: it lies as many behind the last; a ninth unit is of another line), and elements of a line
    int left;               // of the summed index

    SKEW_BOTH Lines(const uint16_t *p, int64_t ld, int64_t l0, int64_t l_end, int64_t s0, int64_t s_end, int from, int lane) {
        const int64_t mine = from % (MAJOR ? kOperandLines : 64) + lane / 8, elem = MAJOR ? s0 : l0 + from / 64 * 64;
        at = reinterpret_cast<const char *>(p + ((MAJOR ? l0 : s0) + mine) * ld + elem);
        four = ld * 8;
        stage = MAJOR ? 128 : ld * 128;
        left = int(within(0, s_end - s0, 1 << 30));
        if (MAJOR) {
            lines = int(within(-N, l_end - l0 - mine, N));
            n = left < 64 ? left : 64;
        } else {
            lines = left - int(mine);
            n = int(within(0, l_end - elem, 64));
        }
    }

    SKEW_BOTH void next() {
        at += stage;
        left -= 64;
        if (MAJOR) n = int(within(0, left, 64)); else lines -= 64;
    }

    // The units that the lane reads, of 144 bytes for each of the warp's lines: ask(its place there, its address, whether it holds an element that is there).
    // Those that do not are asked for too, as zeros.
    template <typename Ask>
    SKEW_BOTH void units(int lane, Ask ask) const {
        const uint32_t to = lane / 8 * kRawLine + lane % 8 * 16;
        const char *p = at;
#ifdef __CUDACC__
#pragma unroll
#endif
        for (int i = 0; i < N / 4; ++i, p += four) {
            const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 15;
            ask(to + i * 4 * kRawLine, p - off + lane % 8 * 16, i * 4 < lines && n > 0 && lane % 8 * 16 < int(off) + n * 2);
        }
        // the ninth units, a line to a lane
        const int line = lane % N;
        const char *q = at + (four >> 2) * (line - lane / 8);
        const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(q)) & 15;
        ask(line * kRawLine + 128, q - off + 128, line - lane / 8 < lines && int(off) + n * 2 > 128);
    }
};

}  // namespace skew
