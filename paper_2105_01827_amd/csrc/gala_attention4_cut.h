// How a call of attention over the paged 4-bit cache is cut up: by its sizes and types alone, on the host.
#pragma once
#include <algorithm>
#include <cmath>

#include "gala_decode.h"

namespace gala {
namespace {

// queries that a wavefront's products take at once, and those of a workgroup, where a sequence brings many
constexpr int kWide = 32, kWavesOf = 4, kColumnsOf = kWide * kWavesOf;

// Whether weights are in half precision.  A score times log2(e) and the logarithm of a scale share an accumulator then: neither may
// drown the other.
inline bool in_halves(float scale, int q_type, int out_type) {
    const float unit = std::fabs(scale) * kLog2E;
    return q_type != GALA_F32 && q_type != GALA_RESIDUE && out_type != GALA_F32 && out_type != GALA_RESIDUE && unit >= 0x1p-20f && unit <= 0x1p20f;
}
// f16 queries of more than 192 channels, in two parts, do not fit the registers beside a wide tile's sums
inline bool fits_wide(int q_type, int dim) { return q_type != GALA_F16 || dim <= 192; }

// How a call is cut up.
struct Cut {
    bool many;
    int tiles, splits, columns, waves;
    long places() const { return (long)tiles * splits * columns; }
};
inline Cut cut_of(const KvArgs &kv, int heads_q, int window, int sinks, bool fine) {
    Cut c;
    const long columns = (long)kv.max_new * (heads_q / kv.heads);
    const long reach = std::min<long>(kv.max_len, (long)kv.table_stride * kKvBlock);
    const long keys = window ? std::min(reach, (long)window + kv.max_new + sinks + 2 * kKvBlock) : reach;
    const long blocks = std::max(1l, (keys + kKvBlock - 1) / kKvBlock);
    const long groups = (columns + kColumnsOf - 1) / kColumnsOf * kv.count * kv.heads;
    // Wide tiles take their time whatever the groups are until those fill the card, narrow ones with shares of the keys grow with them.  128
    // channels of bf16, 1000 tokens: 64 groups 27 us and 17, 128 27 and 27, 160 27 and 31; 6000 tokens: 160 groups 114 and 95, 256 120 and
    // 149.  64 channels, 1000 tokens: 160 groups 21 and 21; 256 channels: 64 groups 47 and 39, 96 47 and 57.
    const int g32 = kv4_groups(kv.dim), fives = g32 <= 2 ? 6 : g32 <= 4 ? 5 : 3;
    c.many = !fine && columns >= kColumnsOf && groups >= std::min(192l, 96 + 2 * blocks) * fives / 5;
    if (c.many) {
        c.tiles = (int)((columns + kColumnsOf - 1) / kColumnsOf), c.splits = 1, c.columns = 0;
        return c;
    }
    c.tiles = (int)((columns + kColumns - 1) / kColumns);
    c.columns = (int)std::min<long>(columns, kColumns);
    // A block takes a wavefront 1.2 us after the other, joining shares 5 us.  Eight wavefronts a workgroup where that leaves CUs with one:
    // 32 windows of 1024 tokens take 12.3 us so and 14.5 with four, one sequence of 131072 25.0 and 26.4; 64 of 8192 in 512
    // workgroups of 32 bits 121 and 114.  Shares for one round of the card, of 8 blocks at least, where there are 48: 4000 tokens take 18.5 us
    // whole and 11.6 in shares.  Wide heads leave room for one wavefront a SIMD.
    const long units = std::max(1l, (long)kv.count * kv.heads * c.tiles);
    const bool wide = g32 > 4;
    const bool few = !wide && (units <= 128 || (units <= 256 && blocks < 128));
    const long room = few || wide ? 256 : 512;
    c.waves = few ? 8 : 4;
    c.splits = blocks < 48 ? 1 : (int)std::max(1l, std::min(room / units, blocks / 8));
    return c;
}

}  // namespace
}  // namespace gala
