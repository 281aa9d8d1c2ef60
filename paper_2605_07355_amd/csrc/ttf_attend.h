// What the attention kernels share: which keys a row sees, where they lie in the cache, and how the work of a ragged batch
// is dealt out on the device (the host knows no lengths).
#pragma once

#include "ttf_device.h"
#include "ttf_serve.h"

namespace ttf {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// One sequence of the batch.
struct Sequence {
    int first, rows;       // rows in the buffers
    int cached, length;    // entries before these rows; entries that any of them may see (0 where `cached` makes no sense)
    int begin;             // lowest entry that a row's window reaches, in whole blocks of 32
};

__device__ __forceinline__ Sequence sequence_of(const ttf_attention_params& p, const ttf_kv_cache& c, int b)
{
    Sequence s;
    const int2 r = rows_of(p.row_offsets, b, p.rows);
    s.first = r.x;
    s.rows = r.y;
    s.cached = p.cached[b];
    const long long room = (long long)c.page_size * c.table_width, all = (long long)s.cached + s.rows;
    s.length = s.cached < 0 ? 0 : (int)min(min(all, room), 0x7ff00000ll);
    s.begin = p.window > 0 && s.cached >= p.window ? (s.cached - p.window + 1) & ~31 : 0;
    return s;
}

// How the work is dealt out.  A tile is up to `columns` (row, query head of the key head's group) pairs of one sequence,
// its work the 32-entry blocks of the sequence's context.  Every tile of a sequence is cut into the same number of parts along the
// context, so many that no part is longer than `per` blocks, where all parts together are about `target` workgroups.
//   part id -> key head fastest, then part, then tile, then sequence: workgroups that run together read neighbouring heads
//   of the same slots.
// Tiles of more than one part leave (sum, maximum, unnormalised row) of each part in the workspace; `slot` counts those.
struct Deal {
    int b, tile, part, parts;
    long long slot;        // first workspace slot of the tile (times kv_heads), where parts > 1
};

__device__ __forceinline__ long long wave_total(long long v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}
__device__ __forceinline__ long long wave_prefix(long long v, int lane)   // sum over the lanes up to this one
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const long long below = __shfl_up(v, m, 64);
        if (lane >= m) v += below;
    }
    return v;
}

__device__ __forceinline__ int tiles_of(int rows, int group, int columns)
{
    return (int)(((long long)rows * group + columns - 1) / columns);
}

// The deal of unit `unit` (of parts if `by_part`, else of tiles).  Every wave works it out by itself from the lengths: two passes
// over the batch, 64 sequences at a time.  False where there is no such unit.
__device__ inline bool deal_out(const ttf_attention_params& p, const ttf_kv_cache& c, int columns, int step, int target, long long unit,
                                bool by_part, Deal& d)
{
    const int lane = threadIdx.x & 63, group = p.heads / p.kv_heads;
    const auto blocks = [&](const Sequence& s) { return max(0, (int)(((long long)s.length - s.begin + step - 1) / step)); };
    long long total = 0;
    for (int i = 0; i < p.batch; i += 64) {
        long long work = 0;
        if (i + lane < p.batch) {
            const Sequence s = sequence_of(p, c, i + lane);
            work = (long long)tiles_of(s.rows, group, columns) * blocks(s);
        }
        total += wave_total(work);
    }
    const long long share = (total * p.kv_heads + target - 1) / target;
    const int per = (int)max(1ll, min(share, 0x7fffffffll));
    long long units = 0, slots = 0;
    for (int i = 0; i < p.batch; i += 64) {
        int tiles = 0, parts = 1;
        if (i + lane < p.batch) {
            const Sequence s = sequence_of(p, c, i + lane);
            tiles = tiles_of(s.rows, group, columns);
            parts = max(1, (blocks(s) + per - 1) / per);
        }
        const long long mine = (long long)tiles * (by_part ? parts : 1), held = parts > 1 ? (long long)tiles * parts : 0;
        const long long upto = units + wave_prefix(mine, lane), slots_upto = slots + wave_prefix(held, lane);
        const unsigned long long after = __ballot(upto > unit);
        if (after) {
            const int at = __ffsll(after) - 1;
            const long long start = __shfl(upto - mine, at, 64);
            d.b = i + at;
            d.parts = __shfl(parts, at, 64);
            const int in = (int)(unit - start);
            d.tile = by_part ? in / d.parts : in;
            d.part = by_part ? in - d.tile * d.parts : 0;
            d.slot = __shfl(slots_upto - held, at, 64) + (long long)d.tile * d.parts;
            return true;
        }
        units = __shfl(upto, 63, 64);
        slots = __shfl(slots_upto, 63, 64);
    }
    return false;
}

}  // namespace ttf
