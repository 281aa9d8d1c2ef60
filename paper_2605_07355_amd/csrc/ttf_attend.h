// What the attention kernels share: which keys a row sees, where they lie in the cache, and how the work of a ragged batch
// is dealt out on the device (the host knows no lengths).
#pragma once

#include "ttf_device.h"
#include "ttf_places.h"
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
// its work the blocks of `keys` entries of the sequence's context.  A workgroup's four waves either take turns with the blocks of
// one key head, or (`neighbours`, where there is enough work) each walk along the same blocks for a key head of its own: then
// the workgroup reads four neighbouring heads of a slot, 1 KiB where one head is 256 bytes, which the memory likes better.  Every tile of a
// sequence is cut into the same number of parts along the context, so many that no part is longer than `per` turns, where all parts
// together are about `target` workgroups (a power of two; `even`: a little less than it or than twice as many).
//   part id -> key head (four of them) fastest, then part, then tile, then sequence.
// Tiles of more than one part leave (maximum, sum, unnormalised row) of each part and head in the workspace, and part 0 a note for
// the join.  With n key heads a workgroup, those rows' tiles are at most 2 n target (parts of cut tiles are more than per / 2 turns long
// on average, also after the last turn of four blocks is rounded up), and the notes at most half as many.
struct Deal {
    int b, tile, part, parts;
    int heads;             // key heads of a workgroup: 1 or 4
    int slot;              // first workspace slot of the tile (times kv_heads), where parts > 1
    int note;              // its number among the tiles of more than one part
    Sequence seq;
};
// (Times in this file and beside it, without further word: bf16, 32 query heads on 8 of 128 entries, ragged batches of up to the sizes given.)
// Whether no tile is cut into parts, and none joined, because table or window leave no long context: up to 512 entries, 256 in fp32 (8 clips
// of 200 rows 28.5 us cut, 14.8 not, 64 tokens over 400 entries 25.7 and 21.6; fp32, 10 x 15 rows over 200 27.0 and 21.0, but one token over 400
// 15.1 and 17.6).  It goes by the room in the table, which the host knows, and not by the lengths.
__host__ __device__ inline bool uncut(const ttf_attention_params& p, const ttf_kv_cache& c)
{
    const long long room = (long long)c.page_size * c.table_width;
    const long long reach = p.window > 0 ? (long long)p.window + p.rows : room;    // (a sequence has at most all the rows)
    return (room < reach ? room : reach) <= (p.dtype == TTF_BF16 ? 512 : 256);
}
constexpr int kNeighbours = 4, kNeighbourTurns = 8;          // least turns a part that make it worth it
struct JoinNote { int b, tile, parts, slot; };
struct JoinNotes { int count, pad[3]; JoinNote note[1]; };

// Sum over the lanes up to this one, at VALU rate: within rows of 16, then lane 15 of each row into the next, then lane 31 on.
__device__ __forceinline__ int wave_prefix(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
    return v;
}

__device__ __forceinline__ int tiles_of(int rows, int group, int columns)
{
    return (int)((unsigned)(rows * group + columns - 1) / (unsigned)columns);    // (rows * heads <= 2^27)
}

// Turns a part at most, so that the workgroups come out in whole rounds of `target`: one that runs alone at the end costs as much as a full
// round of them.  64 lengths are tried, a lane each, from half of an even `share` on, for the least sum of the rounds' longest parts and
// what a part costs besides (kPartTurns: its start, and its rows to the workspace and back; 5 and 14 choose alike).  At most 2 target
// workgroups, or the share stays.  `tiles` and `turns`: of sequence `lane`, at most 64 of them.
//   with the even share and here: 300 rows over 100k keys 779 and 558 us, 4 x 128 over 8k 73 and 56, 2000 over 31k 1057 and 1029, 20 over 8k 23.6 and 24.3
constexpr float kPartTurns = 9.0f;
__device__ inline int even_turns(int batch, int kv_heads, int target, double share, int per, int tiles, int turns)
{
    const int lane = threadIdx.x & 63;
    if (__ballot(turns >= 1 << 18) || wave_sum((float)tiles) * kv_heads > 2.0f * target) return per;    // (past it the quotients below may be off)
    const double aim = share * 0.5 * (1.0 + lane / 16.0);
    const int mine = aim < 1.0 ? 1 : (int)__builtin_ceil(aim);
    const float inverse = 1.0f / mine * (1.0f - 0x1p-21f);   // n / mine, rounded up: 1 / n at least above a whole number, or that number
    float all = 0.0f, most = 0.0f;
    for (int b = 0; b < batch; ++b) {
        const float n = (float)__builtin_amdgcn_readlane(turns, b), parts = fmaxf(1.0f, __builtin_ceilf(n * inverse));
        const float many = (float)__builtin_amdgcn_readlane(tiles, b);
        all += many * parts;
        if (many > 0.0f) most = fmaxf(most, n / parts);
    }
    all *= kv_heads;
    const float cost = all <= 2.0f * target ? __builtin_ceilf(all / target) * (most + kPartTurns) : INFINITY;
    float least = cost;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) least = fminf(least, __shfl_xor(least, d, 64));
    const unsigned long long best = __ballot(cost == least);
    return least == INFINITY || !best ? per : __builtin_amdgcn_readlane(mine, __ffsll(best) - 1);
}

// The deal of workgroup `block`.  Every wave works it out by itself from the lengths, 64 sequences at a time (batches of up to 64
// read them once).  False where nothing is left for it.  With `notes`, counts the tiles of more than one part as well.
__device__ inline bool deal_out(const ttf_attention_params& p, const ttf_kv_cache& c, int columns, int keys, bool neighbours, bool even, int target,
                                int block, JoinNotes* notes, Deal& d)
{
    const int lane = threadIdx.x & 63, group = p.heads / p.kv_heads;
    int tiles = 0, blocks = 0;                               // of sequence i + lane
    Sequence s{};
    const auto look = [&](int i) {
        tiles = blocks = 0;
        if (i + lane < p.batch) {
            s = sequence_of(p, c, i + lane);
            tiles = tiles_of(s.rows, group, columns);
            blocks = (int)((unsigned)(max(0, s.length - s.begin) + keys - 1) / (unsigned)keys);
        }
    };
    double total = 0.0;                                      // (whole numbers below 2^53)
    for (int i = 0; i < p.batch; i += 64) {
        look(i);
        total += wave_sum((double)tiles * blocks);
    }
    // a part of `per` turns: per blocks of one wave and four heads, or 4 per blocks of four waves and one head
    const double share = total * p.kv_heads / (4.0 * target);
    int per = __builtin_amdgcn_readfirstlane(share < 1.0 ? 1 : share > 1e9 ? 1000000000 : (int)__builtin_ceil(share));
    // few rows: parts of up to 3 turns where a third of the workgroups is left then (8 tokens over 3000 entries 23.3 us with shorter ones, 20.8; 12 over a
    // window of 8192 entries 39.3 either way)
    if (!even) per = max(per, __builtin_amdgcn_readfirstlane((int)__builtin_fmin(3.0, __builtin_ceil(3.0 * share))));
    if (even && p.batch <= 64) per = even_turns(p.batch, p.kv_heads, target, share, per, tiles, (blocks + 3) >> 2);
    d.heads = neighbours && per >= kNeighbourTurns ? kNeighbours : 1;
    const int waves = 4 / d.heads, unit = __builtin_amdgcn_readfirstlane(block / (p.kv_heads / d.heads));
    const bool whole = uncut(p, c);
    int units = 0, slots = 0, split = 0;
    bool found = false;
    for (int i = 0; i < p.batch; i += 64) {
        if (p.batch > 64) look(i);
        const int turns = (int)((unsigned)(blocks + waves - 1) / (unsigned)waves);
        // One column's parts are joined one after the other: of a long context they get longer with its root (one token over 10^6 entries of one
        // key head 127 us without, 119 with; over 16796 of two 16.3 and 16.2)
        const int least = even ? per : max(per, (int)__builtin_amdgcn_sqrtf(0.03f * turns));
        const int parts = whole || turns == 0 ? 1 : (int)((unsigned)(turns + least - 1) / (unsigned)least), mine = tiles * parts;
        const int upto = units + wave_prefix(mine), held = parts > 1 ? mine : 0, notes_held = parts > 1 ? tiles : 0;
        const int slots_upto = slots + wave_prefix(held), split_upto = split + wave_prefix(notes_held);
        const unsigned long long after = __ballot(upto > unit);
        if (after && !found) {
            const int at = __builtin_amdgcn_readfirstlane(__ffsll(after) - 1);
            const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, at); };
            d.b = i + at;
            d.parts = of(parts);
            const int in = unit - of(upto - mine);
            if ((unsigned)in >= (unsigned)of(mine)) return false;    // (sums past 32 bits: offsets that make no sense)
            d.tile = __builtin_amdgcn_readfirstlane(in / d.parts);      // (a division leaves it in a vector register)
            d.part = in - d.tile * d.parts;
            d.slot = of(slots_upto - held) + d.tile * d.parts;
            d.note = of(split_upto - notes_held) + d.tile;
            d.seq = Sequence{of(s.first), of(s.rows), of(s.cached), of(s.length), of(s.begin)};
            found = true;
            if (!notes) return true;
        }
        units = __builtin_amdgcn_readlane(upto, 63);
        slots = __builtin_amdgcn_readlane(slots_upto, 63);
        split = __builtin_amdgcn_readlane(split_upto, 63);
    }
    if (notes && threadIdx.x == 0) notes->count = split;
    return found;
}

}  // namespace ttf
