// Attention over a paged cache for chunks of many rows (bf16): the kernel that the matrix cores bound.
//
// The products and the softmax are those of k_attend (S^T = K Q^T, O^T = V^T P^T, the group's query heads of neighbouring rows
// side by side as columns), on 32x32x16 products.  A workgroup of four waves takes 128 columns, 32 a wave, and walks over blocks of 64
// keys, which it stages in LDS for all four: two buffers, filled by loads that go to LDS without passing through registers, one block ahead of
// the products.  Every lane of such a load names its own 16 bytes of memory, so pages may have any size, and lanes whose slot or
// entry does not exist read zeros.
//
// Layout in LDS: rows of 2 D bytes, the 16-byte pieces of row r swapped by XOR with a number made of r's low bits.  A product's
// left operand K is read a row a lane, 16 bytes each: sixteen neighbouring rows fall on sixteen different pieces.  Its left operand
// V^T is read four rows by 16 entries for 16 lanes, transposed by the LDS on the way: the four rows of each of two
// such groups, 64 bytes of each, fall on four different quarters of the 64 banks, twice each.
// A 32x32 product leaves lane (h, m) = (lane / 32, lane % 32) the keys 8a + 4h + b (a, b < 4) of column m; slot j of the next product's right operand
// is given key 16 s + 8 (j / 4) + 4 h + j % 4, so P stays in its lane.
#include "ttf_attend.h"

namespace ttf {
namespace {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(8))) short s16x8;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) char lds_char;

__device__ const uint4 kZeros = {0, 0, 0, 0};

constexpr int kWideColumns = 128, kWideKeys = 64;

// 16 bytes a lane from memory straight to LDS: lane l's to byte 16 l from `to` on.  Written out, because the compiler, which cannot tell the
// buffer being filled from the one being read, would wait for it before every read of LDS.  Whoever reads the bytes has waited for the loads of
// every wave before (wait_for_loads and a barrier).  No register is written.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"               // (m0 counts as reserved; the compiler puts nothing there that outlives this)
__device__ __forceinline__ void load_to_lds(unsigned long long from, unsigned to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ unsigned lds_offset(const char* p) { return (unsigned)(uintptr_t)(const lds_char*)p; }

// Whether either of two bf16 values is infinite or NaN; one of the two in fp32.
__device__ __forceinline__ bool not_finite(uint32_t w) { return ((w & 0x7f800000u) == 0x7f800000u) | ((w & 0x7f80u) == 0x7f80u); }
__device__ __forceinline__ float half_of(uint32_t w, int i) { return __builtin_bit_cast(float, i ? w & 0xffff0000u : w << 16); }

// Number that row r's 16-byte pieces are swapped by.
template <int DP>
__device__ __forceinline__ int swizzle(int r)
{
    if constexpr (DP == 64) return (r >> 1 & 1) << 2 | (r >> 2 & 3);    // 128-byte rows: two share the 64 banks
    return (r & 3) << 2 | (r >> 2 & 3);
}

// A wave's 32 columns over the entries from .. to - 1 again, key by key on the vector units.
template <int DP, typename Slot>
__device__ __forceinline__ void by_keys(int head_dim, const bf16_t* kc, const bf16_t* vc, const Slot& slot_of, int from, int to, int limit,
                                        int lower, float factor, const bf16x8 (&q)[DP / 16], float& top, float& sum, f32x16 (&o)[DP / 32])
{
    constexpr int NT = DP / 32, KS = DP / 16;
    const int h = threadIdx.x >> 5 & 1;
    top = -INFINITY;
    sum = 0.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
#pragma unroll 1
            for (int u = from; u < to; ++u) {
                const long long at = slot_of(u);
                if (at < 0) continue;
                float dot = 0.0f;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int e0 = s * 16 + h * 8;
                    if (e0 >= head_dim) continue;
                    const u32x4 x = __builtin_bit_cast(u32x4, q[s]), y = *reinterpret_cast<const u32x4*>(kc + at + e0);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        dot = __builtin_fmaf(half_of(x[e / 2], e % 2), half_of(y[e / 2], e % 2), dot);
                }
                dot += __shfl_xor(dot, 32, 64);
                const bool sees = (u < limit) & (u >= lower);
                const float score = sees ? dot * factor : -INFINITY, most = fmaxf(top, score);
                const float by = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - most);
                const float weight = __builtin_amdgcn_exp2f(score - (most == -INFINITY ? 0.0f : most));
                top = most;
                sum = sum * by + (h == 0 ? weight : 0.0f);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int a = 0; a < 4; ++a) {
                        const int e0 = 32 * t + 8 * a + 4 * h;
                        const uint2 y = *reinterpret_cast<const uint2*>(vc + at + (e0 < head_dim ? e0 : 0));
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const float v = half_of(b < 2 ? y.x : y.y, b % 2);
                            o[t][4 * a + b] = o[t][4 * a + b] * by + (sees ? weight * v : 0.0f);
                        }
                    }
            }
}

// A wave's 32 columns into the workspace (parts) or the outputs; h, row, qh, is: this lane's half, row, query head and whether it has one.
template <int DP>
__device__ __forceinline__ void finish_wide(const ttf_attention_params& p, const Deal& d, const Sequence& seq, int head, int columns, int col,
                                            int h, int row, long long qh, bool is, int target, float top, float sum, const f32x16 (&o)[DP / 32],
                                            float* ws_out, float2* ws_stat)
{
    constexpr int NT = DP / 32;
    sum += __shfl_xor(sum, 32, 64);
    if (!is) return;
    if (d.parts > 1) {
        const int at = (d.slot + d.part) * p.kv_heads + head;
        if ((unsigned)at >= 2u * target) return;             // (cannot be with offsets that do not decrease)
        const int part_row = at * columns + col;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<float4*>(ws_out + (size_t)part_row * DP + 32 * t + 8 * a + 4 * h) =
                    float4{o[t][4 * a], o[t][4 * a + 1], o[t][4 * a + 2], o[t][4 * a + 3]};
        if (h == 0) ws_stat[part_row] = float2{top, sum};
        return;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    bf16_t* to = (bf16_t*)p.out + (seq.first + row) * p.o_row + qh * p.o_head;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int e = 32 * t + 8 * a + 4 * h;
            if (e < p.head_dim)
                *reinterpret_cast<uint2*>(to + e) =
                    uint2{__builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[t][4 * a] * inv, o[t][4 * a + 1] * inv}, bf16x2)),
                          __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{o[t][4 * a + 2] * inv, o[t][4 * a + 3] * inv}, bf16x2))};
        }
    if (p.lse && h == 0) p.lse[(long long)(seq.first + row) * p.heads + qh] = sum == 0.0f ? -INFINITY : top * kLn2 + logf(sum);
}

template <int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attend_wide(ttf_attention_params p, ttf_kv_cache c, int target, float* ws_out,
                                                                        float2* ws_stat, JoinNotes* notes)
{
    constexpr int PIECES = DP / 8, ROW = 2 * DP, HALF = kWideKeys * ROW;       // 16-byte pieces of a row; bytes of a row, of K's block
    constexpr int CALLS = HALF / 4096, ROWS = 1024 / ROW;                      // loads of 1 KiB a wave makes for K, and for V; rows of one
    constexpr int NT = DP / 32, KS = DP / 16;
    __shared__ __attribute__((aligned(1024))) char buffer[4 * HALF];           // two of K and V
    __shared__ int tainted;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, m = lane & 31;
    const int head = blockIdx.x % p.kv_heads, group = p.heads / p.kv_heads;
    Deal d;
    if (!deal_out(p, c, kWideColumns, kWideKeys / 4, false, true, target, blockIdx.x, blockIdx.x == 0 ? notes : nullptr, d)) return;
    const Sequence& seq = d.seq;
    const int pairs = seq.rows * group;
    // later rows see more keys: they go first
    const int tile = tiles_of(seq.rows, group, kWideColumns) - 1 - d.tile, col0 = tile * kWideColumns;
    d.slot += (tile - d.tile) * d.parts;
    if (d.parts > 1 && d.part == 0 && head == 0 && threadIdx.x == 0 && d.note < target) notes->note[d.note] = JoinNote{d.b, tile, d.parts, d.slot};

    const auto limit_of = [&](int row) { return p.causal ? (int)min((long long)seq.cached + row + 1, (long long)seq.length) : seq.length; };
    const auto lower_of = [&](int row) {
        return p.window > 0 ? (int)max(0ll, min((long long)seq.cached + row + 1 - p.window, 0x7fffffffll)) : 0;
    };
    // what all and what any of the workgroup's and of this wave's rows see
    const int row_a = col0 / group, row_z = min(col0 + kWideColumns - 1, pairs - 1) / group;
    const int begin0 = lower_of(row_a) & ~31, end = limit_of(row_z);
    const int all = max(0, (int)(((long long)end - begin0 + kWideKeys - 1) / kWideKeys));
    const int step0 = (int)((long long)all * d.part / d.parts), blocks = (int)((long long)all * (d.part + 1) / d.parts) - step0;
    const int begin = begin0 + step0 * kWideKeys, stop = min(seq.length, begin + blocks * kWideKeys);

    // Where the loads come from.  Lane l keeps the page number of page `window0` + l, read again when the blocks have passed it (a load
    // whose result is needed in every block would be waited for together with all the younger ones, that go to LDS).  The block whose
    // loads come next starts at entry `next_in` of page `next_page`.
    const bf16_t *kc = (const bf16_t*)c.k + head * c.head_stride, *vc = (const bf16_t*)c.v + head * c.head_stride;
    const int32_t* table = c.page_table + d.b * c.table_stride;
    int next_page = (unsigned)begin / (unsigned)c.page_size, next_in = begin - next_page * c.page_size, next_base = begin;
    int window0 = 0, window = -1;
    bool holes = false;                                      // pages of the window that are not there
    const auto open = [&](int page) {
        window0 = page;
        window = page_begins(page, lane, c.page_size, stop) ? table[page + lane] : -1;
    };
    const auto opened = [&] {
        asm volatile("" : "+v"(window));                     // (waited for here)
        holes = __ballot((window < 0 || window >= c.pages) && page_begins(window0, lane, c.page_size, stop)) != 0;
    };
    open(next_page);

    // this lane's column
    const int pair = col0 + wave * 32 + m, row = pair / group;
    const bool is = pair < pairs;
    const int limit = is ? limit_of(row) : 0x7fffffff, lower = is ? lower_of(row) : 0;
    const long long qh = (long long)head * group + pair % group;
    u32x4 q_bits[KS];                                        // (on their way while the first keys and values are)
    {
        const bf16_t* from = (const bf16_t*)p.q + (seq.first + (is ? row : 0)) * p.q_row + qh * p.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int at = s * 16 + h * 8;
            q_bits[s] = *reinterpret_cast<const u32x4*>(from + (at < p.head_dim ? at : 0));
        }
    }
    const int wave0 = col0 + wave * 32, wave_row_z = min(wave0 + 31, pairs - 1) / group;
    const bool wave_is = wave0 < pairs;
    const int all_limit = limit_of(wave0 / group), any_limit = wave_is ? limit_of(wave_row_z) : 0;
    const int all_lower = lower_of(wave_row_z), any_lower = lower_of(wave0 / group);
    const int block_limit = limit_of(row_a), block_lower = lower_of(row_z);    // what all rows of the workgroup see

    const auto slot_of = [&](int u) -> long long {           // element offset of entry u's slot, -1 where there is none
        if (u >= seq.length) return -1;
        const unsigned at = (unsigned)u / (unsigned)c.page_size;
        const int page = table[at];
        return page >= 0 && page < c.pages ? page * c.page_stride + (u - (int)at * c.page_size) * c.slot_stride : -1;
    };
    // Loads of a block, call i of this wave the KiB 4 i + wave: ROWS neighbouring rows.  Where these lie in one page (pages of whole
    // ROWS slots), are all there and the head fills the row, their address is one for the wave and the lanes' part of it a constant.
    unsigned lane_bytes[CALLS];
    const bool plain = c.page_size % ROWS == 0 && p.head_dim == DP && c.slot_stride < (1ll << 24);
#pragma unroll
    for (int i = 0; i < CALLS; ++i) {
        const int piece = (4 * i + wave) * 64 + lane, r = piece / PIECES;
        lane_bytes[i] = (unsigned)(r % ROWS) * (unsigned)c.slot_stride * 2 + (piece % PIECES ^ swizzle<DP>(r)) * 16;
    }
    // The next block's sources: a lane's addresses in K, and which lanes read keys and values (the others: zeros).
    unsigned long long source[CALLS], reads[CALLS];
    const long long k_to_v = (const char*)vc - (const char*)kc;
    const auto aim = [&] {
        const int last = next_in + kWideKeys - 1;
        int pages_on = 0, in_last = last;                    // pages that the block reaches beyond its first
        while (in_last >= c.page_size) {
            in_last -= c.page_size;
            ++pages_on;
        }
        if (next_page + pages_on >= window0 + 64) {
            open(next_page);
            opened();
        }
        if (plain && next_base + kWideKeys <= stop && !holes) {
            int page = next_page, in = next_in + ROWS * wave;
#pragma unroll
            for (int i = 0; i < CALLS; ++i) {
                while (in >= c.page_size) {
                    in -= c.page_size;
                    ++page;
                }
                source[i] = (unsigned long long)kc + 2 * (__builtin_amdgcn_readlane(window, page - window0) * c.page_stride + in * c.slot_stride) +
                            lane_bytes[i];
                reads[i] = ~0ull;
                in += 4 * ROWS;
            }
        } else {
            const long long slot = next_base + lane < stop ? slot_of(next_base + lane) : -1;
#pragma unroll
            for (int i = 0; i < CALLS; ++i) {
                const int piece = (4 * i + wave) * 64 + lane, r = piece / PIECES, e = (piece % PIECES ^ swizzle<DP>(r)) * 8;
                const long long at = __shfl(slot, r, 64);
                const bool there = at >= 0 && e < p.head_dim;
                source[i] = there ? (unsigned long long)(kc + at + e) : (unsigned long long)&kZeros;
                reads[i] = __ballot(there);
            }
        }
        next_base += kWideKeys;
        next_page += pages_on;
        next_in = in_last + 1;
        if (next_in == c.page_size) {
            next_in = 0;
            ++next_page;
        }
    };

    // load n of the 2 CALLS of a block: of K, then of V
    const auto load = [&](int n, int to) {
        const int i = n % CALLS;
        unsigned long long from = source[i];
        if (n >= CALLS) from = reads[i] >> lane & 1 ? from + k_to_v : from;
        load_to_lds(from, lds_offset(buffer) + to + n / CALLS * HALF + (4 * i + wave) * 1024);
    };

    const float factor = p.scale == 0.0f ? 1.0f : fabsf(p.scale) * kLog2e;
    float top = -INFINITY, sum = 0.0f;
    f32x16 o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;

    // A lane's places in a block.  The pieces' swap is an XOR of bits inside a row, so the place of another piece is an XOR with a
    // constant, another row's an offset.  They are worked out anew every block (`hide`): kept, they would take 16 registers.
    const int vr = (lane & 15) >> 2, low = (lane >> 4 & 1) * 2 + ((lane & 3) >> 1);
    const int v_place = HALF + (4 * h + vr) * ROW + (DP == 64 ? vr >> 1 : vr) * 64 + (low ^ h) * 16 + (lane & 1) * 8;
    const int k_place = m * ROW + (h ^ swizzle<DP>(m)) * 16;
    const auto hide = [](int at) {
        asm volatile("" : "+v"(at));
        return at;
    };

    bf16x8 q[KS];
    // Block at place `at` of the buffer.  The next block's loads are spread over its first products: issued all at once they hold
    // up the waves until the last is taken (2000 rows over 31k keys 1086 us, spread out 1030; 8 clips of 3600 rows 396 and 379).
    // Of a SIMD's two waves the one that multiplies goes first, the other takes its weights in between (the same clips 397 us without, 382 with,
    // 394 the other way round; with one wave a SIMD it only costs).
    const auto first = [&](bool it) {
        if constexpr (DP == 256) return;
        if (it) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
    };
    // Operands are read from LDS four products with K, three with V ahead (the same clips 398 us in the compiler's own order, 387 so; 16 heads of 256
    // entries on 4 547 and 512).
    const auto work = [&](int at, int to, int base, bool gaps) {
        const int kp = hide(k_place + at), vp = hide(v_place + at);
        first(true);
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
        const auto k_frag = [&](int n) { return *reinterpret_cast<const bf16x8*>(buffer + (kp ^ (n / 2 * 32)) + 32 * (n % 2) * ROW); };
        constexpr int KA = 4, VA = 3;
        bf16x8 k[KA];
#pragma unroll
        for (int n = 0; n < KA; ++n) k[n] = k_frag(n);
#pragma unroll
        for (int n = 0; n < 2 * KS; ++n) {
            __builtin_amdgcn_sched_barrier(0);
            s[n % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[n % KA], q[n / 2], s[n % 2], 0, 0, 0);
            if (n + KA < 2 * KS) k[n % KA] = k_frag(n + KA);
            if (n % 2 == 1) load(n / 2, to);
        }
        first(false);
        static_assert(KS == 2 * CALLS, "a load for every pair of products");
        if (!(base + kWideKeys <= all_limit && base >= all_lower && !gaps)) {
            // bit k: this column sees the block's key k + 4 h
            const unsigned long long gone = gaps ? __ballot(slot_of(base + lane) < 0) : 0ull;
            const int from = min(max(lower - base, 0), 64), to = min(max(limit - base, 0), 64);
            const unsigned long long below = to == 64 ? ~0ull : (1ull << to) - 1, above = from == 64 ? 0ull : ~0ull << from;
            const unsigned long long sees = (below & above & ~gone) >> (4 * h);
            const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][r] = half[t] >> (8 * (r / 4) + r % 4) & 1 ? s[t][r] : -INFINITY;
        }
        // The weights against the maximum so far; where they get large, or there is none, against the block's own over again.
        // Each is rounded to one bf16 value for its product, half a step of 2^-8 of it; their sum is not.  A second value for what the first leaves
        // would make the output as good as rounded once (8 clips of up to 3600 rows: rms error 1.88e-3 with one, 1.68e-3 with two), but the
        // matrix cores bound this kernel: 387 -> 495 us there, 4 x 512 rows over 8192 entries 162 -> 205 us.
        bf16x8 w[4];
        float added;
        bool last = false;
        for (;;) {
            const float from = top == -INFINITY ? 0.0f : top;
            float part[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                u32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 8 * (i % 2) + 2 * e;
                    const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][r], factor, -from));
                    const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][r + 1], factor, -from));
                    part[0] += a;
                    part[1] += b;
                    y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
                }
                w[i] = __builtin_bit_cast(bf16x8, y);
            }
            added = part[0] + part[1];
            if (last || !__ballot(!(added <= 256.0f) | (top == -INFINITY))) break;
            float most = s[0][0];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[t][r]);
            most = fmaxf(most, __shfl_xor(most, 32, 64)) * factor;
            most = fmaxf(top, most);
            const float by = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - most);
            top = most;
            sum *= by;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][r] *= by;
            last = true;
        }
        sum += added;
        first(true);
        const auto v_frag = [&](int n) {
            s16x4 part[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
                part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s16x4*)((lds_char*)buffer + (vp ^ (n % NT * 64 + j * 32)) + (16 * (n / NT) + 8 * j) * ROW));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        };
        bf16x8 v[VA];
#pragma unroll
        for (int n = 0; n < VA; ++n) v[n] = v_frag(n);
#pragma unroll
        for (int n = 0; n < 4 * NT; ++n) {
            __builtin_amdgcn_sched_barrier(0);
            o[n % NT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[n % VA], w[n / NT], o[n % NT], 0, 0, 0);
            if (n + VA < 4 * NT) v[n % VA] = v_frag(n + VA);
        }
        first(false);
    };
    // notes an infinite or NaN value in a block that not all rows see whole
    const auto look = [&](const char* block) {
        bool odd = false;
#pragma unroll
        for (int i = 0; i < HALF / 4096; ++i) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(block + HALF + i * 4096 + threadIdx.x * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= not_finite(v[e]);
        }
        if (odd) tainted = 1;
    };
    if (threadIdx.x == 0) tainted = 0;                       // (before the first block's barrier)

    // two buffers: block j + 1 is on its way while block j is worked on; one barrier a block
    if (blocks > 0) {
        opened();
        aim();
        bool gaps = holes;
#pragma unroll
        for (int n = 0; n < 2 * CALLS; ++n) load(n, 0);
        const uint32_t flip = p.scale < 0.0f ? 0x80008000u : 0u, keep = p.scale == 0.0f ? 0u : ~0u;
#pragma unroll
        for (int s = 0; s < KS; ++s)
            q[s] = __builtin_bit_cast(bf16x8, is && s * 16 + h * 8 < p.head_dim ? (q_bits[s] ^ flip) & keep : u32x4{0, 0, 0, 0});
#pragma unroll 1
        for (int j = 0; j < blocks; ++j) {
            const int at = j % 2 * 2 * HALF, base = begin + j * kWideKeys;
            wait_for_loads();
            __syncthreads();                                 // block j is there, and nobody reads the other buffer any more
            const bool now = gaps;
            aim();                                           // (past the last block: zeros)
            gaps = holes;
            if (!(base + kWideKeys <= block_limit && base >= block_lower)) look(buffer + at);
            if (base < any_limit && base + kWideKeys > any_lower) {
                work(at, 2 * HALF - at, base, now);
            } else {
#pragma unroll
                for (int n = 0; n < 2 * CALLS; ++n) load(n, 2 * HALF - at);
            }
        }
        wait_for_loads();                                 // (no load to LDS outlives the wave)
    }

    __syncthreads();
    // An infinite or NaN value that some rows see and others do not: 0 times it is no 0.  Rare, and done over again key by key
    // on the vector units, which leave out what a column does not see.
    if (__builtin_amdgcn_readfirstlane(tainted)) {
        asm volatile("" ::: "memory");                       // (keeps this path out of the common one)
        const int from = max(begin, any_lower), to = min(begin + blocks * kWideKeys, any_limit);
        by_keys<DP>(p.head_dim, kc, vc, slot_of, from, to, limit, lower, factor, q, top, sum, o);
    }
    finish_wide<DP>(p, d, seq, head, kWideColumns, wave * 32 + m, h, row, qh, is, target, top, sum, o, ws_out, ws_stat);
}

}  // namespace

hipError_t launch_attention_wide(const ttf_attention_params& p, const ttf_kv_cache& c, int width, int target, unsigned grid, float* ws_out,
                                 float2* ws_stat, JoinNotes* notes, hipStream_t s)
{
    const auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, s>>>(p, c, target, ws_out, ws_stat, notes);
        return hipGetLastError();
    };
    return width == 64 ? go(k_attend_wide<64>) : width == 128 ? go(k_attend_wide<128>) : go(k_attend_wide<256>);
}

}  // namespace ttf
