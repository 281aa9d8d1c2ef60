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

template <int DP>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void k_attend_wide(ttf_attention_params p, ttf_kv_cache c, int target, float* ws_out,
                                                                        float2* ws_stat, JoinNotes* notes)
{
    constexpr int PIECES = DP / 8, ROW = 2 * DP, HALF = kWideKeys * ROW;       // 16-byte pieces of a row; bytes of a row, of K's block
    constexpr int CALLS = PIECES / 4;                                          // loads of 1 KiB a wave makes for K, and for V
    constexpr int NT = DP / 32, KS = DP / 16;
    __shared__ __attribute__((aligned(1024))) char buf0[2 * HALF], buf1[2 * HALF];
    __shared__ int tainted;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, m = lane & 31;
    const int head = blockIdx.x % p.kv_heads, group = p.heads / p.kv_heads;
    Deal d;
    if (!deal_out(p, c, kWideColumns, kWideKeys / 4, false, target, blockIdx.x, blockIdx.x == 0 ? notes : nullptr, d)) return;
    const Sequence seq = sequence_of(p, c, d.b);
    const int pairs = seq.rows * group;
    // later rows see more keys: they go first
    const int tile = tiles_of(seq.rows, group, kWideColumns) - 1 - d.tile, col0 = tile * kWideColumns;
    d.slot += (tile - d.tile) * d.parts;
    if (d.parts > 1 && d.part == 0 && head == 0 && threadIdx.x == 0 && d.note < target) notes->note[d.note] = JoinNote{d.b, tile, d.parts, d.slot};

    const auto limit_of = [&](int row) { return p.causal ? (int)min((long long)seq.cached + row + 1, (long long)seq.length) : seq.length; };
    const auto lower_of = [&](int row) {
        return p.window > 0 ? (int)max(0ll, min((long long)seq.cached + row + 1 - p.window, 0x7fffffffll)) : 0;
    };
    // this lane's column
    const int pair = col0 + wave * 32 + m, row = pair / group;
    const bool is = pair < pairs;
    const int limit = is ? limit_of(row) : 0x7fffffff, lower = is ? lower_of(row) : 0;
    const long long qh = (long long)head * group + pair % group;
    const float factor = p.scale == 0.0f ? 1.0f : fabsf(p.scale) * kLog2e;
    bf16x8 q[KS];
    {
        const bf16_t* from = (const bf16_t*)p.q + (seq.first + row) * p.q_row + qh * p.q_head;
        const uint32_t flip = p.scale < 0.0f ? 0x80008000u : 0u, keep = p.scale == 0.0f ? 0u : ~0u;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int at = s * 16 + h * 8;
            u32x4 y = {0, 0, 0, 0};
            if (is && at < p.head_dim) y = *reinterpret_cast<const u32x4*>(from + at);
            q[s] = __builtin_bit_cast(bf16x8, (y ^ flip) & keep);
        }
    }
    // what all and what any of the workgroup's and of this wave's rows see
    const int row_a = col0 / group, row_z = min(col0 + kWideColumns - 1, pairs - 1) / group;
    const int begin = lower_of(row_a) & ~31, end = limit_of(row_z);
    const int steps = max(0, (int)(((long long)end - begin + kWideKeys - 1) / kWideKeys));
    const int step0 = (int)((long long)steps * d.part / d.parts), step1 = (int)((long long)steps * (d.part + 1) / d.parts);
    const int wave0 = col0 + wave * 32, wave_row_z = min(wave0 + 31, pairs - 1) / group;
    const bool wave_is = wave0 < pairs;
    const int block_limit = limit_of(row_a), block_lower = lower_of(row_z);    // what all rows of the workgroup see
    const int all_limit = limit_of(wave0 / group), any_limit = wave_is ? limit_of(wave_row_z) : 0;
    const int all_lower = lower_of(wave_row_z), any_lower = lower_of(wave0 / group);

    // staging: call i of this wave fills the KiB (4 i + wave) of a block
    const bf16_t *kc = (const bf16_t*)c.k + head * c.head_stride, *vc = (const bf16_t*)c.v + head * c.head_stride;
    const int32_t* table = c.page_table + d.b * c.table_stride;
    const auto slot_of = [&](int u) -> long long {           // element offset of entry u's slot, -1 where there is none
        if (u >= seq.length) return -1;
        const unsigned at = (unsigned)u / (unsigned)c.page_size;
        const int page = table[at];
        return page >= 0 && page < c.pages ? page * c.page_stride + (u - (int)at * c.page_size) * c.slot_stride : -1;
    };
    const auto stage = [&](char* to, long long slot) {       // lane l: slot of key l of the block
#pragma unroll
        for (int i = 0; i < CALLS; ++i) {
            const int piece = (4 * i + wave) * 64 + lane, r = piece / PIECES, e = (piece % PIECES ^ swizzle<DP>(r)) * 8;
            const long long at = __shfl(slot, r, 64);
            const bool there = at >= 0 && e < p.head_dim;
            const void* kf = there ? (const void*)(kc + at + e) : (const void*)&kZeros;
            const void* vf = there ? (const void*)(vc + at + e) : (const void*)&kZeros;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)kf,
                                             (__attribute__((address_space(3))) void*)(to + (4 * i + wave) * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)vf,
                                             (__attribute__((address_space(3))) void*)(to + HALF + (4 * i + wave) * 1024), 16, 0, 0);
        }
    };

    float top = -INFINITY, sum = 0.0f;
    f32x16 o[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;

    // V^T of 16 keys by 32 entries: product t, keys 16 s ..
    const int vr = (lane & 15) >> 2, vc16 = lane >> 4 & 1, low = vc16 * 2 + ((lane & 3) >> 1);
    const auto v_frag = [&](const char* block, int s, int t) -> bf16x8 {
        s16x4 part[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = 16 * s + 8 * j + 4 * h + vr;
            const int at = HALF + r * ROW + (((t * 4 + low) ^ swizzle<DP>(r)) << 4) + (lane & 1) * 8;
            part[j] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((lds_char*)block + at));
        }
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };

    const auto work = [&](const char* block, int base, unsigned long long gone) {
        if (base >= any_limit || base + kWideKeys <= any_lower) return;
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int at = (32 * t + m) * ROW + (((2 * i + h) ^ swizzle<DP>(m)) << 4);
                const bf16x8 k = *reinterpret_cast<const bf16x8*>(block + at);
                s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[i], s[t], 0, 0, 0);
            }
        const bool full = base + kWideKeys <= all_limit && base >= all_lower && gone == 0;
        if (!full) {
            // bit k: this column sees the block's key k + 4 h
            const int from = min(max(lower - base, 0), 64), to = min(max(limit - base, 0), 64);
            const unsigned long long below = to == 64 ? ~0ull : (1ull << to) - 1, above = from == 64 ? 0ull : ~0ull << from;
            const unsigned long long sees = (below & above & ~gone) >> (4 * h);
            const uint32_t half[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][r] = half[t] >> (8 * (r / 4) + r % 4) & 1 ? s[t][r] : -INFINITY;
        }
        float most = s[0][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[t][r]);
        most *= factor;
        if (__ballot(most > top + 8.0f)) {                   // (the maximum moves only where a block beats it by more than 8)
            most = fmaxf(top, fmaxf(most, __shfl_xor(most, 32, 64)));
            const float by = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - most);
            top = most;
            sum *= by;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[t][r] *= by;
        }
        const float from = top == -INFINITY ? 0.0f : top;
        bf16x8 w[4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 8 * j + 2 * e;
                    const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r], factor, -from));
                    const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r + 1], factor, -from));
                    sum += a + b;
                    y[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
                }
                w[2 * t + j] = __builtin_bit_cast(bf16x8, y);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t)
                o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag(block, i, t), w[i], o[t], 0, 0, 0);
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

    // two buffers: block n+1 is on its way while block n is worked on; one barrier a block
    if (step0 < step1) {
        long long slot = slot_of(begin + step0 * kWideKeys + lane);
        unsigned long long gone = __ballot(slot < 0), gone_next = 0;
        stage(buf0, slot);
        long long ahead = step0 + 1 < step1 ? slot_of(begin + (step0 + 1) * kWideKeys + lane) : -1;
        const auto turn = [&](int step, char* now, char* next) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();                                 // block `step` is there, and nobody reads the other buffer any more
            if (step + 1 < step1) {
                gone_next = __ballot(ahead < 0);
                stage(next, ahead);
                if (step + 2 < step1) ahead = slot_of(begin + (step + 2) * kWideKeys + lane);
            }
            const int base = begin + step * kWideKeys;
            if (!(base + kWideKeys <= block_limit && base >= block_lower)) look(now);
            work(now, base, gone);
            gone = gone_next;
        };
#pragma unroll 1
        for (int step = step0; step < step1; step += 2) {
            turn(step, buf0, buf1);
            if (step + 1 < step1) turn(step + 1, buf1, buf0);
        }
    }

    __syncthreads();
    // An infinite or NaN value that some rows see and others do not: 0 times it is no 0.  Rare, and done over again key by key
    // on the vector units, which leave out what a column does not see.
    if (__builtin_amdgcn_readfirstlane(tainted)) {
        asm volatile("" ::: "memory");                       // (keeps this path out of the common one)
        top = -INFINITY;
        sum = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t][r] = 0.0f;
        const int from = max(begin + step0 * kWideKeys, any_lower), to = min(begin + step1 * kWideKeys, any_limit);
#pragma unroll 1
        for (int u = from; u < to; ++u) {
            const long long at = slot_of(u);
            if (at < 0) continue;
            float dot = 0.0f;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int e0 = s * 16 + h * 8;
                if (e0 >= p.head_dim) continue;
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
                    const uint2 y = *reinterpret_cast<const uint2*>(vc + at + (e0 < p.head_dim ? e0 : 0));
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const float v = half_of(b < 2 ? y.x : y.y, b % 2);
                        o[t][4 * a + b] = o[t][4 * a + b] * by + (weight == 0.0f ? 0.0f : weight * v);
                    }
                }
        }
    }

    sum += __shfl_xor(sum, 32, 64);
    if (!is) return;
    if (d.parts > 1) {
        const int at = (d.slot + d.part) * p.kv_heads + head;
        if ((unsigned)at >= 2u * target) return;             // (cannot be with offsets that do not decrease)
        const int part_row = at * kWideColumns + wave * 32 + m;
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

}  // namespace

hipError_t launch_attention_wide(const ttf_attention_params& p, const ttf_kv_cache& c, int width, int target, unsigned grid, float* ws_out,
                                 float2* ws_stat, JoinNotes* notes, hipStream_t s)
{
    if (width == 64) k_attend_wide<64><<<grid, 256, 0, s>>>(p, c, target, ws_out, ws_stat, notes);
    else if (width == 128) k_attend_wide<128><<<grid, 256, 0, s>>>(p, c, target, ws_out, ws_stat, notes);
    else k_attend_wide<256><<<grid, 256, 0, s>>>(p, c, target, ws_out, ws_stat, notes);
    return hipGetLastError();
}

}  // namespace ttf
