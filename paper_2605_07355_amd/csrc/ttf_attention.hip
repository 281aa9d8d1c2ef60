// Attention of a chunk of new rows, or of single tokens, over a paged cache (ttf_paged_attention): the kernel for few
// rows, the join of parts, and the choice of kernel.
//
// Online softmax over blocks of keys: with s_u = scale log2(e) <q, k_u>, running maximum m and p_u = 2^(s_u - m),
// l = sum p_u and o = sum p_u v_u are carried along and both multiplied by 2^(m - m') where the maximum moves to m'.  m moves
// only where a block beats it by more than 8: p stays below 2^8, sums in fp32 lose nothing by that, and most blocks need neither
// the maximum over their lanes nor the product.
//
// Layout: the group's query heads of up to `columns` rows stand side by side as the columns of S^T = K Q^T and O^T = V^T P^T.
// A 16x16 product leaves lane (g, m) = (lane / 16, lane % 16) the keys 4g .. 4g+3 of column m.  That is what the second product wants of
// its right operand, if slot j of lane group g stands for key 16 (j / 4) + 4 g + j % 4: P goes from one product into the next without
// leaving its lane, and so do m and l.  The left operand V^T wants eight such keys of one entry d.  A lane loads NI = D/16
// neighbouring entries of its keys, 16 lanes whole rows of 2 D bytes, and turns its own 8 x NI values round with byte
// permutes; product i then holds the entries d = NI c + i, c = 0..15.  So neither K nor V goes through LDS.
//
// Few rows are bound by the bytes of the cache: 16 KiB of K and V a wave in flight while the block before is worked on.
#include <algorithm>
#include <type_traits>

#include "ttf_attend.h"

namespace ttf {

hipError_t launch_attention_wide(const ttf_attention_params& p, const ttf_kv_cache& c, int width, int target, unsigned grid, float* ws_out,
                                 float2* ws_stat, JoinNotes* notes, hipStream_t s);

namespace {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Whether a 32-bit word holds an infinite or NaN value (one fp32, or either of two bf16).
template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return (w & 0x7f800000u) == 0x7f800000u;
    return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
}

template <typename T> constexpr int kBlockTiles = sizeof(T) == 2 ? 2 : 1;    // 16-key tiles a wave works on at once

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
// Four values to memory in one access, rounded to T.
__device__ __forceinline__ void store4(float* to, const float* v) { *reinterpret_cast<float4*>(to) = float4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void store4(bf16_t* to, const float* v)
{
    *reinterpret_cast<uint2*>(to) = uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// The factor 2^(m - M) of a share of a row in the join: 0 where the share saw nothing, and is left out; above 0 otherwise, also where the
// power underflows, so that an infinite or NaN value in it stays.
__device__ __forceinline__ float share_of(float m, float most)
{
    return m == -INFINITY ? 0.0f : fmaxf(__builtin_amdgcn_exp2f(m - most), 0x1p-126f);
}

// Keys and values are read once a call as a rule: non-temporal (64 tokens over 32000 entries 834 us without, 768 with; a window of 8192 over 12
// sequences 37 and 39).
template <typename V>
__device__ __forceinline__ V load_once(const char* p) { return __builtin_nontemporal_load(reinterpret_cast<const V*>(p)); }

// A workgroup of four waves works on one part of one tile.  Either its waves take turns with the blocks of 16 or 32 keys of one
// key head, and their (m, l, O) are joined in LDS at the end, or each has a key head to itself (see Deal).
//   DP     head dimension rounded up to 64, 128 or 256;  NM  column tiles of 16;  WAVES  a SIMD has registers for
//   WHOLE  pages hold whole 16-key tiles: a tile's address is one for all its keys, and only a lane's place in it goes by vector
//          registers.  Otherwise every key's page is looked up.
//   CUT    the head is shorter than DP: lanes past its end read its start, and take 0
template <typename T, int DP, int NM, bool WHOLE, bool CUT, int WAVES>
__global__ __launch_bounds__(256, WAVES) void k_attend(ttf_attention_params p, ttf_kv_cache c, int columns, bool neighbours,
                                                       int target, float* ws_out, float2* ws_stat, JoinNotes* notes)
{
    constexpr int E = sizeof(T), TILES = kBlockTiles<T>, KB = 16 * TILES;
    constexpr int KS = DP * E / 64;                          // 16-byte pieces of K a lane holds per tile
    constexpr int NI = DP / 16, VW = NI * E / 4;             // entries of V, in 32-bit words, a lane holds per key
    constexpr int PAD = DP + 4;
    __shared__ __attribute__((aligned(16))) float lds[4 * 16 * PAD];
    __shared__ float2 stat[4][16 * NM];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, m = lane & 15;
    const int group = p.heads / p.kv_heads;
    Deal d;
    if (!deal_out(p, c, columns, KB, neighbours, false, target, blockIdx.x, blockIdx.x == 0 ? notes : nullptr, d)) return;
    const int first_head = blockIdx.x % (p.kv_heads / d.heads) * d.heads, waves = 4 / d.heads;    // `waves` share a head
    const int head = first_head + (d.heads > 1 ? wave : 0), turn = d.heads > 1 ? 0 : wave;
    const Sequence& seq = d.seq;
    const int col0 = d.tile * columns, pairs = min(seq.rows * group, col0 + columns);   // (pairs of the sequence up to this tile's end)

    // the columns of this lane, and what they see: entries lower <= u < limit
    int limit[NM], lower[NM];
    u32x4 q[NM][KS];
    const auto limit_of = [&](int row) { return p.causal ? (int)min((long long)seq.cached + row + 1, (long long)seq.length) : seq.length; };
    const auto lower_of = [&](int row) {
        return p.window > 0 ? (int)max(0ll, min((long long)seq.cached + row + 1 - p.window, 0x7fffffffll)) : 0;
    };
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        const int pair = col0 + 16 * n + m, row = pair / group;
        const bool is = pair < pairs;
        limit[n] = is ? limit_of(row) : 0x7fffffff;
        lower[n] = is ? lower_of(row) : 0;
        const T* from = (const T*)p.q + (seq.first + row) * p.q_row + ((long long)head * group + pair % group) * p.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int at = (s * 64 + g * 16) / E;
            q[n][s] = is && (!CUT || at < p.head_dim) ? *reinterpret_cast<const u32x4*>(from + at) : u32x4{0, 0, 0, 0};
        }
    }
    // what all and what any of the tile's rows see (rows in ascending order: so are their limits)
    const int row_a = col0 / group, row_z = (pairs - 1) / group;
    const int all_limit = limit_of(row_a), all_lower = lower_of(row_z), any_limit = limit_of(row_z);
    const int begin = lower_of(row_a) & ~31;
    const int steps = max(0, (int)(((long long)any_limit - begin + waves * KB - 1) / (waves * KB)));
    const int step0 = (int)((long long)steps * d.part / d.parts), step1 = (int)((long long)steps * (d.part + 1) / d.parts);
    const auto base_of = [&](int step) { return begin + (step * waves + turn) * KB; };

    float top[NM], sum[NM];                                  // m and this lane's share of l
    f32x4 o[NM][NI];
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < NI; ++i) o[n][i] = f32x4{0, 0, 0, 0};
    }

    // element offset of entry u's slot, -1 where there is none
    const int32_t* table = c.page_table + d.b * c.table_stride;
    const auto slot_of = [&](int u) -> long long {
        if (u >= seq.length) return -1;                      // (so u / page_size < table_width)
        const unsigned at = (unsigned)u / (unsigned)c.page_size;
        const int page = table[at];
        return page >= 0 && page < c.pages ? page * c.page_stride + (u - (int)at * c.page_size) * c.slot_stride : -1;
    };

    // Where the keys of a step lie.  WHOLE: lane j holds the offset of tile j % TILES of the j / TILES-th step from the last
    // refill on, every 64 / TILES steps, and `tile` those of the step at hand, in scalar registers.  Otherwise lane j holds key j % KB's.
    struct Place { long long tile[WHOLE ? TILES : 1]; };
    long long mine = -1;
    const auto locate = [&](int step) -> Place {
        Place x;
        if constexpr (WHOLE) {
            const int j = (step - step0) % (64 / TILES);
            if (j == 0) mine = slot_of(base_of(step + lane / TILES) + lane % TILES * 16);
#pragma unroll
            for (int t = 0; t < TILES; ++t)
                x.tile[t] = (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(mine >> 32), j * TILES + t) << 32 |
                                        (unsigned)__builtin_amdgcn_readlane((int)mine, j * TILES + t));
        } else {
            x.tile[0] = slot_of(base_of(step) + lane % KB);
        }
        return x;
    };
    const char *kc = (const char*)((const T*)c.k + head * c.head_stride), *vc = (const char*)((const T*)c.v + head * c.head_stride);
    const unsigned slot_bytes = (unsigned)c.slot_stride * E;
    const int piece = CUT && DP == 64 ? first_piece(g, p.head_dim, E) : 16 * g;    // (longer ones have a first piece for every group)
    const unsigned k_at = m * slot_bytes + piece, v_at = 4 * g * slot_bytes + (!CUT || m * NI < p.head_dim ? m * NI * E : 0);

    u32x4 k[TILES][KS];
    uint32_t v[4 * TILES][VW];
    const auto fetch_k = [&](const Place& x) {
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const char* from;
            if constexpr (WHOLE) from = kc + max(0ll, x.tile[t]) * E + k_at;
            else from = kc + max(0ll, __shfl(x.tile[0], 16 * t + m, 64)) * E + piece;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                k[t][s] = load_once<u32x4>(from + (CUT ? next_piece(s, g, p.head_dim, E) : s * 64));
                if (CUT && !has_piece(s, g, p.head_dim, E)) k[t][s] = u32x4{0, 0, 0, 0};
            }
        }
    };
    const auto fetch_v = [&](const Place& x) {
#pragma unroll
        for (int j = 0; j < 4 * TILES; ++j) {
            const char* from;
            if constexpr (WHOLE) from = vc + max(0ll, x.tile[j / 4]) * E + (j % 4) * slot_bytes + v_at;
            else from = vc + max(0ll, __shfl(x.tile[0], 16 * (j / 4) + 4 * g + j % 4, 64)) * E + (!CUT || m * NI < p.head_dim ? m * NI * E : 0);
            constexpr int W = VW < 4 ? VW : 4;               // words a load brings
#pragma unroll
            for (int w = 0; w < VW; w += W) {
                const bool in = !CUT || m * NI + w * 4 / E < p.head_dim;
                if constexpr (W == 4) {
                    const u32x4 y = load_once<u32x4>(from + (in ? 4 * w : 0));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j][w + e] = in ? y[e] : 0;
                } else {
                    const u32x2 y = load_once<u32x2>(from);
#pragma unroll
                    for (int e = 0; e < 2; ++e) v[j][w + e] = in ? y[e] : 0;
                }
            }
        }
    };

    const float factor = p.scale * kLog2e;
    bool tainted = false;                                    // an infinite or NaN value in a block that not all rows see whole
    Place now{}, next{};
    if (step0 < step1) {
        now = locate(step0);
        fetch_k(now);
        fetch_v(now);
    }
#pragma unroll 1
    for (int step = step0; step < step1; ++step) {
        // K of the next step is on its way as soon as this one's is used up, and so is V
        const int base = base_of(step);
        f32x4 s[NM][TILES];
#pragma unroll
        for (int n = 0; n < NM; ++n)
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f32x4 a = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    if constexpr (E == 2) {
                        a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][i]),
                                                                    __builtin_bit_cast(bf16x8, q[n][i]), a, 0, 0, 0);
                    } else {
                        const f32x4 y = __builtin_bit_cast(f32x4, k[t][i]), z = __builtin_bit_cast(f32x4, q[n][i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_16x16x4f32(y[e], z[e], a, 0, 0, 0);
                    }
                }
                s[n][t] = a * factor;
            }
        if (step + 1 < step1) {
            next = locate(step + 1);
            fetch_k(next);
        }
        bool full = base + KB <= all_limit && base >= all_lower;
        if constexpr (WHOLE) {
#pragma unroll
            for (int t = 0; t < TILES; ++t) full = full && now.tile[t] >= 0;
        } else {
            full = full && !__ballot(now.tile[0] < 0);
        }
        if (!full) {
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 4 * TILES; ++j) {
                const int u = base + 16 * (j / 4) + 4 * g + j % 4;
                bool gone;
                if constexpr (WHOLE) gone = (now.tile[j / 4] < 0) | (u >= seq.length);
                else gone = __shfl((int)(now.tile[0] < 0), 16 * (j / 4) + 4 * g + j % 4, 64);
#pragma unroll
                for (int n = 0; n < NM; ++n) s[n][j / 4][j % 4] = (gone | (u >= limit[n]) | (u < lower[n])) ? -INFINITY : s[n][j / 4][j % 4];
                if (gone) {                                  // whatever the slot holds: weight 0 times that has to be 0
#pragma unroll
                    for (int w = 0; w < VW; ++w) v[j][w] = 0;
                }
#pragma unroll
                for (int w = 0; w < VW; ++w) odd |= not_finite<T>(v[j][w]);
            }
            tainted |= __ballot(odd) != 0;
        }
        // the maximum moves where a lane's own has gone past it by more than 8
        bool moves = false;
#pragma unroll
        for (int n = 0; n < NM; ++n)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) moves |= s[n][t][r] > top[n] + 8.0f;
        if (__ballot(moves)) {
#pragma unroll
            for (int n = 0; n < NM; ++n) {
                float most = top[n];
#pragma unroll
                for (int t = 0; t < TILES; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) most = fmaxf(most, s[n][t][r]);
                most = fmaxf(most, __shfl_xor(most, 16, 64));
                most = fmaxf(most, __shfl_xor(most, 32, 64));
                const float by = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[n] - most);
                top[n] = most;
                sum[n] *= by;
#pragma unroll
                for (int i = 0; i < NI; ++i) o[n][i] *= by;
            }
        }
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            const float from = top[n] == -INFINITY ? 0.0f : top[n];
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[n][t][r] = __builtin_amdgcn_exp2f(s[n][t][r] - from);
                    sum[n] += s[n][t][r];
                }
        }
        if constexpr (E == 2) {
            // The weights as two bf16 values each, the second what the first leaves: with one, its rounding adds to that of the output (64 tokens over
            // up to 32000 entries: rms error 1.81e-3 with one, 1.78e-3 with two, as much as rounding the exact output once).  Bytes bound these calls:
            // the second product costs nothing there (the same tokens 776 us with one, 768 with two), 2 x 8 rows over 500 entries 12.4 -> 12.9 us.
            bf16x8 weight[2][NM];
#pragma unroll
            for (int n = 0; n < NM; ++n) {
                u32x4 w[2];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = s[n][e / 2][e % 2 * 2], y = s[n][e / 2][e % 2 * 2 + 1];
                    w[0][e] = pack_bf16(x, y);
                    w[1][e] = pack_bf16(x - __builtin_bit_cast(float, w[0][e] << 16), y - __builtin_bit_cast(float, w[0][e] & 0xffff0000u));
                }
                weight[0][n] = __builtin_bit_cast(bf16x8, w[0]);
                weight[1][n] = __builtin_bit_cast(bf16x8, w[1]);
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                u32x4 a;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    a[e] = __builtin_amdgcn_perm(v[2 * e + 1][i / 2], v[2 * e][i / 2], i % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int n = 0; n < NM; ++n)
                        o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), weight[w][n], o[n][i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int n = 0; n < NM; ++n)
                        o[n][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, v[r][i]), s[n][0][r], o[n][i], 0, 0, 0);
        }
        if (step + 1 < step1) {
            fetch_v(next);
            now = next;
        }
    }

    // An infinite value that met the second piece of a weight, which may be 0 or negative, is NaN now.  (NaN weights are not the values' doing.)
    if constexpr (E == 2) {
        bool odd = false;
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            f32x4 x = o[n][0];
#pragma unroll
            for (int i = 1; i < NI; ++i) x += o[n][i];
            const float all = x[0] + x[1] + (x[2] + x[3]);
            float l = sum[n];
            l += __shfl_xor(l, 16, 64);
            l += __shfl_xor(l, 32, 64);
            odd |= all != all && l == l && limit[n] != 0x7fffffff;
        }
        tainted |= __ballot(odd) != 0;
    }

    // An infinite or NaN value that some rows see and others do not: 0 times it is no 0.  Rare, and done over again key by key
    // on the vector units, which leave out what a column does not see.
    if (tainted) {
        asm volatile("" ::: "memory");                       // (keeps this path out of the common one)
#pragma unroll
        for (int n = 0; n < NM; ++n) {
            top[n] = -INFINITY;
            sum[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < NI; ++i) o[n][i] = f32x4{0, 0, 0, 0};
        }
#pragma unroll 1
        for (int x = 0; x < (step1 - step0) * KB; ++x) {
            const int u = base_of(step0 + x / KB) + x % KB;
            const long long at = slot_of(u);
            if (at < 0) continue;
            const T *kr = reinterpret_cast<const T*>(kc) + at, *vr = reinterpret_cast<const T*>(vc) + at;
            float y[NI][4];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int e = (4 * g + r) * NI + i;
                    y[i][r] = widen(vr[!CUT || e < p.head_dim ? e : 0]);
                }
#pragma unroll
            for (int n = 0; n < NM; ++n) {
                float dot = 0.0f;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int e0 = (s * 64 + g * 16) / E;
                    if (CUT && e0 >= p.head_dim) continue;
#pragma unroll
                    for (int e = 0; e < 16 / E; ++e) {
                        const uint32_t w = q[n][s][e * E / 4];
                        const float z = E == 4 ? __builtin_bit_cast(float, w) : __builtin_bit_cast(float, e % 2 ? w & 0xffff0000u : w << 16);
                        dot = __builtin_fmaf(z, widen(kr[e0 + e]), dot);
                    }
                }
                dot += __shfl_xor(dot, 16, 64);
                dot += __shfl_xor(dot, 32, 64);
                if (u >= limit[n] || u < lower[n]) continue;
                const float score = dot * factor, most = fmaxf(top[n], score);
                const float by = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top[n] - most);
                const float weight = __builtin_amdgcn_exp2f(score - (most == -INFINITY ? 0.0f : most));
                top[n] = most;
                sum[n] = sum[n] * by + (g == 0 ? weight : 0.0f);
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[n][i][r] = o[n][i][r] * by + weight * y[i][r];
            }
        }
    }

    // join the four waves, one column tile after the other
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        sum[n] += __shfl_xor(sum[n], 16, 64);
        sum[n] += __shfl_xor(sum[n], 32, 64);
        if (g == 0) stat[wave][16 * n + m] = float2{top[n], sum[n]};
    }
    if (d.parts > 1 && d.part == 0 && first_head == 0 && threadIdx.x == 0 && d.note < d.heads * target) notes->note[d.note] = JoinNote{d.b, d.tile, d.parts, d.slot};
    const int col = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * NI;
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        __syncthreads();                                     // (the first one: also the rare blocks' use of the same LDS)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < NI; i += 4)
                *reinterpret_cast<float4*>(lds + (wave * 16 + m) * PAD + (4 * g + r) * NI + i) =
                    float4{o[n][i][r], o[n][i + 1][r], o[n][i + 2][r], o[n][i + 3][r]};
        __syncthreads();
        const int in = 16 * n + col, pair = col0 + in;
        if (pair >= pairs) continue;
#pragma unroll 1
        for (int x = 0; x < d.heads; ++x) {                  // one head of all waves, or every wave's own
            float most = -INFINITY, by[4], l = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (d.heads == 1 || w == x) most = fmaxf(most, stat[w][in].x);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float2 t = d.heads == 1 || w == x ? stat[w][in] : float2{-INFINITY, 0.0f};
                by[w] = share_of(t.x, most);
                l += by[w] * t.y;                            // (a wave without a maximum has summed 0, or NaN)
            }
            float y[NI];
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                y[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < 4; ++w)
                    y[i] += by[w] == 0.0f ? 0.0f : by[w] * lds[(w * 16 + col) * PAD + e0 + i];
            }
            if (d.parts > 1) {
                const int at = (d.slot + d.part) * p.kv_heads + first_head + x;
                if ((unsigned)at >= 2u * d.heads * target) continue;      // (cannot be with offsets that do not decrease)
                const int row = at * columns + in;
#pragma unroll
                for (int i = 0; i < NI; i += 4) store4(ws_out + (size_t)row * DP + e0 + i, y + i);
                if ((threadIdx.x & 15) == 0) ws_stat[row] = float2{most, l};
            } else {
                const int row = seq.first + pair / group, h = (first_head + x) * group + pair % group;
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
                for (int i = 0; i < NI; ++i) y[i] *= inv;
                T* to = (T*)p.out + row * p.o_row + h * p.o_head;
#pragma unroll
                for (int i = 0; i < NI; i += 4)
                    if (e0 + i < p.head_dim) store4(to + e0 + i, y + i);
                if (p.lse && (threadIdx.x & 15) == 0) p.lse[(long long)row * p.heads + h] = l == 0.0f ? -INFINITY : most * kLn2 + logf(l);
            }
        }
    }
}

// Joins the parts of a tile: out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s, in the order of the parts.  Workgroups go by
// the notes that the parts' kernel left.  A wave takes `each` columns, one after the other, or where each is 0 a workgroup one column, a
// quarter of the parts a wave.
//   EACH  entries of a column a lane;  AHEAD  parts whose rows are on their way at once
template <typename T, int EACH, int AHEAD>
__global__ __launch_bounds__(256) void k_attend_join(ttf_attention_params p, int columns, int each, int slots,
                                                     const float* __restrict__ ws_out, const float2* __restrict__ ws_stat,
                                                     const JoinNotes* __restrict__ notes)
{
    constexpr int DP = 64 * EACH;
    __shared__ float quarter[4][EACH + 2][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), group = p.heads / p.kv_heads;
    const int head = blockIdx.x % p.kv_heads, n = blockIdx.x / p.kv_heads;
    const JoinNote d = notes->note[n];
    if (n >= notes->count) return;                           // (what the note holds was not written by this call)
    // (with offsets that decrease, workgroups past the grid have left theirs unwritten: any bits)
    if ((unsigned)d.b >= (unsigned)p.batch || d.slot < 0 || d.parts < 1 || ((long long)d.slot + d.parts) * p.kv_heads > slots) return;
    const int2 rows = rows_of(p.row_offsets, d.b, p.rows);
    if ((unsigned)d.tile >= (unsigned)tiles_of(rows.y, group, columns)) return;
    const int q = each ? d.parts : (max(4 * AHEAD, d.parts) + 4 * AHEAD - 1) / (4 * AHEAD) * AHEAD;    // parts a wave, whole batches
    const int from = each ? 0 : min(wave * q, d.parts), to = min(from + q, d.parts);
    for (int x = 0; x < max(each, 1); ++x) {
        const int col = each ? (blockIdx.y * 4 + wave) * each + x : blockIdx.y, pair = d.tile * columns + col;
        if (col >= columns || pair >= rows.y * group) return;
        const auto at = [&](int part) { return ((d.slot + part) * p.kv_heads + head) * columns + col; };
        float most = -INFINITY;
        for (int s = from + lane; s < to; s += 64) most = fmaxf(most, ws_stat[at(s)].x);
#pragma unroll
        for (int y = 1; y < 64; y <<= 1) most = fmaxf(most, __shfl_xor(most, y, 64));
        float l = 0.0f, v[EACH] = {};
        for (int s0 = from; s0 < to; s0 += 64) {
            const int parts = min(64, to - s0);
            float by = 0.0f;
            if (lane < parts) {
                const float2 t = ws_stat[at(s0 + lane)];
                by = share_of(t.x, most);
                l += by * t.y;
            }
            for (int s1 = 0; s1 < parts; s1 += AHEAD) {      // (parts past the last: the last again, with a weight of 0)
                float y[AHEAD][EACH];
#pragma unroll
                for (int s = 0; s < AHEAD; ++s)
#pragma unroll
                    for (int i = 0; i < EACH; ++i) y[s][i] = ws_out[(size_t)at(s0 + min(s1 + s, parts - 1)) * DP + lane * EACH + i];
#pragma unroll
                for (int s = 0; s < AHEAD; ++s) {
                    const float w = s1 + s < parts ? __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, by), s1 + s)) : 0.0f;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) v[i] += w == 0.0f ? 0.0f : w * y[s][i];
                }
            }
        }
        l = wave_sum(l);
        if (!each && d.parts > AHEAD) {                      // the quarters, in their order
            quarter[wave][EACH][lane] = most;
            quarter[wave][EACH + 1][lane] = l;
#pragma unroll
            for (int i = 0; i < EACH; ++i) quarter[wave][i][lane] = v[i];
            __syncthreads();
            l = 0.0f;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, quarter[w][EACH][lane]);
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float by = share_of(quarter[w][EACH][lane], top);
                l += by * quarter[w][EACH + 1][lane];
#pragma unroll
                for (int i = 0; i < EACH; ++i) v[i] += by == 0.0f ? 0.0f : by * quarter[w][i][lane];
            }
            most = top;
        }
        if (!each && wave > 0) return;
        const int row = rows.x + pair / group, h = head * group + pair % group;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        T* to_row = (T*)p.out + row * p.o_row + h * p.o_head + lane * EACH;
        if (lane * EACH < p.head_dim) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if constexpr (sizeof(T) == 2) to_row[i].bits = __builtin_bit_cast(uint16_t, (__bf16)(v[i] * inv));
                else to_row[i] = v[i] * inv;
            }
        }
        if (p.lse && lane == 0) p.lse[(long long)row * p.heads + h] = l == 0.0f ? -INFINITY : most * kLn2 + logf(l);
    }
}

}  // namespace

namespace {

// The kernel of a call and its sizes.
struct Choice {
    bool wide;      // the kernel for many rows
    bool neighbours;// workgroups may take four key heads
    int width;      // head dimension the kernel is built for
    int tiles;      // column tiles of 16 of the kernel for few rows
    int columns;    // columns of a tile
    int target;     // workgroups that fill the chip, a power of two
    int slots;      // tiles of parts that the workspace has room for
};

// Pairs of a row and a query head that the longest sequence brings to a key head.
// (max_rows below the mean would give tiles of few columns to many rows: a grid past what a launch may have)
long long pairs_of(const ttf_attention_params& p)
{
    const int mean = (int)(((long long)p.rows + p.batch - 1) / p.batch), most = p.max_rows < p.rows ? p.max_rows : p.rows;
    return (long long)(most > mean ? most : mean) * (p.heads / p.kv_heads);
}

Choice choose(const ttf_attention_params& p, long long pairs)
{
    Choice x{};
    x.width = p.head_dim <= 64 ? 64 : p.head_dim <= 128 ? 128 : 256;
    // Between 17 and 32 columns either kernel may win with heads of up to 128 entries (32 x 8 rows over 8000 entries 138 us with the one for few, 131 with that
    // for many; 64 x 6 over 400 24 and 32, 16 x 5 over 3000 the same); with 256, 16 columns are all that the one for few has registers for (16 heads on 4,
    // 32 x 8 rows over 8000 entries 237 and 146 us).
    x.wide = p.dtype == TTF_BF16 && pairs > (x.width == 256 ? 16 : 32);
    if (x.wide) {
        x.columns = 128;
        x.target = x.width == 256 ? 256 : 512;               // (one and two workgroups a CU)
        x.slots = 2 * x.target;
        return x;
    }
    // (fp32 of 128 entries: four spill, 20 x 29 rows over 14000 keys 887 us, two 787)
    x.tiles = pairs <= 16 ? 1 : (pairs <= 32 || p.dtype == TTF_BF16 || x.width > 64) ? 2 : 4;
    if (x.width == 256 && p.dtype == TTF_F32) x.tiles = 1;
    x.columns = pairs < 16 * x.tiles ? (int)pairs : 16 * x.tiles;    // no more than there are: the parts' rows take that much less room
    x.neighbours = p.kv_heads % kNeighbours == 0;
    x.target = 2048 / x.tiles;
    x.slots = 2 * x.target * (x.neighbours ? kNeighbours : 1);
    return x;
}

// Workspace: rows of the parts, their statistics, the notes for the join.
struct Parts {
    float* out;
    float2* stat;
    JoinNotes* notes;
    size_t bytes;
};

Parts carve_parts(const Choice& x, void* workspace)
{
    char* at = static_cast<char*>(workspace);
    const size_t rows = (size_t)x.slots * x.columns, out = rows * x.width * sizeof(float), stat = (rows * sizeof(float2) + 15) / 16 * 16;
    return Parts{reinterpret_cast<float*>(at), reinterpret_cast<float2*>(at + out), reinterpret_cast<JoinNotes*>(at + out + stat),
                 out + stat + sizeof(JoinNotes) + sizeof(JoinNote) * (x.slots / 2)};
}

unsigned most_tiles(const ttf_attention_params& p, const Choice& x)
{
    return (unsigned)((long long)p.rows * (p.heads / p.kv_heads) / x.columns + p.batch);
}

template <typename T, int DP, int NM>
hipError_t launch(const ttf_attention_params& p, const ttf_kv_cache& c, const Choice& x, const Parts& w, hipStream_t s)
{
    constexpr int WAVES = NM == 1 && DP * sizeof(T) <= 256 ? 3 : NM * DP * sizeof(T) <= 512 ? 2 : 1;
    // (heads of 65 to 127 entries: a third wave spills, 32 tokens over 8000 entries of 72 172 us with three, 150 with two)
    constexpr int CUT_WAVES = sizeof(T) == 2 && NM == 1 && DP == 128 ? 2 : WAVES;
    const unsigned grid = most_tiles(p, x) * p.kv_heads + x.target;
    const bool neighbours = x.neighbours && c.head_stride < c.slot_stride;      // (heads of a slot side by side)
    // (the offsets inside a tile are held in 32 bits)
    const auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(p, c, x.columns, neighbours, x.target, w.out, w.stat, w.notes); };
    if (c.page_size % 16 != 0 || c.slot_stride >= (1ll << 24)) go(k_attend<T, DP, NM, false, true, CUT_WAVES>);
    else if (p.head_dim < DP) go(k_attend<T, DP, NM, true, true, CUT_WAVES>);
    else go(k_attend<T, DP, NM, true, false, WAVES>);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_join(const ttf_attention_params& p, const Choice& x, const Parts& w, hipStream_t s)
{
    // Few columns: a workgroup to each.  More: a wave to each.  Many tiles, few of which are cut as a rule: up to four to a wave (20 rows
    // over 8192 entries 24 us with one, 41 with four; 8 clips of 1000 rows 60 and 57, 4 x 512 rows over 8192 entries 166 and 159).
    const unsigned tiles = most_tiles(p, x) * p.kv_heads;
    const int each = x.columns <= 16 ? 0 : tiles <= 256 ? 1 : tiles <= 512 ? 2 : 4;
    const dim3 grid(tiles < (unsigned)x.slots / 2 ? tiles : (unsigned)x.slots / 2, (unsigned)(each ? (x.columns + 4 * each - 1) / (4 * each) : x.columns));
    const auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, s>>>(p, x.columns, each, x.slots, w.out, w.stat, w.notes);
        return hipGetLastError();
    };
    // Where there are many tiles, each is in few parts (4 x 512 rows over 8192 entries, two to four: with eight on their way 162 us, with four 159).
    if (each > 1) return x.width == 64 ? go(k_attend_join<T, 1, 4>) : x.width == 128 ? go(k_attend_join<T, 2, 4>) : go(k_attend_join<T, 4, 4>);
    return x.width == 64 ? go(k_attend_join<T, 1, 8>) : x.width == 128 ? go(k_attend_join<T, 2, 8>) : go(k_attend_join<T, 4, 8>);
}

}  // namespace

size_t attention_workspace_used(const ttf_attention_params& p) { return carve_parts(choose(p, pairs_of(p)), nullptr).bytes; }

// Fewer pairs may take more: the kernel for few rows has more workgroups.  With one kernel and number of column tiles the room
// grows with the pairs, so it is greatest at the most pairs of one of them.
size_t attention_workspace_bytes(const ttf_attention_params& p)
{
    const long long pairs = pairs_of(p);
    size_t most = 0;
    for (const long long n : {pairs, 16ll, 32ll, 64ll}) most = std::max(most, carve_parts(choose(p, std::min(n, pairs)), nullptr).bytes);
    return most;
}

hipError_t launch_attention(const ttf_attention_params& p, const ttf_kv_cache& c, void* workspace, hipStream_t s)
{
    const Choice x = choose(p, pairs_of(p));
    const Parts w = carve_parts(x, workspace);
    const auto few = [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int DP = decltype(width)::value;
        if (x.tiles == 1) return launch<T, DP, 1>(p, c, x, w, s);
        if constexpr (DP < 256) {
            if (x.tiles == 2) return launch<T, DP, 2>(p, c, x, w, s);
        }
        if constexpr (sizeof(T) == 4 && DP == 64) return launch<T, DP, 4>(p, c, x, w, s);
        return hipErrorInvalidValue;                         // (choose() names no other)
    };
    const auto of_width = [&](auto type) {
        if (x.width == 64) return few(type, std::integral_constant<int, 64>());
        if (x.width == 128) return few(type, std::integral_constant<int, 128>());
        return few(type, std::integral_constant<int, 256>());
    };
    const hipError_t e = x.wide ? launch_attention_wide(p, c, x.width, x.target, std::max(2u * x.target, most_tiles(p, x) * p.kv_heads + x.target), w.out, w.stat, w.notes, s)
                       : p.dtype == TTF_BF16 ? of_width(bf16_t{}) : of_width(float{});
    if (e != hipSuccess) return e;
    if (uncut(p, c)) return hipSuccess;
    return p.dtype == TTF_BF16 ? launch_join<bf16_t>(p, x, w, s) : launch_join<float>(p, x, w, s);
}

}  // namespace ttf
