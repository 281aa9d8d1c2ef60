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
#include <type_traits>

#include "ttf_attend.h"

namespace ttf {

hipError_t launch_attention_join(const ttf_attention_params& p, const ttf_kv_cache& c, int columns, int step, int target,
                                 int width, const float* ws_out, const float* ws_stat, hipStream_t s);
hipError_t launch_attention_wide(const ttf_attention_params& p, const ttf_kv_cache& c, int width, int target, float* ws_out,
                                 float* ws_stat, hipStream_t s);

namespace {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

template <typename T> constexpr int kBlockTiles = sizeof(T) == 2 ? 2 : 1;    // 16-key tiles a wave works on at once

template <typename T>
__device__ __forceinline__ void store_row_chunk(T* to, const float* v, int n);   // n % 4 == 0
template <>
__device__ __forceinline__ void store_row_chunk<float>(float* to, const float* v, int n)
{
    for (int i = 0; i < n; i += 4) *reinterpret_cast<float4*>(to + i) = float4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}
template <>
__device__ __forceinline__ void store_row_chunk<bf16_t>(bf16_t* to, const float* v, int n)
{
    for (int i = 0; i < n; i += 4)
        *reinterpret_cast<uint2*>(to + i) = uint2{pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3])};
}

// Whether a 32-bit word holds an infinite or NaN value (one fp32, or either of two bf16).
template <typename T>
__device__ __forceinline__ bool not_finite(uint32_t w)
{
    if constexpr (sizeof(T) == 4) return (w & 0x7f800000u) == 0x7f800000u;
    return (w & 0x7f800000u) == 0x7f800000u || (w & 0x7f80u) == 0x7f80u;
}

// A workgroup of four waves works on one part of one tile for one key head; its waves take turns with the blocks of
// 16 or 32 keys, and their (m, l, O) are joined in LDS at the end.
//   DP     head dimension rounded up to 64, 128 or 256;  NM  column tiles of 16
//   WHOLE  pages hold whole 16-key tiles: a tile's address is one for all its keys.  Otherwise every key's page is looked up.
template <typename T, int DP, int NM, bool WHOLE>
__global__ __launch_bounds__(256) void k_attend(ttf_attention_params p, ttf_kv_cache c, int target, float* ws_out, float* ws_stat)
{
    constexpr int E = sizeof(T), TILES = kBlockTiles<T>, KB = 16 * TILES, COLUMNS = 16 * NM;
    constexpr int KS = DP * E / 64;                          // 16-byte pieces of K a lane holds per tile
    constexpr int NI = DP / 16, VW = NI * E / 4;             // entries of V, in 32-bit words, a lane holds per key
    constexpr int PAD = DP + 4;
    constexpr int JOIN = 4 * 16 * PAD, WEIGHTS = 4 * KB * COLUMNS;
    __shared__ __attribute__((aligned(16))) float lds[JOIN > WEIGHTS ? JOIN : WEIGHTS];
    __shared__ float stat[2][4][COLUMNS];

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, m = lane & 15;
    const int head = blockIdx.x % p.kv_heads, group = p.heads / p.kv_heads;
    Deal d;
    if (!deal_out(p, c, COLUMNS, 4 * KB, target, blockIdx.x / p.kv_heads, true, d)) return;
    const Sequence seq = sequence_of(p, c, d.b);
    const int pairs = seq.rows * group, col0 = d.tile * COLUMNS;   // (rows * heads is bounded by the host)

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
        const long long h = (long long)head * group + pair % group;
        const T* from = (const T*)p.q + (seq.first + row) * p.q_row + h * p.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int at = (s * 64 + g * 16) / E;
            q[n][s] = is && at < p.head_dim ? *reinterpret_cast<const u32x4*>(from + at) : u32x4{0, 0, 0, 0};
        }
    }
    // what all and what any of the tile's rows see (rows in ascending order: so are their limits)
    const int row_a = col0 / group, row_z = min(col0 + COLUMNS - 1, pairs - 1) / group;
    const int all_limit = limit_of(row_a), all_lower = lower_of(row_z), any_limit = limit_of(row_z);
    const int begin = lower_of(row_a) & ~31;
    const int steps = max(0, (int)(((long long)any_limit - begin + 4 * KB - 1) / (4 * KB)));
    const int step0 = (int)((long long)steps * d.part / d.parts), step1 = (int)((long long)steps * (d.part + 1) / d.parts);

    float top[NM], sum[NM];                                  // m and this lane's share of l
    f32x4 o[NM][NI];
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        top[n] = -INFINITY;
        sum[n] = 0.0f;
#pragma unroll
        for (int i = 0; i < NI; ++i) o[n][i] = f32x4{0, 0, 0, 0};
    }

    const T *kc = (const T*)c.k + head * c.head_stride, *vc = (const T*)c.v + head * c.head_stride;
    const int32_t* table = c.page_table + d.b * c.table_stride;
    // element offset of entry u's slot, -1 where there is none
    const auto slot_of = [&](int u) -> long long {
        if (u >= seq.length) return -1;                      // (so u / page_size < table_width)
        const unsigned at = (unsigned)u / (unsigned)c.page_size;
        const int page = table[at];
        return page >= 0 && page < c.pages ? page * c.page_stride + (u - (int)at * c.page_size) * c.slot_stride : -1;
    };
    const auto base_of = [&](int step) { return begin + (step * 4 + wave) * KB; };

    // WHOLE: lane j holds the offset of tile j % TILES of step `held` + j / TILES; a new set every 64 / TILES steps
    long long mine = -1;
    struct Block { u32x4 k[TILES][KS]; uint32_t v[4 * TILES][VW]; bool there[TILES]; unsigned bad; };
    const float factor = p.scale * kLog2e;

    const auto fetch = [&](int step, Block& x) {
        const int base = base_of(step);
        long long ko[TILES], vo[4 * TILES];
        x.bad = 0;                                           // bit j: key slot j of this lane is not there
        if constexpr (WHOLE) {
            if ((step - step0) % (64 / TILES) == 0) mine = slot_of(base_of(step + lane / TILES) + lane % TILES * 16);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const int j = (step - step0) % (64 / TILES) * TILES + t;
                const long long at = ((long long)__builtin_amdgcn_readlane((int)(mine >> 32), j) << 32) |
                                     (uint32_t)__builtin_amdgcn_readlane((int)mine, j);
                x.there[t] = at >= 0;
                if (at < 0) x.bad |= 15u << 4 * t;
                const long long tile = at >= 0 ? at : 0;
                ko[t] = tile + m * c.slot_stride;
#pragma unroll
                for (int r = 0; r < 4; ++r) vo[4 * t + r] = tile + (4 * g + r) * c.slot_stride;
            }
        } else {
            const long long at = slot_of(base + lane % KB);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                x.there[t] = __ballot(at < 0) == 0;
                ko[t] = max(0ll, __shfl(at, 16 * t + m, 64));
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    vo[4 * t + r] = __shfl(at, 16 * t + 4 * g + r, 64);
                    if (vo[4 * t + r] < 0) x.bad |= 1u << (4 * t + r);
                    vo[4 * t + r] = max(0ll, vo[4 * t + r]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int at = (s * 64 + g * 16) / E;
                const bool in = at < p.head_dim;
                x.k[t][s] = *reinterpret_cast<const u32x4*>(kc + ko[t] + (in ? at : 0));
                if (!in) x.k[t][s] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
        for (int j = 0; j < 4 * TILES; ++j) {
            constexpr int W = VW < 4 ? VW : 4;               // words a load brings
#pragma unroll
            for (int w = 0; w < VW; w += W) {
                const int at = m * NI + w * 4 / E;
                const bool in = at < p.head_dim;
                const T* from = vc + vo[j] + (in ? at : 0);
                if constexpr (W == 4) {
                    const u32x4 y = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.v[j][w + e] = in ? y[e] : 0;
                } else {
                    const u32x2 y = *reinterpret_cast<const u32x2*>(from);
#pragma unroll
                    for (int e = 0; e < 2; ++e) x.v[j][w + e] = in ? y[e] : 0;
                }
            }
        }
    };

    const auto work = [&](int step, Block& x) {
        const int base = base_of(step);
        if (base >= any_limit) return;
        f32x4 s[NM][TILES];
#pragma unroll
        for (int n = 0; n < NM; ++n)
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                f32x4 a = {0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < KS; ++i) {
                    if constexpr (E == 2) {
                        a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x.k[t][i]),
                                                                    __builtin_bit_cast(bf16x8, q[n][i]), a, 0, 0, 0);
                    } else {
                        const f32x4 y = __builtin_bit_cast(f32x4, x.k[t][i]), z = __builtin_bit_cast(f32x4, q[n][i]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_16x16x4f32(y[e], z[e], a, 0, 0, 0);
                    }
                }
                s[n][t] = a * factor;
            }
        bool full = base + KB <= all_limit && base >= all_lower;
#pragma unroll
        for (int t = 0; t < TILES; ++t) full = full && x.there[t];
        if (!full) {
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int u = base + 16 * t + 4 * g + r, j = 4 * t + r;
                    const bool gone = (x.bad >> j & 1) || u >= seq.length;
#pragma unroll
                    for (int n = 0; n < NM; ++n)
                        if (gone || u >= limit[n] || u < lower[n]) s[n][t][r] = -INFINITY;
                    if (gone) {                              // whatever the slot holds: weight 0 times that has to be 0
#pragma unroll
                        for (int w = 0; w < VW; ++w) x.v[j][w] = 0;
                    }
                }
        }
        // the maximum moves where a lane's own has gone past it by more than 8
        bool moves = false;
#pragma unroll
        for (int n = 0; n < NM; ++n)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) moves = moves || s[n][t][r] > top[n] + 8.0f;
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
        if (!full) {
            // An infinite or NaN value that some rows see and others do not: 0 times it is no 0, so such a block goes by the
            // vector units, key by key, and leaves out weights of 0.
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 4 * TILES; ++j)
#pragma unroll
                for (int w = 0; w < VW; ++w) odd = odd || not_finite<T>(x.v[j][w]);
            if (__ballot(odd)) {
                float* weights = lds + wave * KB * COLUMNS;
#pragma unroll
                for (int n = 0; n < NM; ++n)
#pragma unroll
                    for (int t = 0; t < TILES; ++t)
#pragma unroll
                        for (int r = 0; r < 4; ++r) weights[(16 * t + 4 * g + r) * COLUMNS + 16 * n + m] = s[n][t][r];
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll 1
                for (int u = 0; u < KB; ++u) {
                    const long long at = slot_of(base + u);
                    if (at < 0) continue;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            const int e = (4 * g + r) * NI + i;
                            const float v = e < p.head_dim ? widen(vc[at + e]) : 0.0f;
#pragma unroll
                            for (int n = 0; n < NM; ++n) {
                                const float weight = weights[u * COLUMNS + 16 * n + m];
                                if (weight != 0.0f) o[n][i][r] += weight * v;
                            }
                        }
                }
                __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                __builtin_amdgcn_wave_barrier();
                return;
            }
        }
        if constexpr (E == 2) {
            bf16x8 weight[NM];
#pragma unroll
            for (int n = 0; n < NM; ++n) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack_bf16(s[n][e / 2][e % 2 * 2], s[n][e / 2][e % 2 * 2 + 1]);
                weight[n] = __builtin_bit_cast(bf16x8, w);
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                u32x4 a;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    a[e] = __builtin_amdgcn_perm(x.v[2 * e + 1][i / 2], x.v[2 * e][i / 2], i % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int n = 0; n < NM; ++n)
                    o[n][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), weight[n], o[n][i], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int n = 0; n < NM; ++n)
                        o[n][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, x.v[r][i]), s[n][0][r],
                                                                       o[n][i], 0, 0, 0);
        }
    };

    Block a, b;
    int step = step0;
    if (step < step1) fetch(step, a);
#pragma unroll 1
    while (step < step1) {
        if (step + 1 < step1) fetch(step + 1, b);
        work(step, a);
        if (++step >= step1) break;
        if (step + 1 < step1) fetch(step + 1, a);
        work(step, b);
        ++step;
    }

    // join the four waves, one column tile after the other
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        sum[n] += __shfl_xor(sum[n], 16, 64);
        sum[n] += __shfl_xor(sum[n], 32, 64);
        if (g == 0) {
            stat[0][wave][16 * n + m] = top[n];
            stat[1][wave][16 * n + m] = sum[n];
        }
    }
    const int tid = threadIdx.x, col = tid >> 4;
#pragma unroll
    for (int n = 0; n < NM; ++n) {
        __syncthreads();                                     // (the first one: also the slow blocks' use of the same LDS)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < NI; i += 4)
                *reinterpret_cast<float4*>(lds + (wave * 16 + m) * PAD + (4 * g + r) * NI + i) =
                    float4{o[n][i][r], o[n][i + 1][r], o[n][i + 2][r], o[n][i + 3][r]};
        __syncthreads();
        const int pair = col0 + 16 * n + col;
        if (pair >= pairs) continue;
        float most = -INFINITY, by[4], l = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) most = fmaxf(most, stat[0][w][16 * n + col]);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float t = stat[0][w][16 * n + col];
            by[w] = t == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(t - most);
            l += by[w] * stat[1][w][16 * n + col];           // (a wave without a maximum has summed 0, or NaN)
        }
        const int e0 = (tid & 15) * NI;
        float v[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                if (by[w] != 0.0f) v[i] += by[w] * lds[(w * 16 + col) * PAD + e0 + i];
            }
        }
        if (d.parts > 1) {
            const long long at = ((d.slot + d.part) * p.kv_heads + head) * COLUMNS + 16 * n + col;
            if (at >= 2ll * target * COLUMNS) continue;      // (cannot be with offsets that do not decrease)
            store_row_chunk<float>(ws_out + at * DP + e0, v, NI);
            if ((tid & 15) == 0) {
                ws_stat[2 * at] = most;
                ws_stat[2 * at + 1] = l;
            }
        } else {
            const int row = seq.first + pair / group, h = head * group + pair % group;
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int i = 0; i < NI; ++i) v[i] *= inv;
            T* to = (T*)p.out + row * p.o_row + h * p.o_head;
#pragma unroll
            for (int i = 0; i < NI; i += 4)
                if (e0 + i < p.head_dim) store_row_chunk<T>(to + e0 + i, v + i, 4);
            if (p.lse && (tid & 15) == 0) p.lse[(long long)row * p.heads + h] = l == 0.0f ? -INFINITY : most * kLn2 + logf(l);
        }
    }
}

// Joins the parts of a tile: out = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s, in the order of the parts.  A wave per
// column; the parts' statistics are read 64 at a time.
template <typename T, int EACH>
__global__ __launch_bounds__(256) void k_attend_join(ttf_attention_params p, ttf_kv_cache c, int columns, int step, int target,
                                                     const float* __restrict__ ws_out, const float* __restrict__ ws_stat)
{
    constexpr int DP = 64 * EACH;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, head = blockIdx.x % p.kv_heads, group = p.heads / p.kv_heads;
    Deal d;
    if (!deal_out(p, c, columns, step, target, blockIdx.x / p.kv_heads, false, d) || d.parts == 1) return;
    const Sequence seq = sequence_of(p, c, d.b);
    const int col = blockIdx.y * 4 + wave, pair = d.tile * columns + col;
    if (pair >= seq.rows * group) return;
    if (((d.slot + d.parts - 1) * p.kv_heads + head) >= 2ll * target) return;
    const auto at = [&](int part) { return ((d.slot + part) * p.kv_heads + head) * columns + col; };
    float most = -INFINITY;
    for (int s = lane; s < d.parts; s += 64) most = fmaxf(most, ws_stat[2 * at(s)]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) most = fmaxf(most, __shfl_xor(most, x, 64));
    float l = 0.0f, v[EACH] = {};
    for (int s0 = 0; s0 < d.parts; s0 += 64) {
        const int n = min(64, d.parts - s0);
        float by = 0.0f;
        if (lane < n) {
            const float t = ws_stat[2 * at(s0 + lane)], part = ws_stat[2 * at(s0 + lane) + 1];
            by = t == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(t - most);
            l += by * part;
        }
        for (int s = 0; s < n; ++s) {
            const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, by), s));
            const float* from = ws_out + at(s0 + s) * DP + lane * EACH;
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] += w == 0.0f ? 0.0f : w * from[i];
        }
    }
    l = wave_sum(l);
    const int row = seq.first + pair / group, h = head * group + pair % group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    T* to = (T*)p.out + row * p.o_row + h * p.o_head + lane * EACH;
    if (lane * EACH < p.head_dim) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if constexpr (sizeof(T) == 2) to[i].bits = __builtin_bit_cast(uint16_t, (__bf16)(v[i] * inv));
            else to[i] = v[i] * inv;
        }
    }
    if (p.lse && lane == 0) p.lse[(long long)row * p.heads + h] = l == 0.0f ? -INFINITY : most * kLn2 + logf(l);
}

}  // namespace

hipError_t launch_attention_join(const ttf_attention_params& p, const ttf_kv_cache& c, int columns, int step, int target,
                                 int width, const float* ws_out, const float* ws_stat, hipStream_t s)
{
    const long long tiles = (long long)p.rows * (p.heads / p.kv_heads) / columns + p.batch;
    const dim3 grid((unsigned)(tiles * p.kv_heads), (unsigned)(columns / 4));
    const auto go = [&](auto kernel) {
        kernel<<<grid, 256, 0, s>>>(p, c, columns, step, target, ws_out, ws_stat);
        return hipGetLastError();
    };
    if (p.dtype == TTF_BF16)
        return width == 64 ? go(k_attend_join<bf16_t, 1>) : width == 128 ? go(k_attend_join<bf16_t, 2>) : go(k_attend_join<bf16_t, 4>);
    return width == 64 ? go(k_attend_join<float, 1>) : width == 128 ? go(k_attend_join<float, 2>) : go(k_attend_join<float, 4>);
}

namespace {

// The kernel of a call and its sizes.
struct Choice {
    bool wide;      // the kernel for many rows
    int width;      // head dimension the kernel is built for
    int columns;    // columns of a tile
    int step;       // keys a workgroup takes a step
    int target;     // workgroups that fill the chip
};

Choice choose(const ttf_attention_params& p)
{
    Choice x;
    x.width = p.head_dim <= 64 ? 64 : p.head_dim <= 128 ? 128 : 256;
    const long long pairs = (long long)(p.max_rows < p.rows ? p.max_rows : p.rows) * (p.heads / p.kv_heads);
    x.wide = p.dtype == TTF_BF16 && pairs > 32;
    if (x.wide) {
        x.columns = 128;
        x.step = 64;
        x.target = 512;
        return x;
    }
    x.columns = pairs <= 16 ? 16 : (pairs <= 32 || p.dtype == TTF_BF16) ? 32 : 64;
    if (x.width == 256 && p.dtype == TTF_F32) x.columns = 16;
    x.step = p.dtype == TTF_BF16 ? 128 : 64;
    x.target = 1024;
    return x;
}

template <typename T, int DP, int NM>
hipError_t launch(const ttf_attention_params& p, const ttf_kv_cache& c, const Choice& x, float* ws_out, float* ws_stat, hipStream_t s)
{
    const long long tiles = (long long)p.rows * (p.heads / p.kv_heads) / (16 * NM) + p.batch;
    const unsigned grid = (unsigned)(tiles * p.kv_heads + x.target);
    if (c.page_size % 16 == 0) k_attend<T, DP, NM, true><<<grid, 256, 0, s>>>(p, c, x.target, ws_out, ws_stat);
    else k_attend<T, DP, NM, false><<<grid, 256, 0, s>>>(p, c, x.target, ws_out, ws_stat);
    return hipGetLastError();
}

}  // namespace

size_t attention_workspace_bytes(const ttf_attention_params& p)
{
    const Choice x = choose(p);
    return (size_t)2 * x.target * x.columns * (x.width + 2) * sizeof(float);
}

hipError_t launch_attention(const ttf_attention_params& p, const ttf_kv_cache& c, void* workspace, hipStream_t s)
{
    const Choice x = choose(p);
    float *ws_out = static_cast<float*>(workspace), *ws_stat = ws_out + (size_t)2 * x.target * x.columns * x.width;
    const auto few = [&](auto type, auto width) {
        using T = decltype(type);
        constexpr int DP = decltype(width)::value;
        if (x.columns == 16) return launch<T, DP, 1>(p, c, x, ws_out, ws_stat, s);
        if constexpr (sizeof(T) == 2 || DP < 256) {
            if (x.columns == 32) return launch<T, DP, 2>(p, c, x, ws_out, ws_stat, s);
        }
        if constexpr (sizeof(T) == 4 && DP < 256) return launch<T, DP, 4>(p, c, x, ws_out, ws_stat, s);
        return hipErrorInvalidValue;                         // (choose() names no other)
    };
    const auto of_width = [&](auto type) {
        if (x.width == 64) return few(type, std::integral_constant<int, 64>());
        if (x.width == 128) return few(type, std::integral_constant<int, 128>());
        return few(type, std::integral_constant<int, 256>());
    };
    const hipError_t e = x.wide ? launch_attention_wide(p, c, x.width, x.target, ws_out, ws_stat, s)
                       : p.dtype == TTF_BF16 ? of_width(bf16_t{}) : of_width(float{});
    if (e != hipSuccess) return e;
    return launch_attention_join(p, c, x.columns, x.step, x.target, x.width, ws_out, ws_stat, s);
}

}  // namespace ttf
