// Norm and rotation of queries and keys by their rows' positions, alone (ttf_qk_norm_rope) or on the way into a
// paged cache (ttf_cache_append).
//
// A row's heads are independent and each entry is read and written once, so the bytes bound it: 2 T (Hq + Hk) D e, with the
// values of an append 2 T (Hq + 2 Hk) D e.  What could cost more is the angles, D/2 a row: position times frequency
// is formed in 64 bits (a position of 10^6 times a frequency of 1 has lost 2^-5 rad in 32) and reduced to turns in [-1/2, 1/2] there; sine and
// cosine are taken in 64 bits too and rounded once, since an angle rounded to 32 before errs by up to 2^-23.3 rad (16 clips 115.3 -> 116.1 us,
// one token the same).  A wave takes a row's share of the heads, forms every angle once, one a
// lane, and hands them to its heads through LDS; 8 lanes then hold one head of 128, the two halves of every pair in the same lane.
// Measured: 648 MB of 16 clips' queries and keys 116 us (5.6 TB/s), 778 MB appended 139 us (5.6 TB/s), fp32 103 MB 20 us (5.1 TB/s).
#include "ttf_device.h"
#include "ttf_serve.h"

namespace ttf {
namespace {

__device__ __forceinline__ void store_as(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_as(bf16_t* p, float v)
{
    p->bits = __builtin_bit_cast(uint16_t, (__bf16)v);
}

template <int BYTES> struct Word;
template <> struct Word<16> { typedef __attribute__((ext_vector_type(4))) uint32_t type; };
template <> struct Word<8> { typedef __attribute__((ext_vector_type(2))) uint32_t type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

// V elements from memory into fp32 and back (rounded to nearest even), in one access of V * sizeof(T) bytes.  Written without a place in the
// caches (16 clips 122 us with one, 116 so, two clips 20 either way; reading likewise 115 on the 16, but 23 on the two).
template <typename T, int V>
__device__ __forceinline__ void load_chunk(const T* p, float* v)
{
    T raw[V];
    __builtin_memcpy(raw, __builtin_assume_aligned(p, V * sizeof(T)), V * sizeof(T));
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = widen(raw[i]);
}
template <typename T, int V>
__device__ __forceinline__ void store_chunk(T* p, const float* v)
{
    T raw[V];
#pragma unroll
    for (int i = 0; i < V; ++i) store_as(&raw[i], v[i]);
    typename Word<V * sizeof(T)>::type w;
    __builtin_memcpy(&w, raw, sizeof(w));
    __builtin_nontemporal_store(w, reinterpret_cast<decltype(w)*>(p));
}

// One wave per row and share of its heads.  V = entries a lane moves at once: a head's pairs are dealt out in units of 2 V
// entries (V first and V second ones of V pairs, or V + V entries that are not rotated).  `group` lanes hold one head, UNITS units each.
template <typename T, int V, int UNITS>
__global__ __launch_bounds__(256) void k_qk(ttf_qk_params p, ttf_kv_cache c, bool append, int group, int shares)
{
    __shared__ float2 turn[4][kMaxHeadDim / 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long id = (long long)blockIdx.x * 4 + wave;
    const int row = (int)(id / shares), share = (int)(id % shares);
    if (row >= p.rows) return;                               // (no barrier below: a wave only reads what it wrote itself)

    // the sequence the row belongs to: as many sequences as have ended at or before it
    long long slot = -1;                                     // element offset of the row's slot in the cache
    if (append) {
        int b = 0;
        for (int i = 0; i < p.batch; i += 64) {
            const bool ended = i + lane < p.batch && p.row_offsets[i + lane + 1] <= row;
            const int n = __popcll(__ballot(ended));
            b += n;
            if (n < 64) break;
        }
        if (b >= p.batch) return;
        const int first = p.row_offsets[b], have = p.cached[b];
        if (first < 0 || row < first) return;
        const uint32_t t = (uint32_t)have + (uint32_t)(row - first), at = t / (uint32_t)c.page_size;   // (below 2^32)
        if (have >= 0 && at < (uint32_t)c.table_width) {
            const int page = c.page_table[b * c.table_stride + at];
            if (page >= 0 && page < c.pages) slot = page * c.page_stride + (t - at * c.page_size) * c.slot_stride;
        }
    } else if (p.row_offsets) {
        if (row < p.row_offsets[0] || row >= p.row_offsets[p.batch]) return;
    }

    const int half = p.rotary_dim / 2;
    for (int j = lane; j < half; j += 64) {
        int a = p.axis ? p.axis[j] : 0;
        if (a < 0 || a >= p.axes) a = 0;
        const double turns = (double)p.pos[a * p.pos_stride + row] * (p.inv_freq[j] * 0.15915494309189533577);   // 1 / 2 pi
        double s, co;
        sincospi(2.0 * (turns - __builtin_rint(turns)), &s, &co);
        turn[wave][j] = float2{(float)(p.attention_factor * co), (float)(p.attention_factor * s)};
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");

    const int rotated = half / V, units = p.head_dim / (2 * V);
    const int sub = lane & (group - 1), per = 64 / group;     // heads a wave holds at once
    const int values = append ? p.kv_heads : 0, all = p.heads + p.kv_heads + values;
    for (int h0 = share * per; h0 < all; h0 += shares * per) {
        const int h = h0 + lane / group;
        // where the head comes from and goes to; `to` stays null where there is nothing to write
        const T *from = nullptr, *weight = nullptr;
        T* to = nullptr;
        bool value = false;
        if (h < p.heads) {
            from = (const T*)p.q + row * p.q_row + h * p.q_head;
            to = (T*)p.q_out + row * p.qo_row + h * p.qo_head;
            weight = (const T*)p.q_weight;
        } else if (h < p.heads + p.kv_heads) {
            const int g = h - p.heads;
            from = (const T*)p.k + row * p.k_row + g * p.k_head;
            weight = (const T*)p.k_weight;
            if (!append) to = (T*)p.k_out + row * p.ko_row + g * p.ko_head;
            else if (slot >= 0) to = (T*)c.k + slot + g * c.head_stride;
        } else if (h < all) {
            const int g = h - p.heads - p.kv_heads;
            value = true;
            from = (const T*)p.v + row * p.v_row + g * p.v_head;
            if (slot >= 0) to = (T*)c.v + slot + g * c.head_stride;
        }
        float x[UNITS][2][V];
        int lo[UNITS], hi[UNITS];
        float squares = 0.0f;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = sub + i * group;
            if (u < rotated && p.layout == TTF_ROPE_HALF) {
                lo[i] = u * V;
                hi[i] = half + u * V;
            } else {
                lo[i] = u * 2 * V;
                hi[i] = lo[i] + V;
            }
            if (to && u < units) {
                load_chunk<T, V>(from + lo[i], x[i][0]);
                load_chunk<T, V>(from + hi[i], x[i][1]);
#pragma unroll
                for (int e = 0; e < V; ++e) squares += x[i][0][e] * x[i][0][e] + x[i][1][e] * x[i][1][e];
            }
        }
        for (int m = 1; m < group; m <<= 1) squares += __shfl_xor(squares, m, 64);
        float mean = squares / (float)p.head_dim + p.eps;
        // Squares that overflow, or are so small that they lose bits and eps does not cover them: the head over again, lifted by a power of two
        // (below it all entries are below 2^-46, and 2^100 times as much has squares between 2^-98 and 2^116).  Rare, and the same for the head's lanes.
        if (weight && !(mean >= 0x1p-100f && mean < INFINITY)) {
            const float lift = mean < 0x1p-100f ? 0x1p100f : 0x1p-70f;
            squares = 0.0f;
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                if (!to || sub + i * group >= units) continue;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    x[i][0][e] *= lift;
                    x[i][1][e] *= lift;
                    squares += x[i][0][e] * x[i][0][e] + x[i][1][e] * x[i][1][e];
                }
            }
            for (int m = 1; m < group; m <<= 1) squares += __shfl_xor(squares, m, 64);
            mean = squares / (float)p.head_dim + p.eps * lift * lift;
        }
        const float scale = weight ? 1.0f / sqrtf(mean) : 1.0f;
        if (!to) continue;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) {
            const int u = sub + i * group;
            if (u >= units) continue;
            float (&a)[V] = x[i][0], (&b)[V] = x[i][1];
            if (weight) {
                float w[2][V];
                load_chunk<T, V>(weight + lo[i], w[0]);
                load_chunk<T, V>(weight + hi[i], w[1]);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    a[e] = a[e] * scale * w[0][e];
                    b[e] = b[e] * scale * w[1][e];
                }
            }
            if (u < rotated && !value) {
                const float2* t = turn[wave] + u * V;
                if (p.layout == TTF_ROPE_HALF) {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float y = a[e], z = b[e];
                        a[e] = y * t[e].x - z * t[e].y;
                        b[e] = z * t[e].x + y * t[e].y;
                    }
                } else if constexpr (V == 1) {
                    const float y = a[0], z = b[0];
                    a[0] = y * t[0].x - z * t[0].y;
                    b[0] = z * t[0].x + y * t[0].y;
                } else {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        float y = a[e], z = a[e + 1];
                        float2 r = t[e / 2];
                        a[e] = y * r.x - z * r.y;
                        a[e + 1] = z * r.x + y * r.y;
                        y = b[e];
                        z = b[e + 1];
                        r = t[V / 2 + e / 2];
                        b[e] = y * r.x - z * r.y;
                        b[e + 1] = z * r.x + y * r.y;
                    }
                }
            }
            store_chunk<T, V>(to + lo[i], a);
            store_chunk<T, V>(to + hi[i], b);
        }
    }
}

template <typename T, int V, int UNITS>
hipError_t launch(const ttf_qk_params& p, const ttf_kv_cache* cache, hipStream_t s)
{
    const int units = p.head_dim / (2 * V);
    int group = 1;
    while (group * UNITS < units) group *= 2;
    const int per = 64 / group, all = p.heads + p.kv_heads * (cache ? 2 : 1), rounds = (all + per - 1) / per;
    // Two waves share the heads of a row, more where that leaves the chip empty.  Every one of them forms the angles, but has less to wait for (16
    // clips of up to 3600 rows 115.5 us with one, 115 with two, 125 with four; appended 145, 139, 152).
    int shares = 1;
    while (shares * 2 <= rounds && (shares < 2 || (long long)p.rows * shares < 2048)) shares *= 2;
    const long long waves = (long long)p.rows * shares;
    k_qk<T, V, UNITS><<<(unsigned)((waves + 3) / 4), 256, 0, s>>>(p, cache ? *cache : ttf_kv_cache{}, cache != nullptr, group,
                                                                  shares);
    return hipGetLastError();
}

}  // namespace

// Entries a lane moves at once: 16 bytes where the rotated and the other part of a head are whole units of 2 V entries, so
// that no unit is half rotated and every access is aligned; 4 entries for parts of 8 entries; single entries for the rest.
hipError_t launch_qk(const ttf_qk_params& p, const ttf_kv_cache* cache, hipStream_t s)
{
    const auto whole = [&](int n) { return p.rotary_dim % n == 0 && (p.head_dim - p.rotary_dim) % n == 0; };
    if (p.dtype == TTF_BF16) {
        if (whole(16)) return launch<bf16_t, 8, 1>(p, cache, s);
        if (whole(8)) return launch<bf16_t, 4, 1>(p, cache, s);
        return launch<bf16_t, 1, 2>(p, cache, s);
    }
    if (whole(8)) return launch<float, 4, 1>(p, cache, s);
    return launch<float, 1, 2>(p, cache, s);
}

}  // namespace ttf
