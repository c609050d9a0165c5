// Operators on a paged cache that several sequences live in: rotary append, attention by a rule, page copies.
#include "kernels.h"
#include "device_utils.h"

#include <type_traits>

namespace sb {

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// The newest rows of a sequence and where they stand.
struct SeqRows { int b, r0, n, len; };   // sequence (-1: none), first row, rows, keys

__device__ __forceinline__ int row_at(const PagedKv& kv, int b) { return clampi(kv.row_start[b], 0, kv.n_rows); }

// The sequence of item t, where sequence b owns the items first(r0, b) .. of its first row r0 up to the next sequence's: the last b with
// first(row_start[b], b) <= t, `first` ascending.  64 sequences are looked at at once, a lane each, with all that is asked of them in one
// trip to memory; more are first searched 64 ways at a time.  All lanes of the wave are active, t is uniform.
template <typename First>
__device__ __forceinline__ SeqRows find_rows(const PagedKv& kv, First first, int t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = kv.n_seq;   // the answer is lo .. lo + n - 1 (or none, while lo is 0)
    while (n > 64) {
        const int step = (n + 63) / 64, b = lo + lane * step;
        const int c = __popcll(__builtin_amdgcn_ballot_w64(b < lo + n && first(row_at(kv, b < lo + n ? b : lo), b) <= t));
        if (c == 0) return SeqRows{-1, 0, 0, 0};
        const int end = lo + n;
        lo += (c - 1) * step;
        n = (lo + step < end ? lo + step : end) - lo;
    }
    const int b = lo + (lane < n ? lane : 0);
    const int r0 = row_at(kv, b), r1 = row_at(kv, b + 1), len = clampi(kv.kv_len[b], 0, kv.max_len);
    const int c = __popcll(__builtin_amdgcn_ballot_w64(lane < n && first(r0, b) <= t));
    SeqRows s{-1, 0, 0, 0};
    if (c == 0) return s;
    s.r0 = __builtin_amdgcn_readlane(r0, c - 1);
    s.n = __builtin_amdgcn_readlane(r1, c - 1) - s.r0;
    s.len = __builtin_amdgcn_readlane(len, c - 1);
    s.b = s.n > 0 ? lo + c - 1 : -1;
    return s;
}

__device__ __forceinline__ uint16_t round_bf16(float v) { return (uint16_t)pack_bf16(v, v); }   // (NaN stays one)
__device__ __forceinline__ void store_x(void* x, int64_t i, bool fp32, float v) {
    if (fp32) reinterpret_cast<float*>(x)[i] = v;
    else reinterpret_cast<uint16_t*>(x)[i] = round_bf16(v);
}

// ---------------------------------------------------------------- rotary append
// Four neighbouring values of a row.
__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
// The same of rows that are read once: past the caches' usual replacement (8100 rows of 48 heads 51 -> 47 us).
typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void load_row4(const float* p, float (&x)[4]) {
    const f32x4v v = __builtin_nontemporal_load(reinterpret_cast<const f32x4v*>(p));
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void load_row4(const uint16_t* p, float (&x)[4]) {
    const u32x2v v = __builtin_nontemporal_load(reinterpret_cast<const u32x2v*>(p));
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4]) { *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]); }
__device__ __forceinline__ void store4(uint16_t* p, const float (&x)[4]) { *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])); }
// Two, rounded to a pair of bf16.
__device__ __forceinline__ uint32_t load_pair(const float* p) {
    const float2 v = *reinterpret_cast<const float2*>(p);
    return pack_bf16(v.x, v.y);
}
__device__ __forceinline__ uint32_t load_pair(const uint16_t* p) { return *reinterpret_cast<const uint32_t*>(p); }

// A block takes the new rows of one page of one sequence (16 at most) and, by blockIdx.y, some of the heads: ROPE_QK q and k
// heads, or ROPE_V v heads.  Sequence b's pages are tiles row_start[b] / 16 + 2 b .., as many as its rows can touch.
//   q and k: HD / 8 lanes a head, eight values a lane -- the two ends of four pairs, so that norm and rotation stay within
// the lane but for the sum of squares; ROPE_U heads a thread in flight.
//   v: a thread takes two dims and eight slots, which leave as 16-byte pieces of the transposed slab; where not all eight are new, the
// others are read and written back (stored by two bytes, 220 rows in 48 sequences of 32 v heads took 13.0 us, so 10.4; 5.8
// without v: two pages a sequence are touched all over for them).
constexpr int ROPE_U = 2;

template <int HD, typename XT>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeAppendArgs a, int qk_heads, int qk_slices) {
    constexpr int ROPE_V = 256 / HD;   // v heads of a block: one item a thread
    const int tid = threadIdx.x, Hq = a.n_heads, Hkv = a.kv.n_kv_heads, rot = a.rot_dim, half = rot / 2;
    const int t = blockIdx.x;
    const SeqRows s = find_rows(a.kv, [](int r0, int b) { return r0 / SB_KV_BLOCK + 2 * b; }, t);
    if (s.b < 0) return;
    const int pos0 = s.len - s.n, from = pos0 > 0 ? pos0 : 0;
    const int page = from / SB_KV_BLOCK + t - (s.r0 / SB_KV_BLOCK + 2 * s.b);
    const int lo = page * SB_KV_BLOCK > from ? page * SB_KV_BLOCK : from;
    int hi = (page + 1) * SB_KV_BLOCK < s.len ? (page + 1) * SB_KV_BLOCK : s.len;
    if (rot && hi > a.n_pos) hi = a.n_pos;
    if (lo >= hi) return;
    const int nr = hi - lo, row0 = s.r0 + lo - pos0;   // rows row0 .. at positions lo ..
    const int pg = a.kv.table[(int64_t)s.b * a.kv.table_ld + page];
    const bool in_pool = pg >= 0 && pg < a.kv.n_pages;
    const XT* const x = reinterpret_cast<const XT*>(a.qkv);
    const int64_t slab = (int64_t)(in_pool ? pg : 0) * Hkv * SB_KV_BLOCK * HD;

    if ((int)blockIdx.y < qk_slices) {
        constexpr int L = HD / 8, SIDE = 256 / L;
        const int c = tid % L, h0 = blockIdx.y * qk_heads;
        const int nh = Hq + Hkv - h0 < qk_heads ? Hq + Hkv - h0 : qk_heads, n = nr * nh;
        const bool turns = c < rot / 8;
        const int dA = a.interleaved ? 8 * c : turns ? 4 * c : rot + 8 * (c - rot / 8);
        const int dB = a.interleaved || !turns ? dA + 4 : dA + half;
        for (int i0 = tid / L; i0 < n; i0 += SIDE * ROPE_U) {
            float u[ROPE_U][2][4];
            int head[ROPE_U], r[ROPE_U];
#pragma unroll
            for (int k = 0; k < ROPE_U; ++k) {   // (past the end: the last one again, not stored)
                const int i = i0 + k * SIDE < n ? i0 + k * SIDE : n - 1;
                r[k] = i / nh;
                head[k] = h0 + i - r[k] * nh;
                const XT* p = x + (row0 + r[k]) * a.ld_qkv + head[k] * HD;
                load_row4(p + dA, u[k][0]);
                load_row4(p + dB, u[k][1]);
            }
#pragma unroll
            for (int k = 0; k < ROPE_U; ++k) {
                float (&A)[4] = u[k][0], (&B)[4] = u[k][1];
                const bool is_q = head[k] < Hq;
                const float* gain = is_q ? a.q_gain : a.k_gain;
                if (a.q_gain || a.k_gain) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) ss += A[e] * A[e] + B[e] * B[e];
                    ss = lanes_sum<L / 2>(ss);
                    if (gain) {
                        const float inv = 1.0f / sqrtf(ss * (1.0f / HD) + a.eps);
                        float ga[4], gb[4];
                        load4(gain + dA, ga);
                        load4(gain + dB, gb);
#pragma unroll
                        for (int e = 0; e < 4; ++e) { A[e] = A[e] * inv * ga[e]; B[e] = B[e] * inv * gb[e]; }
                    }
                }
                if (turns) {
                    float cs[4], sn[4];
                    load4(a.cos + (int64_t)(lo + r[k]) * half + 4 * c, cs);
                    load4(a.sin + (int64_t)(lo + r[k]) * half + 4 * c, sn);
                    if (a.interleaved) {   // pairs are neighbours: (A0, A1), (A2, A3), (B0, B1), (B2, B3)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const float a0 = A[e], a1 = A[e + 1], b0 = B[e], b1 = B[e + 1];
                            A[e] = a0 * cs[e / 2] - a1 * sn[e / 2]; A[e + 1] = a1 * cs[e / 2] + a0 * sn[e / 2];
                            B[e] = b0 * cs[2 + e / 2] - b1 * sn[2 + e / 2]; B[e + 1] = b1 * cs[2 + e / 2] + b0 * sn[2 + e / 2];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float v = A[e], w = B[e];
                            A[e] = v * cs[e] - w * sn[e];
                            B[e] = w * cs[e] + v * sn[e];
                        }
                    }
                }
                if (i0 + k * SIDE >= n) continue;
                if (is_q) {
                    XT* p = reinterpret_cast<XT*>(a.q_out) + (row0 + r[k]) * a.ld_q + head[k] * HD;
                    store4(p + dA, A);
                    store4(p + dB, B);
                } else if (in_pool) {
                    uint16_t* p = a.kv.k + slab + ((head[k] - Hq) * SB_KV_BLOCK + (lo + r[k]) % SB_KV_BLOCK) * HD;
                    store4(p + dA, A);
                    store4(p + dB, B);
                }
            }
        }
        return;
    }
    if (!in_pool) return;
    const int g = (blockIdx.y - qk_slices) * ROPE_V + tid / HD, d = tid % HD & ~1, t0 = (tid & 1) * 8;
    const int s_lo = lo % SB_KV_BLOCK, s_hi = s_lo + nr;   // new slots of the page
    if (g >= Hkv || t0 >= s_hi || t0 + 8 <= s_lo) return;
    const XT* p = x + (Hq + Hkv + g) * HD + d;
    uint32_t w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {   // (no condition, so the eight go out together)
        const int sl = t0 + e < s_lo ? s_lo : t0 + e < s_hi ? t0 + e : s_hi - 1;
        w[e] = load_pair(p + (row0 + sl - s_lo) * a.ld_qkv);
    }
    uint16_t* dst = a.kv.v + slab + (g * HD + d) * SB_KV_BLOCK + t0;
    if (t0 >= s_lo && t0 + 8 <= s_hi) {
        uint32_t lo2[4], hi2[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo2[e] = (w[2 * e] & 0xffffu) | (w[2 * e + 1] << 16);
            hi2[e] = (w[2 * e] >> 16) | (w[2 * e + 1] & 0xffff0000u);
        }
        *reinterpret_cast<uint4*>(dst) = make_uint4(lo2[0], lo2[1], lo2[2], lo2[3]);
        *reinterpret_cast<uint4*>(dst + SB_KV_BLOCK) = make_uint4(hi2[0], hi2[1], hi2[2], hi2[3]);
    } else {
        const uint4 a0 = *reinterpret_cast<const uint4*>(dst), a1 = *reinterpret_cast<const uint4*>(dst + SB_KV_BLOCK);
        uint32_t x0[4] = {a0.x, a0.y, a0.z, a0.w}, x1[4] = {a1.x, a1.y, a1.z, a1.w};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (t0 + e >= s_lo && t0 + e < s_hi) {
                const int sh = (e & 1) * 16;
                x0[e >> 1] = (x0[e >> 1] & ~(0xffffu << sh)) | ((w[e] & 0xffffu) << sh);
                x1[e >> 1] = (x1[e >> 1] & ~(0xffffu << sh)) | ((w[e] >> 16) << sh);
            }
        *reinterpret_cast<uint4*>(dst) = make_uint4(x0[0], x0[1], x0[2], x0[3]);
        *reinterpret_cast<uint4*>(dst + SB_KV_BLOCK) = make_uint4(x1[0], x1[1], x1[2], x1[3]);
    }
}

hipError_t launch_rope_append(const RopeAppendArgs& a, hipStream_t st) {
    // q and k heads of a block: about ROPE_U a thread (16 threads a head of 128) for as many rows as a page gets on average.
    const int64_t rows = a.kv.n_rows / a.kv.n_seq;
    const int qk_heads = rows >= 8 ? 4 : rows >= 3 ? 8 : 16, v_heads = 256 / a.kv.head_dim;
    const int qk = (a.n_heads + a.kv.n_kv_heads + qk_heads - 1) / qk_heads, v = (a.kv.n_kv_heads + v_heads - 1) / v_heads;
    const dim3 grid(a.kv.n_rows / SB_KV_BLOCK + 2 * a.kv.n_seq, qk + v);
    const auto go = [&](auto hd_c) {
        constexpr int HD = decltype(hd_c)::value;
        return launch(a.x_dtype == SB_FP32 ? &rope_append_kernel<HD, float> : &rope_append_kernel<HD, uint16_t>, grid, 256, st, a, qk_heads, qk);
    };
    return a.kv.head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

// ---------------------------------------------------------------- attention
// out = sum_k 2^(s_k - m) v_k / sum_k 2^(s_k - m) over the keys k that a row sees, s_k its scores in units of log 2, in one pass over the
// keys: o and l, the two sums so far, are scaled by 2^(m - m') when the reference point moves from m to m'.  Both products are
// 32x32x16 matrix instructions, S^T = K Q^T and O^T = V^T P^T: a lane holds 16 scores of one query, its maximum and sum need one exchange
// between the halves of the wave, and with the keys of a tile in the order of reg_key (bits 2 and 3 of a tile's rows swapped when K is
// read) what comes out of the first product is the right operand of the second as it stands.  Float rows go through
// the same instructions as three bf16 parts (8 + 8 + 8 bits: all of theirs), keys and values have bf16 already.
//   Two forms: blocks of 32 queries that read keys straight into registers, bound by memory (decode, verification, short prompts), and
// blocks of 128 queries that share staged keys, bound by exponentials and matrix instructions (prompts); attn_plan chooses.
// Keys that a row sees: a0 .. a1 - 1 (of the prefix) and b0 .. b1 - 1 (of its own past).
struct Sees { int a0, a1, b0, b1; };
__device__ __forceinline__ Sees row_sees(const PagedAttnArgs& a, const SeqRows& s, int row, int pos) {
    Sees v;
    v.a0 = v.b0 = a.doc_start ? clampi(a.doc_start[row], 0, s.len) : 0;
    v.a1 = a.prefix_len ? clampi(a.prefix_len[s.b], 0, s.len) : 0;
    v.b1 = clampi(pos + 1, 0, s.len);
    if (a.window > 0 && pos + 1 - a.window > v.b0) v.b0 = pos + 1 - a.window;
    return v;
}

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef uint16_t u16x2v __attribute__((ext_vector_type(2)));
constexpr float LOG2E = 1.4426950408889634f;

// least / largest over the 32 lanes of a half wave
template <int O = 16>
__device__ __forceinline__ int half_min(int v) {
    uint32_t x, y;
    lane_pair<O>((uint32_t)v, x, y);
    const int m = (int)x < (int)y ? (int)x : (int)y;
    if constexpr (O > 1) return half_min<O / 2>(m);
    else return __builtin_amdgcn_readfirstlane(m);
}
__device__ __forceinline__ int half_max(int v) { return -half_min(-v); }

// Query tiles of TQ (row, head of the group) pairs each, by sequence: sequence b's tiles start at row_start[b] G / TQ + b, which
// leaves each at least as many as it needs whatever the row counts are (a tile past them has no query).
template <int TQ>
__device__ __forceinline__ SeqRows tile_seq(const PagedAttnArgs& a, int t, int& q0) {
    const int G = a.group;
    SeqRows s = find_rows(a.kv, [G](int r0, int b) { return r0 * G / TQ + b; }, t);
    q0 = 0;
    if (s.b >= 0) {
        q0 = (t - (s.r0 * G / TQ + s.b)) * TQ;
        if ((unsigned)q0 >= (unsigned)(s.n * G)) s.b = -1;   // (below 0: only where row_start does not ascend)
    }
    return s;
}

// Sum over the wave, a scalar.
template <int O = 32>
__device__ __forceinline__ int wave_total(int v) {
    uint32_t x, y;
    lane_pair<O>((uint32_t)v, x, y);
    if constexpr (O > 1) return wave_total<O / 2>((int)(x + y));
    else return __builtin_amdgcn_readfirstlane((int)(x + y));
}
// The p-th longest tile of TQ queries among 64 R sequences at most, R a lane: a tile's length is its sequence's past, in tiles, and its number there,
// so sequence b has tiles of lengths B_b .. B_b + c_b - 1; `lo` ends as the largest length that more than p tiles reach.
template <int TQ, int R>
__device__ __forceinline__ SeqRows tile_by_length(const PagedAttnArgs& a, int p, int& q0) {
    const int lane = threadIdx.x & 63;
    int r0[R], n[R], len[R], c[R], B[R];
    int all = 0, least = 0x7fffffff, most = 0;
#pragma unroll
    for (int u = 0; u < R; ++u) {
        const int b = 64 * u + lane < a.kv.n_seq ? 64 * u + lane : 0;
        const int r1 = row_at(a.kv, b + 1);
        r0[u] = row_at(a.kv, b);
        len[u] = clampi(a.kv.kv_len[b], 0, a.kv.max_len);
        n[u] = 64 * u + lane < a.kv.n_seq && r1 > r0[u] ? r1 - r0[u] : 0;
    }
#pragma unroll
    for (int u = 0; u < R; ++u) {
        c[u] = (n[u] * a.group + TQ - 1) / TQ;
        const int64_t past = (int64_t)(len[u] > n[u] ? len[u] - n[u] : 0) * a.group / TQ;
        B[u] = past < (1 << 28) ? (int)past : 1 << 28;
        all += c[u];
        if (c[u] && B[u] < least) least = B[u];
        if (c[u] && B[u] + c[u] > most) most = B[u] + c[u];
    }
    const auto reach = [&](int x) {
        int v = 0;
#pragma unroll
        for (int u = 0; u < R; ++u) v += clampi(B[u] + c[u] - x, 0, c[u]);
        return wave_total(v);
    };
    SeqRows s{-1, 0, 0, 0};
    q0 = 0;
    if (p >= wave_total(all)) return s;
    int lo = half_min<32>(least), hi = -half_min<32>(-most);   // reach(lo) > p >= reach(hi)
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (reach(mid) > p) lo = mid;
        else hi = mid;
    }
    int nth = p - reach(lo + 1);   // among the sequences that have a tile of this length
#pragma unroll
    for (int u = 0; u < R; ++u) {
        const bool has = B[u] <= lo && lo < B[u] + c[u];
        const uint64_t have = __builtin_amdgcn_ballot_w64(has);
        const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(have >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)have, 0));
        const uint64_t it = __builtin_amdgcn_ballot_w64(has && before == nth);
        nth -= __popcll(have);
        if (it == 0) continue;
        const int l = __builtin_ctzll(it);
        s.b = 64 * u + l;
        s.r0 = __builtin_amdgcn_readlane(r0[u], l);
        s.n = __builtin_amdgcn_readlane(n[u], l);
        s.len = __builtin_amdgcn_readlane(len[u], l);
        q0 = (lo - __builtin_amdgcn_readlane(B[u], l)) * TQ;
    }
    return s;
}
// Tile t of a call: longest first where there are LEAST sequences or more (256 at most: every block sorts them, 0.6 to 1.2 us) that may be long, else as they
// lie.  As they lie / longest first, us: one row each of 64 sequences of up to 8000 keys 255 / 240, 3000 108 / 92, 500 21.7 / 20.4, 200 13.6 / 14.1, of 16 of up
// to 3000 40.7 / 41.8, of 128 of up to 3000 191 / 176, 100 17.9 / 19.7; five capped float prompts 89 / 82, five of 100 to 2000 bf16 rows 62 / 56; 10 to 100 rows
// of 80 sequences behind up to 1500 139 / 116, up to 200 rows of 100 with no past 71 / 78.
template <int TQ, int LEAST, bool LAST_FIRST>
__device__ __forceinline__ SeqRows tile_of(const PagedAttnArgs& a, int t, int tiles, int& q0) {
    if (a.kv.n_seq >= LEAST && a.kv.max_len >= 512) {
        if (a.kv.n_seq <= 64) return tile_by_length<TQ, 1>(a, t, q0);
        if (a.kv.n_seq <= 256) return tile_by_length<TQ, 4>(a, t, q0);
    }
    return tile_seq<TQ>(a, LAST_FIRST ? tiles - 1 - t : t, q0);
}

// Row of query qq of a sequence (heads of one kv head's group per row).
__device__ __forceinline__ int row_of(const PagedAttnArgs& a, int qq) { return a.group_shift >= 0 ? qq >> a.group_shift : qq / a.group; }

// A lane's query: where it is, and the keys that it sees as two ranges [a0, a0 + an), [b0, b0 + bn).
struct Query {
    int row, head, pos, a0, b0;
    uint32_t an, bn;
    bool valid;
    float slope2;   // in units of log 2
};
// What all 32 queries of a wave see (whole ranges), and bounds of what any of them does; scalars.
struct Reach { int a_lo, a_hi, b_lo, b_hi, a0_max, a1_min, b0_max, b1_min; };

// Of query qw + lane % 32 of the sequence; qw is the wave's first, uniform.
__device__ __forceinline__ Query lane_query(const PagedAttnArgs& a, const SeqRows& s, int g, int qw, int li, Reach& w) {
    Query q;
    const int G = a.group, qq = qw + li, nq = s.n * G, r = row_of(a, qq);
    q.valid = qq < nq;
    q.row = s.r0 + (q.valid ? r : 0);
    q.head = g * G + (q.valid ? qq - r * G : 0);
    q.pos = s.len - s.n + q.row - s.r0;
    const Sees v = row_sees(a, s, q.row, q.pos);
    q.a0 = v.a0; q.b0 = v.b0;
    q.an = q.valid && v.a1 > v.a0 ? v.a1 - v.a0 : 0;
    q.bn = q.valid && v.b1 > v.b0 ? v.b1 - v.b0 : 0;
    q.slope2 = a.slopes ? a.slopes[q.head] * LOG2E : 0.f;
    const int big = 0x7fffffff;
    if (a.doc_start) {
        w.a_lo = half_min(q.an ? v.a0 : big); w.a_hi = half_max(q.an ? v.a1 : 0);
        w.b_lo = half_min(q.bn ? v.b0 : big); w.b_hi = half_max(q.bn ? v.b1 : 0);
        w.a0_max = half_max(q.valid ? v.a0 : 0); w.a1_min = half_min(q.valid ? v.a1 : big);
        w.b0_max = half_max(q.valid ? v.b0 : 0); w.b1_min = half_min(q.valid ? v.b1 : big);
    } else {   // without documents the first and the last row tell (eight reductions over the lanes less)
        const bool any = qw < nq;
        const int last = s.len - s.n + row_of(a, qw + 31 < nq ? qw + 31 : nq - 1), first = s.len - s.n + row_of(a, qw);
        const int pre = a.prefix_len ? clampi(a.prefix_len[s.b], 0, s.len) : 0, win = a.window > 0 ? a.window : big;
        const auto from = [&](int p) { return p >= win ? p + 1 - win : 0; };
        w.a_lo = any && pre ? 0 : big; w.a_hi = any ? pre : 0;
        w.b_lo = any && last >= 0 ? from(first) : big; w.b_hi = any && last >= 0 ? last + 1 : 0;
        w.a0_max = 0; w.a1_min = any ? pre : big;
        w.b0_max = any ? from(last) : 0; w.b1_min = any ? (first >= 0 ? first + 1 : 0) : big;
    }
    return q;
}
__device__ __forceinline__ bool all_see(const Reach& w, int k0, int k1) {   // keys k0 .. k1 - 1, every query
    return (w.b0_max <= k0 && k1 <= w.b1_min) || (w.a0_max <= k0 && k1 <= w.a1_min);
}
__device__ __forceinline__ bool some_see(const Reach& w, int k0, int k1) {
    return (k0 < w.b_hi && k1 > w.b_lo) || (k0 < w.a_hi && k1 > w.a_lo);
}

// The steps of C keys that hold a key which some query sees, in ascending order: two runs of them (prefix, own past), one
// where they touch.
struct Steps {
    int s1, n1, s2, n;
    __device__ __forceinline__ int at(int i) const { return i < n1 ? s1 + i : s2 + i - n1; }
};
template <int C>
__device__ __forceinline__ Steps steps_of(const Reach& w) {
    const int sa = w.a_hi > 0 ? w.a_lo / C : 0, ea = w.a_hi > 0 ? (w.a_hi + C - 1) / C : 0;
    const int sb = w.b_hi > 0 ? w.b_lo / C : 0, eb = w.b_hi > 0 ? (w.b_hi + C - 1) / C : 0;
    Steps t;
    if (ea == 0) { t.s1 = sb; t.n1 = t.n = eb - sb; t.s2 = 0; return t; }
    if (eb == 0) { t.s1 = sa; t.n1 = t.n = ea - sa; t.s2 = 0; return t; }
    if (sb <= ea && sa <= eb) {   // they overlap or touch
        t.s1 = sa < sb ? sa : sb;
        t.n1 = t.n = (ea > eb ? ea : eb) - t.s1;
        t.s2 = 0;
        return t;
    }
    const bool first = ea < sb;
    t.s1 = first ? sa : sb; t.n1 = first ? ea - sa : eb - sb;
    t.s2 = first ? sb : sa; t.n = t.n1 + (first ? eb - sb : ea - sa);
    return t;
}

// Eight floats as PARTS bf16 operands: with three, all of their 24 bits (8 + 8 + 8).
template <int PARTS>
__device__ __forceinline__ void split8(float4 x, float4 y, bf16x8 (&op)[PARTS]) {
    float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[e] = pack_bf16(f[2 * e], f[2 * e + 1]);
            f[2 * e] -= __uint_as_float(w[e] << 16);
            f[2 * e + 1] -= __uint_as_float(w[e] & 0xffff0000u);
        }
        op[i] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}
// Register r of a key tile's scores in lane (li, lh): query li, key key0 + 16 (r / 8) + 8 lh + r % 8.
__device__ __forceinline__ int reg_key(int r) { return (r >> 3) * 16 + (r & 7); }

// A capped score c2 tanh(s k), in units of log 2, to a few units in the last place.  Where |s k| < 0.3 it is z (1 + y (a1 + y (a2 + y a3))), y = (s k)^2, z = c2 k s: the
// polynomial of this form nearest to tanh x / x there (1.3e-8 of it), its coefficients times powers of k^2, so that s k itself is not needed; else
// 1 - 2 / (exp(2 |s k|) + 1).  A score's bits do not depend on the scores beside it.
struct Cap {
    float k, c2, z, b1, b2, b3;
    __device__ __forceinline__ Cap(float k_, float c2_) : k(k_), c2(c2_), z(k_ * c2_) {
        const float kk = k * k;
        b1 = -0.33333060f * kk; b2 = 0.13314833f * (kk * kk); b3 = -0.050366241f * (kk * kk * kk);
    }
    __device__ __forceinline__ float low(float s) const {
        const float y = s * s, w = s * z;
        return fmaf(w * y, fmaf(y, fmaf(y, b3, b2), b1), w);
    }
    __device__ __forceinline__ float any(float s) const {
        const float x = fabsf(s) * k;
        const float e = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (2.f * LOG2E)) + 1.f), 1.f);
        return x < 0.3f ? low(s) : copysignf(c2 * e, s);
    }
};
// Cap and bias, where there are any: scores in units of log 2 then, raw products else.
template <int PARTS, int KT, bool SHAPED>
__device__ __forceinline__ void shape_scores(const PagedAttnArgs& a, const Query& q, int key0, int lh, f32x16 (&st)[KT]) {
    if constexpr (!SHAPED) return;
    if (a.cap > 0.f) {
        const float c2 = a.cap * LOG2E;
        if (PARTS == 1 && a.cap <= 512.f) {   // tanh x = 1 - 2 / (exp 2x + 1): 2e-7 off at most, so a score of bf16 rows 1e-4
            const float k = 2.f * LOG2E * a.scale / a.cap;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    st[t][r] = fmaf(-2.f * c2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(st[t][r] * k) + 1.f), c2);
        } else {   // (mostly all scores of a tile are far below the cap, where the polynomial alone does)
            float k = a.scale / a.cap;
            if (k < 1e-3f) {   // (k^6 and the squares of such scores leave float's range)
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) st[t][r] *= k;
                k = 1.f;
            }
            const Cap cap(k, c2);
            float top = 0.f;
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = __builtin_elementwise_maximum(top, fabsf(st[t][r]));
            if (__builtin_amdgcn_ballot_w64(!(top * cap.k < 0.3f)) == 0) {
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) st[t][r] = cap.low(st[t][r]);
            } else {
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) st[t][r] = cap.any(st[t][r]);
            }
        }
    } else if (a.slopes) {
        const float c2 = a.scale * LOG2E;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[t][r] *= c2;
    }
    if (a.slopes) {
        const float d0 = (float)(q.pos - key0 - 8 * lh);
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[t][r] = fmaf(-q.slope2, fabsf(d0 - (float)(32 * t + reg_key(r))), st[t][r]);
    }
}
__device__ __forceinline__ float score_mul(const PagedAttnArgs& a) { return a.cap > 0.f || a.slopes ? 1.f : a.scale * LOG2E; }

template <int KT>
__device__ __forceinline__ void mask_scores(const Query& q, const Reach& w, int key0, int lh, f32x16 (&st)[KT]) {
    const uint32_t db = (uint32_t)(key0 + 8 * lh - q.b0), da = (uint32_t)(key0 + 8 * lh - q.a0);
    if (w.a_hi == 0) {   // (no query of the wave has a prefix)
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (db + (uint32_t)(32 * t + reg_key(r)) >= q.bn) st[t][r] = -SB_INF;
    } else {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t k = 32 * t + reg_key(r);
                if (db + k >= q.bn && da + k >= q.an) st[t][r] = -SB_INF;
            }
    }
}

// Running soft-max over KT key tiles of this lane's query (what it does not see is -inf): exponentials as PARTS bf16 B operands
// of 16 keys each, this lane's part of their sum (of the float values), the output rescaled where needed.  The reference
// point follows the maximum only when that has grown by more than 2^8 (any reference gives the same quotient).
template <int PARTS, int KT, int DT>
__device__ __forceinline__ void soft_max(f32x16 (&st)[KT], float mul, f32x16 (&o)[DT], float& m_run, float& l_run, bf16x8 (&p)[PARTS][2 * KT]) {
    float mx = -SB_INF;   // (the maximum that a NaN passes through: fmaxf first multiplies every score by 1 to quiet it)
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int r = 0; r < 16; r += 2) mx = __builtin_elementwise_maximum(mx, __builtin_elementwise_maximum(st[kt][r], st[kt][r + 1]));
    mx = lanes_max<32, 32>(mx) * mul;
    const float m_new = mx > m_run + 8.0f ? mx : m_run;
    const bool large = fabsf(mx) > 1e6f && mx != -SB_INF;
    if (__builtin_amdgcn_ballot_w64(large) != 0) {
        // (the reference point is a rounded product, and the exponents below are not: with such scores they would be far from 0 at the maximum)
        const float f = large ? mul : 1.f;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[kt][r] *= f;
        mul = large ? 1.f : mul;
    }
    if (__builtin_amdgcn_ballot_w64(m_new != m_run) != 0) {
        const float alpha = m_new == m_run ? 1.0f : __builtin_amdgcn_exp2f(m_run - m_new);
        l_run *= alpha;
        m_run = m_new;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[dt][r] *= alpha;
    }
    const float ref = m_new == -SB_INF ? 0.f : m_new;   // (nothing seen so far)
    float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
    for (int s = 0; s < KT * 2; ++s) {
        uint32_t w[PARTS][4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float p0 = __builtin_amdgcn_exp2f(fmaf(st[s >> 1][(s & 1) * 8 + 2 * e], mul, -ref));
            float p1 = __builtin_amdgcn_exp2f(fmaf(st[s >> 1][(s & 1) * 8 + 2 * e + 1], mul, -ref));
            sum0 += p0;
            sum1 += p1;
#pragma unroll
            for (int i = 0; i < PARTS; ++i) {
                w[i][e] = pack_bf16(p0, p1);
                p0 -= __uint_as_float(w[i][e] << 16);
                p1 -= __uint_as_float(w[i][e] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int i = 0; i < PARTS; ++i) p[i][s] = __builtin_bit_cast(bf16x8, make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]));
    }
    l_run += sum0 + sum1;
}

// Mask of the first n of eight bf16 values (n < 0: none, n > 8: all).
__device__ __forceinline__ uint4 first_keys(int n) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = n > 2 * e + 1 ? 0xffffffffu : n > 2 * e ? 0xffffu : 0u;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Among eight bf16 values an infinity or NaN is one with all exponent bits set: the largest magnitudes so far, pairwise.
__device__ __forceinline__ void most(uint4 v, u16x2v& top) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2v, w[e] & 0x7fff7fffu));
}
__device__ __forceinline__ bool not_finite(u16x2v top) { return __builtin_amdgcn_ballot_w64(top.x >= 0x7f80 || top.y >= 0x7f80) != 0; }

// Where some value is infinite or NaN and not every query sees its key, the product must not be taken as it is (0 x NaN is not 0):
// the value becomes zero, and the largest float stands in `bad` for it (zero for all others).  bad x sight, with the largest
// float in `sight` for the keys that a query sees, is infinite for the queries that see the value and zero for the others.
__device__ __forceinline__ void set_apart(uint4& v, uint4& bad) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w}, n[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        n[e] = ((w[e] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w[e] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
        w[e] &= ~n[e];
        n[e] &= 0x7f7f7f7fu;
    }
    v = make_uint4(w[0], w[1], w[2], w[3]);
    bad = make_uint4(n[0], n[1], n[2], n[3]);
}
__device__ __forceinline__ bf16x8 sight(const Query& q, int key) {   // of keys key .. key + 7
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t k = key + e;
        if (k - q.b0 < q.bn || k - q.a0 < q.an) w[e >> 1] |= e & 1 ? 0x7f7f0000u : 0x7f7fu;
    }
    return __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
}

template <int HD>
__device__ __forceinline__ void store_out4(const PagedAttnArgs& a, const Query& q, int col, float4 v) {
    const int64_t at = (int64_t)q.row * a.ld_out + q.head * HD + col;
    if (a.x_dtype == SB_FP32) *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = v;
    else *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + at) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// Partial results of a (row, head) pair's key chunks, where the key axis is split over blocks: outputs, then {reference point,
// sum}, then the number of chunks.
struct Partials {
    float *o, *ml;
    int* count;
    __host__ __device__ Partials(float* scratch, int64_t pairs, int chunks, int hd) {
        o = scratch;
        ml = o + pairs * chunks * hd;
        count = reinterpret_cast<int*>(ml + pairs * chunks * 2);
    }
    static size_t bytes(int64_t pairs, int chunks, int hd) { return ((size_t)pairs * chunks * (hd + 2) + pairs) * 4; }
};

// A block owns 32 queries of one kv head and (blockIdx.y) `steps_per_chunk` of the 32-key steps that they see; its four waves take the steps in
// turn with a running soft-max each, operands straight from the cache into registers, the next step's keys requested when
// this step's scores are done and its values when its products are; the waves' results are added in wave order through LDS.
//   Bound by the cache's bytes: six float rows of 32 heads behind 131000 keys of 8 heads (537 MB) 103 us, 5.2 TB/s; 64 bf16 rows behind 4400
// keys each on average (1.14 GB) 226 us, 5.0 TB/s (5.2 to 5.5 where all are equally long: the last blocks end apart); matrix instructions
// take 20 % of the float rows' cycles.  A short context is a chain of trips: 520 keys 9 to 10 us, of which the keys are 2.
// Four waves a block and two blocks a CU: eight steps in flight hide a trip; 8 waves on one chunk took 15.7 us for 520 keys, four and a join 13.9.
template <int HD, int PARTS>
__global__ __launch_bounds__(256, 2) void paged_attn_apart_kernel(PagedAttnArgs a, int steps_per_chunk) {
    constexpr int W = 4, KS = HD / 16, DT = HD / 32, SLAB = SB_KV_BLOCK * HD, NS = DT * 4;
    __shared__ __attribute__((aligned(16))) float o_s[W][NS][64][4];
    __shared__ float m_s[W][32], l_s[W][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int li = lane & 31, lh = lane >> 5;
    const int Hkv = a.kv.n_kv_heads, g = blockIdx.x % Hkv;
    int q0;
    const SeqRows s = tile_of<32, 32, false>(a, blockIdx.x / Hkv, gridDim.x / Hkv, q0);
    if (s.b < 0) return;
    Reach w;
    const Query q = lane_query(a, s, g, q0, li, w);
    const Steps steps = steps_of<32>(w);
    const bool split = gridDim.y > 1;
    const Partials part(a.scratch, (int64_t)a.kv.n_rows * a.n_heads, gridDim.y, HD);
    const int64_t pair = (int64_t)q.row * a.n_heads + q.head;
    const int first = blockIdx.y * steps_per_chunk;
    if (split && blockIdx.y == 0 && wave == 0 && lh == 0 && q.valid) part.count[pair] = (steps.n + steps_per_chunk - 1) / steps_per_chunk;
    if (first >= steps.n && (split || blockIdx.y > 0)) return;
    const int last = first + steps_per_chunk < steps.n ? first + steps_per_chunk : steps.n;

    const int64_t page_elems = (int64_t)Hkv * SLAB;
    const uint16_t* const kbase = a.kv.k + (int64_t)g * SLAB;
    const uint16_t* const vbase = a.kv.v + (int64_t)g * SLAB;
    const int32_t* const table = a.kv.table + (int64_t)s.b * a.kv.table_ld;
    const int krow = (li & 19) | ((li & 4) << 1) | ((li & 8) >> 1);   // row li of a tile is key krow of it
    const uint32_t koff = (uint32_t)((krow & 15) * HD + lh * 8), voff = (uint32_t)(li * SB_KV_BLOCK + lh * 8);
    uint4 kr[KS], vr[2][DT];
    int pg0 = 0, pg1 = 0;   // pages of the step whose operands are requested next; -1: none (nothing is read, zeros)
    auto lookup = [&](int i) {
        const int t = steps.at(i);
        pg0 = table[2 * t];
        pg1 = (2 * t + 1) * SB_KV_BLOCK < s.len ? table[2 * t + 1] : -1;
        if (pg0 >= a.kv.n_pages) pg0 = -1;
        if (pg1 >= a.kv.n_pages) pg1 = -1;
    };
    auto load_k = [&]() {
        const int pg = li & 16 ? pg1 : pg0;
        const uint16_t* p = kbase + (pg < 0 ? 0 : pg) * page_elems + koff;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kr[ks] = *reinterpret_cast<const uint4*>(p + ks * 16);
    };
    auto load_v = [&](int p0, int p1) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int pg = x ? p1 : p0;
            const uint16_t* p = vbase + (pg < 0 ? 0 : pg) * page_elems + voff;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) vr[x][dt] = *reinterpret_cast<const uint4*>(p + dt * 32 * SB_KV_BLOCK);
        }
    };
    // The queries: bf16 rows in registers; the three parts of float rows in LDS, made once for the four waves (in registers they would leave
    // one block per CU), where the results go later.  They are requested before the first keys, so that they are not waited for behind them.
    constexpr int NQ = PARTS == 1 ? KS : HD / 64;
    bf16x8 qo[KS];
    float4 qf[NQ][2];
    bf16x8* const q_s = reinterpret_cast<bf16x8*>(&o_s[0][0][0][0]);   // [PARTS][KS][64 lanes]
    static_assert(PARTS * KS * 64 * 16 <= (int)sizeof(o_s), "the queries fit where the results go");
    if constexpr (PARTS == 1) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            qo[ks] = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const uint16_t*>(a.q) + (int64_t)q.row * a.ld_q + q.head * HD + lh * 8 + ks * 16);
    } else {
        const int x = tid / 8, qq = q0 + x < s.n * a.group ? q0 + x : q0, r = row_of(a, qq);   // (past the end: the first one, not stored)
        const float* p = reinterpret_cast<const float*>(a.q) + (int64_t)(s.r0 + r) * a.ld_q + (g * a.group + qq - r * a.group) * HD + tid % 8 * 8;
#pragma unroll
        for (int y = 0; y < NQ; ++y) {
            qf[y][0] = *reinterpret_cast<const float4*>(p + 64 * y);
            qf[y][1] = *reinterpret_cast<const float4*>(p + 64 * y + 4);
        }
    }
    int i = first + wave;
    const bool any = i < last;
    int cp0 = 0, cp1 = 0;   // pages of the step being worked on
    if (any) {
        lookup(i);
        load_k();
        load_v(pg0, pg1);
        cp0 = pg0; cp1 = pg1;
        if (i + W < last) lookup(i + W);
    }
    if constexpr (PARTS > 1) {
#pragma unroll
        for (int y = 0; y < NQ; ++y) {
            bf16x8 t[PARTS];
            split8<PARTS>(qf[y][0], qf[y][1], t);
            const int at = tid % 8 + 8 * y;   // dims 8 at ..
#pragma unroll
            for (int z = 0; z < PARTS; ++z) q_s[(z * KS + at / 2) * 64 + (at & 1) * 32 + tid / 8] = t[z];
        }
        __syncthreads();
    }
    const float mul = score_mul(a);
    f32x16 o[DT];
    float m_run = -SB_INF, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    for (; i < last; i += W) {
        const int key0 = steps.at(i) * 32;
        if (cp0 < 0 || cp1 < 0) {   // (uniform) keys without a page: zeros
            const bool none = (li & 16 ? cp1 : cp0) < 0;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                if (none) kr[ks] = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                if (cp0 < 0) vr[0][dt] = make_uint4(0, 0, 0, 0);
                if (cp1 < 0) vr[1][dt] = make_uint4(0, 0, 0, 0);
            }
        }
        f32x16 st[1];
#pragma unroll
        for (int r = 0; r < 16; ++r) st[0][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int x = 0; x < PARTS; ++x) {
                const bf16x8 qx = PARTS == 1 ? qo[ks] : q_s[(x * KS + ks) * 64 + lane];
                st[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[ks]), qx, st[0], 0, 0, 0);
            }
            if (PARTS > 1 && ks % 2) __builtin_amdgcn_sched_barrier(0);   // (six operands from LDS at a time: registers)
        }
        const bool more = i + W < last;
        const int np0 = pg0, np1 = pg1;
        if (more) {
            load_k();
            if (i + 2 * W < last) lookup(i + 2 * W);
        }
        shape_scores<PARTS, 1, true>(a, q, key0, lh, st);
        const bool masked = !all_see(w, key0, key0 + 32);
        if (masked) mask_scores<1>(q, w, key0, lh, st);
        if (key0 + 32 > s.len) {   // slots past the last key
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint4 keep = first_keys(s.len - key0 - 16 * x - 8 * lh);   // of this lane's 8 keys, those that exist
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
                    vr[x][dt] = make_uint4(vr[x][dt].x & keep.x, vr[x][dt].y & keep.y, vr[x][dt].z & keep.z, vr[x][dt].w & keep.w);
            }
        }
        bf16x8 p[PARTS][2];
        soft_max<PARTS, 1, DT>(st, mul, o, m_run, l_run, p);
        bool sick = false;
        if (masked) {
            u16x2v top = {0, 0};
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) most(vr[x][dt], top);
            sick = not_finite(top);
        }
        if (sick) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const bf16x8 see = sight(q, key0 + 16 * x + 8 * lh);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    uint4 bad;
                    set_apart(vr[x][dt], bad);
                    o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, bad), see, o[dt], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < PARTS; ++y)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vr[x][dt]), p[y][x], o[dt], 0, 0, 0);
        if (more) load_v(np0, np1);
        cp0 = np0; cp1 = np1;
    }
    // ---- the waves' results, brought to one reference point and added in wave order
    l_run = lanes_sum<32, 32>(l_run);
    if (lh == 0) { m_s[wave][li] = m_run; l_s[wave][li] = l_run; }
    __syncthreads();
    float mx = m_s[0][li];
#pragma unroll
    for (int v = 1; v < W; ++v) mx = fmaxf(mx, m_s[v][li]);
    const float ref = mx == -SB_INF ? 0.f : mx;
    float l = 0.f;
#pragma unroll
    for (int v = 0; v < W; ++v) l += l_s[v][li] * __builtin_amdgcn_exp2f(m_s[v][li] - ref);
    const float f = __builtin_amdgcn_exp2f(m_run - ref);
    if (any) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *reinterpret_cast<f32x4*>(o_s[wave][dt * 4 + r / 4][lane]) = f32x4{o[dt][r] * f, o[dt][r + 1] * f, o[dt][r + 2] * f, o[dt][r + 3] * f};
    }
    __syncthreads();
    if (!q.valid) return;
    const int nw = last - first < W ? last - first : W;   // waves that had a step
    const float inv_l = split ? 1.f : l == 0.f ? 0.f : 1.0f / l;
    const int64_t at = pair * gridDim.y + blockIdx.y;
    if (split && wave == 0 && lh == 0) { part.ml[2 * at] = mx; part.ml[2 * at + 1] = l; }
    f32x4 sum[NS / W];   // (a lane finishes its own query: slot n holds dims 32 (n / 4) + 8 (n % 4) + 4 lh ..; a wave takes slots wave, wave + W ..)
#pragma unroll
    for (int k = 0; k < NS / W; ++k) sum[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int x = 0; x < nw; ++x)
#pragma unroll
        for (int k = 0; k < NS / W; ++k) sum[k] += *reinterpret_cast<const f32x4*>(o_s[x][wave + k * W][lane]);
#pragma unroll
    for (int k = 0; k < NS / W; ++k) {
        const int n = wave + k * W, col = (n >> 2) * 32 + (n & 3) * 8 + 4 * lh;
        const float4 r = make_float4(sum[k][0] * inv_l, sum[k][1] * inv_l, sum[k][2] * inv_l, sum[k][3] * inv_l);
        if (split) *reinterpret_cast<float4*>(part.o + at * HD + col) = r;
        else store_out4<HD>(a, q, col, r);
    }
}

// A block per (row, head): its chunks' results at one reference point, added in a fixed order.  All loads of a usual number of chunks (32
// of 128 dims) go out in one trip: 2.3 us for 32 pairs, 4.9 for 192 pairs of 64 chunks.
template <int HD>
__global__ __launch_bounds__(256) void paged_attn_merge_kernel(PagedAttnArgs a, int chunks) {
    constexpr int L = HD / 4, NG = 256 / L;   // lanes (four dims each) of a group, groups
    __shared__ float red[4];
    __shared__ float ls[NG];
    __shared__ __attribute__((aligned(16))) float os[NG][HD];
    const int tid = threadIdx.x, row = blockIdx.x / a.n_heads, head = blockIdx.x % a.n_heads, grp = tid / L, d = tid % L * 4;
    const Partials part(a.scratch, (int64_t)a.kv.n_rows * a.n_heads, chunks, HD);
    const int64_t pair = blockIdx.x, at = pair * chunks;
    // All that the first rounds may need is requested at once, before it is known how many chunks there are (what lies in the others is not used).
    constexpr int U = 4;
    const int n_all = part.count[pair];
    const float m0 = part.ml[2 * (at + (tid < chunks ? tid : 0))];
    float2 ml[U];
    float4 pv[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = grp + NG * u < chunks ? grp + NG * u : 0;
        ml[u] = *reinterpret_cast<const float2*>(part.ml + 2 * (at + c));
        pv[u] = *reinterpret_cast<const float4*>(part.o + (at + c) * HD + d);
    }
    const SeqRows s = find_rows(a.kv, [](int r0, int) { return r0; }, row);
    if (s.b < 0 || row < s.r0 || row >= s.r0 + s.n) return;
    const int n = n_all < chunks ? n_all : chunks;   // (never more, unless what lies on the device changed since)
    float mx = tid < n ? m0 : -SB_INF;
    for (int c = tid + 256; c < n; c += 256) mx = fmaxf(mx, part.ml[2 * (at + c)]);
    mx = wave_max(mx);
    if ((tid & 63) == 0) red[tid >> 6] = mx;
    __syncthreads();
    mx = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float ref = mx == -SB_INF ? 0.f : mx;
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const auto take = [&](float2 x, float4 v) {
        const float f = __builtin_amdgcn_exp2f(x.x - ref);
        l += x.y * f;
        o.x += v.x * f; o.y += v.y * f; o.z += v.z * f; o.w += v.w * f;
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (grp + NG * u < n) take(ml[u], pv[u]);
#pragma unroll 4
    for (int c = grp + NG * U; c < n; c += NG) take(*reinterpret_cast<const float2*>(part.ml + 2 * (at + c)), *reinterpret_cast<const float4*>(part.o + (at + c) * HD + d));
    *reinterpret_cast<float4*>(&os[grp][d]) = o;
    if (d == 0) ls[grp] = l;
    __syncthreads();
    if (tid >= HD) return;
    float t = 0.f, v = 0.f;
#pragma unroll
    for (int x = 0; x < NG; ++x) { t += ls[x]; v += os[x][tid]; }
    store_x(a.out, (int64_t)row * a.ld_out + head * HD + tid, a.x_dtype == SB_FP32, t == 0.f ? 0.f : v / t);
}

// For many rows: a block owns 128 queries of one kv head, 32 a wave, and walks the steps of CH keys that any of them sees.  The four waves of a
// group share a step's keys and values in LDS, two steps deep, by direct global -> LDS loads issued a step ahead (lane l of a
// wave lands 16 l bytes after the wave's base).  Which piece lands where is chosen so that operand reads are free of bank conflicts: a K piece
// (key, p) sits at piece p ^ f(key) of its key's row; the two halves (8 keys each) of a V row change places in every second group of 8 dims.
//   Two waves a SIMD cover for each other: two blocks of one group, or (float rows at head_dim 128, whose three parts would leave one block
// per CU: the second and third lie in LDS then) one block whose two groups take the steps in turn and add their results at the
// end.  Such groups are out of step: where one multiplies its keys, the other takes exponentials (group 0 goes keys, soft-max, values;
// group 1 soft-max, values, the next keys).
//   2048 bf16 rows of 32 heads of 128 behind as many keys (103 GFLOP as counted, 105 with the steps cut by the diagonal) 136 us, 0.76
// PFLOP/s; 8000 rows of 32 heads over 8, a window of 1024 in documents of 900, 116 us; five float prompts of 16 heads of 64, capped, 60 us.
// The first takes 87 us without its exponentials, 58 with those alone, and 111 without loads: matrix instructions 34 % of the cycles, vector
// ones 38 %, no bank conflicts; the two waves of a SIMD overlap them in part, and the clock falls (with zeros for operands 126 where it takes 156).
// 128 queries a block: with 64 a wave there is no room in the registers (218 us), with 256 a block the last blocks leave the card
// idle (152 us; from 8000 rows on 4 % faster).
template <int HD, int PARTS>
struct SharedForm {
    static constexpr int GROUPS = PARTS > 1 && HD == 128 ? 2 : 1;
    static constexpr int KT = PARTS == 1 ? 2 : 1;        // 32-key tiles whose scores are held at once
    static constexpr int CH = GROUPS == 2 ? 32 : 64;     // keys of a step
};
template <int HD, int PARTS, bool SHAPED>
__global__ __launch_bounds__((256 * SharedForm<HD, PARTS>::GROUPS), 2) void paged_attn_shared_kernel(PagedAttnArgs a) {
    using F = SharedForm<HD, PARTS>;
    constexpr int NT = 256, BQ = 128, GROUPS = F::GROUPS, KT = F::KT, CH = F::CH;
    static_assert(GROUPS == 1 || CH == 32 * KT, "a group that runs ahead holds the scores of a whole step");
    constexpr int KS = HD / 16, DT = HD / 32, PPK = HD / 8, SLAB = SB_KV_BLOCK * HD, NPG = CH / SB_KV_BLOCK;
    constexpr int NL = NPG * SLAB / (NT * 8);   // 16-byte pieces per thread, operand and step
    constexpr int PD = 4;                       // operands are read from LDS PD ahead of their MFMAs
    constexpr int NK = KT * KS, NV = 2 * KT * DT, STAGE = CH * HD, IN_LDS = GROUPS == 2 ? PARTS - 1 : 0;   // (parts of the queries)
    __shared__ __attribute__((aligned(16))) uint16_t kv_s[GROUPS][2][2][STAGE];   // [group][keys, values][turn % 2]
    __shared__ __attribute__((aligned(16))) bf16x8 q_s[IN_LDS ? IN_LDS * KS * 256 : 1];
    __shared__ float ml_s[GROUPS][4][32][2];
    __shared__ int reach_s[4][8];
    __shared__ int sick_s;
    static_assert(GROUPS == 1 || sizeof(kv_s) >= 8 * (DT / 2) * 4 * 64 * 16, "the groups' results fit where the steps were");
    const int lane = threadIdx.x & 63, wave8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = GROUPS == 2 ? wave8 >> 2 : 0, wave = wave8 & 3, tid = threadIdx.x & 255;
    const int li = lane & 31, lh = lane >> 5;
    const int Hkv = a.kv.n_kv_heads, tiles = gridDim.x / Hkv;
    const int g = blockIdx.x % Hkv;
    int q0;
    const SeqRows s = tile_of<BQ, 2, true>(a, blockIdx.x / Hkv, tiles, q0);   // (a prompt's last rows see most: they start first)
    if (s.b < 0) return;
    Reach w;
    const Query q = lane_query(a, s, g, q0 + wave * 32, li, w);
    // The queries go out now, their trip runs beside the search for the steps and the first pages.
    using Raw = std::conditional_t<PARTS == 1, bf16x8, float4>;
    constexpr int RAW = PARTS == 1 ? 1 : 2;
    Raw raw[KS][RAW];
    const int64_t q_at = ((int64_t)q.row * a.ld_q + q.head * HD + lh * 8) * (2 * RAW);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int x = 0; x < RAW; ++x)
            raw[ks][x] = reinterpret_cast<const Raw*>(reinterpret_cast<const char*>(a.q) + q_at + ks * 32 * RAW)[x];
    if (lane == 0 && grp == 0) {
        int* const r = reach_s[wave];
        r[0] = w.a_lo; r[1] = w.b_lo; r[2] = w.a1_min; r[3] = w.b1_min;
        r[4] = w.a_hi; r[5] = w.b_hi; r[6] = w.a0_max; r[7] = w.b0_max;
    }
    if (threadIdx.x == 0) sick_s = 0;
    __syncthreads();
    int e8[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        int v = reach_s[0][k];
#pragma unroll
        for (int i = 1; i < 4; ++i) v = k < 4 ? (reach_s[i][k] < v ? reach_s[i][k] : v) : (reach_s[i][k] > v ? reach_s[i][k] : v);
        e8[k] = __builtin_amdgcn_readfirstlane(v);
    }
    const Reach all{e8[0], e8[4], e8[1], e8[5], e8[6], e8[2], e8[7], e8[3]};
    const Steps steps = steps_of<CH>(all);
    const int turns = (steps.n + GROUPS - 1) / GROUPS;   // of a group; its step in turn j is GROUPS j + grp

    const int64_t page_elems = (int64_t)Hkv * SLAB;
    const uint16_t* const kbase = a.kv.k + (int64_t)g * SLAB;
    const uint16_t* const vbase = a.kv.v + (int64_t)g * SLAB;
    const int32_t* const table = a.kv.table + (int64_t)s.b * a.kv.table_ld;
    // A wave's 64 pieces lie in one page, so the page is a scalar: lane i < NPG holds the i-th page of a turn's step (-1: no key
    // there, or no such page: zeros).  A thread's place within a page is the same for all its pieces.
    auto lookup = [&](int j) {
        const int i = GROUPS * j + grp, page = (i < steps.n ? steps.at(i) : 0) * NPG + (lane & (NPG - 1));
        const int pg = i < steps.n && page * SB_KV_BLOCK < s.len ? table[page] : -1;
        return pg >= a.kv.n_pages ? -1 : pg;
    };
    const int slot_p = (wave * 64 + lane) % (SB_KV_BLOCK * PPK), key_p = slot_p / PPK;
    const uint32_t koff = (uint32_t)(key_p * HD + ((slot_p % PPK) ^ (PPK == 16 ? key_p : (key_p >> 1) & 7)) * 8) * 2;
    const uint32_t voff = (uint32_t)(slot_p ^ ((slot_p >> 4) & 1)) * 16;
    auto issue = [&](const uint16_t* base, uint32_t off, uint16_t* lds, int pages) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int slot0 = i * NT + wave * 64;   // the wave's place in LDS
            const int page = __builtin_amdgcn_readlane(pages, slot0 / (SB_KV_BLOCK * PPK));
            uint16_t* const at = lds + slot0 * 8;
            if (page >= 0) __builtin_amdgcn_global_load_lds(reinterpret_cast<const char*>(base + page * page_elems) + off, at, 16, 0, 0);
            else *reinterpret_cast<uint4*>(at + lane * 8) = make_uint4(0, 0, 0, 0);
        }
    };
    int pages_v = lookup(0), pages_k = pages_v;   // of the steps whose values / keys are requested next
    if (turns > 0) {
        issue(kbase, koff, kv_s[grp][0][0], pages_k);
        issue(vbase, voff, kv_s[grp][1][0], pages_v);
        pages_v = pages_k = lookup(1);
        if (grp == 1) {   // (its keys are a turn further ahead)
            issue(kbase, koff, kv_s[grp][0][1], pages_k);
            pages_k = lookup(2);
        }
    }
    bf16x8 qo[PARTS - IN_LDS][KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        bf16x8 t[PARTS];
        if constexpr (PARTS == 1) t[0] = raw[ks][0];
        else split8<PARTS>(raw[ks][0], raw[ks][1], t);
#pragma unroll
        for (int x = 0; x < PARTS; ++x)
            if (x < PARTS - IN_LDS) qo[x][ks] = t[x];
            else if (grp == 0) q_s[((x - 1) * KS + ks) * 256 + wave * 64 + lane] = t[x];
    }
    const float mul = score_mul(a);
    f32x16 o[DT];
    float m_run = -SB_INF, l_run = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[dt][r] = 0.f;
    const int krow = (li & 19) | ((li & 4) << 1) | ((li & 8) >> 1);   // row li of a key tile is key krow of it
    const int kswz = PPK == 16 ? (krow & 15) : ((krow >> 1) & 7);
    const auto seen = [&](int j, int t) {   // tiles t .. of turn j, by a query of the wave
        if (GROUPS * j + grp >= steps.n) return false;
        const int k = steps.at(GROUPS * j + grp) * CH + 32 * t;
        return some_see(w, k, k + 32 * KT);
    };

    f32x16 st[KT];
    bf16x8 op[PD];
    auto scores = [&](int j, int t) {   // of the keys of turn j's tiles t ..
        const uint16_t* const k = kv_s[grp][0][j & 1] + t * 32 * HD;
        auto read = [&](int n) {   // k step n / KT of tile n % KT
            op[n % PD] = *reinterpret_cast<const bf16x8*>(&k[((n % KT) * 32 + krow) * HD + (((n / KT) * 2 + lh) ^ kswz) * 8]);
        };
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) st[kt][r] = 0.f;
#pragma unroll
        for (int n = 0; n < PD; ++n) read(n);
#pragma unroll
        for (int n = 0; n < NK; n += KT) {
#pragma unroll
            for (int x = 0; x < PARTS; ++x) {
                const bf16x8 qx = x < PARTS - IN_LDS ? qo[x < PARTS - IN_LDS ? x : 0][n / KT] : q_s[IN_LDS ? ((x - 1) * KS + n / KT) * 256 + wave * 64 + lane : 0];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) st[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[(n + kt) % PD], qx, st[kt], 0, 0, 0);
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
                if (n + kt + PD < NK) read(n + kt + PD);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if constexpr (GROUPS == 2) {
        if (grp == 1 && turns > 0 && seen(0, 0)) scores(0, 0);
        __syncthreads();   // (every wave is done with the first keys of group 1)
    }
#pragma unroll 1
    for (int j = 0; j < turns; ++j) {
        const int buf = j & 1;
        // K: group 0 the next turn's, group 1 the one's after that, whose place this turn's scores have left
        issue(kbase, koff, kv_s[grp][0][grp ? buf : buf ^ 1], pages_k);
        issue(vbase, voff, kv_s[grp][1][buf ^ 1], pages_v);
        pages_v = grp ? pages_k : lookup(j + 2);
        pages_k = grp ? lookup(j + 3) : pages_v;
        const int ka = steps.at(GROUPS * j) * CH, kb = steps.at(GROUPS == 2 && 2 * j + 1 < steps.n ? 2 * j + 1 : GROUPS * j) * CH;   // the groups' keys
        const int key0 = grp ? kb : ka;
        uint16_t* const v_s = kv_s[grp][1][buf];
        auto v_at = [&](int n) {   // page n / DT, dims 32 (n % DT) + li, keys 8 lh ..
            const int slot = ((n % DT) * 32 + li) * 2 + lh;
            return *reinterpret_cast<const bf16x8*>(&v_s[(n / DT) * SLAB + (slot ^ ((slot >> 4) & 1)) * 8]);
        };
        if (!all_see(all, ka, ka + CH) || !all_see(all, kb, kb + CH)) {
            // Some query does not see some key: its value must not be an infinity or NaN in the product.  Slots past the last key are
            // made zeros; if a value that some query sees is one (a thread looks at the pieces that it staged), its product
            // with who sees it is taken here and a zero left in its place.
            u16x2v top = {0, 0};
#pragma unroll
            for (int k = 0; k < NL; ++k) {
                const int slot = k * NT + tid;
                const int vk = key0 + (slot / (SB_KV_BLOCK * PPK)) * SB_KV_BLOCK + ((slot ^ (slot >> 4)) & 1) * 8;   // keys vk .. vk + 7 of one dim
                uint4 v = *reinterpret_cast<uint4*>(&v_s[slot * 8]);
                if (vk + 8 > s.len) {
                    const uint4 keep = first_keys(s.len - vk);
                    v = make_uint4(v.x & keep.x, v.y & keep.y, v.z & keep.z, v.w & keep.w);
                    *reinterpret_cast<uint4*>(&v_s[slot * 8]) = v;
                }
                most(v, top);
            }
            if (not_finite(top) && lane == 0) sick_s = j + 1;
            __syncthreads();
            if (sick_s == j + 1) {
#pragma unroll 1
                for (int x = 0; x < NPG; ++x) {
                    const bf16x8 see = sight(q, key0 + 16 * x + 8 * lh);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        uint4 v = __builtin_bit_cast(uint4, v_at(x * DT + dt)), bad;
                        set_apart(v, bad);
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, bad), see, o[dt], 0, 0, 0);
                    }
                }
                __syncthreads();
#pragma unroll 1
                for (int k = 0; k < NL; ++k) {
                    uint4* const at = reinterpret_cast<uint4*>(&v_s[(k * NT + tid) * 8]);
                    uint4 v = *at, bad;
                    set_apart(v, bad);
                    *at = v;
                }
                __syncthreads();
            }
        }
#pragma unroll 1
        for (int t = 0; t < CH / 32; t += KT) {
            if (!seen(j, t)) continue;
            const int tk = key0 + 32 * t;
            if (grp == 0) scores(j, t);
            shape_scores<PARTS, KT, SHAPED>(a, q, tk, lh, st);
            if (!all_see(w, tk, tk + 32 * KT)) mask_scores<KT>(q, w, tk, lh, st);
            auto read = [&](int n) { op[n % PD] = v_at(2 * t * DT + n); };
#pragma unroll
            for (int n = 0; n < PD; ++n) read(n);
            bf16x8 p[PARTS][2 * KT];
            soft_max<PARTS, KT, DT>(st, mul, o, m_run, l_run, p);
#pragma unroll
            for (int n = 0; n < NV; n += 2) {
#pragma unroll
                for (int y = 0; y < PARTS; ++y)
#pragma unroll
                    for (int x = 0; x < 2; ++x) o[(n + x) % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[(n + x) % PD], p[y][n / DT], o[(n + x) % DT], 0, 0, 0);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (n + x + PD < NV) read(n + x + PD);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (GROUPS == 2 && grp == 1 && seen(j + 1, 0)) scores(j + 1, 0);
        __builtin_amdgcn_s_waitcnt(0);   // this wave's pieces have landed
        __syncthreads();                 // ... and everybody's; every wave is done with this turn
    }
    const float l_own = lanes_sum<32, 32>(l_run);
    if constexpr (GROUPS == 1) {
        const float inv_l = l_own == 0.f ? 0.f : 1.0f / l_own;
        // Rows leave whole: a wave turns its own in LDS (piece p of row r at p ^ r % 16), so that a store covers whole lines.
        constexpr int P = HD * (PARTS == 1 ? 2 : 4) / 16, RPI = 64 / P;   // 16-byte pieces of a row, rows of a store
        char* const t_s = reinterpret_cast<char*>(&kv_s[0][0][0][0]) + wave * 32 * P * 16;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const float4 v = make_float4(o[dt][r] * inv_l, o[dt][r + 1] * inv_l, o[dt][r + 2] * inv_l, o[dt][r + 3] * inv_l);
                if constexpr (PARTS == 1)
                    *reinterpret_cast<uint2*>(t_s + (li * P + ((dt * 4 + r / 4) ^ (li & (P - 1)))) * 16 + lh * 8) =
                        make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
                else *reinterpret_cast<float4*>(t_s + (li * P + ((dt * 8 + r / 2 + lh) ^ (li & (P - 1)))) * 16) = v;
            }
        const int nq = s.n * a.group - (q0 + wave * 32);   // queries of this wave from here on
#pragma unroll
        for (int i = 0; i < 32 / RPI; ++i) {
            const int x = i * RPI + lane / P, p = lane % P;
            const uint4 v = *reinterpret_cast<const uint4*>(t_s + (x * P + (p ^ (x & (P - 1)))) * 16);
            if (x >= nq) continue;
            const int qq = q0 + wave * 32 + x, r = row_of(a, qq);
            char* const to = reinterpret_cast<char*>(a.out) + ((int64_t)(s.r0 + r) * a.ld_out + (g * a.group + qq - r * a.group) * HD) * (PARTS == 1 ? 2 : 4);
            *reinterpret_cast<uint4*>(to + p * 16) = v;
        }
        return;
    }
    // ---- the groups' results at one reference point: each keeps half of the dims and gives the other half away
    if (lh == 0) { ml_s[grp][wave][li][0] = m_run; ml_s[grp][wave][li][1] = l_own; }
    f32x4* const x_s = reinterpret_cast<f32x4*>(&kv_s[0][0][0][0]);   // [group][wave][dims][64 lanes]
    constexpr int HALF = DT / 2 * 4;
#pragma unroll
    for (int dt = 0; dt < DT / 2; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = grp ? o[dt][r + e] : o[dt + DT / 2][r + e];
            x_s[((grp * 4 + wave) * HALF + dt * 4 + r / 4) * 64 + lane] = v;
        }
    __syncthreads();
    const float mx = fmaxf(m_run, ml_s[GROUPS - 1 - grp][wave][li][0]), ref = mx == -SB_INF ? 0.f : mx;
    const float f = __builtin_amdgcn_exp2f(m_run - ref), h = __builtin_amdgcn_exp2f(ml_s[GROUPS - 1 - grp][wave][li][0] - ref);
    const float l = l_own * f + ml_s[GROUPS - 1 - grp][wave][li][1] * h, inv_l = l == 0.f ? 0.f : 1.0f / l;
    if (!q.valid) return;
#pragma unroll
    for (int dt = 0; dt < DT / 2; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 u = x_s[(((GROUPS - 1 - grp) * 4 + wave) * HALF + dt * 4 + r / 4) * 64 + lane];
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ((grp ? o[dt + DT / 2][r + e] : o[dt][r + e]) * f + u[e] * h) * inv_l;
            store_out4<HD>(a, q, (dt + grp * (DT / 2)) * 32 + 2 * r + 4 * lh, make_float4(v[0], v[1], v[2], v[3]));
        }
}

// Which form a call takes, and how its keys are split.  Blocks of 128 queries read a quarter of what blocks of 32 do, but a few of them leave the card
// idle and a long one to wait for.  From 192 of them on for bf16 rows, 512 for float rows (whose products take three times as long for the
// same reads).  Shared / apart, us, a prompt of 512, 1024, 2048 rows (128, 256, 512 blocks), 32 heads over 8: bf16, heads of 128 18.6 / 16.8,
// 34.4 / 42.5, 65 / 118, of 64 13.5 / 11.3, 22.6 / 24.6, 48 / 65; float, of 128 32.8 / 21.7, 56.2 / 53.7, 121 / 152, of 64 21.6 / 13.4, 40.2 / 31.6, 79 / 83.
//   Sequences of a few rows leave most of such a block empty: 32 queries a sequence on average for bf16 rows, 192 for float rows (whose
// blocks, one a CU at head_dim 128, wait longer for keys that nobody else reads).  Shared / apart behind 1000 keys, four queries a row:
// bf16, 512 sequences of 2 rows 397 / 383, 256 of 4 206 / 212, 128 of 8 111 / 164, 128 of 32 205 / 263; float, 128 of 16 281 / 186, 128 of 32
// 487 / 306, 64 of 64 282 / 294, 32 of 128 261 / 290; float, heads of 64, 32 of 64 64 / 80, 16 of 128 63 / 75.
//   Taken apart, a block has as many 32-key steps (a multiple of its four waves) as give some 512 blocks, 64 at most: six rows behind
// 131000 keys, 16 / 32 / 64 / 128 steps 138 / 121 / 112 / 136 us; 64 sequences of up to 8000 keys 257 / 258 / 256 / 275; one row behind 520 keys, 4
// steps 11.8, all in one block 18.8.
struct AttnPlan { bool shared; int64_t tiles; int steps, chunks; };
static AttnPlan attn_plan(const PagedKv& kv, int32_t n_heads, bool fp32) {
    const int64_t G = n_heads / kv.n_kv_heads, total = (kv.max_len + 31) / 32;
    AttnPlan p;
    p.shared = (int64_t)kv.n_rows * n_heads / 128 >= (fp32 ? 512 : 192) && kv.n_rows * G >= (fp32 ? 192 : 32) * (int64_t)kv.n_seq;
    if (p.shared) {
        p.tiles = kv.n_rows * G / 128 + kv.n_seq;
        p.steps = 0;
        p.chunks = 1;
        return p;
    }
    p.tiles = kv.n_rows * G / 32 + kv.n_seq;
    const int64_t want = (p.tiles * kv.n_kv_heads * total + 511) / 512;
    p.steps = (int)(want < 4 ? 4 : want > 64 ? 64 : (want + 3) / 4 * 4);
    const int64_t most = 4096 / (p.tiles * kv.n_kv_heads) + 1;   // chunks: what they leave stays below some 70 MB
    if (total > most * p.steps) p.steps = (int)((total + most - 1) / most + 3) / 4 * 4;
    p.chunks = (int)((total + p.steps - 1) / p.steps);
    return p;
}

size_t paged_attention_scratch(const PagedKv& kv, int32_t n_heads) {   // (of either type: float rows are taken apart longer)
    const AttnPlan p = attn_plan(kv, n_heads, true);
    return p.chunks > 1 ? Partials::bytes((int64_t)kv.n_rows * n_heads, p.chunks, kv.head_dim) : 0;
}

hipError_t launch_paged_attention(const PagedAttnArgs& args, hipStream_t st) {
    PagedAttnArgs a = args;
    a.group_shift = (a.group & (a.group - 1)) == 0 ? __builtin_ctz(a.group) : -1;
    const AttnPlan p = attn_plan(a.kv, a.n_heads, a.x_dtype == SB_FP32);
    const auto go = [&](auto hd_c) {
        constexpr int HD = decltype(hd_c)::value;
        const dim3 grid((unsigned)(p.tiles * a.kv.n_kv_heads), p.chunks);
        const bool shaped = a.cap > 0.f || a.slopes;
        if (p.shared && a.x_dtype == SB_FP32)
            return launch(shaped ? &paged_attn_shared_kernel<HD, 3, true> : &paged_attn_shared_kernel<HD, 3, false>, grid, 256 * SharedForm<HD, 3>::GROUPS, st, a);
        if (p.shared) return launch(shaped ? &paged_attn_shared_kernel<HD, 1, true> : &paged_attn_shared_kernel<HD, 1, false>, grid, 256, st, a);
        const hipError_t e = launch(a.x_dtype == SB_FP32 ? &paged_attn_apart_kernel<HD, 3> : &paged_attn_apart_kernel<HD, 1>, grid, 256, st, a, p.steps);
        if (e != hipSuccess || p.chunks == 1) return e;
        return launch(&paged_attn_merge_kernel<HD>, dim3(a.kv.n_rows * a.n_heads), 256, st, a, p.chunks);
    };
    return a.kv.head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

// ---------------------------------------------------------------- page copies
// 16 bytes a thread, nothing more: with four loads a thread in flight (16 KB pieces) a fork of 10 MB took 16.7 us and a compaction of 870 MB
// (read and written) 160, with one 4.2 and 145 (6.0 TB/s; a plain copy of 1 GB to the next runs at 4.7).  grid (pages x pieces of a page, slabs).
constexpr int COPY_PIECE = 4096;
__global__ __launch_bounds__(256) void copy_pages_kernel(CopyPagesArgs a, int pieces) {
    const int page = blockIdx.x / pieces, piece = blockIdx.x - page * pieces;
    const uint4* s = reinterpret_cast<const uint4*>(a.src + blockIdx.y * a.src_slab + a.from[page] * a.page_bytes);
    uint4* d = reinterpret_cast<uint4*>(a.dst + blockIdx.y * a.dst_slab + a.to[page] * a.page_bytes);
    const size_t i = (size_t)piece * (COPY_PIECE / 16) + threadIdx.x;
    if (i < a.page_bytes / 16) d[i] = s[i];
}
hipError_t launch_copy_pages(const CopyPagesArgs& a, int32_t n, int32_t n_slabs, hipStream_t st) {
    const size_t pieces = (a.page_bytes + COPY_PIECE - 1) / COPY_PIECE;
    if (pieces > 0x7fffffff / (size_t)n) return hipErrorInvalidValue;
    return launch(&copy_pages_kernel, dim3((unsigned)(pieces * n), n_slabs), 256, st, a, (int)pieces);
}

}  // namespace sb
