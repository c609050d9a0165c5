// Operators on a paged cache that several sequences live in: rotary append, attention by a rule, page copies.
#include "kernels.h"
#include "device_utils.h"

namespace sb {

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// The newest rows of a sequence and where they stand.
struct SeqRows { int b, r0, n, len; };   // sequence (-1: none), first row, rows, keys

// Sequence of item t where sequence b owns the items first(b) .. first(b + 1) - 1 of an ascending `first`: the last b
// with first(b) <= t, by a search 64 ways wide (one load a lane and step).  All lanes of the wave are active, t is uniform.
template <typename First>
__device__ __forceinline__ int find_seq(int n_seq, First first, int t) {
    const int lane = threadIdx.x & 63;
    int lo = 0, n = n_seq;   // the answer is lo - 1 .. lo + n - 1 (lo - 1 only while lo is 0)
    while (n > 0) {
        const int step = (n + 63) / 64, b = lo + lane * step;
        const int c = __popcll(__builtin_amdgcn_ballot_w64(b < lo + n && first(b) <= t));
        if (c == 0) return lo - 1;
        const int end = lo + n;
        lo += (c - 1) * step;
        if (step == 1) return lo;
        n = (lo + step < end ? lo + step : end) - lo;
    }
    return -1;
}

__device__ __forceinline__ int row_at(const PagedKv& kv, int b) { return clampi(kv.row_start[b], 0, kv.n_rows); }

__device__ __forceinline__ SeqRows seq_rows(const PagedKv& kv, int b) {
    SeqRows s{b, 0, 0, 0};
    if (b < 0) return s;
    s.r0 = row_at(kv, b);
    s.n = row_at(kv, b + 1) - s.r0;
    s.len = clampi(kv.kv_len[b], 0, kv.max_len);
    if (s.n <= 0) s.b = -1;
    return s;
}

__device__ __forceinline__ float load_x(const void* x, int64_t i, bool fp32) {
    return fp32 ? reinterpret_cast<const float*>(x)[i] : bf2f(reinterpret_cast<const uint16_t*>(x)[i]);
}
__device__ __forceinline__ uint16_t round_bf16(float v) { return (uint16_t)pack_bf16(v, v); }   // (NaN stays one)
__device__ __forceinline__ void store_x(void* x, int64_t i, bool fp32, float v) {
    if (fp32) reinterpret_cast<float*>(x)[i] = v;
    else reinterpret_cast<uint16_t*>(x)[i] = round_bf16(v);
}

// ---------------------------------------------------------------- rotary append
// A wave per row and head, grid (rows, ceil(heads / 4)).
template <int HD>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeAppendArgs a) {
    __shared__ float xs[4][HD];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.x;
    const int Hq = a.n_heads, Hkv = a.kv.n_kv_heads, head = blockIdx.y * 4 + wave;
    const SeqRows s = seq_rows(a.kv, find_seq(a.kv.n_seq, [&](int b) { return row_at(a.kv, b); }, row));
    const int pos = s.len - s.n + row - s.r0, rot = a.rot_dim, half = rot / 2;
    const bool fp32 = a.x_dtype == SB_FP32;
    const bool on = s.b >= 0 && row < s.r0 + s.n && head < Hq + 2 * Hkv && pos >= 0 && (rot == 0 || pos < a.n_pos);
    const bool is_v = head >= Hq + Hkv;
    const float* gain = head < Hq ? a.q_gain : is_v ? nullptr : a.k_gain;
    float x[HD / 64], ss = 0.f;
    if (on) {
        for (int i = 0; i < HD / 64; ++i) {
            x[i] = load_x(a.qkv, (int64_t)row * a.ld_qkv + head * HD + i * 64 + lane, fp32);
            ss += x[i] * x[i];
        }
        if (gain) {
            const float inv = 1.0f / sqrtf(wave_sum(ss) / (float)HD + a.eps);
            for (int i = 0; i < HD / 64; ++i) x[i] = x[i] * inv * gain[i * 64 + lane];
        }
        for (int i = 0; i < HD / 64; ++i) xs[wave][i * 64 + lane] = x[i];
    }
    __syncthreads();
    if (!on) return;
    const int page = pos / SB_KV_BLOCK, slot = pos % SB_KV_BLOCK;
    const int pg = a.kv.table[(int64_t)s.b * a.kv.table_ld + page];
    for (int i = 0; i < HD / 64; ++i) {
        const int d = i * 64 + lane;
        float y = x[i];
        if (!is_v && d < rot) {
            const bool second = a.interleaved ? d & 1 : d >= half;
            const int p = a.interleaved ? d >> 1 : second ? d - half : d;
            const float o = xs[wave][a.interleaved ? d ^ 1 : second ? d - half : d + half];
            const float c = a.cos[(int64_t)pos * half + p], n = a.sin[(int64_t)pos * half + p];
            y = second ? x[i] * c + o * n : x[i] * c - o * n;
        }
        if (head < Hq) {
            store_x(a.q_out, (int64_t)row * a.ld_q + head * HD + d, fp32, y);
        } else if (pg >= 0 && pg < a.kv.n_pages) {
            const int g = is_v ? head - Hq - Hkv : head - Hq;
            const int64_t slab = ((int64_t)pg * Hkv + g) * SB_KV_BLOCK * HD;
            if (is_v) a.kv.v[slab + d * SB_KV_BLOCK + slot] = round_bf16(y);
            else a.kv.k[slab + slot * HD + d] = round_bf16(y);
        }
    }
}

hipError_t launch_rope_append(const RopeAppendArgs& a, hipStream_t st) {
    const dim3 grid(a.kv.n_rows, (a.n_heads + 2 * a.kv.n_kv_heads + 3) / 4);
    return a.kv.head_dim == 128 ? launch(&rope_append_kernel<128>, grid, 256, st, a) : launch(&rope_append_kernel<64>, grid, 256, st, a);
}

// ---------------------------------------------------------------- attention
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

// A wave per row and head: 64 keys at a time, a lane each, with a running maximum and sum; then a lane holds HD / 64 dims.
template <int HD>
__global__ __launch_bounds__(64) void paged_attn_kernel(PagedAttnArgs a) {
    __shared__ float qs[HD];
    const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y, Hkv = a.kv.n_kv_heads, g = head / a.group;
    const SeqRows s = seq_rows(a.kv, find_seq(a.kv.n_seq, [&](int b) { return row_at(a.kv, b); }, row));
    if (s.b < 0 || row >= s.r0 + s.n) return;
    const int pos = s.len - s.n + row - s.r0;
    const bool fp32 = a.x_dtype == SB_FP32;
    for (int d = lane; d < HD; d += 64) qs[d] = load_x(a.q, (int64_t)row * a.ld_q + head * HD + d, fp32);
    __syncthreads();
    const Sees see = row_sees(a, s, row, pos);
    float m = -SB_INF, l = 0.f, o[HD / 64] = {};
    for (int k0 = 0; k0 < s.len; k0 += 64) {
        const int key = k0 + lane;
        float sc = -SB_INF;
        if ((key >= see.a0 && key < see.a1) || (key >= see.b0 && key < see.b1)) {
            const int pg = a.kv.table[(int64_t)s.b * a.kv.table_ld + key / SB_KV_BLOCK];
            float z = 0.f;
            if (pg >= 0 && pg < a.kv.n_pages) {
                const uint16_t* kp = a.kv.k + (((int64_t)pg * Hkv + g) * SB_KV_BLOCK + key % SB_KV_BLOCK) * HD;
                for (int d = 0; d < HD; ++d) z = fmaf(qs[d], bf2f(kp[d]), z);
            }
            sc = z * a.scale;
            if (a.cap > 0.f) sc = a.cap * tanhf(sc / a.cap);
            if (a.slopes) sc -= a.slopes[head] * fabsf((float)(pos - key));
        }
        const float m1 = fmaxf(m, wave_max(sc)), ref = m1 == -SB_INF ? 0.f : m1;
        const float p = expf(sc - ref), f = expf((m == -SB_INF ? ref : m) - ref);
        l = l * f + wave_sum(p);
        for (int i = 0; i < HD / 64; ++i) o[i] *= f;
        m = m1;
        for (int j = 0; j < 64 && k0 + j < s.len; ++j) {
            const float pj = __shfl(p, j, 64), sj = __shfl(sc, j, 64);
            if (sj == -SB_INF) continue;
            const int kj = k0 + j, pg = a.kv.table[(int64_t)s.b * a.kv.table_ld + kj / SB_KV_BLOCK];
            if (pg < 0 || pg >= a.kv.n_pages) continue;
            const uint16_t* vp = a.kv.v + ((int64_t)pg * Hkv + g) * SB_KV_BLOCK * HD + kj % SB_KV_BLOCK;
            for (int i = 0; i < HD / 64; ++i) o[i] = fmaf(pj, bf2f(vp[(i * 64 + lane) * SB_KV_BLOCK]), o[i]);
        }
    }
    for (int i = 0; i < HD / 64; ++i) store_x(a.out, (int64_t)row * a.ld_out + head * HD + i * 64 + lane, fp32, l == 0.f ? 0.f : o[i] / l);
}

size_t paged_attention_scratch(const PagedKv&, int32_t) { return 0; }

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t st) {
    const dim3 grid(a.kv.n_rows, a.n_heads);
    return a.kv.head_dim == 128 ? launch(&paged_attn_kernel<128>, grid, 64, st, a) : launch(&paged_attn_kernel<64>, grid, 64, st, a);
}

// ---------------------------------------------------------------- page copies
// grid (pages, slabs).
__global__ __launch_bounds__(256) void copy_pages_kernel(CopyPagesArgs a) {
    const uint4* s = reinterpret_cast<const uint4*>(a.src + blockIdx.y * a.src_slab + a.from[blockIdx.x] * a.page_bytes);
    uint4* d = reinterpret_cast<uint4*>(a.dst + blockIdx.y * a.dst_slab + a.to[blockIdx.x] * a.page_bytes);
    for (size_t i = threadIdx.x; i < a.page_bytes / 16; i += 256) d[i] = s[i];
}
hipError_t launch_copy_pages(const CopyPagesArgs& a, int32_t n, int32_t n_slabs, hipStream_t st) {
    return launch(&copy_pages_kernel, dim3(n, n_slabs), 256, st, a);
}

}  // namespace sb
