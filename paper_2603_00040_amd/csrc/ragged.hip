// Attention over the NVFP4 KV cache for a step whose sequences bring different numbers of queries: O = softmax(scale Q K^T + mask) V with K and V
// the values that the pages stand for.  Only the cache is in 4 bits: Q enters as it is, the probabilities are not quantized.
//
// The G query heads of a kv head and the queries of a sequence are one run of rows (row = query * G + head of the group), cut into tiles of
// rows that share every key that is read.  Scores are computed transposed, S^T = K Q^T: in the accumulator a lane owns one row, so that the running
// maximum and sum of the softmax are per-lane numbers, and its four consecutive keys are, without being moved, what the matrix instruction takes
// of P^T in O^T += V^T P^T (any order of the keys will do as long as V's rows come in the same one).
//
// Numbers: a cached value has at most 6 significant bits and lies in [2^-10, 2688], exact in fp16.  A row of Q, bf16, is multiplied by the power of
// two that brings its largest element to [2^14, 2^15) and is exact in fp16 but for elements 2^-28 of the largest and less, which lose
// what lies below 2^-39 of the largest.  Scores, maxima, sums and O are fp32.  P is rounded to fp16 (11 bits, P <= 1) for the product with V: a
// relative 2^-12 per probability, an eighth of what rounding the output to bf16 costs; the sum that divides O is of the unrounded ones.
#include "common.hpp"
#include "kernels.hpp"
#include "nvfp4.hpp"

namespace aq {

namespace {

constexpr int kFewRows = 32;          // most rows of a (sequence, kv head) that the kernel for few rows takes
constexpr int kWideRows = 128;        // rows of a tile of the other one

struct Seq { int first, n, len; };    // first query of the step, number of queries, keys
__device__ inline Seq seq_of(const RaggedArgs& a, int b)
{
    const int s = min(max(a.cu_q[b], 0), a.T), e = min(max(a.cu_q[b + 1], s), a.T);
    return Seq{s, min(e - s, a.max_q), max(0, min(a.kv_lens[b], a.max_pages * 128))};
}

// Keys [lo, hi) that some row of a tile sees, its rows being queries ta .. tb of the sequence.
__device__ inline void keys_of(const RaggedArgs& a, const Seq& s, int ta, int tb, int& lo, int& hi)
{
    hi = a.causal ? min(max(s.len - s.n + tb + 1, 0), s.len) : s.len;
    lo = a.window > 0 ? max(0, s.len - s.n + ta + 1 - a.window) : 0;
    hi = max(lo, hi);
}

// The units of work of the kernel for few rows: the pages that the rows of a sequence see, once per kv head, sequence by sequence, head by head, page by
// page.  Sequences with more rows than `most` have none here.
struct Few { int rows, first_page, pages; };
__device__ inline Few few_of(const RaggedArgs& a, int b, int G, int most)
{
    const Seq s = seq_of(a, b);
    const int rows = s.n <= most ? s.n * G : most + 1;
    int lo, hi;
    keys_of(a, s, 0, s.n - 1, lo, hi);
    const bool on = rows > 0 && rows <= most && hi > lo;
    return Few{rows, lo >> 7, on ? ((hi + 127) >> 7) - (lo >> 7) : 0};
}

// Sums over a workgroup of 256: inclusive, and of all.
__device__ inline int wg_scan256(int v, int* red /* [4], LDS */, int& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) { const int u = __shfl_up(v, d); if (lane >= d) v += u; }
    __syncthreads();
    if (lane == 63) red[wave] = v;
    __syncthreads();
    total = (red[0] + red[1]) + (red[2] + red[3]);
    return v + (wave > 0 ? red[0] : 0) + (wave > 1 ? red[1] : 0) + (wave > 2 ? red[2] : 0);
}

// The tile number `item` of the step: sequence by sequence, each with ceil(n G / kWideRows) tiles, none where the kernel for few rows (at most `few`)
// takes it.  By a workgroup of 256; false behind the last one.
__device__ inline bool find_tile(const RaggedArgs& a, int G, int few, int item, int& b_out, int& tile_out, int* lds /* [8] */)
{
    const int tid = threadIdx.x;
    if (tid == 0) lds[4] = -1;
    for (int b0 = 0; b0 < a.B; b0 += 256) {
        const int b = b0 + tid;
        const long long rows = b < a.B ? (long long)seq_of(a, b).n * G : 0;
        const int tiles = rows > few ? (int)((rows + kWideRows - 1) / kWideRows) : 0;
        int total;
        const int upto = wg_scan256(tiles, lds, total);
        if (item < upto && item >= upto - tiles) { lds[4] = b; lds[5] = item - (upto - tiles); }
        if (item < total) break;
        item -= total;
    }
    __syncthreads();
    b_out = __builtin_amdgcn_readfirstlane(lds[4]);
    tile_out = __builtin_amdgcn_readfirstlane(lds[5]);
    return b_out >= 0;
}

// Codes and scale bytes of D / 4 values of one key: lane (key cc of 16, group g) holds d = (D/4) g .. + D/4 - 1.
template <int D> struct Raw { uint32_t w[D / 32]; uint32_t sc; };
template <int D>
__device__ inline Raw<D> load_raw(const unsigned char* part /* K or V part of a page's head */, int key, int g)
{
    Raw<D> r;
    if constexpr (D == 128) {
        const uint4v c = *reinterpret_cast<const uint4v*>(part + key * 64 + 16 * g);
        r.w[0] = c[0]; r.w[1] = c[1]; r.w[2] = c[2]; r.w[3] = c[3];
        r.sc = *reinterpret_cast<const uint16_t*>(part + 128 * 64 + key * 8 + 2 * g);
    } else {
        const uint2v c = *reinterpret_cast<const uint2v*>(part + key * 32 + 8 * g);
        r.w[0] = c[0]; r.w[1] = c[1];
        r.sc = part[128 * 32 + key * 4 + g];
    }
    return r;
}
// The block scales of those values as an fp16 pair (one for D = 64).  Not live: 0, whatever the bytes are (a stale scale byte may be NaN).
template <int D>
__device__ inline half2v scales_of(const Raw<D>& r, bool live) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(live ? r.sc : 0u, 1.0f, false); }
// Values 8 s .. 8 s + 7 of the lane's as fp16.
template <int D>
__device__ inline half8 values8(const Raw<D>& r, half2v sc, int s)
{
    const half_t sv = (D == 128 && s >= 2) ? sc[1] : sc[0];
    const half2v sc2 = {sv, sv};
    const uint32_t w = r.w[s];
    uint4v v;
    v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0) * sc2);
    v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1) * sc2);
    v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2) * sc2);
    v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3) * sc2);
    return __builtin_bit_cast(half8, v);
}

// The power of two that brings a row's largest magnitude to [2^14, 2^15), and its inverse (magnitudes below 2^-112 count as that).
__device__ inline void row_factor(float amax, float& f, float& inv)
{
    const uint32_t e = max(__float_as_uint(amax) >> 23, 15u);
    f = __uint_as_float((268u - e) << 23);
    inv = __uint_as_float((e - 14u) << 23);
}

// What the launches of a step hand over: how many pages each workgroup takes, the pages (of one head) in front of every sequence, and, of a unit whose
// pages are shared by several workgroups, each one's O, maximum and sum.
struct FewWs { int* quota; int* front /* [B + 1] */; float* part_o /* [workgroup][2][rows][D] */; float* part_ml /* [workgroup][2][rows][2] */; };

// Few rows (decode steps, drafted tokens): bound by reading the cache, so the pages of all units are dealt out evenly, `quota` consecutive ones to a
// workgroup, however uneven the sequences are.  Which of them are its own a workgroup finds from the lengths itself (one trip to memory and a scan; a
// launch that makes a list would cost more).  Its four waves take 32 keys of every page, each with its own maximum, sum and O; the pages of
// the next iteration are requested before the present ones are used.
template <int D, int RT /* 16-row groups of a unit */>
__global__ __launch_bounds__(256, RT == 1 ? 3 : 2) void ragged_few_kernel(const RaggedArgs a, const FewWs ws)
{
    constexpr int NS = D / 32, NDT = D / 16, ROWS = 16 * RT;
    constexpr int RS = 2 * D + 16;                                // bytes per key of the V tile
    constexpr size_t VOFF = (size_t)128 * (D / 2 + D / 16);
    __shared__ __align__(16) unsigned char stage[4 * 32 * RS];     // per wave: V of 32 keys [key][d]; at the end the waves' sums [4][16][D]
    __shared__ float ml[2][4][ROWS];
    __shared__ int red[4], found[2];

    const int tid = threadIdx.x, lane = tid & 63, cc = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.Hkv;
    unsigned char* stg = stage + wave * (32 * RS);
    const uint32_t tr_base = lds_addr_of(stg) + (uint32_t)((4 * g + (cc >> 2)) * RS + 8 * (cc & 3));

    // this workgroup's pages [w, w_end) of all units', and the sequence that the first of them belongs to
    int all = 0, total;
    for (int b0 = 0; b0 < a.B; b0 += 256) {
        const int n = b0 + tid < a.B ? few_of(a, b0 + tid, G, ROWS).pages : 0;
        const int upto = all + wg_scan256(n, red, total);
        if (blockIdx.x == 0) {
            if (b0 + tid < a.B) ws.front[b0 + tid + 1] = upto;
            if (b0 + tid == 0) ws.front[0] = 0;
        }
        all += total;
    }
    const long long work = (long long)all * a.Hkv;
    const int quota = (int)((work + gridDim.x - 1) / gridDim.x);
    if (blockIdx.x == 0 && tid == 0) *ws.quota = quota;
    long long w = (long long)blockIdx.x * quota;
    const long long w_end = min(w + quota, work);
    if (w >= w_end) return;
    int b = 0, front = 0;
    {
        int at = 0;
        for (int b0 = 0; b0 < a.B; b0 += 256) {
            const int n = b0 + tid < a.B ? few_of(a, b0 + tid, G, ROWS).pages : 0;
            const int upto = at + wg_scan256(n, red, total);
            if (n > 0 && w < (long long)upto * a.Hkv && w >= (long long)(upto - n) * a.Hkv) { found[0] = b0 + tid; found[1] = upto - n; }
            at += total;
            if (w < (long long)at * a.Hkv) break;
        }
        __syncthreads();
        b = __builtin_amdgcn_readfirstlane(found[0]);
        front = __builtin_amdgcn_readfirstlane(found[1]);
    }

    while (w < w_end) {
        Few u = few_of(a, b, G, ROWS);
        while (u.pages == 0 && b + 1 < a.B) u = few_of(a, ++b, G, ROWS);          // (there is one: w < work)
        if (u.pages == 0) return;
        const Seq s = seq_of(a, b);
        const int in_seq = (int)(w - (long long)front * a.Hkv), h = in_seq / u.pages, off = in_seq % u.pages;
        const int cnt = (int)min((long long)(u.pages - off), w_end - w), rows = u.rows;
        const int groups = RT == 1 ? 1 : (rows + 15) / 16;        // of 16 rows

        // Q: row cc of a group of 16, d = (D/4) g + 8 s .. + 7
        half8 qreg[RT][NS];
        float c_row[RT];
        int k_first[RT], k_last[RT];                              // keys that this lane's rows see
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = min(16 * rt + cc, rows - 1), tok = row / G, head = h * G + row % G, pos = s.len - s.n + tok;
            k_first[rt] = a.window > 0 ? pos - a.window + 1 : 0;
            k_last[rt] = a.causal ? min(pos, s.len - 1) : s.len - 1;
            uint4v x[NS];
            float amax = 0.0f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                x[i] = *reinterpret_cast<const uint4v*>(a.q + (size_t)(s.first + tok) * a.q_token + (size_t)head * a.q_head + (D / 4) * g + 8 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(x[i][j] << 16)), fabsf(__uint_as_float(x[i][j] & 0xFFFF0000u))));
            }
            amax = lanes_max<16, 32>(amax);
            float f, inv;
            row_factor(amax, f, inv);
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    qreg[rt][i][2 * j]     = (half_t)(__uint_as_float(x[i][j] << 16) * f);
                    qreg[rt][i][2 * j + 1] = (half_t)(__uint_as_float(x[i][j] & 0xFFFF0000u) * f);
                }
            c_row[rt] = a.c * inv;
        }
        // keys that every row sees: a page inside [see_first, see_last] needs no mask
        const int see_first = a.window > 0 ? s.len - a.window : 0, see_last = a.causal ? s.len - s.n : s.len - 1;

        floatx4 o[RT][NDT];
        float m[RT], l[RT];                                       // the maximum in units of the exponent of 2
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY; l[rt] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[rt][dt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int first = u.first_page + off;
        const int* ids = a.table + (size_t)b * a.max_pages + first;
        int id_lane = 0;

        struct Tile { Raw<D> k[2], v[2]; bool live; };
        auto load = [&](Tile& t, int i) __attribute__((always_inline)) {
            if ((i & 63) == 0) {                                  // 64 page ids at a time, waited for here and not at every use
                id_lane = ids[min(i + lane, cnt - 1)];
                asm volatile("" : "+v"(id_lane));
            }
            const int page = __builtin_amdgcn_readlane(id_lane, i & 63);
            t.live = page >= 0 && page < a.num_pages;
            const unsigned char* part = a.cache + ((size_t)(t.live ? page : 0) * a.Hkv + h) * (2 * VOFF);
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) t.k[blk] = load_raw<D>(part, 32 * wave + 16 * blk + cc, g);
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) t.v[blk] = load_raw<D>(part + VOFF, 32 * wave + 16 * blk + cc, g);
        };
        auto step = [&](const Tile& t, int i) __attribute__((always_inline)) {
            const int kt = (first + i) * 128 + 32 * wave;
            const bool masked = kt < see_first || kt + 31 > see_last;
            floatx4 sc[RT][2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const half2v ks = scales_of<D>(t.k[blk], t.live);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) sc[rt][blk] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < NS; ++j) {
                    const half8 kv = values8<D>(t.k[blk], ks, j);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) if (rt < groups) sc[rt][blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, qreg[rt][j], sc[rt][blk], 0, 0, 0);
                }
            }
            // V through LDS: written key by key, read back with four keys of one d in a lane
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const half2v vs = scales_of<D>(t.v[blk], t.live && kt + 16 * blk + cc < s.len);
#pragma unroll
                for (int j = 0; j < NS; ++j) *reinterpret_cast<half8*>(stg + (16 * blk + cc) * RS + (D / 2) * g + 16 * j) = values8<D>(t.v[blk], vs, j);
            }
            __builtin_amdgcn_wave_barrier();
            half8 pt[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (rt >= groups) break;
                if (masked) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = kt + 16 * (j >> 2) + 4 * g + (j & 3);
                        if (key < k_first[rt] || key > k_last[rt]) sc[rt][j >> 2][j & 3] = -INFINITY;
                    }
                }
                float mx = max_nc(max_nc(max_nc(sc[rt][0][0], sc[rt][0][1]), max_nc(sc[rt][0][2], sc[rt][0][3])),
                                  max_nc(max_nc(sc[rt][1][0], sc[rt][1][1]), max_nc(sc[rt][1][2], sc[rt][1][3])));
                mx = lanes_max<16, 32>(mx) * c_row[rt];
                const float m_new = fmaxf(m[rt], mx), m_at = m_new == -INFINITY ? 0.0f : m_new, alpha = __builtin_amdgcn_exp2f(m[rt] - m_at);
                m[rt] = m_new;
                float add = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[rt][j >> 2][j & 3], c_row[rt], -m_at));
                    add += x;
                    pt[rt][j] = (half_t)x;
                }
                l[rt] = fmaf(l[rt], alpha, add);
                if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) o[rt][dt] *= alpha;
                }
            }
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                const uint2v x = lds_read_tr16_at(tr_base + 32 * dt), y = lds_read_tr16_at(tr_base + 32 * dt + 16 * RS);
                const uint4v av = {x[0], x[1], y[0], y[1]};
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) if (rt < groups) o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, av), pt[rt], o[rt][dt], 0, 0, 0);
            }
        };
        // (two sets of registers by name, and requests that depend on nothing: rotated by copies the compiler waits for everything in flight)
        Tile ta, tb;
        load(ta, 0);
        for (int i = 0; i < cnt; i += 2) {
            load(tb, min(i + 1, cnt - 1));
            step(ta, i);
            if (i + 1 >= cnt) break;
            load(ta, min(i + 2, cnt - 1));
            step(tb, i + 1);
        }

        // the four waves' sums, in units of their common maximum
        const bool whole = cnt == u.pages;
        const size_t slot = (size_t)blockIdx.x * 2 + (off == 0 ? 1 : 0);
        float* sums = reinterpret_cast<float*>(stage);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = lanes_sum<16, 32>(l[rt]);
            if (g == 0) { ml[0][wave][16 * rt + cc] = m[rt]; ml[1][wave][16 * rt + cc] = l[rt]; }
        }
        __syncthreads();
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (16 * rt >= rows) break;
            const int r = 16 * rt + cc;
            const float top = fmaxf(fmaxf(ml[0][0][r], ml[0][1][r]), fmaxf(ml[0][2][r], ml[0][3][r])), f = __builtin_amdgcn_exp2f(m[rt] - (top == -INFINITY ? 0.0f : top));
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) *reinterpret_cast<floatx4*>(sums + (wave * 16 + cc) * D + 16 * dt + 4 * g) = o[rt][dt] * f;
            __syncthreads();
            for (int e = tid; e < min(16, rows - 16 * rt) * (D / 4); e += 256) {
                const int q = e / (D / 4), d = e % (D / 4) * 4, rr = 16 * rt + q;
                const float tp = fmaxf(fmaxf(ml[0][0][rr], ml[0][1][rr]), fmaxf(ml[0][2][rr], ml[0][3][rr])), at = tp == -INFINITY ? 0.0f : tp;
                float lt = 0.0f;
                floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    lt += ml[1][x][rr] * __builtin_amdgcn_exp2f(ml[0][x][rr] - at);
                    v += *reinterpret_cast<const floatx4*>(sums + (x * 16 + q) * D + d);
                }
                if (whole) {
                    const int tk = rr / G, hd = h * G + rr % G;
                    v *= lt != 0.0f ? 1.0f / lt : 0.0f;
                    const uint2v y = {pack_bf16x2_cvt(v[0], v[1]), pack_bf16x2_cvt(v[2], v[3])};
                    *reinterpret_cast<uint2v*>(a.o + (size_t)(s.first + tk) * a.o_token + (size_t)hd * a.o_head + d) = y;
                    if (d == 0 && a.lse) a.lse[(size_t)(s.first + tk) * a.Hq + hd] = lt != 0.0f ? tp * 0.6931471805599453f + logf(lt) : -INFINITY;
                } else {
                    *reinterpret_cast<floatx4*>(ws.part_o + (slot * ROWS + rr) * D + d) = v;
                    if (d == 0) { ws.part_ml[(slot * ROWS + rr) * 2] = tp; ws.part_ml[(slot * ROWS + rr) * 2 + 1] = lt; }
                }
            }
            __syncthreads();
        }
        w += cnt;
        if (off + cnt == u.pages && h == a.Hkv - 1) { front += u.pages; ++b; }
    }
}

// O and lse of the units whose pages were shared, and of rows that see no key: a workgroup per unit and row, whose groups of D / 4 threads take the
// partial sums in turn.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void ragged_few_merge_kernel(const RaggedArgs a, const FewWs ws)
{
    constexpr int NG = 256 / (D / 4);
    __shared__ __align__(16) float acc[NG][D];
    __shared__ float ml[NG][2];
    const int G = a.Hq / a.Hkv, b = blockIdx.x / a.Hkv, h = blockIdx.x % a.Hkv, r = blockIdx.y;
    const int tid = threadIdx.x, grp = tid / (D / 4), d = tid % (D / 4) * 4;
    const Few u = few_of(a, b, G, ROWS);
    if (r >= u.rows || u.rows > ROWS) return;
    const Seq s = seq_of(a, b);
    const int tk = r / G, hd = h * G + r % G;
    uint16_t* dst = a.o + (size_t)(s.first + tk) * a.o_token + (size_t)hd * a.o_head;
    if (u.pages == 0) {
        if (grp == 0) *reinterpret_cast<uint2v*>(dst + d) = uint2v{0u, 0u};
        if (tid == 0 && a.lse) a.lse[(size_t)(s.first + tk) * a.Hq + hd] = -INFINITY;
        return;
    }
    const int quota = *ws.quota;
    const long long w0 = (long long)ws.front[b] * a.Hkv + (long long)h * u.pages, w1 = w0 + u.pages - 1;
    const int f = (int)(w0 / quota), n = (int)(w1 / quota) - f + 1;
    if (n < 2) return;
    float M = -INFINITY, l = 0.0f;
    floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = grp; i0 < n; i0 += 4 * NG) {                      // four at a time: one trip to memory
        floatx4 po[4];
        float pm[4], pl[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = min(i0 + k * NG, n - 1);
            const size_t at = ((size_t)(f + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + r;
            po[k] = *reinterpret_cast<const floatx4*>(ws.part_o + at * D + d);
            pm[k] = i0 + k * NG < n ? ws.part_ml[at * 2] : -INFINITY;
            pl[k] = ws.part_ml[at * 2 + 1];
        }
        const float top = fmaxf(fmaxf(fmaxf(pm[0], pm[1]), fmaxf(pm[2], pm[3])), M), at = top == -INFINITY ? 0.0f : top;
        const float al = __builtin_amdgcn_exp2f(M - at);
        M = top; l *= al; v *= al;
#pragma unroll
        for (int k = 0; k < 4; ++k) { const float x = __builtin_amdgcn_exp2f(pm[k] - at); l = fmaf(pl[k], x, l); v += po[k] * x; }
    }
    *reinterpret_cast<floatx4*>(&acc[grp][d]) = v;
    if (d == 0) { ml[grp][0] = M; ml[grp][1] = l; }
    __syncthreads();
    if (grp != 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < NG; ++k) top = fmaxf(top, ml[k][0]);
    const float at = top == -INFINITY ? 0.0f : top;
    l = 0.0f; v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NG; ++k) { const float x = __builtin_amdgcn_exp2f(ml[k][0] - at); l = fmaf(ml[k][1], x, l); v += *reinterpret_cast<const floatx4*>(&acc[k][d]) * x; }
    v *= l != 0.0f ? 1.0f / l : 0.0f;
    *reinterpret_cast<uint2v*>(dst + d) = uint2v{pack_bf16x2_cvt(v[0], v[1]), pack_bf16x2_cvt(v[2], v[3])};
    if (d == 0 && a.lse) a.lse[(size_t)(s.first + tk) * a.Hq + hd] = l != 0.0f ? top * 0.6931471805599453f + logf(l) : -INFINITY;
}

// Many rows (pieces of prompts): bound by the matrix instructions and the softmax between them.  A workgroup takes a tile of 128 rows, 32 to a wave, and
// walks tiles of 64 keys that its waves unpack together into LDS, K in swizzled rows of fp16, V key by key (padded rows), one tile ahead of the products;
// the codes of the tile after that are in flight meanwhile.
template <int D>
__global__ __launch_bounds__(256, 2) void ragged_wide_kernel(const RaggedArgs a, int most /* rows of a sequence that the kernel for few takes */)
{
    constexpr int ND = D / 16, NB = D / 32, CH = D / 8;           // contraction steps of S, 32-d blocks of O, 16-byte chunks per key
    constexpr int RS = 2 * D + 16;
    constexpr int KB = 64 * 2 * D, VB = 64 * RS;                  // bytes of a tile of K, of V
    constexpr size_t VOFF = (size_t)128 * (D / 2 + D / 16);
    extern __shared__ __align__(256) unsigned char lds[];          // two tiles of K, two of V
    __shared__ int find[8];
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.Hkv, h = blockIdx.y;
    int b, tile;
    if (!find_tile(a, G, most, blockIdx.x, b, tile, find)) return;
    const Seq s = seq_of(a, b);
    const int rows = s.n * G, r0 = tile * kWideRows;
    int lo, hi, wlo = 0, whi = 0;                                 // keys that rows of the workgroup, of this wave see
    keys_of(a, s, r0 / G, (min(r0 + kWideRows, rows) - 1) / G, lo, hi);
    const int w0 = r0 + 32 * wave, row = min(w0 + col, rows - 1);
    if (w0 < rows) keys_of(a, s, w0 / G, (min(w0 + 32, rows) - 1) / G, wlo, whi);
    const int tok = row / G, head = h * G + row % G, pos = s.len - s.n + tok;
    const int k_first = a.window > 0 ? pos - a.window + 1 : 0, k_last = a.causal ? min(pos, s.len - 1) : s.len - 1;
    const int see_first = a.window > 0 ? s.len - s.n + (min(w0 + 32, rows) - 1) / G - a.window + 1 : 0;
    const int see_last = a.causal ? min(s.len - s.n + w0 / G, s.len - 1) : s.len - 1;

    // Q: row col, d = 16 i + 8 half .. + 7
    half8 qreg[ND];
    float c_row;
    {
        uint4v x[ND];
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            x[i] = *reinterpret_cast<const uint4v*>(a.q + (size_t)(s.first + tok) * a.q_token + (size_t)head * a.q_head + 16 * i + 8 * half);
#pragma unroll
            for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(x[i][j] << 16)), fabsf(__uint_as_float(x[i][j] & 0xFFFF0000u))));
        }
        amax = lanes_max<32, 32>(amax);
        float f, inv;
        row_factor(amax, f, inv);
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                qreg[i][2 * j]     = (half_t)(__uint_as_float(x[i][j] << 16) * f);
                qreg[i][2 * j + 1] = (half_t)(__uint_as_float(x[i][j] & 0xFFFF0000u) * f);
            }
        c_row = a.c * inv;
    }

    floatx16 o[NB];
    float m = -INFINITY, l = 0.0f;                                 // the maximum in units of the exponent of 2
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;

    const int t0 = lo >> 6, t1 = (hi + 63) >> 6;                   // tiles of 64 keys
    const int key = tid >> 2, g = tid & 3;                         // what this thread unpacks: D / 4 values of one key
    Raw<D> kr, vr;
    bool live = false;
    auto load = [&](int t) __attribute__((always_inline)) {
        t = min(t, t1 - 1);
        const int page = a.table[(size_t)b * a.max_pages + (t >> 1)];
        live = page >= 0 && page < a.num_pages;
        const unsigned char* part = a.cache + ((size_t)(live ? page : 0) * a.Hkv + h) * (2 * VOFF);
        kr = load_raw<D>(part, (t & 1) * 64 + key, g);
        vr = load_raw<D>(part + VOFF, (t & 1) * 64 + key, g);
    };
    auto unpack = [&](int t, int buf) __attribute__((always_inline)) {
        const bool on = live && t * 64 + key < s.len;             // (keys behind the end: zeros, whatever the slots hold)
        const half2v ks = scales_of<D>(kr, on), vs = scales_of<D>(vr, on);
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            *reinterpret_cast<half8*>(lds + buf * KB + (key * CH + swz<CH>(key, (D / 32) * g + j)) * 16) = values8<D>(kr, ks, j);
            *reinterpret_cast<half8*>(lds + 2 * KB + buf * VB + key * RS + (D / 2) * g + 16 * j) = values8<D>(vr, vs, j);
        }
    };
    const uint32_t k_base = lds_addr_of(lds), v_base = lds_addr_of(lds) + 2 * KB + (uint32_t)((4 * half + ((lane & 15) >> 2)) * RS + 32 * ((lane >> 4) & 1) + 8 * (lane & 3));

    if (t0 < t1) {
        load(t0);
        unpack(t0, 0);
        load(t0 + 1);
    }
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        __syncthreads();                                          // this tile is there, and nobody reads the one that is overwritten next
        if (t + 1 < t1) unpack(t + 1, buf ^ 1);
        load(t + 2);
        if (t * 64 >= whi || t * 64 + 63 < wlo) continue;          // (the wave sees none of these keys)
        floatx16 sc[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int j = 0; j < 16; ++j) sc[kb][j] = 0.0f;
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                const uint4v kv = lds_read16_at(k_base + (uint32_t)(buf * KB + ((32 * kb + col) * CH + swz<CH>(32 * kb + col, 2 * i + half)) * 16));
                sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, kv), qreg[i], sc[kb], 0, 0, 0);
            }
        }
        if (t * 64 < see_first || t * 64 + 63 > see_last) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int k = t * 64 + 32 * kb + (j & 3) + 8 * (j >> 2) + 4 * half;
                    if (k < k_first || k > k_last) sc[kb][j] = -INFINITY;
                }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j) mx = max_nc(mx, sc[kb][j]);
        mx = lanes_max<32, 32>(mx) * c_row;
        const float m_new = fmaxf(m, mx), m_at = m_new == -INFINITY ? 0.0f : m_new, alpha = __builtin_amdgcn_exp2f(m - m_at);
        m = m_new;
        float add = 0.0f;
        half8 pt[4];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float x = __builtin_amdgcn_exp2f(fmaf(sc[kb][j], c_row, -m_at));
                add += x;
                pt[2 * kb + (j >> 3)][j & 7] = (half_t)x;
            }
        l = fmaf(l, alpha, add);
        if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {
#pragma unroll
            for (int i = 0; i < NB; ++i) o[i] *= alpha;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < NB; ++i) {
                const uint2v x = lds_read_tr16_at(v_base + (uint32_t)(buf * VB + 16 * q * RS + 64 * i)), y = lds_read_tr16_at(v_base + (uint32_t)(buf * VB + (16 * q + 8) * RS + 64 * i));
                const uint4v av = {x[0], x[1], y[0], y[1]};
                o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, av), pt[q], o[i], 0, 0, 0);
            }
    }
    if (w0 + col >= rows) return;
    l = lanes_sum<32, 32>(l);
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    uint16_t* dst = a.o + (size_t)(s.first + tok) * a.o_token + (size_t)head * a.o_head;
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *reinterpret_cast<uint2v*>(dst + 32 * i + 8 * j + 4 * half) = uint2v{pack_bf16x2_cvt(o[i][4 * j] * inv, o[i][4 * j + 1] * inv), pack_bf16x2_cvt(o[i][4 * j + 2] * inv, o[i][4 * j + 3] * inv)};
    if (half == 0 && a.lse) a.lse[(size_t)(s.first + tok) * a.Hq + head] = l != 0.0f ? m * 0.6931471805599453f + logf(l) : -INFINITY;
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Which kernels a step may need: the host knows only how many rows a sequence has at most.
struct RaggedPlan { int few_groups; bool wide; int few_wgs; };
inline RaggedPlan plan_of(int T, int B, int Hq, int Hkv, int max_q, int max_pages, int cus)
{
    const long long rows = (long long)(max_q < T ? max_q : T) * (Hq / Hkv), units = (long long)B * Hkv * max_pages;
    RaggedPlan p;
    p.few_groups = rows <= 16 ? 1 : 2;
    p.wide = rows > kFewRows;
    const long long wgs = (long long)cus * (p.few_groups == 1 ? 3 : 2);
    p.few_wgs = (int)(units < wgs ? units : wgs);
    return p;
}
inline FewWs carve_few(void* ws, const RaggedPlan& p, int B, int D, size_t& bytes)
{
    unsigned char* base = (unsigned char*)ws;
    size_t off = 0;
    auto take = [&](size_t n) { unsigned char* r = base + off; off += up256(n); return r; };
    const size_t rows = (size_t)p.few_wgs * 2 * 16 * p.few_groups;
    FewWs w;
    w.quota = (int*)take(4);
    w.front = (int*)take(((size_t)B + 1) * 4);
    w.part_o = (float*)take(rows * D * 4);
    w.part_ml = (float*)take(rows * 8);
    bytes = off;
    return w;
}

template <int D, int RT>
int launch_few(const RaggedArgs& a, const RaggedPlan& p, const FewWs& w, hipStream_t st)
{
    hipLaunchKernelGGL((ragged_few_kernel<D, RT>), dim3(p.few_wgs), dim3(256), 0, st, a, w);
    if (hipGetLastError() != hipSuccess) return -1;
    const int rows = (a.max_q < a.T ? a.max_q : a.T) * (a.Hq / a.Hkv);                        // (the host has checked that T Hq fits)
    hipLaunchKernelGGL((ragged_few_merge_kernel<D, 16 * RT>), dim3(a.B * a.Hkv, rows < 16 * RT ? rows : 16 * RT), dim3(256), 0, st, a, w);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int D>
int launch_wide(const RaggedArgs& a, hipStream_t st)
{
    constexpr int bytes = 2 * 64 * (2 * D + 2 * D + 16);
    static unsigned long long done = 0;
    if (!ensure_dynamic_lds((const void*)ragged_wide_kernel<D>, bytes, done)) return -1;
    const int G = a.Hq / a.Hkv;
    const dim3 grid((unsigned)(a.B + (long long)a.T * G / kWideRows), a.Hkv);
    hipLaunchKernelGGL((ragged_wide_kernel<D>), grid, dim3(256), bytes, st, a, kFewRows);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace

size_t ragged_ws_bytes(int T, int B, int Hq, int Hkv, int max_q, int max_pages, int D)
{
    size_t bytes;
    carve_few(nullptr, plan_of(T, B, Hq, Hkv, max_q, max_pages, kChipCus), B, D, bytes);
    return bytes;
}

int launch_ragged(const RaggedArgs& a, int D, void* ws, hipStream_t st)
{
    const RaggedPlan p = plan_of(a.T, a.B, a.Hq, a.Hkv, a.max_q, a.max_pages, kChipCus);
    size_t bytes;
    const FewWs w = carve_few(ws, p, a.B, D, bytes);
    int rc = D == 128 ? (p.few_groups == 1 ? launch_few<128, 1>(a, p, w, st) : launch_few<128, 2>(a, p, w, st))
                      : (p.few_groups == 1 ? launch_few<64, 1>(a, p, w, st) : launch_few<64, 2>(a, p, w, st));
    if (!rc && p.wide) rc = D == 128 ? launch_wide<128>(a, st) : launch_wide<64>(a, st);
    return rc;
}

}  // namespace aq
