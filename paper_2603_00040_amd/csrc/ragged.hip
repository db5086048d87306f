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

constexpr int kFewRows = 16;          // rows of a tile

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

// The tile number `item` of the step: sequence by sequence, each with ceil(n G / rows) tiles.  By a workgroup of 256; false behind the last one.
__device__ inline bool find_tile(const RaggedArgs& a, int G, int rows, int item, int& b_out, int& tile_out, int* lds /* [8] */)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int b0 = 0; b0 < a.B; b0 += 256) {
        const int b = b0 + tid;
        const int tiles = b < a.B ? (int)(((long long)seq_of(a, b).n * G + rows - 1) / rows) : 0;
        int v = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) { const int u = __shfl_up(v, d); if (lane >= d) v += u; }
        if (lane == 63) lds[wave] = v;
        if (tid == 0) lds[4] = -1;
        __syncthreads();
        for (int w = 0; w < wave; ++w) v += lds[w];
        const int total = lds[0] + lds[1] + lds[2] + lds[3];
        if (item < v && item >= v - tiles) { lds[4] = b; lds[5] = item - (v - tiles); }
        __syncthreads();
        const int hit = lds[4], tile = lds[5];
        __syncthreads();
        if (hit >= 0) { b_out = __builtin_amdgcn_readfirstlane(hit); tile_out = __builtin_amdgcn_readfirstlane(tile); return true; }
        item -= total;
    }
    return false;
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

// One workgroup per tile of 16 rows: its four waves take 32 keys of every page, each with its own maximum, sum and O, which are
// added up at the end.
template <int D>
__global__ __launch_bounds__(256, 2) void ragged_few_kernel(const RaggedArgs a)
{
    constexpr int NS = D / 32, NDT = D / 16;
    constexpr int RS = 2 * D + 16;                                // bytes per key of the V tile
    constexpr size_t VOFF = (size_t)128 * (D / 2 + D / 16);
    __shared__ __align__(16) unsigned char stage[4 * 32 * RS];     // per wave: V of 32 keys [key][d]; at the end the waves' sums [4][16][D]
    __shared__ float ml[2][4][kFewRows];
    __shared__ int find[8];

    const int tid = threadIdx.x, lane = tid & 63, cc = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = a.Hq / a.Hkv, h = blockIdx.y;
    int b, tile;
    if (!find_tile(a, G, kFewRows, blockIdx.x, b, tile, find)) return;
    const Seq s = seq_of(a, b);
    const int rows = s.n * G, r0 = tile * kFewRows, row = min(r0 + cc, rows - 1);
    const int tok = row / G, head = h * G + row % G, pos = s.len - s.n + tok;
    int lo, hi;
    keys_of(a, s, r0 / G, (min(r0 + kFewRows, rows) - 1) / G, lo, hi);
    const int k_first = a.window > 0 ? pos - a.window + 1 : 0, k_last = a.causal ? min(pos, s.len - 1) : s.len - 1;      // what this lane's row sees

    // Q: row cc, d = (D/4) g + 8 s .. + 7
    half8 qreg[NS];
    float c_row;
    {
        uint4v w[NS];
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            w[i] = *reinterpret_cast<const uint4v*>(a.q + (size_t)(s.first + tok) * a.q_token + (size_t)head * a.q_head + (D / 4) * g + 8 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(__uint_as_float(w[i][j] << 16)), fabsf(__uint_as_float(w[i][j] & 0xFFFF0000u))));
        }
        amax = lanes_max<16, 32>(amax);
        float f, inv;
        row_factor(amax, f, inv);
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                qreg[i][2 * j]     = (half_t)(__uint_as_float(w[i][j] << 16) * f);
                qreg[i][2 * j + 1] = (half_t)(__uint_as_float(w[i][j] & 0xFFFF0000u) * f);
            }
        c_row = a.c * inv;
    }

    floatx4 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, l = 0.0f;                                 // in units of the exponent of 2
    unsigned char* stg = stage + wave * (32 * RS);
    const uint32_t tr_base = lds_addr_of(stg) + (uint32_t)((4 * g + (cc >> 2)) * RS + 8 * (cc & 3));

    for (int p = lo >> 7; p * 128 < hi; ++p) {
        const int page = a.table[(size_t)b * a.max_pages + p];
        const bool live = page >= 0 && page < a.num_pages;
        const unsigned char* part = a.cache + ((size_t)(live ? page : 0) * a.Hkv + h) * (2 * VOFF);
        const int kt = p * 128 + 32 * wave;
        Raw<D> kr[2], vr[2];
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) { kr[blk] = load_raw<D>(part, 32 * wave + 16 * blk + cc, g); vr[blk] = load_raw<D>(part + VOFF, 32 * wave + 16 * blk + cc, g); }
        floatx4 sc[2];
        float mx = -INFINITY;
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
            const half2v ks = scales_of<D>(kr[blk], live);
#pragma unroll
            for (int i = 0; i < NS; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(values8<D>(kr[blk], ks, i), qreg[i], acc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int key = kt + 16 * blk + 4 * g + i;
                sc[blk][i] = key < k_first || key > k_last ? -INFINITY : acc[i] * c_row;
                mx = fmaxf(mx, sc[blk][i]);
            }
        }
        mx = lanes_max<16, 32>(mx);
        const float m_new = fmaxf(m, mx), m_at = m_new == -INFINITY ? 0.0f : m_new, alpha = __builtin_amdgcn_exp2f(m - m_at);
        m = m_new;
        l *= alpha;
        half8 pt;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = __builtin_amdgcn_exp2f(sc[i >> 2][i & 3] - m_at);
            l += x;
            pt[i] = (half_t)x;
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
        // V through LDS: written key by key, read back with four keys of one d in a lane
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) {
            const half2v vs = scales_of<D>(vr[blk], live && kt + 16 * blk + cc < s.len);
#pragma unroll
            for (int i = 0; i < NS; ++i) *reinterpret_cast<half8*>(stg + (16 * blk + cc) * RS + (D / 2) * g + 16 * i) = values8<D>(vr[blk], vs, i);
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
            const uint2v x = lds_read_tr16_at(tr_base + 32 * dt), y = lds_read_tr16_at(tr_base + 32 * dt + 16 * RS);
            const uint4v av = {x[0], x[1], y[0], y[1]};
            o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, av), pt, o[dt], 0, 0, 0);
        }
    }

    // the four waves' sums, in units of their common maximum
    l = lanes_sum<16, 32>(l);
    if (g == 0) { ml[0][wave][cc] = m; ml[1][wave][cc] = l; }
    __syncthreads();
    const float top = fmaxf(fmaxf(ml[0][0][cc], ml[0][1][cc]), fmaxf(ml[0][2][cc], ml[0][3][cc])), top_at = top == -INFINITY ? 0.0f : top;
    const float f = __builtin_amdgcn_exp2f(m - top_at);
    float* sums = reinterpret_cast<float*>(stage);
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[(wave * kFewRows + cc) * D + 16 * dt + 4 * g + i] = o[dt][i] * f;
    __syncthreads();
    for (int e = tid; e < kFewRows * D; e += 256) {
        const int r = e / D, d = e % D;
        if (r0 + r >= rows) break;
        const float tp = fmaxf(fmaxf(ml[0][0][r], ml[0][1][r]), fmaxf(ml[0][2][r], ml[0][3][r])), ta = tp == -INFINITY ? 0.0f : tp;
        float lt = 0.0f, v = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) { lt += ml[1][w][r] * __builtin_amdgcn_exp2f(ml[0][w][r] - ta); v += sums[(w * kFewRows + r) * D + d]; }
        const int tk = (r0 + r) / G, hd = h * G + (r0 + r) % G;
        a.o[(size_t)(s.first + tk) * a.o_token + (size_t)hd * a.o_head + d] = f32_to_bf16_rne(lt > 0.0f ? v / lt : 0.0f);
        if (d == 0 && a.lse) a.lse[(size_t)(s.first + tk) * a.Hq + hd] = lt > 0.0f ? tp * 0.6931471805599453f + logf(lt) : -INFINITY;
    }
}

}  // namespace

size_t ragged_ws_bytes(int T, int B, int Hq, int Hkv, int max_q, int max_pages, int D) { return 256; }

int launch_ragged(const RaggedArgs& a, int D, void* ws, hipStream_t st)
{
    const int G = a.Hq / a.Hkv;
    const dim3 grid((unsigned)(a.B + (long long)a.T * G / kFewRows), a.Hkv);
    if (D == 128) hipLaunchKernelGGL((ragged_few_kernel<128>), grid, dim3(256), 0, st, a);
    else          hipLaunchKernelGGL((ragged_few_kernel<64>), grid, dim3(256), 0, st, a);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace aq
