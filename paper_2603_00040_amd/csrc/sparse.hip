// Attention over a choice of the pages of the NVFP4 KV cache: for every query and kv head the first pages, the last ones and those whose keys, by their mean,
// look most like what the query asks for (attnqat_kv_summarize, attnqat_kv_select, attnqat_fwd_kv4_sparse).
//
// The choice is made of whole numbers and powers of two, so that it does not depend on the order of sums: means in 8 bits with a power of two per (page, head),
// the queries of a kv head's group in 8 bits with one power of two between them (which no comparison needs), products in int32.
#include "common.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

namespace aq {

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------- means of the keys of a page
// A cached value is a multiple of 2^-10 below 2^12 (one of a block whose scale is NaN counts as 0), the sum S of a page's 128 a whole number of 2^-10 below 2^29: exact in int32, in any order (four of them in
// fp32, where six would fit).  With the largest |S| of a head in [2^(b-1), 2^b) the codes are S 2^-e, e = b - 7, rounded to nearest even, at most 127 in
// magnitude, and the mean is code 2^(e-17).
//
// A wave takes a (page, head), whole: a key's 32 channels lie with one lane, 16 (D = 64: 32) keys side by side, eight (four) times over, all loads under way at once; sums over
// lanes halve what a lane holds at every step.  A workgroup has four heads of its rows' pages: their parts of a page lie one after another.  Bound by memory for long
// prompts (5 prompts, 100 916 rows, 8 heads of 128, 59 MB of K: 15.0 us, 4.0 TB/s with the launch), by launch and two trips to memory for a step of decodes (600 rows, 8 of
// them complete a page: 3.9 us).
__device__ __forceinline__ uint32_t other_of_8(uint32_t x) { return __builtin_amdgcn_update_dpp(0u, x, 0x128, 0xF, 0xF, true); }                 // of lane ^ 8: row_ror 8
__device__ __forceinline__ uint32_t other_of_4(uint32_t x)
{
    const uint32_t a = __builtin_amdgcn_update_dpp(x, x, 0x104, 0xF, 0x5, false);                                                               // row_shl 4 into quads 0 and 2
    return __builtin_amdgcn_update_dpp(a, x, 0x114, 0xF, 0xA, false);                                                                            // row_shr 4 into quads 1 and 3
}
__device__ __forceinline__ uint32_t other_of_2(uint32_t x) { return __builtin_amdgcn_update_dpp(0u, x, 0x4E, 0xF, 0xF, true); }                  // quad_perm 2,3,0,1

template <int D>
__global__ __launch_bounds__(256) void summarize_kernel(const unsigned char* __restrict__ cache, int num_pages, int Hkv, const long long* __restrict__ slots, int T, int rows_per /* <= 128 */,
                                                        unsigned char* __restrict__ summary)
{
    constexpr int NCH = D / 32, KEYS = 64 / NCH;                  // lanes to a key (32 values each), keys at a time
    const int lane = threadIdx.x & 63, ch = lane % NCH, kk = lane / NCH;
    const int h = (int)blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (h >= Hkv) return;
    const int r0 = (int)blockIdx.x * rows_per, r_end = min(r0 + rows_per, T);
    long long slot[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) slot[i] = slots[min(r0 + 64 * i + lane, T - 1)];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool ends = r0 + 64 * i + lane < r_end && slot[i] >= 0 && slot[i] < (long long)num_pages * 128 && (slot[i] & 127) == 127;
        const int page_lane = (int)(slot[i] >> 7);
        for (unsigned long long left = __builtin_amdgcn_ballot_w64(ends); left != 0; left &= left - 1) {
            const int page = __builtin_amdgcn_readlane(page_lane, (int)__builtin_ctzll(left));
            const unsigned char* k = cache + ((size_t)page * Hkv + h) * nvfp4_page_head_bytes(D);
            uint4v c[128 / KEYS];
            uint32_t sc[128 / KEYS];
#pragma unroll
            for (int p = 0; p < 128 / KEYS; ++p) {
                const int key = p * KEYS + kk;
                c[p] = *reinterpret_cast<const uint4v*>(k + key * (D / 2) + 16 * ch);
                sc[p] = *reinterpret_cast<const uint16_t*>(k + 128 * (D / 2) + key * (D / 16) + 2 * ch);
            }
            int sum[32];
#pragma unroll
            for (int q = 0; q < 32 / KEYS; ++q) {                 // four keys at a time in fp32
                float acc[32];
#pragma unroll
                for (int p = 4 * q; p < 4 * q + 4; ++p) {
                    typedef float float2v __attribute__((ext_vector_type(2)));
                    auto scale_of = [](float s) __attribute__((always_inline)) { return s == s ? s : 0.0f; };                      // (a NaN has no whole number)
                    const float s0 = scale_of(__builtin_amdgcn_cvt_scalef32_f32_fp8(sc[p], 1024.0f, 0)), s1 = scale_of(__builtin_amdgcn_cvt_scalef32_f32_fp8(sc[p], 1024.0f, 1));
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float s = w < 2 ? s0 : s1;
#define AQ_ADD2(J) { const float2v v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[p][w], 1.0f, J); float &a = acc[8 * w + 2 * J], &b = acc[8 * w + 2 * J + 1]; \
                     a = p == 4 * q ? v[0] * s : fmaf(v[0], s, a); b = p == 4 * q ? v[1] * s : fmaf(v[1], s, b); }
                        AQ_ADD2(0) AQ_ADD2(1) AQ_ADD2(2) AQ_ADD2(3)
#undef AQ_ADD2
                    }
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[j] = q == 0 ? (int)acc[j] : sum[j] + (int)acc[j];
            }
            // over lanes ^ 32, ^ 16, ^ 8, ^ 4 (^ 2): the lane whose bit is 0 keeps the lower half of what both hold
#pragma unroll
            for (int j = 0; j < 16; ++j) { const auto r = __builtin_amdgcn_permlane32_swap((uint32_t)sum[j], (uint32_t)sum[j + 16], false, false); sum[j] = (int)(r[0] + r[1]); }
#pragma unroll
            for (int j = 0; j < 8; ++j) { const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)sum[j], (uint32_t)sum[j + 8], false, false); sum[j] = (int)(r[0] + r[1]); }
#define AQ_HALVE(N, BIT, OTHER) _Pragma("unroll") for (int j = 0; j < N; ++j) { const int keep = (lane & BIT) ? sum[j + N] : sum[j], send = (lane & BIT) ? sum[j] : sum[j + N]; sum[j] = keep + (int)OTHER((uint32_t)send); }
            AQ_HALVE(4, 8, other_of_8)
            AQ_HALVE(2, 4, other_of_4)
            int d = 32 * ch + 16 * ((lane >> 5) & 1) + 8 * ((lane >> 4) & 1) + 4 * ((lane >> 3) & 1) + 2 * ((lane >> 2) & 1);
            constexpr int N = D == 64 ? 1 : 2;                    // sums that a lane is left with: channels d ..
            if constexpr (D == 64) { AQ_HALVE(1, 2, other_of_2) d += (lane >> 1) & 1; }
#undef AQ_HALVE
            int most = abs(sum[0]);
            if (N == 2) most = max(most, abs(sum[1]));
            for (int w = 1; w < 64; w <<= 1) most = max(most, __shfl_xor(most, w));
            const int e = (most > 0 ? 32 - __builtin_clz((unsigned)most) : 0) - 7;
            uint32_t code[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                int x;
                if (e <= 0) x = sum[j] * (1 << -e);
                else {
                    x = sum[j] >> e;
                    const int rest = sum[j] - (x << e), half = 1 << (e - 1);
                    x += rest > half || (rest == half && (x & 1)) ? 1 : 0;
                }
                code[j] = (uint32_t)min(max(x, -127), 127) & 0xFFu;
            }
            unsigned char* dst = summary + ((size_t)page * Hkv + h) * (D + kSummaryTail);
            if constexpr (N == 2) *reinterpret_cast<uint16_t*>(dst + d) = (uint16_t)(code[0] | code[1] << 8);
            else dst[d] = (unsigned char)code[0];
            if (lane == 0) *reinterpret_cast<float*>(dst + D) = __uint_as_float((uint32_t)(e + 110) << 23);
        }
    }
}

// ---------------------------------------------------------------------------------------------- what a workgroup's tokens are
// Sequence (-1: of none) and position (below 0: before the first key) of tokens t0 .. t0 + nt - 1 (entries behind them: none).
template <int N>
__device__ inline void find_tokens(const StepArgs& a, int t0, int nt, int (&seq)[N], int (&pos)[N])
{
    const int tid = threadIdx.x;
    if (tid < N) { seq[tid] = -1; pos[tid] = -1; }
    __syncthreads();
    for (int b = tid; b < a.B; b += (int)blockDim.x) {
        const int s = min(max(a.cu_q[b], 0), a.T), e = min(max(a.cu_q[b + 1], s), a.T);
        const int len = max(0, min(a.kv_lens[b], a.max_pages * 128));
        for (int t = max(s, t0); t < min(e, t0 + nt); ++t) { seq[t - t0] = b; pos[t - t0] = max(len - e + t, -1); }
    }
    __syncthreads();
}

// ---------------------------------------------------------------------------------------------- the choice
// Order of floats as of unsigned numbers.
__device__ inline uint32_t ordered(float x) { const uint32_t u = __float_as_uint(x); return (u >> 31) ? ~u : (u | 0x80000000u); }

// The limit that the m best of some scores lie at or above, of which `top` is the largest and count(x) says how many are x or more (x > 0).  It lies not far below the largest
// (scores are floats: half of it is 2^23 away): steps down from that double until there are m scores, and the last step is quartered until a limit has exactly m at or above it,
// or is the m-th largest itself, which others equal: then ties of those are taken.  SIDE: two or three limits are counted side by side, since a count waits for the one before
// (the 3751 tokens below 67.6 us without, 66 with; where a count is many instructions, registers run out).
struct Limit { uint32_t at; int ties; };
template <bool SIDE, class Count>
__device__ __forceinline__ Limit limit_of(uint32_t top, int n, int m, const Count& count)
{
    // at: at least m scores; over: fewer (behind the largest none; 2^32 is 0 here)
    uint32_t at = 1, over = top + 1;
    int c = n;
    for (uint32_t step = 1u << 22; step < top; step <<= SIDE ? 2 : 1) {
        if constexpr (SIDE) {
            const uint32_t far = step < top - step ? top - 2 * step : 1;
            const int near = count(top - step), x = count(far);
            if (near >= m) { at = top - step; c = near; break; }
            over = top - step;
            if (x >= m) { at = far; c = x; break; }
            over = far;
        } else {
            const int x = count(top - step);
            if (x >= m) { at = top - step; c = x; break; }
            over = top - step;
        }
        if (step >> 30) break;
    }
    while (c != m && over - at > 1) {
        const uint32_t w = over - at, a2 = at + w / 2;
        if constexpr (!SIDE) {
            const int x = count(a2);
            if (x >= m) { at = a2; c = x; } else over = a2;
            continue;
        }
        const uint32_t a1 = at + w / 4, a3 = a2 + w / 4;
        const int c1 = count(a1), c2 = count(a2), c3 = count(a3);
        if (c3 >= m) { at = a3; c = c3; }
        else if (c2 >= m) { at = a2; c = c2; over = a3; }
        else if (c1 >= m) { at = a1; c = c1; over = a2; }
        else over = a1;
    }
    return Limit{at, c == m ? n : m - (at == top ? 0 : count(at + 1))};
}
__device__ inline uint32_t wave_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, true));          // rows of 16, turned by 8, 4, 2, 1
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xF, 0xF, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xF, 0xF, true));
    const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return (uint32_t)uniform((int)max(b[0], b[1]));
}
// Those of a wave's scores x (0: none) that are taken, to out as numbers, in the order of the lanes.
__device__ __forceinline__ void emit(uint32_t x, int number, uint32_t at, int n, int& ties, int*& out)
{
    const unsigned long long below = (1ull << (threadIdx.x & 63)) - 1;
    bool take = x >= at;
    if (ties < n) {
        const unsigned long long eq = __builtin_amdgcn_ballot_w64(x == at);
        take = x > at || (x == at && (int)__builtin_popcountll(eq & below) < ties);
        ties -= min(ties, (int)__builtin_popcountll(eq));
    }
    const unsigned long long all = __builtin_amdgcn_ballot_w64(take);
    if (take) out[(int)__builtin_popcountll(all & below)] = number;
    out += (int)__builtin_popcountll(all);
}
// The m best of n scores (0 < m < n; scores from `key` on, in LDS), lowest first among equals, to out as page numbers first + index, ascending.  By a wave, with its scores
// in R registers (64 R of them at most; R = 0: read from LDS every time).  The m-th largest of the lanes' largest is no more than the m-th largest of all, and few
// scores beyond the m are as large: these go on alone, one to a lane (best, which: 64 places of the wave's in LDS).
template <int R>
__device__ inline void best_of(const uint32_t* key, int n, int m, int first, int* out, uint32_t* best, uint16_t* which)
{
    const int lane = threadIdx.x & 63;
    uint32_t k[R > 0 ? R : 1];
    uint32_t mine = 0;
    if constexpr (R > 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) { k[r] = 64 * r + lane < n ? key[64 * r + lane] : 0u; mine = max(mine, k[r]); }
    } else
        for (int j = lane; j < n; j += 64) mine = max(mine, key[j]);
    const uint32_t top = wave_max(mine);
    if constexpr (R > 1) {
        if (m <= 64) {
            const uint32_t from = limit_of<true>(top, 64, m, [&](uint32_t x) __attribute__((always_inline)) { return (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(mine >= x)); }).at;
            int c = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const unsigned long long in = __builtin_amdgcn_ballot_w64(k[r] >= from);
                const int at = c + (int)__builtin_popcountll(in & ((1ull << lane) - 1));
                if (k[r] >= from && at < 64) { best[at] = k[r]; which[at] = (uint16_t)(64 * r + lane); }
                c += (int)__builtin_popcountll(in);
            }
            if (c <= 64) {
                __builtin_amdgcn_wave_barrier();
                const uint32_t x = lane < c ? best[lane] : 0u;
                Limit l{from, c};
                if (c > m) l = limit_of<true>(top, c, m, [&](uint32_t f) __attribute__((always_inline)) { return (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(x >= f)); });
                emit(x, first + which[lane], l.at, c, l.ties, out);
                return;
            }
        }
    }
    const Limit l = limit_of<R == 1>(top, n, m, [&](uint32_t from) __attribute__((always_inline)) {
        int c = 0;
        if constexpr (R > 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) c += (int)__builtin_popcountll(__builtin_amdgcn_ballot_w64(k[r] >= from));
        } else {
            for (int j = lane; j < n; j += 64) c += key[j] >= from ? 1 : 0;
            c = lane_total(c);
        }
        return c;
    });
    int ties = l.ties;
    if constexpr (R > 0) {
#pragma unroll
        for (int r = 0; r < R; ++r) if (64 * r < n) emit(k[r], first + 64 * r + lane, l.at, n, ties, out);
    } else
        for (int j0 = 0; j0 < n; j0 += 64) emit(j0 + lane < n ? key[j0 + lane] : 0u, first + j0 + lane, l.at, n, ties, out);
}

// 16 rows of the matrix instruction are the query heads of a kv head's group, padded to GP by heads that are there, for 16 / GP tokens, against 16 pages at a
// time.  Scores stay in LDS; then a wave has a token.  What bounds it: one token over 938 pages, 32/8 heads of 128, 11.6 us, trips to memory that wait for each other
// (lengths, page ids, means) and the search, whose steps are chains of counts over a wave; 32 tokens of 63 - 375 pages 9.2 us; 3751 tokens over up to 470 pages 66 us, vector
// instructions for 33 % of it.
template <int D, int GP>
__global__ __launch_bounds__(1024) void select_kernel(const SelectArgs a, int nt /* tokens of a workgroup */, int tiles)
{
    constexpr int NS = D / 64, NC = D / 8;                        // steps of the contraction, eights of a row
    extern __shared__ uint32_t keys[];                            // [nt][max_pages]
    __shared__ __align__(16) unsigned char q8s[16][D];
    __shared__ uint32_t amax_s[16], best[16][64];
    __shared__ uint16_t which[16][64];
    __shared__ int seq[16], pos[16];
    const StepArgs& s = a.s;
    const int tid = threadIdx.x, lane = tid & 63, cc = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = s.Hq / s.Hkv, subs = (G + 15) / 16, S = s.max_pages, waves = (int)blockDim.x >> 6;
    int h, tile;
    head_tile_of_block((int)blockIdx.x, s.Hkv, tiles, h, tile);
    const int t0 = tile * nt;

    // Q in 8 bits, eight values to a thread of the first four (D = 64: two) waves: one power of two for a token's group brings its largest magnitude to
    // [64, 128) (magnitudes below 2^-121 count as that)
    const int qrow = tid / NC, qtok = min(qrow / GP, nt - 1);
    const bool has_q = qrow < 16;
    uint4v x[1];
    auto load_q = [&](int sub) __attribute__((always_inline)) {
        x[0] = *reinterpret_cast<const uint4v*>(s.q + (size_t)min(t0 + qtok, s.T - 1) * s.q_token + (size_t)(h * G + min(16 * sub + qrow % GP, G - 1)) * s.q_head + 8 * (tid % NC));
    };
    if (tid < 16) amax_s[tid] = 0;
    if (has_q) load_q(0);
    find_tokens(s, t0, nt, seq, pos);                             // (two barriers)
    for (int sub = 0; sub < subs; ++sub) {
        if (!has_q) break;
        if (sub > 0) load_q(sub);
        atomicMax(&amax_s[qtok], __float_as_uint(largest_of(x)));
    }
    const int seq_lane = seq[cc], pos_lane = pos[cc];

    for (int sub = 0; sub < subs; ++sub) {
        __syncthreads();                                          // (amax_s is whole; q8s has been read)
        if (has_q) {
            if (subs > 1) load_q(sub);
            const float f = __uint_as_float((260u - max(amax_s[qtok] >> 23, 6u)) << 23);
            uint2v r;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t p = x[0][2 * i + (j >> 1)];
                    // (1.5 2^23 added: rounded to nearest even, in two's complement in the low bits)
                    v[j] = __float_as_uint(__builtin_amdgcn_fmed3f(__uint_as_float((j & 1) ? p & 0xFFFF0000u : p << 16) * f, -127.0f, 127.0f) + 12582912.0f);
                }
                r[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(v[3], v[2], 0x0C0C0400u), __builtin_amdgcn_perm(v[1], v[0], 0x0C0C0400u), 0x05040100u);
            }
            *reinterpret_cast<uint2v*>(&q8s[qrow][8 * (tid % NC)]) = r;
        }
        __syncthreads();
        intx4 q8[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) q8[i] = *reinterpret_cast<const intx4*>(&q8s[cc][64 * i + 16 * g]);
        for (int i0 = 0, i1; i0 < nt; i0 = i1) {                  // tokens of one sequence
            const int b = __builtin_amdgcn_readlane(seq_lane, i0);
            int hi = 0;                                           // behind the last page that competes
            for (i1 = i0; i1 < nt && __builtin_amdgcn_readlane(seq_lane, i1) == b; ++i1) {
                const int own = __builtin_amdgcn_readlane(pos_lane, i1) >> 7;
                if (own + 1 > a.n_blocks) hi = max(hi, own + 1 - a.last);
            }
            if (b < 0) continue;
            constexpr int U = 2;                                  // sixteens of pages under way at once (the 3751 tokens: 66 us; with one 79, with four 65, but 32 tokens 9.5 instead of 9.2)
            for (int j1 = (a.first & ~15) + 16 * wave; j1 < hi; j1 += 16 * U * waves) {
                // (a lane asks for the id and the scale of a page of sixteen g, and hands them to the lanes that need them: the way to memory takes a load of one
                // dword for sixteen pages as long as one of sixteen bytes)
                const int mine = s.table[(size_t)b * s.max_pages + min(j1 + 16 * (g % U) * waves + cc, s.max_pages - 1)];
                const bool live = mine >= 0 && mine < s.num_pages;
                const int page = live ? mine : 0;
                float scale_mine = *reinterpret_cast<const float*>(a.summary + ((size_t)page * s.Hkv + h) * (D + kSummaryTail) + D);
                intx4 k8[U][NS];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const unsigned char* rec = a.summary + ((size_t)__shfl(page, 16 * u + cc) * s.Hkv + h) * (D + kSummaryTail);
#pragma unroll
                    for (int i = 0; i < NS; ++i) k8[u][i] = *reinterpret_cast<const intx4*>(rec + 64 * i + 16 * g);
                }
                if (!live) scale_mine = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int j = j1 + 16 * u * waves + cc;
                    if (j - cc >= hi) break;
                    const float scale = __shfl(scale_mine, 16 * u + cc);
                    intx4 acc = {0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < NS; ++i) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(q8[i], k8[u][i], acc, 0, 0, 0);
                    // rows 4 g .. 4 g + 3 of page j: the largest of a token's heads
                    auto put = [&](int token, int v) __attribute__((always_inline)) {
                        if (token < i0 || token >= i1 || j >= hi) return;
                        const uint32_t key = max(ordered(fmaf((float)v, scale, 0.0f)), 1u);
                        uint32_t* p = keys + token * S + j;
                        *p = sub == 0 ? key : max(*p, key);
                    };
                    if constexpr (GP == 1) { put(4 * g, acc[0]); put(4 * g + 1, acc[1]); put(4 * g + 2, acc[2]); put(4 * g + 3, acc[3]); }
                    else if constexpr (GP == 2) { put(2 * g, max(acc[0], acc[1])); put(2 * g + 1, max(acc[2], acc[3])); }
                    else {
                        int m = max(max(acc[0], acc[1]), max(acc[2], acc[3]));
                        if constexpr (GP >= 8) { const auto r = __builtin_amdgcn_permlane16_swap((uint32_t)m, (uint32_t)m, false, false); m = max((int)r[0], (int)r[1]); }
                        if constexpr (GP >= 16) { const auto r = __builtin_amdgcn_permlane32_swap((uint32_t)m, (uint32_t)m, false, false); m = max((int)r[0], (int)r[1]); }
                        if (GP == 4 || (GP == 8 && (g & 1) == 0) || g == 0) put(4 * g / GP, m);
                    }
                }
            }
        }
    }
    __syncthreads();

    for (int i = wave; i < nt; i += waves) {
        if (__builtin_amdgcn_readlane(seq_lane, i) < 0) continue;
        const int nb = (__builtin_amdgcn_readlane(pos_lane, i) >> 7) + 1;                  // (position -1: no page)
        int* out = a.blocks + ((size_t)(t0 + i) * s.Hkv + h) * a.n_blocks;
        if (nb <= a.n_blocks) {
            for (int j = lane; j < a.n_blocks; j += 64) out[j] = j < nb ? j : -1;
            continue;
        }
        for (int j = lane; j < a.first; j += 64) out[j] = j;
        for (int j = lane; j < a.last; j += 64) out[a.n_blocks - a.last + j] = nb - a.last + j;
        const int n = nb - a.first - a.last, m = a.n_blocks - a.first - a.last;            // n > m
        if (m == 0) continue;
        const uint32_t* key = keys + i * S + a.first;
        out += a.first;
        // (scores in registers: one token over 938 pages 11.6 us, 23 with all of them read from LDS for every count; the 3751 tokens 66 and 78)
        if (n <= 64) best_of<1>(key, n, m, a.first, out, best[wave], which[wave]);
        else if (n <= 256) best_of<4>(key, n, m, a.first, out, best[wave], which[wave]);
        else if (n <= 512) best_of<8>(key, n, m, a.first, out, best[wave], which[wave]);
        else if (n <= 1024) best_of<16>(key, n, m, a.first, out, best[wave], which[wave]);
        else best_of<0>(key, n, m, a.first, out, best[wave], which[wave]);
    }
}

// ---------------------------------------------------------------------------------------------- attention
constexpr float kNoScore = -0x1p126f; // the reference of a row that has none yet: finite, so that differences of two are, also of waves and pieces without a score; no score lies as low
constexpr int kEntries = 2048;        // (token, page)s of a workgroup at most

// 16 rows: the G query heads of a kv head for nt tokens (rows = token * G + head of the group), or 16 of more heads for one token.  Their pages are taken together, each
// once, whichever of the tokens asked for it; split over `splits` workgroups, or over groups of four waves of one workgroup, where there are few rows.
//
// Scores are computed transposed, S^T = K Q^T, so that a lane has one row, its maximum and sum are the lane's, and P^T is what O^T += V^T P^T takes.  K goes from memory into
// registers, is unpacked (exact in fp16) and multiplied; V goes through LDS, written key by key and read transposed.  A wave has 32 keys of a page, four waves a page, and the next
// page is on its way while one is worked on.  Q is exact in fp16 by a power of two per row; the probabilities are rounded to fp16, by a relative 2^-12 down to 2^-25 of
// a row's largest, because that is the product's type; scores, sums and O are fp32.
//
// What bounds it.  One token, 32 pages, 32/8 heads of 128: 7.5 us and 4.5 to join, trips to memory one after another (choice, lengths, page ids, page).  32 tokens of 32 pages each
// (157 MB): 36 us, 4.3 TB/s, from memory.  Pieces of three prompts, 3751 tokens of 24 pages each, 196 GFLOP: 1.00 ms, the vector instructions: they issue for 81 % of the time
// (exponentials four times as long; matrix instructions 21 %, LDS 37 %), 226 for a wave's 32 keys, of which unpacking K and V, a conversion and a multiplication for two values,
// is 136; a wave's 16 rows cost as much with all four tokens in a page as with one (four tokens visit 66 pages where they asked for 96).  Two sixteens of rows to a wave share the
// unpacking but leave three waves to a SIMD: 5 % slower; four and two: 8 %; rows of 16 or 32 tokens gathered page by page, P through LDS: 6 and 19 %; waves that score and waves
// that add, a barrier between them: 13 %.
struct SparsePlan { int nt, subs, tiles, splits, waves; };
constexpr int sparse_stage(int D, int waves) { return waves * 32 * (2 * D + 32); }        // bytes of LDS beside the list of pages
struct SparseWs { float *part_o /* [unit][split][16][D] */, *part_ml /* [unit][split][16][2]: maximum, sum; a sum below 0: not a row of any sequence */; };

// The pages that any of a workgroup's tokens asks for, each once, sequence by sequence: page of the sequence, and the tokens that ask for it << 16.  tab: `cap` words, 16 bits
// for every page of a sequence, zeros as far as tab_words() says; sequences that do not fit it together take their turns.  first: the choice number threadIdx.x of the
// tokens', asked for ahead.  Returns how many.
__device__ inline int tab_words(const StepArgs& s, int nt, int cap) { return min(nt * ((s.max_pages + 1) / 2), cap); }
__device__ inline int choice_of(const StepArgs& s, const int* __restrict__ blocks, int n_blocks, int h, int t0, int nt, int x)
{
    const int t = t0 + x / n_blocks;
    return x < nt * n_blocks && t < s.T ? blocks[((size_t)t * s.Hkv + h) * n_blocks + x % n_blocks] : -1;
}
template <int NW>
__device__ inline int pages_of_tokens(const StepArgs& s, const int* __restrict__ blocks, int n_blocks, int h, int t0, int nt, const int (&seq)[16], const int (&pos)[16], int first,
                                      uint32_t* tab, int cap, uint32_t* ents, int* red)
{
    const int tid = threadIdx.x, seq_lane = seq[tid & 15], pos_lane = pos[tid & 15];
    int total = 0;
    for (int i0 = 0, i1; i0 < nt; i0 = i1) {
        // where each token's sequence has its words, as many sequences as fit
        int words = 0, base_lane = -1;
        for (i1 = i0; i1 < nt;) {
            const int b = __builtin_amdgcn_readlane(seq_lane, i1);
            int nb = 0, j = i1;
            for (; j < nt && __builtin_amdgcn_readlane(seq_lane, j) == b; ++j) nb = max(nb, (__builtin_amdgcn_readlane(pos_lane, j) >> 7) + 1);
            const int w = b < 0 ? 0 : (nb + 1) / 2;
            if (words + w > cap) break;                           // (one alone fits)
            if (w > 0 && (tid & 15) >= i1 && (tid & 15) < j) base_lane = words;
            words += w;
            i1 = j;
        }
        if (i0 > 0) {
            for (int w = tid; w < words; w += 64 * NW) tab[w] = 0;
            __syncthreads();
        }
        // (waves go round whole: a lane reads what the token's lane has, and one that has left a loop reads as 0)
        for (int x0 = i0 * n_blocks + uniform(tid & ~63); x0 < i1 * n_blocks; x0 += 64 * NW) {
            const int x = x0 + (tid & 63), i = min(x / n_blocks, 15);
            const int base = __shfl(base_lane, i), last = __shfl(pos_lane, i) >> 7;
            if (x >= i1 * n_blocks || base < 0) continue;
            const int blk = x == tid ? first : choice_of(s, blocks, n_blocks, h, t0, nt, x);
            if (blk >= 0 && blk <= last) atomicOr(&tab[base + (blk >> 1)], 1u << (i + 16 * (blk & 1)));
        }
        __syncthreads();
        for (int w0 = 0; w0 < words; w0 += 64 * NW) {
            const uint32_t w = w0 + tid < words ? tab[w0 + tid] : 0u;
            int base = 0;
            for (int i = i0; i < i1; ++i) { const int x = __builtin_amdgcn_readlane(base_lane, i); if (w0 + tid >= x) base = max(base, x); }
            const int page = 2 * (w0 + tid - base), n = ((w & 0xFFFFu) != 0) + ((w >> 16) != 0);
            int all;
            int at = total + wg_scan<NW>(n, red, all) - n;
            if (w & 0xFFFFu) ents[at++] = (uint32_t)page | w << 16;
            if (w >> 16) ents[at] = (uint32_t)(page + 1) | (w & 0xFFFF0000u);
            total += all;
        }
        __syncthreads();
    }
    return total;
}

// Those pages, from the first of `cnt` on: what a wave has of one, 32 keys of K and V, and the lists behind it, 64 entries at a time in the lanes.  Addresses are a
// page's, in scalar registers, and a lane's offsets, made once.
template <int D> struct PageTile { Raw<D> k[2], v[2]; uint32_t ent; int end, all; };
template <int D>
struct PageWalk {
    const StepArgs& s; const unsigned char* cache /* of the head */; const uint32_t* ents; const int *seq, *pos; int cnt;
    uint32_t codes, scales;           // this lane's offsets in a part of a page's head
    int ent_lane, id_lane, end_lane, all_lane, id_end;            // of entry id_end - 64 + lane: itself, its page, the last key that any of its tokens sees, and that all of them see
    __device__ __forceinline__ void ids(int i0)
    {
        ent_lane = (int)ents[min(i0 + (int)(threadIdx.x & 63), cnt - 1)];
        const int last = 15 - __builtin_clz((uint32_t)ent_lane), b = seq[last];            // (tokens of one sequence follow each other: the last sees most)
        end_lane = pos[last];
        all_lane = pos[__builtin_ctz((uint32_t)ent_lane >> 16)];
        id_lane = s.table[(size_t)b * s.max_pages + (ent_lane & 0xFFFF)];
        asm volatile("" : "+v"(id_lane));                         // (waited for here and not at every use)
        id_end = i0 + 64;
    }
    __device__ __forceinline__ void begin(int wave, int cc, int g)
    {
        codes = (uint32_t)((32 * wave + cc) * (D / 2) + (D / 8) * g);
        scales = (uint32_t)(128 * (D / 2) + (32 * wave + cc) * (D / 16) + (D == 128 ? 4 * (g >> 1) : 0));
        ids(0);
    }
    __device__ __forceinline__ Raw<D> raw(const unsigned char* part, uint32_t key) const
    {
        uint32_t codes = this->codes, scales = this->scales;
        asm("" : "+v"(codes), "+v"(scales));                      // (32 bits beside a scalar address; widened in front of the loop they would be added to it by vector instructions)
        Raw<D> r;
        if constexpr (D == 128) {
            const uint4v c = *reinterpret_cast<const uint4v*>(part + key * (D / 2) + codes);
            r.w[0] = c[0]; r.w[1] = c[1]; r.w[2] = c[2]; r.w[3] = c[3];
        } else {
            const uint2v c = *reinterpret_cast<const uint2v*>(part + key * (D / 2) + codes);
            r.w[0] = c[0]; r.w[1] = c[1];
        }
        r.sc = *reinterpret_cast<const uint32_t*>(part + key * (D / 16) + scales);
        return r;
    }
    __device__ __forceinline__ void load(PageTile<D>& t, int i)
    {
        constexpr size_t HALF = (size_t)128 * (D / 2 + D / 16);
        if (i >= id_end) ids(id_end);
        const int at = i - (id_end - 64), page = __builtin_amdgcn_readlane(id_lane, at);
        const bool live = page >= 0 && page < s.num_pages;
        t.ent = (uint32_t)__builtin_amdgcn_readlane(ent_lane, at);
        t.all = __builtin_amdgcn_readlane(all_lane, at);
        t.end = live ? __builtin_amdgcn_readlane(end_lane, at) : -1;                       // (V, and K below, are zeros from here on)
        const unsigned char* part = cache + (size_t)(live ? page : 0) * s.Hkv * (2 * HALF);
        const unsigned char* values = part + HALF;
        asm("" : "+s"(values));                                   // (the distance is more than a load adds)
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) t.k[blk] = raw(part, 16 * blk);
#pragma unroll
        for (int blk = 0; blk < 2; ++blk) t.v[blk] = raw(values, 16 * blk);
    }
};

// NaN scales among a wave's 32 keys of V (lane (cc, g) has those of keys cc and 16 + cc, as scales_of() gives them): the matrix instruction would carry them to every
// row, a probability of 0 times NaN being NaN, so rows that see such a key get their NaN here, and the product zeros.  seen: how many of the keys, from the first on,
// the lane's row sees.
template <int D>
__device__ __forceinline__ void nan_of_v(half2v (&vs)[2], floatx4 (&o)[D / 16], int seen)
{
    constexpr int H = D / 64;                                     // blocks of 16 of a lane
    const uint32_t keys = seen >= 32 ? 0xFFFFFFFFu : (1u << max(seen, 0)) - 1u;
    unsigned long long bad[2][H];
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const bool is = vs[blk][i] != vs[blk][i];
            bad[blk][i] = __builtin_amdgcn_ballot_w64(is);
            if (is) vs[blk][i] = (half_t)0.0f;
        }
#pragma unroll
    for (int dt = 0; dt < D / 16; ++dt) {
        const int sh = 16 * (dt / H), i = dt % H;
        const uint32_t b = ((uint32_t)(bad[0][i] >> sh) & 0xFFFFu) | (uint32_t)(bad[1][i] >> sh) << 16;
        if ((b & keys) != 0) o[dt] = floatx4{NAN, NAN, NAN, NAN};
    }
}

template <int D, int NW /* waves: 4, or 16 where a unit's pages are not split */>
__global__ __launch_bounds__(64 * NW, 4) void sparse_kernel(const SparseArgs a, const SparsePlan p, const SparseWs ws)
{
    constexpr int NS = D / 32, NDT = D / 16;
    constexpr int RS = 2 * D + 32;                                // bytes per key of the V tile
    constexpr size_t VOFF = (size_t)128 * (D / 2 + D / 16);
    // first which tokens ask for a page, 16 bits each; then per wave V of 32 keys; at the end the waves' sums
    extern __shared__ __align__(16) unsigned char stage[];
    constexpr int kStage = sparse_stage(D, NW);
    uint32_t* ents = reinterpret_cast<uint32_t*>(stage + kStage);  // page of the sequence, and the tokens that ask for it << 16
    __shared__ float ml[2][NW][16];
    __shared__ int seq[16], pos[16], red[NW];
    const StepArgs& s = a.s;
    const int tid = threadIdx.x, lane = tid & 63, cc = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = s.Hq / s.Hkv;
    int h, rest;
    head_tile_of_block((int)blockIdx.x, s.Hkv, p.tiles * p.subs * p.splits, h, rest);
    const int split = rest % p.splits, sub = rest / p.splits % p.subs, tile = rest / p.splits / p.subs;
    const int t0 = tile * p.nt, rows = p.subs > 1 ? min(16, G - 16 * sub) : p.nt * G;

    // this lane's row: its token and head
    const int r = min(cc, rows - 1), tok = p.subs > 1 ? 0 : r / G, head = h * G + (p.subs > 1 ? 16 * sub + r : r % G);
    uint4v x[NS];
    {
        const uint16_t* q = s.q + (size_t)min(t0 + tok, s.T - 1) * s.q_token + (size_t)head * s.q_head + (D / 4) * g;
#pragma unroll
        for (int i = 0; i < NS; ++i) x[i] = *reinterpret_cast<const uint4v*>(q + 8 * i);
    }
    const int first = choice_of(s, a.blocks, a.n_blocks, h, t0, p.nt, tid);
    constexpr int cap = sparse_stage(D, 4) / 4;
    static_assert(cap >= 8192 / 2);
    uint32_t* tab = reinterpret_cast<uint32_t*>(stage);
    for (int w = tid; w < tab_words(s, p.nt, cap); w += 64 * NW) tab[w] = 0;
    find_tokens(s, t0, p.nt, seq, pos);
    const int total = pages_of_tokens<NW>(s, a.blocks, a.n_blocks, h, t0, p.nt, seq, pos, first, tab, cap, ents, red);
    const int e0 = (int)((long long)total * split / p.splits), cnt = (int)((long long)total * (split + 1) / p.splits) - e0;

    const int k_last = pos[tok];
    const uint32_t row_bit = 1u << (16 + tok);
    floatx4 o[NDT];
    float m = kNoScore, up_to = -INFINITY, l = 0.0f;
    uint32_t asked = 0;                                           // tokens that asked for any page
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const int group = wave >> 2;                                  // of four waves: pages group, group + NW / 4 ..
    if (group < cnt) {
        unsigned char* stg = stage + wave * (32 * RS);
        // (the two 16-byte pieces of every 32 change places in keys 4 - 7 of 8: a store serves eight lanes, eight keys, at a time on 32 banks)
        const uint32_t tr_base = lds_addr_of(stg) + (uint32_t)((4 * g + (cc >> 2)) * RS + 8 * ((cc & 3) ^ (2 * (g & 1))));
        PageWalk<D> walk{s, a.cache + (size_t)h * (2 * VOFF), ents + e0, seq, pos, cnt};
        walk.begin(wave & 3, cc, g);
        PageTile<D> t;
        walk.load(t, group);

        // Q: row cc, d = (D/4) g + 8 s .. + 7
        half8 qreg[NS];
        float c_row;
        {
            const float amax = lanes_max<16, 32>(largest_of(x));
            float f, inv;
            row_factor(amax, f, inv);
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    qreg[i][2 * j]     = (half_t)(__uint_as_float(x[i][j] << 16) * f);
                    qreg[i][2 * j + 1] = (half_t)(__uint_as_float(x[i][j] & 0xFFFF0000u) * f);
                }
            c_row = fmaxf(a.c * inv, kLeastFactor);
        }
        for (int i = group; i < cnt; i += NW / 4) {
            const uint32_t ent = t.ent;
            const int kt = (int)(ent & 0xFFFFu) * 128 + 32 * (wave & 3), end = t.end, all = t.all;
            const bool member = (ent & row_bit) != 0;
            if (kt + 31 > end) {                                  // behind a sequence's end there may be anything, and a page outside the cache reads as zeros
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    if (kt + 16 * blk + cc > end) t.v[blk].sc = 0;
                    if (end < 0) t.k[blk].sc = 0;
                }
            }
            asked |= ent;
            floatx4 sc[2];
            const half2v ks[2] = {scales_of<D>(t.k[0], g, true), scales_of<D>(t.k[1], g, true)};
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                sc[blk] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < NS; ++j) sc[blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values8<D>(t.k[blk], ks[blk], j), qreg[j], sc[blk], 0, 0, 0);
            }
            // V through LDS: written key by key, read back with four keys of one d in a lane
            __builtin_amdgcn_wave_barrier();
            half2v vs[2] = {scales_of<D>(t.v[0], g, true), scales_of<D>(t.v[1], g, true)};
            // (scales are NaN or finite.  Rows that do not ask for the page: another sequence's keys may be NaN)
            const float any_nan = __builtin_amdgcn_fdot2(vs[0], vs[1], __builtin_amdgcn_fdot2(ks[0], ks[1], 0.0f, false), false);
            if (__builtin_amdgcn_ballot_w64(any_nan != any_nan) != 0) {
                nan_of_v<D>(vs, o, member ? k_last - kt + 1 : 0);
                if (!member) sc[0] = sc[1] = floatx4{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            }
#pragma unroll
            for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                for (int j = 0; j < NS; ++j) *reinterpret_cast<half8*>(stg + (16 * blk + cc) * RS + (D / 2) * g + 16 * (j ^ ((cc >> 2) & 1))) = values8<D>(t.v[blk], vs[blk], j);
            __builtin_amdgcn_wave_barrier();
            walk.load(t, min(i + NW / 4, cnt - 1));
            if (kt + 31 > all) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (kt + 16 * (j >> 2) + 4 * g + (j & 3) > k_last) sc[j >> 2][j & 3] = -INFINITY;
            }
            float mx = max_nc(max_nc(sc[0][0], sc[0][1]), sc[0][2]);                       // (chains of three)
            mx = max_nc(max_nc(mx, sc[0][3]), sc[1][0]);
            mx = max_nc(max_nc(mx, sc[1][1]), sc[1][2]);
            mx = max_nc(mx, sc[1][3]);
            mx = xor_tree<16, 32>(mx, [](float a, float b) __attribute__((always_inline)) { return max_raw(a, b); });
            mx = member ? mx : -INFINITY;
            if (__builtin_amdgcn_ballot_w64(mx > up_to) != 0) {
                const float m_new = fmaxf(m, fmaf(mx, c_row, -kTop)), alpha = __builtin_amdgcn_exp2f(m - m_new);
                m = m_new;
                up_to = score_up_to(m_new, c_row);
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
            }
            const float m_at = member ? m : INFINITY;             // (rows that do not ask for the page: probabilities of 0)
            float add;
            half8 pt;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = __builtin_amdgcn_exp2f(fmaf(sc[j >> 2][j & 3], c_row, -m_at));
                add = j == 0 ? x : add + x;
                pt[j] = (half_t)x;
            }
            l += add;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                const uint2v u = lds_read_tr16_at(tr_base + 32 * dt), w = lds_read_tr16_at(tr_base + 32 * dt + 16 * RS);
                const uint4v av = {u[0], u[1], w[0], w[1]};
                o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, av), pt, o[dt], 0, 0, 0);
            }
        }
    }

    // (a row that asked for nothing has nothing, whatever its query was)
    if ((asked & row_bit) == 0) {
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[dt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    // the waves' sums, in units of their common maximum
    constexpr int SS = D + 4;                                     // floats per row of the sums (16 rows are written side by side)
    static_assert(NW * 16 * SS * 4 <= kStage);
    float* sums = reinterpret_cast<float*>(stage);
    l = lanes_sum<16, 32>(l);
    if (g == 0) { ml[0][wave][cc] = m; ml[1][wave][cc] = l; }
    __syncthreads();
    auto largest = [&](int row) __attribute__((always_inline)) {
        float x = ml[0][0][row];
#pragma unroll
        for (int w = 1; w < NW; ++w) x = fmaxf(x, ml[0][w][row]);
        return x;
    };
    const float top = largest(cc), f = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) *reinterpret_cast<floatx4*>(sums + (wave * 16 + cc) * SS + 16 * dt + 4 * g) = o[dt] * f;
    __syncthreads();
    const size_t slot = (((size_t)tile * s.Hkv + h) * p.subs + sub) * p.splits + split;
    for (int e = tid; e < rows * (D / 4); e += 64 * NW) {
        const int q = e / (D / 4), d = e % (D / 4) * 4, tk = p.subs > 1 ? 0 : q / G, hd = h * G + (p.subs > 1 ? 16 * sub + q : q % G);
        const bool on = seq[tk] >= 0;
        const float tp = largest(q);
        float lt = 0.0f;
        floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            lt += ml[1][x][q] * __builtin_amdgcn_exp2f(ml[0][x][q] - tp);
            v += *reinterpret_cast<const floatx4*>(sums + (x * 16 + q) * SS + d);
        }
        if (p.splits > 1) {
            *reinterpret_cast<floatx4*>(ws.part_o + (slot * 16 + q) * D + d) = v;
            if (d == 0) { ws.part_ml[(slot * 16 + q) * 2] = tp; ws.part_ml[(slot * 16 + q) * 2 + 1] = on ? lt : -1.0f; }
        } else if (on) {
            v *= lt != 0.0f ? 1.0f / lt : 0.0f;
            const uint2v y = {pack_bf16x2_cvt(v[0], v[1]), pack_bf16x2_cvt(v[2], v[3])};
            *reinterpret_cast<uint2v*>(a.o + (size_t)(t0 + tk) * a.o_token + (size_t)hd * a.o_head + d) = y;
            if (d == 0 && a.lse) a.lse[(size_t)(t0 + tk) * s.Hq + hd] = lt != 0.0f ? tp * 0.6931471805599453f + logf(lt) : -INFINITY;
        }
    }
}

// O and lse of rows whose pages were split: `per` groups of D / 4 threads share a row, so that its partial sums take one trip to memory.  Bound by launch and that trip: 4.8 us for 32
// rows of 32 pieces as for 7408 rows of four.
template <int D>
__global__ __launch_bounds__(256) void sparse_merge_kernel(const SparseArgs a, const SparsePlan p, const SparseWs ws, int per)
{
    constexpr int nt = D / 4, NG = 256 / nt, K = 8;               // partial sums of a group at a time
    __shared__ __align__(16) float acc[NG][D];
    __shared__ float ml[NG][2];
    const StepArgs& s = a.s;
    const int grp = threadIdx.x / nt, d = threadIdx.x % nt * 4, G = s.Hq / s.Hkv;
    const long long x = (long long)blockIdx.x * (NG / per) + grp / per;
    const int t = (int)min(x / s.Hq, (long long)s.T - 1), hd = (int)(x % s.Hq), h = hd / G, gh = hd % G;
    const int sub = p.subs > 1 ? gh / 16 : 0, row = p.subs > 1 ? gh % 16 : t % p.nt * G + gh;
    const size_t slot0 = (((size_t)(t / p.nt) * s.Hkv + h) * p.subs + sub) * p.splits;
    float M = -INFINITY, l = 0.0f;
    floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    bool on = x < (long long)s.T * s.Hq;
    for (int i0 = grp % per; i0 < p.splits; i0 += K * per) {
        floatx4 po[K];
        float pm[K], pl[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const size_t at = (slot0 + min(i0 + k * per, p.splits - 1)) * 16 + row;
            po[k] = *reinterpret_cast<const floatx4*>(ws.part_o + at * D + d);
            pm[k] = ws.part_ml[at * 2];
            pl[k] = ws.part_ml[at * 2 + 1];
        }
        if (pl[0] < 0.0f) on = false;                             // (no sequence's row)
        float top = M;
#pragma unroll
        for (int k = 0; k < K; ++k) { if (i0 + k * per >= p.splits) pm[k] = -INFINITY; top = fmaxf(top, pm[k]); }
        const float al = __builtin_amdgcn_exp2f(M - top);          // (every group has a piece: top is finite)
        M = top; l *= al; v *= al;
#pragma unroll
        for (int k = 0; k < K; ++k) { const float f = __builtin_amdgcn_exp2f(pm[k] - top); l = fmaf(pl[k], f, l); v += po[k] * f; }
    }
    if (per > 1) {
        *reinterpret_cast<floatx4*>(&acc[grp][d]) = v;
        if (d == 0) { ml[grp][0] = M; ml[grp][1] = l; }
        __syncthreads();
        if (grp % per != 0) return;
        M = -INFINITY; l = 0.0f; v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < per; ++k) M = fmaxf(M, ml[grp + k][0]);
        for (int k = 0; k < per; ++k) { const float f = __builtin_amdgcn_exp2f(ml[grp + k][0] - M); l = fmaf(ml[grp + k][1], f, l); v += *reinterpret_cast<const floatx4*>(&acc[grp + k][d]) * f; }
    }
    if (!on) return;
    v *= l != 0.0f ? 1.0f / l : 0.0f;
    *reinterpret_cast<uint2v*>(a.o + (size_t)t * a.o_token + (size_t)hd * a.o_head + d) = uint2v{pack_bf16x2_cvt(v[0], v[1]), pack_bf16x2_cvt(v[2], v[3])};
    if (d == 0 && a.lse) a.lse[(size_t)t * s.Hq + hd] = l != 0.0f ? M * 0.6931471805599453f + logf(l) : -INFINITY;
}

inline SparsePlan sparse_plan(int T, int Hq, int Hkv, int max_q, int n_blocks, int cus)
{
    const int G = Hq / Hkv;
    SparsePlan p;
    p.subs = (G + 15) / 16;
    p.nt = p.subs > 1 ? 1 : 16 / G;
    if (p.nt > max_q) p.nt = max_q;
    if (p.nt > kEntries / n_blocks) p.nt = kEntries / n_blocks;
    p.tiles = (T + p.nt - 1) / p.nt;
    const long long units = (long long)p.tiles * Hkv * p.subs, most = (long long)p.nt * n_blocks, wgs = 4ll * cus;
    p.waves = 4; p.splits = 1;
    // Steps of single or drafted tokens, whose units are alike: where units of 16 or 8 waves just fill the chip, or there is little to read, waves share a unit's
    // pages inside a workgroup, and nothing is joined afterwards (32 pages, heads of 128, with the choice: 256 units 47.5 us instead of 50.7, 512 76 instead of 82; 8 pages: 256 25.5
    // instead of 28.7, 96 23.5 instead of 24.5).  Units that are not alike need smaller workgroups (steps of pieces and single tokens: 45 us instead of 53).
    if (p.subs > 1 || max_q <= 16 / G) {
        if (units <= cus && (8 * units >= 7ll * cus || most <= 8)) p.waves = 16;
        else if (units <= 2ll * cus && 8 * units >= 14ll * cus) p.waves = 8;
        if (p.waves > 4) return p;
    }
    // as many workgroups as the chip holds, four to a compute unit; up to twice as many while each has 16 pages, since tiles differ
    long long splits = 1;
    if (units > 0) {
        splits = wgs / units;
        if (splits < 2 * wgs / units && splits < most / 16) splits = 2 * wgs / units < most / 16 ? 2 * wgs / units : most / 16;
        if (splits > most) splits = most;
    }
    p.splits = splits < 2 ? 1 : (int)splits;
    return p;
}
inline SparseWs carve_sparse(void* ws, const SparsePlan& p, int Hkv, int D, size_t& bytes)
{
    const size_t rows = p.splits > 1 ? (size_t)p.tiles * Hkv * p.subs * p.splits * 16 : 0;
    bytes = rows * (D + 2) * 4 + 256;
    return SparseWs{(float*)ws, (float*)ws + rows * D};
}
template <int D>
int launch_sparse_of(const SparseArgs& a, const SparsePlan& p, const SparseWs& w, hipStream_t st)
{
    const dim3 grid((unsigned)p.tiles * a.s.Hkv * p.subs * p.splits);
    const unsigned lds = sparse_stage(D, p.waves) + 4u * p.nt * a.n_blocks;
    if (p.waves == 16) {
        static unsigned long long done = 0;
        if (!ensure_dynamic_lds((const void*)sparse_kernel<D, 16>, sparse_stage(D, 16) + 4 * kEntries, done)) return -1;
        hipLaunchKernelGGL((sparse_kernel<D, 16>), grid, dim3(1024), lds, st, a, p, w);
    } else if (p.waves == 8) {
        static unsigned long long done = 0;
        if (!ensure_dynamic_lds((const void*)sparse_kernel<D, 8>, sparse_stage(D, 8) + 4 * kEntries, done)) return -1;
        hipLaunchKernelGGL((sparse_kernel<D, 8>), grid, dim3(512), lds, st, a, p, w);
    } else hipLaunchKernelGGL((sparse_kernel<D, 4>), grid, dim3(256), lds, st, a, p, w);
    if (hipGetLastError() != hipSuccess) return -1;
    if (p.splits > 1) {
        const int groups = 256 / (D / 4);
        int per = 1;
        while (per < groups && per * 8 < p.splits) per *= 2;
        const int rows = groups / per;
        hipLaunchKernelGGL((sparse_merge_kernel<D>), dim3((unsigned)(((long long)a.s.T * a.s.Hq + rows - 1) / rows)), dim3(256), 0, st, a, p, w, per);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
template <int D, int GP>
int launch_select_of(const SelectArgs& a, int nt, hipStream_t st)
{
    const int tiles = (a.s.T + nt - 1) / nt;
    // few workgroups: more waves each, for the way to memory; not more than there are sixteens of pages (8 workgroups, 938 pages: 11.6 us with 16 waves, 13.6 with 4; 256, up to 375
    // pages: 9.2 with 16, 10.1 with 4; 464, up to 204 pages: 7.2 with 8, 7.4 with 4; 7504, up to 470 pages: 66 with 4, 146 with 16)
    const unsigned wgs = (unsigned)tiles * a.s.Hkv;
    int waves = wgs <= 256 ? 16 : wgs <= 512 ? 8 : 4;
    while (waves > 4 && waves * 16 > a.s.max_pages) waves /= 2;
    hipLaunchKernelGGL((select_kernel<D, GP>), dim3(wgs), dim3(64 * waves), (size_t)nt * a.s.max_pages * 4, st, a, nt, tiles);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}
template <int D>
int launch_select_d(const SelectArgs& a, int max_q, hipStream_t st)
{
    const int G = a.s.Hq / a.s.Hkv;
    int gp = 1;
    while (gp < G && gp < 16) gp *= 2;
    int nt = 16 / gp;
    if (nt > max_q) nt = max_q;
    const int room = 12288 / a.s.max_pages;                       // tokens whose scores fit 48 KiB of LDS
    if (nt > room) nt = room > 1 ? room : 1;                      // (one token of 8192 pages: 32 KiB)
    switch (gp) {
        case 1: return launch_select_of<D, 1>(a, nt, st);
        case 2: return launch_select_of<D, 2>(a, nt, st);
        case 4: return launch_select_of<D, 4>(a, nt, st);
        case 8: return launch_select_of<D, 8>(a, nt, st);
        default: return launch_select_of<D, 16>(a, nt, st);
    }
}

}  // namespace

int launch_summarize(const void* cache, int num_pages, int Hkv, int D, const long long* slots, int T, void* summary, hipStream_t st)
{
    // rows of a workgroup: a page is complete at most once in 128 rows of a prompt, but every row of a step of single tokens may complete one
    const int rows = T > 8192 ? 128 : 16;
    const dim3 grid((T + rows - 1) / rows, (Hkv + 3) / 4);
    if (D == 128) hipLaunchKernelGGL((summarize_kernel<128>), grid, dim3(256), 0, st, (const unsigned char*)cache, num_pages, Hkv, slots, T, rows, (unsigned char*)summary);
    else          hipLaunchKernelGGL((summarize_kernel<64>), grid, dim3(256), 0, st, (const unsigned char*)cache, num_pages, Hkv, slots, T, rows, (unsigned char*)summary);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_select(const SelectArgs& a, int max_q, int D, hipStream_t st) { return D == 128 ? launch_select_d<128>(a, max_q, st) : launch_select_d<64>(a, max_q, st); }

size_t sparse_ws_bytes(int T, int Hq, int Hkv, int max_q, int n_blocks, int D)
{
    size_t bytes;
    carve_sparse(nullptr, sparse_plan(T, Hq, Hkv, max_q, n_blocks, kChipCus), Hkv, D, bytes);
    return bytes;
}

int launch_sparse(const SparseArgs& a, int max_q, int D, void* ws, hipStream_t st)
{
    size_t bytes;
    const SparsePlan p = sparse_plan(a.s.T, a.s.Hq, a.s.Hkv, max_q, a.n_blocks, kChipCus);
    const SparseWs w = carve_sparse(ws, p, a.s.Hkv, D, bytes);
    return D == 128 ? launch_sparse_of<128>(a, p, w, st) : launch_sparse_of<64>(a, p, w, st);
}

}  // namespace aq
