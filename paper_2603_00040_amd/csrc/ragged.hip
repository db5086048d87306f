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
// what lies below 2^-39 of the largest.  Scores, maxima, sums and O are fp32.  P is rounded to fp16 for the product with V, scaled so that a row's largest is
// at least 2^11 (kTop): by a relative 2^-12, an eighth of what rounding the output to bf16 costs, down to 2^-25 of the row's largest so far, and by 2^-36 of that
// largest below (all of them together by less than 2^-16 of the largest |V|, for 2^20 keys).  The sum that divides O is of the unrounded ones.  Scores
// times log2 e that reach 2^27 have no reference in fp32 that is near enough for that: P may leave fp16.
#include "common.hpp"
#include "kernels.hpp"
#include "kv4.hpp"

#include <type_traits>

namespace aq {

namespace {

// Most rows of a (sequence, kv head) that the kernel for few rows takes, in tiles of 16 or 32 that read the keys each for itself; more go to the one that has
// tiles of 256.  Few -> many, 16 sequences of 4096 keys, 8 kv heads of 128: 48 rows 56 against 78 us, 80 rows 76 against 79, 128 rows 84 against 87;
// 4 of 16 000 keys: 40 rows 59 against 75, 120 rows 91 against 81.  (Not measured where a window leaves fewer keys to see.)
constexpr int kFewRows = 96;
// What the start and the end of a row tile weigh in tiles of keys: 13 000 cycles against 3200 (heads of 64: 2600), and a piece of a row tile that ends a
// workgroup's work is joined later.  (Six prompts of 766 - 3846 tokens, heads of 128: with 4 253.6 us, 5 251.7, 6 255.0, 7 255.4.)
constexpr int kWideStart = 5;
constexpr int kWideRows = 256;        // rows of a tile of the other one

// The query heads of a kv head, and whole division by their number: x / G = x mul >> 31 + shift with mul = ceil(2^(31 + shift) / G), 2^shift >= G, exact for
// 0 <= x < 2^31 (x times what mul is too large by stays below 2^(31 + shift)).  Three instructions instead of the two dozen of a division, of
// which the start of a row tile has six.
struct Group { int n; uint32_t mul; int shift; __device__ operator int() const { return n; } };
__device__ inline int operator/(int x, const Group& g) { return (int)(((uint64_t)(uint32_t)x * g.mul) >> (31 + g.shift)); }
__device__ inline int operator%(int x, const Group& g) { return x - (x / g) * g.n; }
__device__ inline Group group_of(const RaggedArgs& a) { return Group{a.group, a.group_mul, a.group_shift}; }

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

// The units of work of the kernel for few rows: the pages that the rows of a sequence see, once per kv head and tile of rows, sequence by sequence, head by
// head, tile by tile, page by page.  What a tile costs besides (its rows of Q, the first trip to its pages, the result) counts as kFewStart pages in
// front of its own.  Sequences with more rows than kFewRows have no units here.
template <int D> constexpr int kFewStart = D == 64 ? 3 : 2;      // (6 000 cycles, against 2 000 and 3 200 for a page)
struct Few { int rows, tiles /* of ROWS rows */, first_page, pages, units /* of a tile */; };
template <int D, int ROWS>
__device__ inline Few few_of(const RaggedArgs& a, const Seq& s, const Group& G)
{
    const int rows = s.n * G;
    int lo, hi;
    keys_of(a, s, 0, s.n - 1, lo, hi);
    const int pages = rows > 0 && rows <= kFewRows && hi > lo ? ((hi + 127) >> 7) - (lo >> 7) : 0;
    return Few{rows, (rows + ROWS - 1) / ROWS, lo >> 7, pages, pages > 0 ? pages + kFewStart<D> : 0};
}
__device__ inline int few_units(const Few& u) { return u.tiles * u.units; }      // of a head
__device__ inline Seq uniform_seq(const Seq& s) { return Seq{uniform(s.first), uniform(s.n), uniform(s.len)}; }
// The first sequence from b on that has work for a kernel (has(s)), and its index: a wave asks 64 at a time, since a step's places that are idle, or the other
// kernel's, may be thousands (three prompts far apart among 4096 idle places: one after the other 770 us, so 224).  a.B: there is none.
template <class Has>
__device__ inline Seq next_seq(const RaggedArgs& a, int& b, const Has& has)
{
    const int lane = threadIdx.x & 63;
    for (; b < a.B; b += 64) {
        const Seq s = b + lane < a.B ? seq_of(a, b + lane) : Seq{0, 0, 0};
        const unsigned long long hit = __builtin_amdgcn_ballot_w64(has(s));
        if (hit != 0) {
            const int src = (int)__builtin_ctzll(hit);
            b += src;
            return Seq{__builtin_amdgcn_readlane(s.first, src), __builtin_amdgcn_readlane(s.n, src), __builtin_amdgcn_readlane(s.len, src)};
        }
    }
    b = a.B;
    return Seq{0, 0, 0};
}

// What the launches of a step hand over: how many pages each workgroup takes, the pages (of one head) in front of every sequence, and, of a unit whose
// pages are shared by several workgroups, each one's O, maximum and sum.
struct FewWs { int* quota; int* front /* [B + 1] */; float* part_o /* [workgroup][2][rows][D] */; float* part_ml /* [workgroup][2][rows][2] */; };

// Few rows (decode steps, drafted tokens): bound by reading the cache, so the pages of all units are dealt out evenly, `quota` consecutive ones to a
// workgroup, however uneven the sequences are.  Which of them are its own a workgroup finds from the lengths itself (one trip to memory and a scan; a
// launch that makes a list would cost more).  Its four waves take 32 keys of every page, each with its own maximum, sum and O; the pages of
// the next iteration are requested before the present ones are used.  One query of 32 sequences of 4096 - 16384 keys, 32/8 heads of 128: 326 MB in 61 us,
// 5.3 TB/s, what a copy reaches.  With more rows and short segments the vector instructions bound it (unpacking, softmax: a wave issues one
// in 9 cycles) and the start of a segment: one to six queries of 40 sequences of 300 - 9000 keys, 16/4 heads of 64, 34 MB in 16.7 us.
template <int D, int RT /* 16-row groups of a unit */>
__global__ __launch_bounds__(256, RT == 1 ? 3 : 2) void ragged_few_kernel(const RaggedArgs a, const FewWs ws)
{
    constexpr int NS = D / 32, NDT = D / 16, ROWS = 16 * RT;
    constexpr int SETS = D == 64 ? 3 : 2;           // pages in registers, the present one included (heads of 64: half the bytes each)
    constexpr int RS = 2 * D + 32;                                // bytes per key of the V tile (eight keys side by side in other banks)
    constexpr size_t VOFF = (size_t)128 * (D / 2 + D / 16);
    __shared__ __align__(16) unsigned char stage[4 * 32 * RS];     // per wave: V of 32 keys [key][d]; at the end the waves' sums [4][16][D + 4]
    __shared__ float ml[2][4][ROWS];
    __shared__ int red[4], found[5];

    const int tid = threadIdx.x, lane = tid & 63, cc = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Group G = group_of(a);
    unsigned char* stg = stage + wave * (32 * RS);
    // (the two 16-byte pieces of every 32 change places in keys 4 - 7 of 8: a store serves eight lanes, eight keys, at a time on 32 banks)
    const uint32_t tr_base = lds_addr_of(stg) + (uint32_t)((4 * g + (cc >> 2)) * RS + 8 * ((cc & 3) ^ (2 * (g & 1))));

    // this workgroup's units [w, w_end) of all, and the sequence that the first of them belongs to
    int all = 0, total, n_b = 0, upto_b = 0;
    Seq s_b{0, 0, 0};
    for (int b0 = 0; b0 < a.B; b0 += 256) {
        s_b = b0 + tid < a.B ? seq_of(a, b0 + tid) : Seq{0, 0, 0};
        n_b = few_units(few_of<D, ROWS>(a, s_b, G));
        upto_b = all + wg_scan<4>(n_b, red, total);
        if (blockIdx.x == 0) {
            if (b0 + tid < a.B) ws.front[b0 + tid + 1] = upto_b;
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
    for (int b0 = 0, at = 0; ; b0 += 256) {
        if (a.B > 256) {                                          // (up to 256 sequences: as found above)
            s_b = b0 + tid < a.B ? seq_of(a, b0 + tid) : Seq{0, 0, 0};
            n_b = few_units(few_of<D, ROWS>(a, s_b, G));
            upto_b = at + wg_scan<4>(n_b, red, total);
            at += total;
        }
        if (n_b > 0 && w < (long long)upto_b * a.Hkv && w >= (long long)(upto_b - n_b) * a.Hkv) {
            found[0] = b0 + tid; found[1] = upto_b - n_b; found[2] = s_b.first; found[3] = s_b.n; found[4] = s_b.len;
        }
        if (a.B <= 256 || w < (long long)at * a.Hkv || b0 + 256 >= a.B) break;
    }
    __syncthreads();
    int b = uniform(found[0]), front = uniform(found[1]);
    Seq s{uniform(found[2]), uniform(found[3]), uniform(found[4])};
    Few u = few_of<D, ROWS>(a, s, G);
    int ht, off;                                                  // head and tile (head * tiles + tile), and its units in front of w
    {
        const long long in_seq = w - (long long)front * a.Hkv;
        ht = (int)(in_seq / u.units); off = (int)(in_seq % u.units);
    }

    while (w < w_end) {
        const int units = (int)min((long long)(u.units - off), w_end - w);
        const int at = max(off - kFewStart<D>, 0), cnt = min(off + units - kFewStart<D>, u.pages) - at;      // pages: where this workgroup begins, how many
        const int h = ht / u.tiles, r0 = ht % u.tiles * ROWS, rows = min(u.rows - r0, ROWS);
        w += units;
        if (cnt <= 0) break;                                      // (the start alone: w is at this workgroup's end)
        const int first = u.first_page + at;
        const int* ids = a.table + (size_t)b * a.max_pages + first;

        // what a segment needs from memory first, asked for at once: page ids (64 at a time: lane x has that of page id_end - 64 + x) and Q
        int id_lane = ids[min(lane, cnt - 1)], id_end = 64;
        uint4v x[RT][NS];
        int k_first[RT], k_last[RT];                              // keys that this lane's rows see
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int row = r0 + min(16 * rt + cc, rows - 1), tok = row / G, head = h * G + row % G, pos = s.len - s.n + tok;
            k_first[rt] = a.window > 0 ? pos - a.window + 1 : 0;
            k_last[rt] = a.causal ? min(pos, s.len - 1) : s.len - 1;
#pragma unroll
            for (int i = 0; i < NS; ++i)
                x[rt][i] = *reinterpret_cast<const uint4v*>(a.q + (size_t)(s.first + tok) * a.q_token + (size_t)head * a.q_head + (D / 4) * g + 8 * i);
        }
        asm volatile("" : "+v"(id_lane));                         // (waited for here and not at every use)

        struct Tile { Raw<D> k[2], v[2]; bool live; };
        auto load = [&](Tile& t, int i) __attribute__((always_inline)) {
            if (i >= id_end) {
                id_lane = ids[min(id_end + lane, cnt - 1)];
                asm volatile("" : "+v"(id_lane));
                id_end += 64;
            }
            const int page = __builtin_amdgcn_readlane(id_lane, i - (id_end - 64));
            t.live = page >= 0 && page < a.num_pages;
            const unsigned char* part = a.cache + ((size_t)(t.live ? page : 0) * a.Hkv + h) * (2 * VOFF);
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) t.k[blk] = load_raw<D>(part, 32 * wave + 16 * blk + cc, g);
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) t.v[blk] = load_raw<D>(part + VOFF, 32 * wave + 16 * blk + cc, g);
        };
        // (sets of registers by name, and requests that depend on nothing: rotated by copies the compiler waits for everything in flight)
        Tile t[SETS];
#pragma unroll
        for (int i = 0; i + 1 < SETS; ++i) load(t[i], min(i, cnt - 1));

        // Q: row cc of a group of 16, d = (D/4) g + 8 s .. + 7
        half8 qreg[RT][NS];
        float c_row[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const float amax = lanes_max<16, 32>(largest_of(x[rt]));
            float f, inv;
            row_factor(amax, f, inv);
#pragma unroll
            for (int i = 0; i < NS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    qreg[rt][i][2 * j]     = (half_t)(__uint_as_float(x[rt][i][j] << 16) * f);
                    qreg[rt][i][2 * j + 1] = (half_t)(__uint_as_float(x[rt][i][j] & 0xFFFF0000u) * f);
                }
            c_row[rt] = fmaxf(a.c * inv, kLeastFactor);
        }
        // keys that every row sees: a page inside [see_first, see_last] needs no mask
        const int see_first = a.window > 0 ? s.len - s.n + (r0 + rows - 1) / G - a.window + 1 : 0, see_last = a.causal ? min(s.len - s.n + r0 / G, s.len - 1) : s.len - 1;

        floatx4 o[RT][NDT];
        float m[RT], up_to[RT], l[RT];                                       // the reference (kTop)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = up_to[rt] = -INFINITY; l[rt] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[rt][dt] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        auto step = [&](auto groups, const Tile& t, int i) __attribute__((always_inline)) {
            constexpr int N = decltype(groups)::value;            // groups of 16 rows that there are
            const int kt = (first + i) * 128 + 32 * wave;
            const bool masked = kt < see_first || kt + 31 > see_last;
            floatx4 sc[N][2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const half2v ks = scales_of<D>(t.k[blk], g, t.live);
#pragma unroll
                for (int rt = 0; rt < N; ++rt) sc[rt][blk] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int j = 0; j < NS; ++j) {
                    const half8 kv = values8<D>(t.k[blk], ks, j);
#pragma unroll
                    for (int rt = 0; rt < N; ++rt) sc[rt][blk] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, qreg[rt][j], sc[rt][blk], 0, 0, 0);
                }
            }
            // V through LDS: written key by key, read back with four keys of one d in a lane
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const half2v vs = scales_of<D>(t.v[blk], g, t.live && kt + 16 * blk + cc < s.len);
#pragma unroll
                for (int j = 0; j < NS; ++j) *reinterpret_cast<half8*>(stg + (16 * blk + cc) * RS + (D / 2) * g + 16 * (j ^ ((cc >> 2) & 1))) = values8<D>(t.v[blk], vs, j);
            }
            __builtin_amdgcn_wave_barrier();
            half8 pt[N];
#pragma unroll
            for (int rt = 0; rt < N; ++rt) {
                if (masked) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = kt + 16 * (j >> 2) + 4 * g + (j & 3);
                        if (key < k_first[rt] || key > k_last[rt]) sc[rt][j >> 2][j & 3] = -INFINITY;
                    }
                }
                float mx = max_nc(max_nc(max_nc(sc[rt][0][0], sc[rt][0][1]), max_nc(sc[rt][0][2], sc[rt][0][3])),
                                  max_nc(max_nc(sc[rt][1][0], sc[rt][1][1]), max_nc(sc[rt][1][2], sc[rt][1][3])));
                mx = lanes_max<16, 32>(mx);
                if (__builtin_amdgcn_ballot_w64(mx > up_to[rt]) != 0) {
                    const float m_new = fmaxf(m[rt], fmaf(mx, c_row[rt], -kTop)), alpha = __builtin_amdgcn_exp2f(m[rt] - (m_new == -INFINITY ? 0.0f : m_new));
                    m[rt] = m_new;
                    up_to[rt] = score_up_to(m_new, c_row[rt]);
                    l[rt] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) o[rt][dt] *= alpha;
                }
                const float m_at = m[rt] == -INFINITY ? 0.0f : m[rt];
                float add = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[rt][j >> 2][j & 3], c_row[rt], -m_at));
                    add += x;
                    pt[rt][j] = (half_t)x;
                }
                l[rt] += add;
            }
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) {
                const uint2v x = lds_read_tr16_at(tr_base + 32 * dt), y = lds_read_tr16_at(tr_base + 32 * dt + 16 * RS);
                const uint4v av = {x[0], x[1], y[0], y[1]};
#pragma unroll
                for (int rt = 0; rt < N; ++rt) o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, av), pt[rt], o[rt][dt], 0, 0, 0);
            }
        };
        // (a loop for either number of groups: asked at every product, the products stand alone between branches)
        auto walk = [&](auto groups) __attribute__((always_inline)) {
            for (int i = 0; i < cnt; i += SETS) {
#pragma unroll
                for (int x = 0; x < SETS; ++x) {
                    if (x > 0 && i + x >= cnt) break;
                    load(t[(x + SETS - 1) % SETS], min(i + x + SETS - 1, cnt - 1));
                    step(groups, t[x], i + x);
                }
            }
        };
        if (RT == 1 || rows <= 16) walk(std::integral_constant<int, 1>{});
        else walk(std::integral_constant<int, RT>{});

        // the four waves' sums, in units of their common maximum
        const bool whole = cnt == u.pages;
        const size_t slot = (size_t)blockIdx.x * 2 + (at == 0 ? 1 : 0);
        constexpr int SS = D + 4;                                 // floats per row of the sums (16 rows are written side by side)
        static_assert(4 * 16 * SS * 4 <= 4 * 32 * RS);
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
            for (int dt = 0; dt < NDT; ++dt) *reinterpret_cast<floatx4*>(sums + (wave * 16 + cc) * SS + 16 * dt + 4 * g) = o[rt][dt] * f;
            __syncthreads();
            for (int e = tid; e < min(16, rows - 16 * rt) * (D / 4); e += 256) {
                const int q = e / (D / 4), d = e % (D / 4) * 4, rr = 16 * rt + q;
                const float tp = fmaxf(fmaxf(ml[0][0][rr], ml[0][1][rr]), fmaxf(ml[0][2][rr], ml[0][3][rr])), at = tp == -INFINITY ? 0.0f : tp;
                float lt = 0.0f;
                floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    lt += ml[1][x][rr] * __builtin_amdgcn_exp2f(ml[0][x][rr] - at);
                    v += *reinterpret_cast<const floatx4*>(sums + (x * 16 + q) * SS + d);
                }
                if (whole) {
                    const int tk = (r0 + rr) / G, hd = h * G + (r0 + rr) % G;
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
        // on to the next head, sequence (there is one while w < w_end; a sequence of the other kernel, or without a key, has no units)
        off = 0;
        if (++ht == a.Hkv * u.tiles) {
            if (w >= w_end) return;
            ht = 0;
            ++b;
            s = next_seq(a, b, [&](const Seq& x) { return few_of<D, ROWS>(a, x, G).units > 0; });
            if (b >= a.B) return;                                 // (lengths that change under the launch)
            u = few_of<D, ROWS>(a, s, G);
        }
    }
}

// O and lse of a unit whose pages were shared, and of rows that see no key, by a workgroup: groups of D / 4 threads have a row each, or, while there are
// fewer rows than groups, several groups share the partial sums of a row.  A launch and two or three trips to memory: 4.7 us.
template <int D, int ROWS>
__device__ void few_merge(const RaggedArgs& a, const FewWs& ws, int unit, int tiles /* of a sequence at most */)
{
    constexpr int NG = 256 / (D / 4);
    __shared__ __align__(16) float acc[NG][D];
    __shared__ float ml[NG][2];
    const Group G = group_of(a);
    const int tile = unit % tiles, b = unit / tiles / a.Hkv, h = unit / tiles % a.Hkv;
    const int tid = threadIdx.x, grp = tid / (D / 4), d = tid % (D / 4) * 4;
    const int quota = *ws.quota, front = ws.front[b];             // (beside the lengths, not behind them)
    const Seq s = seq_of(a, b);
    const Few u = few_of<D, ROWS>(a, s, G);
    if (u.rows > kFewRows || tile >= u.tiles) return;
    const int first_row = tile * ROWS, rows = min(u.rows - first_row, ROWS);
    int f = 0, n = 0;                                             // the first workgroup that had pages of it, how many had
    if (u.pages > 0) {
        const long long w0 = (long long)front * a.Hkv + (long long)(h * u.tiles + tile) * u.units + kFewStart<D>, w1 = w0 + u.pages - 1;
        f = (int)(w0 / quota); n = (int)(w1 / quota) - f + 1;
        if (n < 2) return;
    }
    int per = NG;                                                 // groups to a row
    while (per > 1 && (NG / per) < rows) per >>= 1;
    for (int r0 = 0; r0 < rows; r0 += NG / per) {
        const int r = r0 + grp / per;
        const bool on = r < rows;
        float M = -INFINITY, l = 0.0f;
        floatx4 v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (on) {
            constexpr int K = 8;                                  // at a time: one trip to memory (4: 16 000 keys 16.1 instead of 14.5 us; 16: 64 sequences of 500 17.4 instead of 16.6)
            for (int i0 = grp % per; i0 < n; i0 += K * per) {
                floatx4 po[K];
                float pm[K], pl[K];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const int i = min(i0 + k * per, n - 1);
                    const size_t at = ((size_t)(f + i) * 2 + (i == 0 ? 1 : 0)) * ROWS + r;
                    po[k] = *reinterpret_cast<const floatx4*>(ws.part_o + at * D + d);
                    pm[k] = i0 + k * per < n ? ws.part_ml[at * 2] : -INFINITY;
                    pl[k] = ws.part_ml[at * 2 + 1];
                }
                float top = M;
#pragma unroll
                for (int k = 0; k < K; ++k) top = fmaxf(top, pm[k]);
                const float at = top == -INFINITY ? 0.0f : top, al = __builtin_amdgcn_exp2f(M - at);
                M = top; l *= al; v *= al;
#pragma unroll
                for (int k = 0; k < K; ++k) { const float x = __builtin_amdgcn_exp2f(pm[k] - at); l = fmaf(pl[k], x, l); v += po[k] * x; }
            }
        }
        if (per > 1) {                                            // (then one round is all)
            *reinterpret_cast<floatx4*>(&acc[grp][d]) = v;
            if (d == 0) { ml[grp][0] = M; ml[grp][1] = l; }
            __syncthreads();
            if (grp % per != 0 || !on) return;
            float top = -INFINITY;
            for (int k = 0; k < per; ++k) top = fmaxf(top, ml[grp + k][0]);
            const float at = top == -INFINITY ? 0.0f : top;
            l = 0.0f; v = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < per; ++k) { const float x = __builtin_amdgcn_exp2f(ml[grp + k][0] - at); l = fmaf(ml[grp + k][1], x, l); v += *reinterpret_cast<const floatx4*>(&acc[grp + k][d]) * x; }
            M = top;
        }
        if (!on) continue;
        const int tk = (first_row + r) / G, hd = h * G + (first_row + r) % G;
        v *= l != 0.0f ? 1.0f / l : 0.0f;
        *reinterpret_cast<uint2v*>(a.o + (size_t)(s.first + tk) * a.o_token + (size_t)hd * a.o_head + d) = uint2v{pack_bf16x2_cvt(v[0], v[1]), pack_bf16x2_cvt(v[2], v[3])};
        if (d == 0 && a.lse) a.lse[(size_t)(s.first + tk) * a.Hq + hd] = l != 0.0f ? M * 0.6931471805599453f + logf(l) : -INFINITY;
    }
}

// The units of work of the kernel for many rows: a tile of kWideRows rows and the tiles of 64 keys that it sees, for every kv head, sequence by sequence,
// head by head, tile by tile.  What a row tile costs besides (its rows of Q, the first tiles of K and V, the result) counts as kWideStart
// tiles of keys in front of its own.
__device__ inline void wide_tile(const RaggedArgs& a, const Seq& s, const Group& G, int tile, int& t0, int& nt)
{
    const int r0 = tile * kWideRows;
    int lo, hi;
    keys_of(a, s, r0 / G, (min(r0 + kWideRows, s.n * G) - 1) / G, lo, hi);
    t0 = lo >> 6;
    nt = hi > lo ? ((hi + 63) >> 6) - t0 + kWideStart : 0;
}
// The key tiles (for one head) of all row tiles of sequence b, a thread each: the lanes of a wave go over the row tiles of one of its sequences after
// another.  0 where the kernel for few rows takes the sequence.
__device__ inline long long wide_work(const RaggedArgs& a, const Group& G, int b)
{
    const int lane = threadIdx.x & 63;
    Seq s{0, 0, 0};
    if (b < a.B) s = seq_of(a, b);
    const bool on = s.n * G > kFewRows;
    long long mine = 0;
    for (unsigned long long left = __builtin_amdgcn_ballot_w64(on); left != 0; left &= left - 1) {
        const int src = (int)__builtin_ctzll(left);
        const Seq x{0, __builtin_amdgcn_readlane(s.n, src), __builtin_amdgcn_readlane(s.len, src)};
        const int tiles = (x.n * G + kWideRows - 1) / kWideRows;
        long long sum = 0;
        for (int r = lane; r < tiles; r += 64) { int t0, nt; wide_tile(a, x, G, r, t0, nt); sum += nt; }
        sum = lane_total(sum);
        if (lane == src) mine = sum;
    }
    return mine;
}

// Where the pages of a workgroup begin: a row tile, its head and how many of its key tiles lie in front.
struct WideRec { int b, tile, h, off, nt, pad[3]; };
struct WideWs { long long* quota; WideRec* rec; float* part_o /* [workgroup][2][8 waves][D / 8][64 lanes][4] */; float* part_ml /* [workgroup][2][8][32][2] */; };

// Many rows (pieces of prompts): bound by the matrix instructions and by the softmax between them.  Eight waves have 32 rows each of a tile of 256 and
// walk tiles of 64 keys together; waves 0 - 3 and 4 - 7 are half an iteration apart, between barriers: while one half computes O += V P and the next
// tile's S, and between these products unpacks its half of the keys of a K and a V tile into LDS (K as operands of the matrix instruction, V key by
// key), the other does the softmax, so that every SIMD has a wave for either unit.  The work (row tile, key tile) is dealt out evenly as in the
// kernel for few rows.
// Rates over 20 passes and more, in operations that the mask leaves: 8192 queries and keys, 32/8 heads of 128, 1110 TFLOP/s without a mask (988 us), 1030 causal;
// 8 x 512 queries over 8192 keys each 1040; 16/4 heads of 64, 16384 queries and keys, 870.  The products with their barriers alone would run at 1550, with
// their operands out of LDS and the pages' loads at 1375 (a large library product: 1280).  A wave's phases of a tile, in cycles: heads of 128 vector 1350 and
// 180 of waiting, matrix 1590 (1024 of products) and 75; heads of 64 vector 1165 and 70, matrix 1070 (512) and 310: the matrix phase bounds the one, the
// vector phase the other.  Also tried: softmax and products of a wave in one stream (5 % slower, heads
// of 64 2 %), four waves of 32 rows and two workgroups to a compute unit without phases (10 %), the unpacking shared between the phases (5 %).
template <int D>
__global__ __launch_bounds__(512, 2) void ragged_wide_kernel(const RaggedArgs a, const WideWs ws)
{
    constexpr int ND = D / 16, NB = D / 32;                       // contraction steps of S, 32-d blocks of O
    constexpr int RS = 2 * D + 64;                                // bytes per key of the V tile: the 64 bytes of four keys that are read together in other banks
    constexpr int KB = 64 * 2 * D, VB = 64 * RS;                  // bytes of a tile of K, of V
    constexpr size_t VOFF = (size_t)128 * (D / 2 + D / 16);
    extern __shared__ __align__(256) unsigned char lds[];          // two tiles of K, two of V
    __shared__ long long red[8], found_front, found_per;
    __shared__ int found_b;
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool late = wave >= 4;
    const Group G = group_of(a);

    // this workgroup's key tiles [w, w_end) of all units', and where they begin
    long long all = 0, total, n_b = 0, upto_b = 0;
    for (int b0 = 0; b0 < a.B; b0 += 512) {
        n_b = wide_work(a, G, b0 + tid);
        upto_b = all + wg_scan<8>(n_b, red, total);
        all += total;
    }
    const long long work = all * a.Hkv;
    long long quota = (work + gridDim.x - 1) / gridDim.x;
    if (blockIdx.x == 0 && tid == 0) *ws.quota = quota;
    long long w = (long long)blockIdx.x * quota;
    const long long w_end = min(w + quota, work);
    // (also of a workgroup without work: every record is read when the sums are joined)
    if (tid == 0) ws.rec[blockIdx.x] = WideRec{0, 0, 0, 0, 0, {0, 0, 0}};
    if (w >= w_end) return;
    long long front = 0;                                          // key tiles (of one head) of the sequences in front of b
    for (int b0 = 0; ; b0 += 512) {
        if (a.B > 512) {                                          // (up to 512 sequences: as found above)
            n_b = wide_work(a, G, b0 + tid);
            upto_b = front + wg_scan<8>(n_b, red, total);
            front += total;
        }
        if (n_b > 0 && w < upto_b * a.Hkv && w >= (upto_b - n_b) * a.Hkv) { found_b = b0 + tid; found_front = upto_b - n_b; found_per = n_b; }
        if (a.B <= 512 || w < front * a.Hkv || b0 + 512 >= a.B) break;
    }
    __syncthreads();
    int b = uniform(found_b);
    front = uniform(found_front);
    long long per = uniform(found_per);                           // key tiles of one head of sequence b; 0: to be counted

    const uint32_t lds0 = lds_addr_of(lds);
    // (key 4 half + r of 16, r = (lane & 15) / 4; for the order of the 16-byte pieces of a key see unpack)
    const int r4 = (lane & 15) >> 2;
    const uint32_t v_base = lds0 + 2 * KB + (uint32_t)((4 * half + r4) * RS + 16 * ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ ((D == 128 ? 2 : 1) * (r4 & 1))) + 8 * (lane & 1));
    auto phase_end = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    // Rows of Q and O pass through a place of LDS of the wave's own (of the tiles', which nobody reads before a segment's first barrier and behind its last):
    // in memory the wave takes rows whole, D / 8 lanes to each, where in registers a lane has a piece of every row (one row's 16 bytes
    // beside the next row's: 32 lines of memory to every instruction; 1 % slower).  Behind a row, where it lies.
    constexpr int RO = 2 * D + 16, LR = D / 8, RP = 64 / LR;       // bytes of a row, lanes to a row, rows at a time
    static_assert(8 * 32 * RO <= 2 * KB + 2 * VB && 32 / RP == ND);
    const uint32_t own_row = lds0 + (uint32_t)((wave * 32 + col) * RO), own_piece = lds0 + (uint32_t)((wave * 32 + lane / LR) * RO + 16 * (lane % LR));
    const uint32_t own_where = lds0 + (uint32_t)((wave * 32 + lane / LR) * RO + 2 * D);
    auto row_at = [&](int p) __attribute__((always_inline)) {      // of row RP p + lane / LR, as it was written behind it
        const uint2v w = lds_read8_at(own_where + (uint32_t)(p * RP * RO));
        return (size_t)(((unsigned long long)w[1] << 32) | w[0]);
    };
    auto write_where = [&](size_t at) __attribute__((always_inline)) { lds_write8_at(own_row + 2 * D, uint2v{(uint32_t)at, (uint32_t)(at >> 32)}); };

    int tile = -1, h = 0, off = 0, t0 = 0, nt = 0;                 // tile < 0: to be looked up
    int id_lane = 0, id_b = -1, id_first = 0;                      // lane i: the id of page id_first + i of sequence id_b, -1: outside the cache
    Seq s = uniform_seq(seq_of(a, b));
    while (w < w_end) {
        if (tile < 0) {
            // the row tile of a sequence's work that w lies in
            if (per == 0) {                                       // (of many rows and a key: the last row sees one)
                s = next_seq(a, b, [&](const Seq& x) { return x.n * G > kFewRows && x.len > 0; });
                if (b >= a.B) return;                             // (lengths that change under the launch)
            }
            const int tiles = (s.n * G + kWideRows - 1) / kWideRows;
            if (per == 0) {
                for (int r0 = 0; r0 < tiles; r0 += 64) {
                    int x0, n = 0;
                    if (r0 + lane < tiles) wide_tile(a, s, G, r0 + lane, x0, n);
                    per += lane_total(n);                         // (64 row tiles of at most 2^14 key tiles)
                }
            }
            const long long in_seq = w - front * a.Hkv;
            h = (int)(in_seq / per);
            long long rem = in_seq % per;
            for (int r0 = 0; r0 < tiles && tile < 0; r0 += 64) {
                int x0 = 0, n = 0;
                if (r0 + lane < tiles) wide_tile(a, s, G, r0 + lane, x0, n);
                const int upto = lane_scan(n);
                const unsigned long long hit = __builtin_amdgcn_ballot_w64(rem < upto && rem >= upto - n);
                if (hit != 0) {
                    const int src = (int)__builtin_ctzll(hit);
                    tile = r0 + src;
                    off = (int)(rem - (__builtin_amdgcn_readlane(upto, src) - __builtin_amdgcn_readlane(n, src)));
                    t0 = __builtin_amdgcn_readlane(x0, src); nt = __builtin_amdgcn_readlane(n, src);
                }
                rem -= __builtin_amdgcn_readlane(upto, 63);
            }
            if (tile < 0) return;                                 // (lengths that change under the launch)
            if (tid == 0 && w == (long long)blockIdx.x * quota) ws.rec[blockIdx.x] = WideRec{b, tile, h, off, nt, {0, 0, 0}};
        }
        const int units = (int)min((long long)(nt - off), w_end - w);      // of work, the start included
        const int keys = nt - kWideStart, at = max(off - kWideStart, 0), cnt = min(off + units - kWideStart, keys) - at;      // tiles of keys: all of them, where this workgroup begins, how many
        w += units;
        if (cnt <= 0) { off += units; continue; }                 // (the start alone: w is at this workgroup's end)
        const int rows = s.n * G, r0 = tile * kWideRows, w0 = r0 + 32 * wave;
        const bool mine = w0 < rows;                              // this wave has rows
        const int row = min(w0 + col, rows - 1), tok = row / G, head = h * G + row % G, pos = s.len - s.n + tok;
        const int k_first = a.window > 0 ? pos - a.window + 1 : 0, k_last = a.causal ? min(pos, s.len - 1) : s.len - 1;
        const int see_first = a.window > 0 ? s.len - s.n + (min(w0 + 32, rows) - 1) / G - a.window + 1 : 0;      // what all rows of the wave see
        const int see_last = a.causal ? min(s.len - s.n + w0 / G, s.len - 1) : s.len - 1;

        // what this thread unpacks: 32 d of one key, of K (waves 0, 1, 4, 5) or of V; the early waves have the first 32 keys of a tile
        const int is_v = (wave >> 1) & 1, key = (late ? 32 : 0) + ((tid & 127) >> 2), g = tid & 3;
        const int first = t0 + at, last = first + cnt - 1;
        const int* ids = a.table + (size_t)b * a.max_pages;
        const unsigned char* part0 = a.cache + (size_t)h * (2 * VOFF) + (is_v ? VOFF : 0);      // of page 0
        const uint32_t page_bytes = (uint32_t)a.Hkv * (uint32_t)(2 * VOFF);      // (at most 65535 heads of 18 KiB)
        const uint32_t code_at = (uint32_t)(key * (D / 2) + (D / 8) * g), scale_at = (uint32_t)(128 * (D / 2) + key * (D / 16) + (D == 128 ? 4 * (g >> 1) : 0));
        if (b != id_b) { id_b = b; id_first = 1 << 30; }          // (none of them)
        Raw<D> raw;
        bool raw_on = false;
        // Where tile t lies, and how many positions of its page and sequence there are from its first on (none: a page outside the cache)
        struct Place { const unsigned char* page; uint32_t odd; int have; };
        auto place_of = [&](int t) __attribute__((always_inline)) {
            t = min(t, last);
            const int p = t >> 1;
            if ((uint32_t)(p - id_first) >= 64u) {                // 64 page ids at a time, waited for here and not at every use
                id_first = p;
                id_lane = ids[min(p + lane, a.max_pages - 1)];
                id_lane = id_lane >= 0 && id_lane < a.num_pages ? id_lane : -1;
                asm volatile("" : "+v"(id_lane));
            }
            const int page = __builtin_amdgcn_readlane(id_lane, p - id_first);
            return Place{part0 + (uint64_t)(uint32_t)max(page, 0) * page_bytes, (uint32_t)(t & 1), page >= 0 ? s.len - t * 64 : 0};
        };
        auto load_at = [&](Raw<D>& r, bool& on, const Place& pl) __attribute__((always_inline)) {
            on = key < pl.have;                                   // (keys behind the end: zeros, whatever the slots hold)
            const unsigned char* codes = pl.page + (code_at + pl.odd * (uint32_t)(64 * (D / 2)));
            const unsigned char* scales = pl.page + (scale_at + pl.odd * (uint32_t)(64 * (D / 16)));
            if constexpr (D == 128) {
                const uint4v c = *reinterpret_cast<const uint4v*>(codes);
                r.w[0] = c[0]; r.w[1] = c[1]; r.w[2] = c[2]; r.w[3] = c[3];
            } else {
                const uint2v c = *reinterpret_cast<const uint2v*>(codes);
                r.w[0] = c[0]; r.w[1] = c[1];
            }
            r.sc = *reinterpret_cast<const uint32_t*>(scales);
        };
        auto load_to = [&](Raw<D>& r, bool& on, int t) __attribute__((always_inline)) { load_at(r, on, place_of(t)); };
        auto load = [&](int t) __attribute__((always_inline)) { load_to(raw, raw_on, t); };
        // K: the 16 bytes of d = 16 i + 8 hf .. of a key in place 32 hf + key % 32 of operand (key / 32, i).  V: key after key.  A store serves eight lanes at
        // a time, the four pieces j of two keys, on 32 banks: the places of K's operands are turned by the piece, the 16-byte pieces of V's
        // keys by the key and the piece, so that they are eight different places of 16 bytes of 128.
        uint32_t place[D / 32];
#pragma unroll
        for (int j = 0; j < D / 32; ++j) {
            const int c = (D / 32) * g + j, i = c >> 1;
            place[j] = lds0 + (is_v ? (uint32_t)(2 * KB + key * RS + 16 * (D == 128 ? c ^ (2 * (key & 1)) ^ (g >> 1) : c ^ (key & 1)))
                                    : (uint32_t)((((key >> 5) * ND + i) * 64 + ((32 * (c & 1) + (key & 31)) ^ (2 * ((i >> (D == 128 ? 1 : 0)) & 3)))) * 16));
        }
        // (in D / 8 parts, so that they can stand between products: part 4 j + x makes values 8 j + 2 x, + 1, the last of four stores them)
        struct Unpack { half2v sc; uint32_t buf; uint4v v; };
        auto unpack_part = [&](Unpack& p, const Raw<D>& raw, bool raw_on, int part, int buf_k, int buf_v) __attribute__((always_inline)) {
            const int j = part >> 2, x = part & 3;
            if (part == 0) { p.sc = scales_of<D>(raw, g, raw_on); p.buf = is_v ? (uint32_t)(buf_v * VB) : (uint32_t)(buf_k * KB); }
            const half_t sv = (D == 128 && j >= 2) ? p.sc[1] : p.sc[0];
            const half2v sc2 = {sv, sv};
            if (x == 0) p.v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw.w[j], 1.0f, 0) * sc2);
            if (x == 1) p.v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw.w[j], 1.0f, 1) * sc2);
            if (x == 2) p.v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw.w[j], 1.0f, 2) * sc2);
            if (x == 3) { p.v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(raw.w[j], 1.0f, 3) * sc2); lds_write16_at(place[j] + p.buf, p.v); }
        };
        auto unpack = [&](const Raw<D>& raw, bool raw_on, int buf_k, int buf_v) __attribute__((always_inline)) {
            Unpack p;
#pragma unroll
            for (int part = 0; part < D / 8; ++part) unpack_part(p, raw, raw_on, part, buf_k, buf_v);
        };

        // what a segment needs from memory first, asked for at once: Q, the first tile of V, the first two of K
        uint4v x[ND];
        write_where((size_t)(s.first + tok) * a.q_token + (size_t)head * a.q_head);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < ND; ++i) x[i] = *reinterpret_cast<const uint4v*>(a.q + row_at(i) + 8 * (lane % LR));
        Raw<D> raw0, raw1;
        bool on0, on1;
        load_to(raw0, on0, first);
        load_to(raw1, on1, first + 1);
        if (is_v) { raw = raw1; raw_on = on1; } else load(first + 2);

        // Q: row col, d = 16 i + 8 half .. + 7
        half8 qreg[ND];
        float c_row;
        {
#pragma unroll
            for (int i = 0; i < ND; ++i) lds_write16_at(own_piece + (uint32_t)(i * RP * RO), x[i]);
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < ND; ++i) x[i] = lds_read16_at(own_row + (uint32_t)(32 * i + 16 * half));
            const float amax = lanes_max<32, 32>(largest_of(x));
            float f, inv;
            row_factor(amax, f, inv);
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    qreg[i][2 * j]     = (half_t)(__uint_as_float(x[i][j] << 16) * f);
                    qreg[i][2 * j + 1] = (half_t)(__uint_as_float(x[i][j] & 0xFFFF0000u) * f);
                }
            c_row = fmaxf(a.c * inv, kLeastFactor);
        }
        __syncthreads();                                          // (the segment before has read its tiles)
        unpack(raw0, on0, 0, 0);
        if (!is_v) unpack(raw1, on1, 1, 0);
        floatx16 o[NB], sc[2];
        float m = -INFINITY, up_to = -INFINITY, l = 0.0f;                             // the reference (kTop)
        half8 pt[4];
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.0f;

        // The products of a matrix phase in one run, each operand requested kAhead products before its own: a wave issues in order, and the trip to LDS
        // is as long as four products.  First O += V P of a tile, group of 16 keys by group, then S of the next.  The unpacking begins behind
        // kUnpackAt products, a few instructions to each, so that what it waits for from memory has had its time (from product 2 on 1 % slower).
        constexpr int kUnpackAt = D == 128 ? 8 : 4;
        constexpr int kAhead = 6, NV = 4 * NB, NK = 2 * ND;
        uint32_t k_base[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) k_base[x] = lds0 + 16u * (uint32_t)(lane ^ (2 * x));
        auto products = [&](auto with_values, int buf_v, int buf_k, int next) __attribute__((always_inline)) {
            constexpr int N0 = decltype(with_values)::value ? 0 : NV, N = NV + NK;
            const uint32_t vb[2] = {v_base + (uint32_t)(buf_v * VB), (v_base ^ 16u) + (uint32_t)(buf_v * VB)};
            uint32_t kb4[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) kb4[x] = k_base[x] + (uint32_t)(buf_k * KB);
            half8 ring[kAhead];
            Unpack up;
            Place next_at;
            auto operand = [&](int n) __attribute__((always_inline)) {
                if (n < NV) {
                    const uint32_t at = vb[(n % NB) >> 1] + (uint32_t)((n / NB) * 16 * RS + 64 * (n % NB));
                    const uint2v x = lds_read_tr16_at(at), y = lds_read_tr16_at(at + 8 * RS);
                    return __builtin_bit_cast(half8, uint4v{x[0], x[1], y[0], y[1]});
                }
                const int i = (n - NV) >> 1, kb = (n - NV) & 1;
                return __builtin_bit_cast(half8, lds_read16_at(kb4[(i >> (D == 128 ? 1 : 0)) & 3] + (uint32_t)((kb * ND + i) * 1024)));
            };
#pragma unroll
            for (int n = N0; n < N0 + kAhead; ++n) ring[n % kAhead] = operand(n);
#pragma unroll
            for (int n = N0; n < N; ++n) {
                __builtin_amdgcn_sched_barrier(0);
                if (n < NV) o[n % NB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ring[n % kAhead], pt[n / NB], o[n % NB], 0, 0, 0);
                else {
                    const int i = (n - NV) >> 1, kb = (n - NV) & 1;
                    if (i == 0) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) sc[kb][j] = 0.0f;
                    }
                    sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ring[n % kAhead], qreg[i], sc[kb], 0, 0, 0);
                }
                if (n + kAhead < N) ring[n % kAhead] = operand(n + kAhead);
                if (N0 == 0 && n >= kUnpackAt && n - kUnpackAt < D / 8) unpack_part(up, raw, raw_on, n - kUnpackAt, buf_v, buf_k);
                if (N0 == 0 && n == 4) next_at = place_of(next);
                if (N0 == 0 && n == kUnpackAt + D / 8) load_at(raw, raw_on, next_at);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        auto vector_phase = [&](int t) __attribute__((always_inline)) {
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
            mx = lanes_max<32, 32>(mx);
            if (__builtin_amdgcn_ballot_w64(mx > up_to) != 0) {
                const float m_new = fmaxf(m, fmaf(mx, c_row, -kTop)), alpha = __builtin_amdgcn_exp2f(m - (m_new == -INFINITY ? 0.0f : m_new));
                m = m_new;
                up_to = score_up_to(m_new, c_row);
                l *= alpha;
#pragma unroll
                for (int i = 0; i < NB; ++i) o[i] *= alpha;
            }
            const float m_at = m == -INFINITY ? 0.0f : m;
            float add[2] = {0.0f, 0.0f};
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const float x = __builtin_amdgcn_exp2f(fmaf(sc[kb][j], c_row, -m_at));
                    add[j & 1] += x;
                    pt[2 * kb + (j >> 3)][j & 7] = (half_t)x;
                }
            l += add[0] + add[1];
        };
        // Half-steps: the early waves are in the vector phase of tile i in half-step 2 i and in its matrix phase in 2 i + 1, the late ones one later.
        // K(i + 2) and V(i + 1), needed from half-step 2 i + 3 on, take the places of K(i) and V(i - 1), last read in 2 i: every wave unpacks its share of
        // them in its matrix phase, 2 i + 1 or 2 i + 2, between the products, which leave the vector unit idle three quarters of the time.  (In the
        // vector phase, with that phase at the higher priority: heads of 128 the same within 3 %, heads of 64 20 % slower.)
        phase_end();
        if (mine) products(std::false_type{}, 0, 0, 0);
        if (late) phase_end();
        for (int i = 0; i < cnt; ++i) {
            if (mine) vector_phase(first + i);
            phase_end();
            const int next = first + i + (is_v ? 2 : 3);
            __builtin_amdgcn_s_setprio(1);                        // (the longer of the two phases)
            if (mine) products(std::true_type{}, i & 1, (i + 1) & 1, next);
            else { unpack(raw, raw_on, i & 1, (i + 1) & 1); load(next); }
            __builtin_amdgcn_s_setprio(0);
            phase_end();
        }
        if (!late) phase_end();

        const bool whole = cnt == keys;
        if (mine) {
            l = lanes_sum<32, 32>(l);
            if (whole) {
                const float inv = l != 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        lds_write8_at(own_row + (uint32_t)(64 * i + 16 * j + 8 * half), uint2v{pack_bf16x2_cvt(o[i][4 * j] * inv, o[i][4 * j + 1] * inv), pack_bf16x2_cvt(o[i][4 * j + 2] * inv, o[i][4 * j + 3] * inv)});
                write_where((size_t)(s.first + tok) * a.o_token + (size_t)head * a.o_head);
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int p = 0; p < ND; ++p) {
                    const uint4v y = lds_read16_at(own_piece + (uint32_t)(p * RP * RO));
                    const size_t to = row_at(p);
                    if (w0 + p * RP + lane / LR < rows) *reinterpret_cast<uint4v*>(a.o + to + 8 * (lane % LR)) = y;
                }
                if (half == 0 && w0 + col < rows && a.lse) a.lse[(size_t)(s.first + tok) * a.Hq + head] = l != 0.0f ? m * 0.6931471805599453f + logf(l) : -INFINITY;
                __builtin_amdgcn_wave_barrier();
            } else {
                const size_t slot = ((size_t)blockIdx.x * 2 + (at == 0 ? 1 : 0)) * 8 + wave;
#pragma unroll
                for (int i = 0; i < NB; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<floatx4*>(ws.part_o + ((slot * (D / 8) + 4 * i + j) * 64 + lane) * 4) = floatx4{o[i][4 * j], o[i][4 * j + 1], o[i][4 * j + 2], o[i][4 * j + 3]};
                if (half == 0) { ws.part_ml[(slot * 32 + col) * 2] = m; ws.part_ml[(slot * 32 + col) * 2 + 1] = l; }
            }
        }
        // on to the next row tile, head, sequence
        off = 0;
        const int tiles = (rows + kWideRows - 1) / kWideRows;
        nt = 0;
        while (nt == 0 && ++tile < tiles) wide_tile(a, s, G, tile, t0, nt);
        if (nt == 0) {                                            // this head is done
            tile = -1;
            if (h == a.Hkv - 1) { front += per; per = 0; ++b; }
        }
    }
}

// O and lse of the row tiles whose key tiles were shared: a workgroup per place where one workgroup's work ended and another's began, and 32 rows; of the
// places within a row tile the first has it.  Bound by memory (each of 256 workgroups leaves up to two tiles of 256 rows in fp32: 14 us for heads of 128).
template <int D>
__device__ void wide_merge(const RaggedArgs& a, const WideWs& ws, int place, int wave)
{
    constexpr int NB = D / 32;
    if (place == 0) return;                                       // (nothing in front of the first)
    const long long quota = *ws.quota;
    const WideRec r = ws.rec[place];
    if (quota == 0 || r.off <= kWideStart || r.off - quota > kWideStart) return;      // it begins there, or has begun two workgroups ago
    const Seq s = seq_of(a, r.b);
    const Group G = group_of(a);
    const int rows = s.n * G, lane = threadIdx.x & 63, j = threadIdx.x >> 6;
    const int col = lane & 31, half = lane >> 5, row = r.tile * kWideRows + 32 * wave + col;
    if (r.tile * kWideRows + 32 * wave >= rows) return;
    const int n = 1 + (int)((r.nt - r.off + quota - 1) / quota);
    float M = -INFINITY, l = 0.0f;
    floatx4 v[NB] = {};
    for (int k0 = 0; k0 < n; k0 += 2) {
        floatx4 po[2][NB];
        float pm[2], pl[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int x = min(k0 + k, n - 1);
            const size_t slot = (x == 0 ? (size_t)(place - 1) * 2 + 1 : (size_t)(place + x - 1) * 2) * 8 + wave;
#pragma unroll
            for (int i = 0; i < NB; ++i) po[k][i] = *reinterpret_cast<const floatx4*>(ws.part_o + ((slot * (D / 8) + 4 * i + j) * 64 + lane) * 4);
            pm[k] = k0 + k < n ? ws.part_ml[(slot * 32 + col) * 2] : -INFINITY;
            pl[k] = ws.part_ml[(slot * 32 + col) * 2 + 1];
        }
        const float top = fmaxf(fmaxf(pm[0], pm[1]), M), at = top == -INFINITY ? 0.0f : top;
        const float f0 = __builtin_amdgcn_exp2f(M - at), f1 = __builtin_amdgcn_exp2f(pm[0] - at), f2 = __builtin_amdgcn_exp2f(pm[1] - at);
        M = top;
        l = l * f0 + pl[0] * f1 + pl[1] * f2;
#pragma unroll
        for (int i = 0; i < NB; ++i) v[i] = v[i] * f0 + po[0][i] * f1 + po[1][i] * f2;
    }
    if (row >= rows) return;
    const int tok = row / G, head = r.h * G + row % G;
    const float inv = l != 0.0f ? 1.0f / l : 0.0f;
    uint16_t* dst = a.o + (size_t)(s.first + tok) * a.o_token + (size_t)head * a.o_head + 8 * j + 4 * half;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
        const floatx4 y = v[i] * inv;
        *reinterpret_cast<uint2v*>(dst + 32 * i) = uint2v{pack_bf16x2_cvt(y[0], y[1]), pack_bf16x2_cvt(y[2], y[3])};
    }
    if (j == 0 && half == 0 && a.lse) a.lse[(size_t)(s.first + tok) * a.Hq + head] = l != 0.0f ? M * 0.6931471805599453f + logf(l) : -INFINITY;
}
// O = 0, lse = -inf for row tiles, of sequences with many rows, that see no key: they are nobody's work.  One of n workgroups, which has every n-th sequence
// and asks for the lengths of 64 of them at once.
template <int D>
__device__ void wide_empty(const RaggedArgs& a, int which, int n)
{
    const Group G = group_of(a);
    const int lane = threadIdx.x & 63;
    for (int b0 = which; b0 < a.B; b0 += 64 * n) {
        const Seq mine = b0 + lane * n < a.B ? seq_of(a, b0 + lane * n) : Seq{0, 0, 0};
        int t0, nt = 1;
        if (mine.n * G > kFewRows) wide_tile(a, mine, G, 0, t0, nt);
        for (unsigned long long left = __builtin_amdgcn_ballot_w64(nt == 0); left != 0; left &= left - 1) {
            const int src = (int)__builtin_ctzll(left);
            const Seq s{__builtin_amdgcn_readlane(mine.first, src), __builtin_amdgcn_readlane(mine.n, src), __builtin_amdgcn_readlane(mine.len, src)};
            const int rows = s.n * G;
            for (int tile = 0; tile * kWideRows < rows; ++tile) {
                wide_tile(a, s, G, tile, t0, nt);
                if (nt > 0) break;                                // (the ones behind it see keys as well)
                const int r1 = min((tile + 1) * kWideRows, rows);
                for (int h = 0; h < a.Hkv; ++h)
                    for (int e = threadIdx.x; e < (r1 - tile * kWideRows) * (D / 8); e += 256) {
                        const int row = tile * kWideRows + e / (D / 8), d = e % (D / 8) * 8, head = h * G + row % G;
                        *reinterpret_cast<uint4v*>(a.o + (size_t)(s.first + row / G) * a.o_token + (size_t)head * a.o_head + d) = uint4v{0u, 0u, 0u, 0u};
                        if (d == 0 && a.lse) a.lse[(size_t)(s.first + row / G) * a.Hq + head] = -INFINITY;
                    }
            }
        }
    }
}
// The last launch of a step: what the others left to be joined.
constexpr int kEmptyWgs = 64;
template <int D, int ROWS>
__global__ __launch_bounds__(256) void ragged_merge_kernel(const RaggedArgs a, const FewWs few, int tiles, const WideWs wide, int places)
{
    int x = (int)blockIdx.x;
    if (x < 8 * places) { wide_merge<D>(a, wide, x / 8, x % 8); return; }
    x -= 8 * places;
    if (x < a.B * a.Hkv * tiles) { few_merge<D, ROWS>(a, few, x, tiles); return; }
    wide_empty<D>(a, x - a.B * a.Hkv * tiles, kEmptyWgs);
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

// Which kernels a step may need: the host knows only how many rows a sequence has at most.
struct RaggedPlan { int few_groups, few_tiles, few_wgs, wide_wgs /* 0: no sequence has that many rows */; };
inline RaggedPlan plan_of(int T, int B, int Hq, int Hkv, int max_q, int max_pages, int D, int cus)
{
    const long long most = (long long)(max_q < T ? max_q : T) * (Hq / Hkv), rows = (long long)T * (Hq / Hkv);
    RaggedPlan p;
    p.few_groups = most <= 16 ? 1 : 2;
    p.few_tiles = (int)(((most < kFewRows ? most : kFewRows) + 16 * p.few_groups - 1) / (16 * p.few_groups));
    const long long units = (long long)B * Hkv * p.few_tiles * (max_pages + (D == 64 ? kFewStart<64> : kFewStart<128>)), wgs = (long long)cus * (p.few_groups == 1 ? 3 : 2);
    p.few_wgs = (int)(units < wgs ? units : wgs);
    p.wide_wgs = 0;
    if (most > kFewRows) {
        const long long tiles = ((long long)B + rows / kWideRows) * Hkv * (max_pages * 2 + kWideStart), wide = cus;
        p.wide_wgs = (int)(tiles < wide ? tiles : wide);
    }
    return p;
}
struct RaggedWs { FewWs few; WideWs wide; size_t bytes; };
inline RaggedWs carve_ragged(void* ws, const RaggedPlan& p, int B, int D)
{
    unsigned char* base = (unsigned char*)ws;
    size_t off = 0;
    auto take = [&](size_t n) { unsigned char* r = base + off; off += up256(n); return r; };
    const size_t rows = (size_t)p.few_wgs * 2 * 16 * p.few_groups, wide = (size_t)p.wide_wgs * 2 * kWideRows;
    RaggedWs w;
    w.few.quota = (int*)take(4);
    w.few.front = (int*)take(((size_t)B + 1) * 4);
    w.wide.quota = (long long*)take(8);
    w.wide.rec = (WideRec*)take(p.wide_wgs * sizeof(WideRec));
    // (the two kinds of partial sums follow each other: both launches' are there until they are joined)
    w.few.part_o = (float*)take(rows * D * 4);
    w.few.part_ml = (float*)take(rows * 8);
    w.wide.part_o = (float*)take(wide * D * 4);
    w.wide.part_ml = (float*)take(wide * 8);
    w.bytes = off;
    return w;
}

template <int D, int RT>
int launch_ragged_of(const RaggedArgs& a, const RaggedPlan& p, const RaggedWs& w, hipStream_t st)
{
    hipLaunchKernelGGL((ragged_few_kernel<D, RT>), dim3(p.few_wgs), dim3(256), 0, st, a, w.few);
    if (hipGetLastError() != hipSuccess) return -1;
    if (p.wide_wgs > 0) {
        constexpr int bytes = 2 * 64 * (2 * D + 2 * D + 64);
        static unsigned long long done = 0;
        if (!ensure_dynamic_lds((const void*)ragged_wide_kernel<D>, bytes, done)) return -1;
        hipLaunchKernelGGL((ragged_wide_kernel<D>), dim3(p.wide_wgs), dim3(512), bytes, st, a, w.wide);
        if (hipGetLastError() != hipSuccess) return -1;
    }
    const int wgs = a.B * a.Hkv * p.few_tiles + (p.wide_wgs > 0 ? p.wide_wgs * 8 + kEmptyWgs : 0);
    hipLaunchKernelGGL((ragged_merge_kernel<D, 16 * RT>), dim3(wgs), dim3(256), 0, st, a, w.few, p.few_tiles, w.wide, p.wide_wgs);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace

size_t ragged_ws_bytes(int T, int B, int Hq, int Hkv, int max_q, int max_pages, int D)
{
    return carve_ragged(nullptr, plan_of(T, B, Hq, Hkv, max_q, max_pages, D, kChipCus), B, D).bytes;
}

int launch_ragged(const RaggedArgs& args, int D, void* ws, hipStream_t st)
{
    RaggedArgs a = args;
    if (a.window >= a.max_pages * 128) a.window = 0;              // (hides nothing; below, positions less a window stay within 32 bits)
    a.group = a.Hq / a.Hkv;
    a.group_shift = 0;
    while ((1 << a.group_shift) < a.group) ++a.group_shift;       // (a.group <= 2^28)
    a.group_mul = (uint32_t)(((1ull << (31 + a.group_shift)) + a.group - 1) / a.group);
    const RaggedPlan p = plan_of(a.T, a.B, a.Hq, a.Hkv, a.max_q, a.max_pages, D, kChipCus);
    const RaggedWs w = carve_ragged(ws, p, a.B, D);
    return D == 128 ? (p.few_groups == 1 ? launch_ragged_of<128, 1>(a, p, w, st) : launch_ragged_of<128, 2>(a, p, w, st))
                    : (p.few_groups == 1 ? launch_ragged_of<64, 1>(a, p, w, st) : launch_ragged_of<64, 2>(a, p, w, st));
}

}  // namespace aq
