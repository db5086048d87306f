// Rotary positions: Q and K turned by their positions in up to four axes (attnqat_rope_fwd, and with the opposite angles attnqat_rope_bwd), and the same on
// the way into the NVFP4 KV cache (attnqat_kv_cache_append_rope).
//
// Pair i of a head turns by the angle p f, p the position in the pair's axis and f its frequency: (a, b) -> (a cos - b sin, a sin + b cos).  Angles are kept as
// fractions of a turn in 64 bits of fixed point: f / 2 pi as a fraction F 2^-64 (what it has of whole turns changes nothing, p being whole), and p F modulo
// 2^64 is the angle, off by at most |p| 2^-53 turns of rounding f, however far p is.  Its quadrant and the rest, within an eighth of a turn, go to the Taylor series of
// sine and cosine (the first terms left out are below 2^-29 and 2^-33), so that both are within 2^-23 of what they should be.  The products are fp32, and
// a turned value is rounded once, to bf16.
#include "common.hpp"
#include "kernels.hpp"
#include "nvfp4.hpp"

namespace aq {

namespace {

__device__ __forceinline__ void turn_of(uint64_t f, int pos, float& c, float& s)
{
    const uint32_t u = (uint32_t)((f * (uint64_t)(int64_t)pos + 0x80000000ull) >> 32);      // the angle in units of 2^-32 turns
    const uint32_t q = (u + 0x20000000u) >> 30;
    const float z = (float)(int)(u - (q << 30)) * 1.4629180792671596e-9f /* 2 pi / 2^32 */, z2 = z * z;
    const float sz = fmaf(z * z2, fmaf(z2, fmaf(z2, fmaf(z2, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), z);
    const float cz = fmaf(z2, fmaf(z2, fmaf(z2, fmaf(z2, fmaf(z2, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const float a = (q & 1) ? sz : cz, b = (q & 1) ? cz : sz;
    c = __uint_as_float(__float_as_uint(a) ^ (((q + 1) & 2) << 30));
    s = __uint_as_float(__float_as_uint(b) ^ ((q & 2) << 30));
}

// What a thread has of a row of heads: 8 pairs, which are 16 consecutive values (pairs of neighbours), or 8 values and their 8 partners half the turned part
// away.  Values behind the turned part go to the threads that are left, 16 each, as they are.
template <int D, bool HALVES>
struct Part {
    int lo, hi;                       // first of its 8 + 8 values
    int live;                         // pairs that turn
    float c[8], s[8];
    __device__ __forceinline__ Part(const RopeTable& r, int chunk)
    {
        const int left = r.pairs - 8 * chunk;
        live = min(max(left, 0), 8);
        if (HALVES) {
            lo = left > 0 ? 8 * chunk : 16 * chunk;                      // (pairs is a multiple of 8)
            hi = lo + (left > 0 ? r.pairs : 8);
        } else { lo = 16 * chunk; hi = lo + 8; }
    }
    __device__ __forceinline__ void turn(const RopeTable& r, int chunk, const int* __restrict__ pos /* of the token */)
    {
        int p[kRopeAxes];
#pragma unroll
        for (int a = 0; a < kRopeAxes; ++a) p[a] = a < r.axes ? pos[a] : 0;
        const uint32_t axis = r.axis[chunk >> 1] >> (16 * (chunk & 1));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t a = (axis >> (2 * i)) & 3u;
            turn_of(r.freq[8 * chunk + i], a < 2 ? (a == 0 ? p[0] : p[1]) : (a == 2 ? p[2] : p[3]), c[i], s[i]);
        }
    }
    __device__ __forceinline__ void apply(uint4v& x, uint4v& y) const
    {
        if (live == 0) return;
        auto f = [](uint32_t w, int odd) __attribute__((always_inline)) { return odd ? __uint_as_float(w & 0xFFFF0000u) : __uint_as_float(w << 16); };
        if (HALVES) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a0 = f(x[j], 0), a1 = f(x[j], 1), b0 = f(y[j], 0), b1 = f(y[j], 1);
                x[j] = pack_bf16x2_cvt(a0 * c[2 * j] - b0 * s[2 * j], a1 * c[2 * j + 1] - b1 * s[2 * j + 1]);
                y[j] = pack_bf16x2_cvt(a0 * s[2 * j] + b0 * c[2 * j], a1 * s[2 * j + 1] + b1 * c[2 * j + 1]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t w = j < 4 ? x[j & 3] : y[j & 3];
                const float a = f(w, 0), b = f(w, 1);
                const uint32_t t = j < live ? pack_bf16x2_cvt(a * c[j] - b * s[j], a * s[j] + b * c[j]) : w;
                if (j < 4) x[j & 3] = t; else y[j & 3] = t;
            }
        }
    }
};

// Bound by memory: a value is read once and written once, 4 bytes for 3 operations; a table of sines in memory would add to that, and sixteen multiply-adds for
// a pair's angle are in the shadow of the loads.  A thread has its pairs of several heads of a token: their loads, of 32 bytes a head, are under way at once, and
// they share the sines.  12 + 12 heads of 128, 32760 tokens (403 MB): 83 us, 4.85 TB/s, where a large copy reaches 5.1; of a pass, 84.5 us, one head to a thread makes 94, two 86, eight 86.
// 32 + 8 heads, 16384 tokens (336 MB): 73 us, 4.6 TB/s.  1560 tokens (19 MB) 7.1 us, 512 rows of 64 (0.26 MB) 4.2 us: launch and one trip to memory.
constexpr int kRopeHeads = 4;
template <int D, bool HALVES>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a, const RopeTable r)
{
    constexpr int nt = D / 16;
    const int chunk = threadIdx.x % nt;
    const long long n = (long long)blockIdx.x * (256 / nt) + threadIdx.x / nt;
    const int q_groups = (a.t[0].heads + kRopeHeads - 1) / kRopeHeads;
    const bool is_k = (int)blockIdx.y >= q_groups;
    const RopeTensor& t = a.t[is_k];
    const int h0 = ((int)blockIdx.y - (is_k ? q_groups : 0)) * kRopeHeads;
    if (n >= (long long)a.B * a.L) return;
    const int b = (int)(n / a.L), l = (int)(n % a.L);
    Part<D, HALVES> p(r, chunk);
    uint4v x[kRopeHeads], y[kRopeHeads];
    const uint16_t* src = t.src + b * t.src_batch + l * t.src_token;
#pragma unroll
    for (int i = 0; i < kRopeHeads; ++i) {
        const uint16_t* s = src + min(h0 + i, t.heads - 1) * t.src_head;
        x[i] = *reinterpret_cast<const uint4v*>(s + p.lo);
        y[i] = *reinterpret_cast<const uint4v*>(s + p.hi);
    }
    p.turn(r, chunk, a.positions + b * a.pos_batch + (size_t)l * r.axes);
    uint16_t* dst = t.dst + b * t.dst_batch + l * t.dst_token;
#pragma unroll
    for (int i = 0; i < kRopeHeads; ++i) {
        if (h0 + i >= t.heads) break;
        p.apply(x[i], y[i]);
        uint16_t* d = dst + (h0 + i) * t.dst_head;
        *reinterpret_cast<uint4v*>(d + p.lo) = x[i];
        *reinterpret_cast<uint4v*>(d + p.hi) = y[i];
    }
}

// Into the cache: a group of workgroups has heads of Q (turned, to q_out), of K (turned, rounded to bf16, which is what a model trained on turned bf16 keys
// quantizes, and phi) or of V (phi).  A thread has 16 values of a row; where the partners lie half a row apart the turned K goes through LDS, a row within its
// wave, to come back as the blocks of 16 that phi takes.
// Bound by memory too: Q is read and written, K and V are read (phi leaves 0.28 of their bytes).  Q, K and V of a token are often pieces of one projection's row, so the
// workgroups of a group of tokens follow each other.  32 + 8 + 8 heads of 128, 12172 tokens (pieces of one tensor, 263 MB): 53 us, 5.0 TB/s; all of Q in front of K and V: 67 us.
// 64 rows of a decode step: 5.0 us.
template <int D, bool HALVES>
__global__ __launch_bounds__(256) void append_rope_kernel(const AppendRopeArgs a, const RopeTable r)
{
    constexpr int nt = D / 16, nb = D / 16, RS = 2 * D + 16;
    __shared__ __align__(16) unsigned char rows[HALVES ? 256 / nt * RS : 16];
    const int qg = (a.Hq + kRopeHeads - 1) / kRopeHeads, kg = (a.Hkv + kRopeHeads - 1) / kRopeHeads;
    const int chunk = threadIdx.x % nt, t = (int)(blockIdx.x / (unsigned)(qg + 2 * kg)) * (256 / nt) + threadIdx.x / nt;
    const int g = (int)(blockIdx.x % (unsigned)(qg + 2 * kg)), role = g < qg ? 0 : g < qg + kg ? 1 : 2, h0 = (g - (role == 0 ? 0 : role == 1 ? qg : qg + kg)) * kRopeHeads;
    const Rows& in = role == 0 ? a.q : role == 1 ? a.k : a.v;
    const int heads = role == 0 ? a.Hq : a.Hkv;
    const int tc = min(t, a.T - 1);                               // (whole waves stay: they share LDS rows and lanes)
    Part<D, HALVES> p(r, chunk);
    if (role == 2) { p.lo = 16 * chunk; p.hi = p.lo + 8; p.live = 0; }
    uint4v x[kRopeHeads], y[kRopeHeads];
    const uint16_t* src = (const uint16_t*)in.p + tc * in.token;
#pragma unroll
    for (int i = 0; i < kRopeHeads; ++i) {
        const uint16_t* s = src + min(h0 + i, heads - 1) * in.head;
        x[i] = *reinterpret_cast<const uint4v*>(s + p.lo);
        y[i] = *reinterpret_cast<const uint4v*>(s + p.hi);
    }
    const long long slot = role == 0 ? 0 : a.slots[tc];
    if (role != 2) p.turn(r, chunk, a.positions + (size_t)tc * r.axes);
    if (role == 0) {
        if (t >= a.T) return;
        uint16_t* dst = (uint16_t*)a.q_out.p + t * a.q_out.token;
#pragma unroll
        for (int i = 0; i < kRopeHeads; ++i) {
            if (h0 + i >= heads) break;
            p.apply(x[i], y[i]);
            uint16_t* d = dst + (h0 + i) * a.q_out.head;
            *reinterpret_cast<uint4v*>(d + p.lo) = x[i];
            *reinterpret_cast<uint4v*>(d + p.hi) = y[i];
        }
        return;
    }
    const bool on = t < a.T && slot >= 0 && slot < (long long)a.num_pages * 128;
    const int off = (int)(slot & 127);
#pragma unroll
    for (int i = 0; i < kRopeHeads; ++i) {
        if (h0 + i >= heads) break;
        p.apply(x[i], y[i]);
        if (HALVES && role == 1) {
            unsigned char* row = rows + threadIdx.x / nt * RS;
            __builtin_amdgcn_wave_barrier();
            *reinterpret_cast<uint4v*>(row + 2 * p.lo) = x[i];
            *reinterpret_cast<uint4v*>(row + 2 * p.hi) = y[i];
            __builtin_amdgcn_wave_barrier();
            x[i] = *reinterpret_cast<const uint4v*>(row + 32 * chunk);
            y[i] = *reinterpret_cast<const uint4v*>(row + 32 * chunk + 16);
        }
        float val[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t w = j < 4 ? x[i][j & 3] : y[i][j & 3];
            val[2 * j] = __uint_as_float(w << 16);
            val[2 * j + 1] = __uint_as_float(w & 0xFFFF0000u);
        }
        const Nv16 c = phi_block16_bf16(val);
        // the scale bytes of four neighbouring blocks of a row as one dword
        uint32_t sb = c.sc & 0xFFu;
        sb |= lane_down<1>(sb) << 8;
        sb |= lane_down<2>(sb) << 16;
        if (!on) continue;
        unsigned char* part = a.cache + ((size_t)(slot >> 7) * a.Hkv + h0 + i) * nvfp4_page_head_bytes(D) + (role == 2 ? 128 * (D / 2 + nb) : 0);
        uint2v c2; c2[0] = c.clo; c2[1] = c.chi;
        *reinterpret_cast<uint2v*>(part + off * (D / 2) + chunk * 8) = c2;
        if ((chunk & 3) == 0) *reinterpret_cast<uint32_t*>(part + 128 * (D / 2) + off * nb + chunk) = sb;
    }
}

inline int groups_of(int heads) { return (heads + kRopeHeads - 1) / kRopeHeads; }

}  // namespace

int launch_rope(const RopeArgs& a, const RopeTable& r, int D, bool halves, hipStream_t st)
{
    const int per = 256 / (D / 16);
    const dim3 grid((unsigned)(((long long)a.B * a.L + per - 1) / per), groups_of(a.t[0].heads) + groups_of(a.t[1].heads));
    if (D == 128) {
        if (halves) hipLaunchKernelGGL((rope_kernel<128, true>), grid, dim3(256), 0, st, a, r);
        else        hipLaunchKernelGGL((rope_kernel<128, false>), grid, dim3(256), 0, st, a, r);
    } else {
        if (halves) hipLaunchKernelGGL((rope_kernel<64, true>), grid, dim3(256), 0, st, a, r);
        else        hipLaunchKernelGGL((rope_kernel<64, false>), grid, dim3(256), 0, st, a, r);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_append_rope(const AppendRopeArgs& a, const RopeTable& r, int D, bool halves, hipStream_t st)
{
    const int per = 256 / (D / 16);
    // (all heads of a group of tokens one after another: they lie side by side in memory)
    const dim3 grid((unsigned)((a.T + per - 1) / per) * (groups_of(a.Hq) + 2 * groups_of(a.Hkv)));
    if (D == 128) {
        if (halves) hipLaunchKernelGGL((append_rope_kernel<128, true>), grid, dim3(256), 0, st, a, r);
        else        hipLaunchKernelGGL((append_rope_kernel<128, false>), grid, dim3(256), 0, st, a, r);
    } else {
        if (halves) hipLaunchKernelGGL((append_rope_kernel<64, true>), grid, dim3(256), 0, st, a, r);
        else        hipLaunchKernelGGL((append_rope_kernel<64, false>), grid, dim3(256), 0, st, a, r);
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace aq
