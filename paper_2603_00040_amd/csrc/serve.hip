// A serving step's bookkeeping and its way into and out of the NVFP4 KV cache: page tables and slot maps from request lengths
// (attnqat_page_plan), the rows of a ragged batch into their slots (attnqat_kv_cache_append) and back (attnqat_kv_cache_read).
// A slot is page * 128 + position within the page.
#include "common.hpp"
#include "kernels.hpp"
#include "nvfp4.hpp"

namespace aq {

namespace {

// What the plan keeps between its two launches.  Of a request: the positions it had, the place in the ring of its first new page (-1 where
// the request was refused), and how many pages it gives back, the first of them being number first_give among all.  Of the ring: where the
// pages that are given back go.
struct PlanItem { int old_len, take, give, first_give; };
struct PlanHead { int tail, unused[3]; };

__device__ inline int pages_of(int positions) { return (positions + 127) >> 7; }

// Inclusive sums over a workgroup of 1024 threads, and the sums over all of it.
template <class T>
__device__ inline T wg_scan(T v, T* red /* [16], LDS */, T& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const T a = __shfl_up(v, d);
        if (lane >= d) v += a;
    }
    __syncthreads();                                             // (red of the call before has been read)
    if (lane == 63) red[wave] = v;
    __syncthreads();
    T front = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        front += w < wave ? red[w] : T(0);
        total += red[w];
    }
    return v + front;
}

// One workgroup: who gets what.  A request is served if it fits its row of the page table, its new positions end within the step's capacity
// T, and the pages asked for up to and including it are free; pages given back by this step are for the next one.  The sums run over
// refused requests too, so that nobody waits for a decision: refused for want of pages are then all that ask for any from the first such on,
// and the pages that are taken are a prefix of those asked for.  (64 bits for the positions: what is asked for is not limited by T.)
__global__ __launch_bounds__(1024) void plan_scan_kernel(const int* kv_lens, const int* new_lens, int B, int max_pages, const int* ring_state,
                                                         int ring_size /* 0: no ring, the table is complete */, int T, int* kv_out,
                                                         int* __restrict__ cu, int* state_out, PlanHead* __restrict__ hd, PlanItem* __restrict__ items)
{
    __shared__ long long red_l[16];
    __shared__ int red_i[16], taken, refused;
    const int tid = threadIdx.x;
    const bool ring = ring_size > 0;
    const int head = ring ? min(max(ring_state[0], 0), ring_size - 1) : 0, count = ring ? min(max(ring_state[1], 0), ring_size) : 0;
    if (tid == 0) { taken = 0; refused = 0; cu[0] = 0; }
    long long grown = 0, total_l;
    int needed = 0, given = 0, total;
    for (int b0 = 0; b0 < B; b0 += 1024) {
        const int b = b0 + tid;
        const bool on = b < B;
        const int old = on ? min(max(kv_lens[b], 0), max_pages * 128) : 0, want = on ? max(new_lens[b], 0) : 0;
        const bool bad = want > max_pages * 128;
        const int grow = bad ? 0 : max(want - old, 0), give = ring && !bad ? max(pages_of(old) - pages_of(want), 0) : 0;
        const long long end = grown + wg_scan<long long>(grow, red_l, total_l);
        grown += total_l;
        const bool late = grow > 0 && end > T;
        const int need = !ring || bad || late ? 0 : max(pages_of(want) - pages_of(old), 0);
        const int upto = needed + wg_scan(need, red_i, total);
        needed += total;
        const int give_end = given + wg_scan(give, red_i, total);
        given += total;
        const bool ok = !bad && !late && (need == 0 || upto <= count);
        if (on) {
            cu[b + 1] = (int)min(end, (long long)T);
            kv_out[b] = ok ? want : old;
            items[b] = PlanItem{old, ok ? (ring ? (int)(((long long)head + upto - need) % ring_size) : 0) : -1, give, give_end - give};
            if (need > 0 && ok) atomicMax(&taken, upto);
            if (!ok) atomicAdd(&refused, 1);
        }
    }
    __syncthreads();
    if (tid == 0) {
        hd->tail = ring ? (int)(((long long)head + count) % ring_size) : 0;
        if (state_out) {
            state_out[0] = ring ? (int)(((long long)head + taken) % ring_size) : 0;
            state_out[1] = (int)min((long long)count - taken + given, (long long)ring_size);
            state_out[2] = refused;
        }
    }
}

// The request of position t of the step: the last b with cu[b] <= t (t < cu[B]).
__device__ inline int request_of(const int* cu, int B, int t)
{
    int lo = 0, hi = B;                                          // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= t) lo = mid; else hi = mid;
    }
    return lo;
}

// Slots and positions of the step's tokens, a thread each; the token that begins a new page writes it into the table (every new page begins with
// one).  The last workgroups: pages that are given back, a wave for 64 requests, its lanes over the pages of one request after another.  What
// is read of the ring and what is written to it do not meet: free pages and pages given back together are no more than the ring has places.
__global__ __launch_bounds__(256) void plan_fill_kernel(const int* __restrict__ cu, int B, int* page_table, int max_pages, int* ring,
                                                        int ring_size, int T, int token_wgs, const PlanHead* __restrict__ hd,
                                                        const PlanItem* __restrict__ items, long long* __restrict__ slots, int* __restrict__ positions)
{
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < token_wgs) {
        const int t = (int)blockIdx.x * 256 + tid;
        if (t >= T) return;
        long long slot = -1;
        int pos = 0;
        if (t < cu[B]) {
            const int b = request_of(cu, B, t);
            const PlanItem it = items[b];
            pos = it.old_len + (t - cu[b]);
            if (it.take >= 0) {
                const int j = pos >> 7, fresh = j - pages_of(it.old_len);          // < max_pages: the request fits its row
                int* entry = page_table + (size_t)b * max_pages + j;
                int page;
                if (ring_size > 0 && fresh >= 0) {
                    page = ring[((long long)it.take + fresh) % ring_size];
                    if ((pos & 127) == 0) *entry = page;
                } else page = *entry;
                if (page >= 0) slot = (long long)page * 128 + (pos & 127);
            }
        }
        slots[t] = slot;
        positions[t] = pos;
        return;
    }
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int b0 = (((int)blockIdx.x - token_wgs) * 4 + wave) * 64, b = b0 + lane;
    const PlanItem it = b < B ? items[b] : PlanItem{0, 0, 0, 0};
    const int tail = hd->tail;
    for (unsigned long long m = __builtin_amdgcn_ballot_w64(it.give > 0); m != 0; m &= m - 1) {
        const int src = (int)__builtin_ctzll(m);
        const int give = __builtin_amdgcn_readlane(it.give, src), first = __builtin_amdgcn_readlane(it.first_give, src);
        const int kept = pages_of(__builtin_amdgcn_readlane(it.old_len, src)) - give;
        for (int j = lane; j < give; j += 64)
            ring[((long long)tail + first + j) % ring_size] = page_table[(size_t)(b0 + src) * max_pages + kept + j];
    }
}

// A row (token, kv head) of K or V has D / 16 blocks; a thread takes one block of one row, neighbouring threads the blocks of a row and
// then the rows of the next tokens, whose slots in a page mostly follow each other.
template <int D>
__global__ __launch_bounds__(256) void append_kernel(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, size_t k_token, size_t k_head,
                                                     size_t v_token, size_t v_head, int T, int Hkv, unsigned char* __restrict__ cache, int num_pages,
                                                     const long long* __restrict__ slots)
{
    constexpr int nb = D / 16;
    const int h = blockIdx.y, which = blockIdx.z, cb = threadIdx.x % nb;
    const int t = (int)blockIdx.x * (256 / nb) + threadIdx.x / nb, tc = min(t, T - 1);
    const long long slot = slots[tc];
    const uint4v* src = reinterpret_cast<const uint4v*>((which ? v : k) + (size_t)tc * (which ? v_token : k_token) + (size_t)h * (which ? v_head : k_head) + cb * 16);
    const uint4v a = src[0], b = src[1];
    float val[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        val[2 * i]         = __uint_as_float(a[i] << 16);
        val[2 * i + 1]     = __uint_as_float(a[i] & 0xFFFF0000u);
        val[8 + 2 * i]     = __uint_as_float(b[i] << 16);
        val[8 + 2 * i + 1] = __uint_as_float(b[i] & 0xFFFF0000u);
    }
    const Nv16 q = phi_block16_bf16(val);
    // the scale bytes of four neighbouring blocks of a row as one dword
    uint32_t sb = q.sc & 0xFFu;
    sb |= lane_down<1>(sb) << 8;
    sb |= lane_down<2>(sb) << 16;
    if (t >= T || slot < 0 || slot >= (long long)num_pages * 128) return;
    unsigned char* part = cache + ((size_t)(slot >> 7) * Hkv + h) * nvfp4_page_head_bytes(D) + (which ? 128 * (D / 2 + nb) : 0);
    const int off = (int)(slot & 127);
    uint2v c2; c2[0] = q.clo; c2[1] = q.chi;
    *reinterpret_cast<uint2v*>(part + off * (D / 2) + cb * 8) = c2;
    if ((cb & 3) == 0) *reinterpret_cast<uint32_t*>(part + 128 * (D / 2) + off * nb + cb) = sb;
}

// The same way back; a slot outside the cache reads as zeros.  (A value has at most 6 significant bits: exact in bf16.)
template <int D>
__global__ __launch_bounds__(256) void read_kernel(uint16_t* __restrict__ k, uint16_t* __restrict__ v, size_t k_token, size_t k_head, size_t v_token,
                                                   size_t v_head, int T, int Hkv, const unsigned char* __restrict__ cache, int num_pages,
                                                   const long long* __restrict__ slots)
{
    constexpr int nb = D / 16;
    const int h = blockIdx.y, which = blockIdx.z, cb = threadIdx.x % nb;
    const int t = (int)blockIdx.x * (256 / nb) + threadIdx.x / nb;
    if (t >= T) return;
    const long long slot = slots[t];
    float x[16] = {};
    if (slot >= 0 && slot < (long long)num_pages * 128) {
        const unsigned char* part = cache + ((size_t)(slot >> 7) * Hkv + h) * nvfp4_page_head_bytes(D) + (which ? 128 * (D / 2 + nb) : 0);
        const int off = (int)(slot & 127);
        const uint2v c = *reinterpret_cast<const uint2v*>(part + off * (D / 2) + cb * 8);
        dequant_block16(nv16_of(c[0], c[1], part[128 * (D / 2) + off * nb + cb]), x);
    }
    uint4v* dst = reinterpret_cast<uint4v*>((which ? v : k) + (size_t)t * (which ? v_token : k_token) + (size_t)h * (which ? v_head : k_head) + cb * 16);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint4v w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2_cvt(x[8 * i + 2 * j], x[8 * i + 2 * j + 1]);
        dst[i] = w;
    }
}

}  // namespace

size_t page_plan_ws_bytes(int B) { return sizeof(PlanHead) + (size_t)B * sizeof(PlanItem); }

int launch_page_plan(const int* kv_lens, const int* new_lens, int B, int* page_table, int max_pages, int* ring, int ring_size, const int* ring_state,
                     int T, int* kv_out, int* cu, long long* slots, int* positions, int* state_out, void* ws, hipStream_t st)
{
    PlanHead* hd = (PlanHead*)ws;
    PlanItem* items = (PlanItem*)(hd + 1);
    hipLaunchKernelGGL(plan_scan_kernel, dim3(1), dim3(1024), 0, st, kv_lens, new_lens, B, max_pages, ring_state, ring_size, T, kv_out, cu, state_out, hd, items);
    if (hipGetLastError() != hipSuccess) return -1;
    const int token_wgs = (T + 255) / 256, give_wgs = ring_size > 0 ? (B + 255) / 256 : 0;
    if (token_wgs + give_wgs > 0)
        hipLaunchKernelGGL(plan_fill_kernel, dim3(token_wgs + give_wgs), dim3(256), 0, st, cu, B, page_table, max_pages, ring, ring_size, T, token_wgs, hd, items, slots, positions);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_append(const Rows& k, const Rows& v, int T, int Hkv, int D, void* cache, int num_pages, const long long* slots, hipStream_t st)
{
    const int per = 256 / (D / 16);
    const dim3 grid((T + per - 1) / per, Hkv, 2);
    if (D == 128) hipLaunchKernelGGL((append_kernel<128>), grid, dim3(256), 0, st, (const uint16_t*)k.p, (const uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (unsigned char*)cache, num_pages, slots);
    else          hipLaunchKernelGGL((append_kernel<64>), grid, dim3(256), 0, st, (const uint16_t*)k.p, (const uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (unsigned char*)cache, num_pages, slots);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_read(const Rows& k, const Rows& v, int T, int Hkv, int D, const void* cache, int num_pages, const long long* slots, hipStream_t st)
{
    const int per = 256 / (D / 16);
    const dim3 grid((T + per - 1) / per, Hkv, 2);
    if (D == 128) hipLaunchKernelGGL((read_kernel<128>), grid, dim3(256), 0, st, (uint16_t*)k.p, (uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (const unsigned char*)cache, num_pages, slots);
    else          hipLaunchKernelGGL((read_kernel<64>), grid, dim3(256), 0, st, (uint16_t*)k.p, (uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (const unsigned char*)cache, num_pages, slots);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace aq
