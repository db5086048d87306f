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

// Who gets what, by a workgroup of 1024: of request b (a thread each) what the rest of the plan needs; sums of the requests in front in `in`, which moves on.
// A request is served if it fits its row of the page table, its new positions end within the step's capacity T, and the pages asked for up to and
// including it are free; pages given back by this step are for the next one, and go into places of the ring that no free page has (those of the free ones are
// read by whoever takes them, at the same time): a request whose pages find no such place is refused.  The sums run over refused requests too, so that nobody
// waits for a decision: refused for want of pages are then all that ask for any from the first such on, and the pages that are taken are a prefix
// of those asked for, as those that come back are of those given.  (64 bits for the positions: what is asked for is not limited by T.)
struct PlanArgs {
    const int *kv_lens, *new_lens; int B;
    int* page_table; int max_pages;
    int* ring; int ring_size /* 0: no ring, the table is complete */; const int* ring_state;
    int T;
    int *kv_out, *cu; long long* slots; int *positions, *state_out;
};
struct PlanSums { long long grown; int needed, given; };
struct PlanDone { int taken, given, refused; };      // pages, pages, requests
struct PlanRing { int head, count; };
__device__ inline PlanRing plan_ring(const PlanArgs& a)
{
    if (a.ring_size == 0) return PlanRing{0, 0};
    return PlanRing{min(max(a.ring_state[0], 0), a.ring_size - 1), min(max(a.ring_state[1], 0), a.ring_size)};
}
__device__ inline PlanItem plan_request(const PlanArgs& a, const PlanRing& r, int b, PlanSums& in, int& cu_end, int& kv_new, PlanDone& done /* LDS */,
                                        long long* red_l /* [16], LDS */, int* red_i /* [16], LDS */)
{
    const bool on = b < a.B, ring = a.ring_size > 0;
    const int old = on ? min(max(a.kv_lens[b], 0), a.max_pages * 128) : 0, want = on ? max(a.new_lens[b], 0) : 0;
    const bool bad = want > a.max_pages * 128;
    const int grow = bad ? 0 : max(want - old, 0), give = ring && !bad ? max(pages_of(old) - pages_of(want), 0) : 0;
    long long total_l;
    const long long end = in.grown + wg_scan<16>((long long)grow, red_l, total_l);
    in.grown += total_l;
    const bool late = grow > 0 && end > a.T;
    const int need = !ring || bad || late ? 0 : max(pages_of(want) - pages_of(old), 0);
    int total;
    const int upto = in.needed + wg_scan<16>(need, red_i, total);
    in.needed += total;
    const int give_end = in.given + wg_scan<16>(give, red_i, total);
    in.given += total;
    const bool ok = !bad && !late && (need == 0 || upto <= r.count) && (give == 0 || give_end <= a.ring_size - r.count);
    cu_end = (int)min(end, (long long)a.T);
    kv_new = ok ? want : old;
    if (on && need > 0 && ok) atomicMax(&done.taken, upto);
    if (on && give > 0 && ok) atomicMax(&done.given, give_end);
    if (on && !ok) atomicAdd(&done.refused, 1);
    return PlanItem{old, ok ? (ring ? (int)(((long long)r.head + upto - need) % a.ring_size) : 0) : -1, ok ? give : 0, give_end - give};
}
__device__ inline void plan_state(const PlanArgs& a, const PlanRing& r, const PlanDone& done)
{
    if (!a.state_out) return;
    a.state_out[0] = a.ring_size > 0 ? (int)(((long long)r.head + done.taken) % a.ring_size) : 0;
    a.state_out[1] = r.count - done.taken + done.given;           // (at most r.count + done.given, which the ring has places for)
    a.state_out[2] = done.refused;
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
// Slot and position of row t of the step, which is position pos of request b (b < 0: of none).  The row that begins a new page writes it into the
// table (every new page begins with one).
__device__ inline void plan_row(const PlanArgs& a, int t, int b, int pos, int old_len, int take)
{
    long long slot = -1;
    if (b >= 0 && take >= 0) {
        const int j = pos >> 7, fresh = j - pages_of(old_len);    // j < max_pages: the request fits its row
        int* entry = a.page_table + (size_t)b * a.max_pages + j;
        int page;
        if (a.ring_size > 0 && fresh >= 0) {
            page = a.ring[((long long)take + fresh) % a.ring_size];
            if ((pos & 127) == 0) *entry = page;
        } else page = *entry;
        if (page >= 0) slot = (long long)page * 128 + (pos & 127);
    }
    a.slots[t] = slot;
    a.positions[t] = b >= 0 ? pos : 0;
}
// Pages that 64 requests from b0 on give back, by a wave: its lanes over the pages of one request after another.  What is read of the ring and what is
// written to it do not meet: free pages and pages given back together are no more than the ring has places (plan_request).
__device__ inline void plan_give(const PlanArgs& a, const PlanItem& it /* of request b0 + lane */, int b0, int tail)
{
    const int lane = threadIdx.x & 63;
    for (unsigned long long m = __builtin_amdgcn_ballot_w64(it.give > 0); m != 0; m &= m - 1) {
        const int src = (int)__builtin_ctzll(m);
        const int give = __builtin_amdgcn_readlane(it.give, src), first = __builtin_amdgcn_readlane(it.first_give, src);
        const int kept = pages_of(__builtin_amdgcn_readlane(it.old_len, src)) - give;
        for (int j = lane; j < give; j += 64)
            a.ring[((long long)tail + first + j) % a.ring_size] = a.page_table[(size_t)(b0 + src) * a.max_pages + kept + j];
    }
}

// Up to 1024 requests: one launch, in which every workgroup makes out for itself who gets what and then does its share of the rows.  (Two launches, as
// below, take as long on the GPU, but the second one costs the host its 3.5 us, which is what a step waits for.)  Bound by the launch and a chain of trips
// to memory (lengths, ring, table): 24 requests 4.3 us, 700 with 39 000 rows 6.3 us.
constexpr int kPlanOne = 1024;
constexpr int kPlanOneWg = 4096;      // rows that one workgroup does alone: then nobody else reads what it writes
__global__ __launch_bounds__(1024) void plan_one_kernel(const PlanArgs a)
{
    __shared__ long long red_l[16];
    __shared__ int red_i[16], cu_s[kPlanOne + 1], old_s[kPlanOne], take_s[kPlanOne];
    __shared__ PlanDone done;
    const int tid = threadIdx.x;
    const PlanRing r = plan_ring(a);
    if (tid == 0) { done = PlanDone{0, 0, 0}; cu_s[0] = 0; }
    PlanSums in{0, 0, 0};
    int cu_end, kv_new;
    const PlanItem it = plan_request(a, r, tid, in, cu_end, kv_new, done, red_l, red_i);
    cu_s[tid + 1] = cu_end; old_s[tid] = it.old_len; take_s[tid] = it.take;
    __syncthreads();                                              // (every input but the ring and the table has been read: outputs may lie over them)
    if (blockIdx.x == 0) {
        if (tid < a.B) { a.kv_out[tid] = kv_new; a.cu[tid + 1] = cu_end; }
        if (tid == 0) { a.cu[0] = 0; plan_state(a, r, done); }
        if (a.ring_size > 0) plan_give(a, it, tid & ~63, (int)(((long long)r.head + r.count) % a.ring_size));
    }
    for (int t = (int)blockIdx.x * 1024 + tid; t < a.T; t += (int)gridDim.x * 1024) {
        int b = -1, pos = 0;
        if (t < cu_s[a.B]) { b = request_of(cu_s, a.B, t); pos = old_s[b] + (t - cu_s[b]); }
        plan_row(a, t, b, pos, b >= 0 ? old_s[b] : 0, b >= 0 ? take_s[b] : -1);
    }
}

// More requests, or outputs that lie over inputs that other workgroups would still read: one workgroup makes out who gets what, a second launch does the rows.
__global__ __launch_bounds__(1024) void plan_scan_kernel(const PlanArgs a, PlanHead* __restrict__ hd, PlanItem* __restrict__ items)
{
    __shared__ long long red_l[16];
    __shared__ int red_i[16];
    __shared__ PlanDone done;
    const int tid = threadIdx.x;
    const PlanRing r = plan_ring(a);
    if (tid == 0) { done = PlanDone{0, 0, 0}; a.cu[0] = 0; }
    PlanSums in{0, 0, 0};
    for (int b0 = 0; b0 < a.B; b0 += 1024) {
        int cu_end, kv_new;
        const PlanItem it = plan_request(a, r, b0 + tid, in, cu_end, kv_new, done, red_l, red_i);
        if (b0 + tid < a.B) { a.cu[b0 + tid + 1] = cu_end; a.kv_out[b0 + tid] = kv_new; items[b0 + tid] = it; }
    }
    __syncthreads();
    if (tid == 0) {
        hd->tail = a.ring_size > 0 ? (int)(((long long)r.head + r.count) % a.ring_size) : 0;
        plan_state(a, r, done);
    }
}
__global__ __launch_bounds__(256) void plan_fill_kernel(const PlanArgs a, int row_wgs, const PlanHead* __restrict__ hd, const PlanItem* __restrict__ items)
{
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < row_wgs) {
        const int t = (int)blockIdx.x * 256 + tid;
        if (t >= a.T) return;
        if (t >= a.cu[a.B]) { plan_row(a, t, -1, 0, 0, -1); return; }
        const int b = request_of(a.cu, a.B, t);
        const PlanItem it = items[b];
        plan_row(a, t, b, it.old_len + (t - a.cu[b]), it.old_len, it.take);
        return;
    }
    const int b0 = (((int)blockIdx.x - row_wgs) * 4 + (tid >> 6)) * 64, b = b0 + (tid & 63);
    plan_give(a, b < a.B ? items[b] : PlanItem{0, 0, 0, 0}, b0, hd->tail);
}

// A row (token, kv head) of K or V is D / 16 blocks; a thread takes a block of kAppendRows rows, which are under way at once.  Rows are taken token by
// token, all heads of a token after each other: they lie side by side in memory.  Bound by memory: 21 300 tokens, 8 heads of 128, 87 MB read, 25 MB
// written: 26.7 us, 4.2 TB/s, of rows that no cache holds, 21.3 us again on the same ones; 40 tokens 2.6 us, a launch.  (Half a block per thread, to store 1 KiB at once: the same.)
constexpr int kAppendRows = 2;
template <int D>
__global__ __launch_bounds__(256) void append_kernel(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v, size_t k_token, size_t k_head,
                                                     size_t v_token, size_t v_head, int T, int Hkv, unsigned char* __restrict__ cache, int num_pages,
                                                     const long long* __restrict__ slots)
{
    constexpr int nb = D / 16, per = 256 / nb;                    // threads to a row, rows at a time
    const int which = blockIdx.y, c = threadIdx.x % nb, r0 = (int)blockIdx.x * (per * kAppendRows) + threadIdx.x / nb, rows = T * Hkv;
    const uint16_t* src = (which ? v : k) + 16 * c;
    const size_t token = which ? v_token : k_token, head = which ? v_head : k_head;
    uint4v x[kAppendRows][2];
    long long slot[kAppendRows];
    int h[kAppendRows];
#pragma unroll
    for (int i = 0; i < kAppendRows; ++i) {
        const int r = min(r0 + i * per, rows - 1), t = r / Hkv;
        h[i] = r % Hkv;
        const uint4v* p = reinterpret_cast<const uint4v*>(src + (size_t)t * token + (size_t)h[i] * head);
        x[i][0] = p[0]; x[i][1] = p[1];
        slot[i] = slots[t];
    }
#pragma unroll
    for (int i = 0; i < kAppendRows; ++i) {
        float val[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            val[2 * j]     = __uint_as_float(x[i][j >> 2][j & 3] << 16);
            val[2 * j + 1] = __uint_as_float(x[i][j >> 2][j & 3] & 0xFFFF0000u);
        }
        const Nv16 q = phi_block16_bf16(val);
        // the scale bytes of four neighbouring blocks of a row as one dword
        uint32_t sb = q.sc & 0xFFu;
        sb |= lane_down<1>(sb) << 8;
        sb |= lane_down<2>(sb) << 16;
        if (r0 + i * per >= rows || slot[i] < 0 || slot[i] >= (long long)num_pages * 128) continue;
        unsigned char* part = cache + ((size_t)(slot[i] >> 7) * Hkv + h[i]) * nvfp4_page_head_bytes(D) + (which ? 128 * (D / 2 + nb) : 0);
        const int off = (int)(slot[i] & 127);
        uint2v c2; c2[0] = q.clo; c2[1] = q.chi;
        *reinterpret_cast<uint2v*>(part + off * (D / 2) + c * 8) = c2;
        if ((c & 3) == 0) *reinterpret_cast<uint32_t*>(part + 128 * (D / 2) + off * nb + c) = sb;
    }
}

// The same way back; a slot outside the cache reads as zeros.  (A value has at most 6 significant bits: exact in bf16.)  Bound by what it writes: a thread
// makes 8 values, so that a wave stores 1 KiB in one piece per instruction, and has kReadRows rows under way at once.  116 000 tokens, 8 heads of 128:
// 609 MB in 121.6 us, 5.0 TB/s (16 values per thread 136 us); 777 tokens 3.4 us.
constexpr int kReadRows = 4;
template <int D>
__global__ __launch_bounds__(256) void read_kernel(uint16_t* __restrict__ k, uint16_t* __restrict__ v, size_t k_token, size_t k_head, size_t v_token,
                                                   size_t v_head, int T, int Hkv, const unsigned char* __restrict__ cache, int num_pages,
                                                   const long long* __restrict__ slots)
{
    constexpr int nt = D / 8, per = 256 / nt;                     // threads to a row, rows at a time
    const int which = blockIdx.y, c = threadIdx.x % nt, r0 = (int)blockIdx.x * (per * kReadRows) + threadIdx.x / nt, rows = T * Hkv;
    long long slot[kReadRows];
    uint32_t codes[kReadRows], sc[kReadRows];
    int t[kReadRows], h[kReadRows];
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) {
        const int r = min(r0 + i * per, rows - 1);
        t[i] = r / Hkv; h[i] = r % Hkv;
        slot[i] = slots[t[i]];
    }
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) {
        const bool in = slot[i] >= 0 && slot[i] < (long long)num_pages * 128;
        const long long at = in ? slot[i] : 0;
        const unsigned char* part = cache + ((size_t)(at >> 7) * Hkv + h[i]) * nvfp4_page_head_bytes(D) + (which ? 128 * (D / 2 + D / 16) : 0);
        const int off = (int)(at & 127);
        codes[i] = *reinterpret_cast<const uint32_t*>(part + off * (D / 2) + 4 * c);
        sc[i] = part[128 * (D / 2) + off * (D / 16) + (c >> 1)];
        if (!in) { codes[i] = 0; sc[i] = 0; }
    }
    uint16_t* dst = (which ? v : k) + 8 * c;
    const size_t token = which ? v_token : k_token, head = which ? v_head : k_head;
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) {
        typedef float float2v __attribute__((ext_vector_type(2)));
        const float f = __builtin_amdgcn_cvt_scalef32_f32_fp8(sc[i], 1.0f, 0);
        uint4v w;
#define AQ_VALUES(J) { const float2v x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[i], 1.0f, J); w[J] = pack_bf16x2_cvt(x[0] * f, x[1] * f); }
        AQ_VALUES(0) AQ_VALUES(1) AQ_VALUES(2) AQ_VALUES(3)
#undef AQ_VALUES
        if (r0 + i * per < rows) *reinterpret_cast<uint4v*>(dst + (size_t)t[i] * token + (size_t)h[i] * head) = w;
    }
}

}  // namespace

size_t page_plan_ws_bytes(int B) { return sizeof(PlanHead) + (size_t)B * sizeof(PlanItem); }

int launch_page_plan(const int* kv_lens, const int* new_lens, int B, int* page_table, int max_pages, int* ring, int ring_size, const int* ring_state,
                     int T, int* kv_out, int* cu, long long* slots, int* positions, int* state_out, bool in_place, void* ws, hipStream_t st)
{
    const PlanArgs a{kv_lens, new_lens, B, page_table, max_pages, ring, ring_size, ring_state, T, kv_out, cu, slots, positions, state_out};
    const int wgs = T <= kPlanOneWg ? 1 : (T + 1023) / 1024;
    if (B <= kPlanOne && (wgs == 1 || !in_place)) {
        hipLaunchKernelGGL(plan_one_kernel, dim3(wgs < 256 ? wgs : 256), dim3(1024), 0, st, a);
        return hipGetLastError() == hipSuccess ? 0 : -1;
    }
    PlanHead* hd = (PlanHead*)ws;
    PlanItem* items = (PlanItem*)(hd + 1);
    hipLaunchKernelGGL(plan_scan_kernel, dim3(1), dim3(1024), 0, st, a, hd, items);
    if (hipGetLastError() != hipSuccess) return -1;
    const int row_wgs = (T + 255) / 256, give_wgs = ring_size > 0 ? (B + 255) / 256 : 0;
    if (row_wgs + give_wgs > 0)
        hipLaunchKernelGGL(plan_fill_kernel, dim3(row_wgs + give_wgs), dim3(256), 0, st, a, row_wgs, hd, items);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_append(const Rows& k, const Rows& v, int T, int Hkv, int D, void* cache, int num_pages, const long long* slots, hipStream_t st)
{
    const int per = 256 / (D / 16) * kAppendRows;
    const dim3 grid((T * Hkv + per - 1) / per, 2);
    if (D == 128) hipLaunchKernelGGL((append_kernel<128>), grid, dim3(256), 0, st, (const uint16_t*)k.p, (const uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (unsigned char*)cache, num_pages, slots);
    else          hipLaunchKernelGGL((append_kernel<64>), grid, dim3(256), 0, st, (const uint16_t*)k.p, (const uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (unsigned char*)cache, num_pages, slots);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_kv_read(const Rows& k, const Rows& v, int T, int Hkv, int D, const void* cache, int num_pages, const long long* slots, hipStream_t st)
{
    const int per = 256 / (D / 8) * kReadRows;
    const dim3 grid((T * Hkv + per - 1) / per, 2);
    if (D == 128) hipLaunchKernelGGL((read_kernel<128>), grid, dim3(256), 0, st, (uint16_t*)k.p, (uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (const unsigned char*)cache, num_pages, slots);
    else          hipLaunchKernelGGL((read_kernel<64>), grid, dim3(256), 0, st, (uint16_t*)k.p, (uint16_t*)v.p, k.token, k.head, v.token, v.head, T, Hkv, (const unsigned char*)cache, num_pages, slots);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace aq
