// Pages of a step of continuous batching, built on the GPU: block tables, slot maps and positions from the lengths that requests
// have and get (vq_kv_pages_assign).  Integer work of a few kilobytes: bound by the latency of a launch and of the
// dependent trips to memory in it (lengths, free pages, table, slots), so one workgroup does all of it: a lane per request, one scan where
// everyone is served, pages and tokens dealt out to all lanes by a search in the scan's sums.  Slots of many tokens are a second
// launch, over the chip.  A step of 16 requests takes 4.9 us, of 256 with eight chunks of 1000 tokens and eight that ended 9.4 and 1.9;
// 16 thousand page ids (64 prompts of 1024 tokens, 100 long requests that ended) 20.8 and 4.2: 1.3 ns an id, by one workgroup's memory requests.
#include "vq_common.h"

namespace vq {

namespace {

constexpr int kAssignThreads = 1024, kAssignWaves = kAssignThreads / kWave;
constexpr int kEndsInLds = 4096;      // requests whose ends a workgroup keeps in LDS
constexpr int kSlotThreads = 256;
// Tokens that the one workgroup takes along: two a lane.  Alone and with the second launch, us (graph replay): 16 tokens 5.7 and 6.8, 1000 7.0 and 8.6,
// 2000 7.6 and 8.8, 4000 9.3 and 8.9, 8000 12.3 and 9.0, 64000 62 and 12.
constexpr int kFewTokens = 2 * kAssignThreads;

struct AssignArgs {
    vq_page_step_t p;
    int log_ps;
};

// Inclusive sum over the workgroup's threads and the sum of all of them (xs: kAssignWaves values of LDS).
__device__ __forceinline__ unsigned long long scan(unsigned long long x, unsigned long long *xs, unsigned long long *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned long long y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
    }
    __syncthreads();   // (xs may still be read from the last scan)
    if (lane == 63) xs[wave] = x;
    __syncthreads();
    unsigned long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kAssignWaves; ++w) {
        if (w < wave) before += xs[w];
        all += xs[w];
    }
    *total = all;
    return before + x;
}

__device__ __forceinline__ long long pages_of(long long tokens, int log_ps) { return (tokens + (1ll << log_ps) - 1) >> log_ps; }

// The first of n ascending ends that lies behind t.
__device__ __forceinline__ int owner_of(const int *ends, int n, int t) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > t) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Things 0 .. n - 1 of a chunk of requests, number j of request l where upto (the requests' sums) says so, dealt out to the lanes, a
// wavefront a run of them: load(l, j) and then store(i, l, j, what was loaded), eight of a lane's at once (no load here reads what a store
// writes).  A lane looks for the owner of its first thing and for another one where the run leaves that: the ten dependent reads of LDS of a
// search take longer than a trip to L2.
template <typename Load, typename Store>
__device__ __forceinline__ void deal(int n, const int *upto, Load load, Store store) {
    const int per = (n + kAssignThreads - 1) / kAssignThreads, from = (int)(threadIdx.x >> 6) * 64 * per;
    const int end = min(from + 64 * per, n);
    int i = from + (int)(threadIdx.x & 63);
    if (i >= end) return;
    int at = owner_of(upto, kAssignThreads, i);
    for (; i < end; i += 8 * 64) {
        int l[8], j[8], x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + 64 * k < end) {
                if (upto[at] <= i + 64 * k) at += 1 + owner_of(upto + at + 1, kAssignThreads - at - 1, i + 64 * k);
                l[k] = at;
                j[k] = i + 64 * k - (at ? upto[at - 1] : 0);
                x[k] = load(at, j[k]);
            }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i + 64 * k < end) store(i + 64 * k, l[k], j[k], x[k]);
    }
}

// Slot and position of new token t of `tokens`; ends: cu_new + 1.
__device__ __forceinline__ void write_slot(const AssignArgs &a, const int *ends, int tokens, int t) {
    const vq_page_step_t &p = a.p;
    int slot = -1, pos = -1;
    if (t < tokens) {
        const int b = owner_of(ends, p.B, t);
        pos = p.seq_lens[b] - (ends[b] - t);
        const int page = p.block_table[(size_t)b * p.max_pages + (pos >> a.log_ps)];
        if ((unsigned)page < (unsigned)p.n_pages) slot = (page << a.log_ps) + (pos & ((1 << a.log_ps) - 1));
    }
    p.slots[t] = slot;
    if (p.positions) p.positions[t] = pos;
}

__global__ __launch_bounds__(kAssignThreads) void kv_pages_assign_kernel(AssignArgs a) {
    __shared__ unsigned long long xs[kAssignWaves];
    __shared__ int upto[kAssignThreads], base[kAssignThreads], ends[kEndsInLds];
    const vq_page_step_t &p = a.p;
    const int tid = threadIdx.x;
    const long long row = (long long)p.max_pages << a.log_ps;   // tokens of a row of the table
    const int n_free = min(max(p.n_free[0], 0), p.n_pages);
    auto len_of = [&](int b) { return (long long)min((long long)max(p.lens[b], 0), row); };
    unsigned long long total;
    // 1. pages of the requests that have ended (where any has)
    long long freed = 0;
    for (int b0 = 0; b0 < p.B; b0 += kAssignThreads) {
        const int b = b0 + tid;
        const bool gone = b < p.B && p.new_lens[b] < 0;
        if (!__syncthreads_or(gone)) continue;
        const int count = gone ? (int)pages_of(len_of(b), a.log_ps) : 0;
        upto[tid] = (int)scan(count, xs, &total);
        __syncthreads();
        deal((int)total, upto, [&](int l, int j) { return p.block_table[(size_t)(b0 + l) * p.max_pages + j]; },
             [&](int i, int, int, int page) {
                 if (n_free + freed + i < p.n_pages) p.free_pages[n_free + freed + i] = page;
             });
        freed += total;
        __syncthreads();
    }
    const long long pool = min(n_free + freed, (long long)p.n_pages);
    __syncthreads();
    // 2. new tokens
    unsigned long long asked = 0, needed = 0, served = 0, tokens = 0;   // tokens asked for and pages needed so far, pages and tokens given so far
    for (int b0 = 0; b0 < p.B; b0 += kAssignThreads) {
        const int b = b0 + tid;
        const bool live = b < p.B;
        const int n = live ? p.new_lens[b] : 0;
        const long long len = live && n >= 0 ? len_of(b) : 0, have = pages_of(len, a.log_ps);
        const bool room = n <= 0 || len + n <= row;
        const unsigned long long ask = room && n > 0 ? n : 0, want = ask ? pages_of(len + n, a.log_ps) - have : 0;
        // Both sums in one: 1024 requests ask for less than 2^41 tokens and want fewer pages than are in the table, 2^31; the tokens are counted
        // up to 2^21 each, more than a step takes.
        const unsigned long long both = scan((want << 32) | min(ask, 1ull << 21), xs, &total);
        unsigned long long ask_to = asked + (both & 0xFFFFFFFFull), want_to = needed + (both >> 32);
        bool fits = room;
        unsigned long long give = ask, need = want, give_to = ask_to - asked, need_to = want_to - needed;
        if (asked + (total & 0xFFFFFFFFull) <= (unsigned long long)p.n_tokens && needed + (total >> 32) <= (unsigned long long)pool) {   // everyone is served
            asked += total & 0xFFFFFFFFull;
            needed += total >> 32;
        } else {
            unsigned long long t;
            fits = fits && (ask == 0 || ask_to <= (unsigned long long)p.n_tokens);
            asked += total & 0xFFFFFFFFull;
            need = fits ? want : 0;
            want_to = needed + scan(need, xs, &t);
            needed += t;
            fits = fits && (need == 0 || want_to <= (unsigned long long)pool);
            need = fits ? need : 0;
            give = fits ? ask : 0;
            const unsigned long long given = scan((need << 32) | give, xs, &total);
            give_to = given & 0xFFFFFFFFull;
            need_to = given >> 32;
        }
        if (live) {
            const int end = (int)(tokens + give_to);
            p.status[b] = fits ? 0 : 1;
            p.seq_lens[b] = (int)(len + give);
            p.cu_new[b + 1] = end;
            if (b < kEndsInLds) ends[b] = end;
        }
        // (requests are served in order: what those before this chunk got is what they needed, up to the first that was refused for want of pages, behind
        // whom nobody gets any)
        upto[tid] = (int)need_to;
        base[tid] = (int)have;
        __syncthreads();
        const int pages = (int)(total >> 32);
        deal(pages, upto, [&](int l, int j) { return p.free_pages[pool - 1 - (long long)served - ((l ? upto[l - 1] : 0) + j)]; },
             [&](int, int l, int j, int page) { p.block_table[(size_t)(b0 + l) * p.max_pages + base[l] + j] = page; });
        served += pages;
        tokens += total & 0xFFFFFFFFull;
        __syncthreads();
    }
    if (tid == 0) {
        p.cu_new[0] = 0;
        p.n_free_out[0] = (int)(pool - (long long)served);
    }
    // 3. slots and positions
    if (p.n_tokens > kFewTokens) return;
    const int *e = p.B <= kEndsInLds ? ends : p.cu_new + 1;
    for (int t = tid; t < p.n_tokens; t += kAssignThreads) write_slot(a, e, (int)tokens, t);
}

__global__ __launch_bounds__(kSlotThreads) void kv_pages_slots_kernel(AssignArgs a) {
    __shared__ int ends[kEndsInLds];
    const vq_page_step_t &p = a.p;
    const int tokens = p.cu_new[p.B];
    const int *e = p.cu_new + 1;
    if (p.B <= kEndsInLds) {
        for (int b = threadIdx.x; b < p.B; b += kSlotThreads) ends[b] = e[b];
        __syncthreads();
        e = ends;
    }
    const int t = blockIdx.x * kSlotThreads + threadIdx.x;
    if (t < p.n_tokens) write_slot(a, e, tokens, t);
}

}  // namespace

int launch_kv_pages_assign(const vq_page_step_t *step, hipStream_t s) {
    AssignArgs a;
    a.p = *step;
    a.log_ps = __builtin_ctz(step->page_tokens);
    kv_pages_assign_kernel<<<1, kAssignThreads, 0, s>>>(a);
    if (step->n_tokens > kFewTokens) kv_pages_slots_kernel<<<(step->n_tokens + kSlotThreads - 1) / kSlotThreads, kSlotThreads, 0, s>>>(a);
    return launch_status();
}

}  // namespace vq
