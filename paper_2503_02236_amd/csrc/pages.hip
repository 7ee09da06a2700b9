// Pages of a step of continuous batching, built on the GPU: block tables, slot maps and positions from the lengths that requests
// have and get (vq_kv_pages_assign).  Integer work of a few kilobytes: bound by the latency of a launch and of the
// dependent trips to memory in it, so one workgroup does all of it, with one lane per request and three scans.
#include "vq_common.h"

namespace vq {

namespace {

constexpr int kAssignThreads = 1024, kAssignWaves = kAssignThreads / kWave;

struct AssignArgs {
    vq_page_step_t p;
    int log_ps;
};

// Inclusive sum over the workgroup's threads and the sum of all of them (xs: kAssignWaves values of LDS).
__device__ __forceinline__ long long scan(long long x, long long *xs, long long *total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long y = __shfl_up(x, d, 64);
        if (lane >= d) x += y;
    }
    __syncthreads();   // (xs may still be read from the last scan)
    if (lane == 63) xs[wave] = x;
    __syncthreads();
    long long before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kAssignWaves; ++w) {
        if (w < wave) before += xs[w];
        all += xs[w];
    }
    *total = all;
    return before + x;
}

__device__ __forceinline__ long long pages_of(long long tokens, int log_ps) { return (tokens + (1ll << log_ps) - 1) >> log_ps; }

__global__ __launch_bounds__(kAssignThreads) void kv_pages_assign_kernel(AssignArgs a) {
    __shared__ long long xs[kAssignWaves];
    const vq_page_step_t &p = a.p;
    const int tid = threadIdx.x, lane = tid & 63;
    const long long row = (long long)p.max_pages << a.log_ps;   // tokens of a row of the table
    const int n_free = min(max(p.n_free[0], 0), p.n_pages);
    auto len_of = [&](int b) { return (long long)min((long long)max(p.lens[b], 0), row); };
    // 1. pages of the requests that have ended
    long long freed = 0, total;
    for (int b0 = 0; b0 < p.B; b0 += kAssignThreads) {
        const int b = b0 + tid;
        const bool gone = b < p.B && p.new_lens[b] < 0;
        const int count = gone ? (int)pages_of(len_of(b), a.log_ps) : 0;
        const long long at = n_free + freed + scan(count, xs, &total) - count;
        for (unsigned long long left = __ballot(count > 0); left; left &= left - 1) {   // a wavefront copies one request's pages at a time
            const int l = __ffsll((long long)left) - 1, c = __shfl(count, l, 64);
            const long long to = __shfl(at, l, 64);
            const int *from = p.block_table + (size_t)__shfl(b, l, 64) * p.max_pages;
            for (int j = lane; j < c; j += 64)
                if (to + j < p.n_pages) p.free_pages[to + j] = from[j];
        }
        freed += total;
    }
    const long long pool = min(n_free + freed, (long long)p.n_pages);
    __syncthreads();
    // 2. new tokens
    long long asked = 0, needed = 0, served = 0, tokens = 0;   // asked and needed so far, pages and tokens given so far
    for (int b0 = 0; b0 < p.B; b0 += kAssignThreads) {
        const int b = b0 + tid;
        const bool live = b < p.B;
        const int n = live ? p.new_lens[b] : 0;
        const long long len = live && n >= 0 ? len_of(b) : 0;
        bool fits = n <= 0 || len + n <= row;
        const long long ask = fits && n > 0 ? n : 0;
        const long long ask_to = asked + scan(ask, xs, &total);
        asked += total;
        fits = fits && (ask == 0 || ask_to <= p.n_tokens);
        const long long have = pages_of(len, a.log_ps), want = fits && n > 0 ? pages_of(len + n, a.log_ps) - have : 0;
        const long long want_to = needed + scan(want, xs, &total);
        needed += total;
        fits = fits && (want == 0 || want_to <= pool);
        const int need = fits ? (int)want : 0, give = fits && n > 0 ? n : 0;
        const long long give_to = tokens + scan(give, xs, &total);
        tokens += total;
        scan(need, xs, &total);
        served += total;
        if (live) {
            p.status[b] = fits ? 0 : 1;
            p.seq_lens[b] = (int)(len + give);
            p.cu_new[b + 1] = (int)give_to;
        }
        // (requests are served in order, so those served before b needed want_to - want pages)
        const long long first = pool - 1 - (want_to - want);
        for (unsigned long long left = __ballot(need > 0); left; left &= left - 1) {
            const int l = __ffsll((long long)left) - 1, c = __shfl(need, l, 64);
            const long long from = __shfl(first, l, 64);
            int *to = p.block_table + (size_t)__shfl(b, l, 64) * p.max_pages + __shfl((int)have, l, 64);
            for (int j = lane; j < c; j += 64) to[j] = p.free_pages[from - j];
        }
    }
    if (tid == 0) {
        p.cu_new[0] = 0;
        p.n_free_out[0] = (int)(pool - served);
    }
    __syncthreads();
    // 3. slots and positions
    for (int t = tid; t < p.n_tokens; t += kAssignThreads) {
        int slot = -1, pos = -1;
        if (t < tokens) {
            int lo = 0, hi = p.B - 1;   // the request: the first whose end lies behind t
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (p.cu_new[mid + 1] > t) hi = mid;
                else lo = mid + 1;
            }
            pos = p.seq_lens[lo] - (p.cu_new[lo + 1] - t);
            const int page = p.block_table[(size_t)lo * p.max_pages + (pos >> a.log_ps)];
            if ((unsigned)page < (unsigned)p.n_pages) slot = (page << a.log_ps) + (pos & ((1 << a.log_ps) - 1));
        }
        p.slots[t] = slot;
        if (p.positions) p.positions[t] = pos;
    }
}

}  // namespace

int launch_kv_pages_assign(const vq_page_step_t *step, hipStream_t s) {
    AssignArgs a;
    a.p = *step;
    a.log_ps = __builtin_ctz(step->page_tokens);
    kv_pages_assign_kernel<<<1, kAssignThreads, 0, s>>>(a);
    return launch_status();
}

}  // namespace vq
