// Attention of the new tokens of a batch of requests over a paged cache of VQ codes (vq_attn_paged).
#include <cfloat>

#include "vq_common.h"

namespace vq {

namespace {



struct PagedArgs {
    const uint8_t *k_codes, *v_codes;
    const half_t *k_cb, *v_cb;
    const int *table, *cu_new, *seq_lens, *prefix_lens;
    const float *slopes;
    const half_t *q;
    half_t *out;
    size_t q_stride, out_stride;
    int B, H, group, E, G, n_pages, max_pages, log_ps, n_tokens, window;
    float scale, softcap;
};

// A wavefront per new token and query head; a lane per channel pair, keys one after the other.
template <int D>
__global__ __launch_bounds__(64) void attn_paged_row_kernel(PagedArgs a, int V) {
    const int lane = threadIdx.x, row = blockIdx.x, hq = blockIdx.y, h = hq / a.group;
    if (row >= min(a.cu_new[a.B], a.n_tokens)) return;
    int lo = 0, hi = a.B - 1;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (a.cu_new[mid + 1] > row) hi = mid;
        else lo = mid + 1;
    }
    const int b = lo, ps = 1 << a.log_ps, P = D / V, PG = P / a.G;
    const int len = a.n_pages > 0 ? min(max(a.seq_lens[b], 0), a.max_pages << a.log_ps) : 0;
    const int pos = len - (a.cu_new[b + 1] - row);
    const int prefix = a.prefix_lens ? a.prefix_lens[b] : 0;
    constexpr int C = D / 64;
    float q[C], o[C], m = -FLT_MAX, l = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        q[c] = (float)a.q[(size_t)row * a.q_stride + (size_t)hq * D + lane * C + c];
        o[c] = 0.f;
    }
    for (int t = 0; t < len; ++t) {
        if (!((t <= pos && (a.window == 0 || t > pos - a.window)) || t < prefix)) continue;
        const int page = min(max(a.table[(size_t)b * a.max_pages + (t >> a.log_ps)], 0), a.n_pages - 1), off = t & (ps - 1);
        const size_t base = ((size_t)page * a.H + h) * ps * P;
        float k[C], v[C], s = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int ch = lane * C + c, p = ch / V, i = ch % V, g = p / PG;
            const int kc = min((int)a.k_codes[base + (size_t)off * P + p], a.E - 1);
            const int vc = min((int)a.v_codes[base + (size_t)(off / 16) * P * 16 + p * 16 + off % 16], a.E - 1);
            k[c] = (float)a.k_cb[(((size_t)h * a.G + g) * a.E + kc) * V + i];
            v[c] = (float)a.v_cb[(((size_t)h * a.G + g) * a.E + vc) * V + i];
            s += q[c] * k[c];
        }
        s = wave_sum(s) * a.scale;
        if (a.softcap > 0.f) s = a.softcap * tanhf(s / a.softcap);
        if (a.slopes) s -= a.slopes[hq] * fabsf((float)(pos - t));
        const float m_new = fmaxf(m, s), f = expf(m - m_new), p = expf(s - m_new);
        m = m_new;
        l = l * f + p;
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] = o[c] * f + p * v[c];
    }
#pragma unroll
    for (int c = 0; c < C; ++c) a.out[(size_t)row * a.out_stride + (size_t)hq * D + lane * C + c] = (half_t)(l == 0.f ? 0.f : o[c] / l);
}

}  // namespace

bool attn_paged_supported(const vq_kv_pages_t *kv) {
    const int PG = kv->D / kv->v / kv->cb_groups;
    return (kv->D == 64 || kv->D == 128) && (PG & (PG - 1)) == 0;
}

size_t attn_paged_workspace(const vq_kv_pages_t *, const vq_paged_batch_t *) { return 0; }

int launch_attn_paged(const vq_kv_pages_t *kv, const vq_paged_batch_t *b, const void *q, size_t q_stride, float sm_scale, void *out,
                      size_t out_stride, void *, hipStream_t s) {
    PagedArgs a;
    a.k_codes = (const uint8_t *)kv->k_codes;
    a.v_codes = (const uint8_t *)kv->v_codes;
    a.k_cb = (const half_t *)kv->k_codebooks;
    a.v_cb = (const half_t *)kv->v_codebooks;
    a.table = b->block_table;
    a.cu_new = b->cu_new;
    a.seq_lens = b->seq_lens;
    a.prefix_lens = b->prefix_lens;
    a.slopes = b->slopes;
    a.q = (const half_t *)q;
    a.out = (half_t *)out;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.B = b->B;
    a.H = kv->H;
    a.group = b->Hq / kv->H;
    a.E = kv->n_entries;
    a.G = kv->cb_groups;
    a.n_pages = kv->n_pages;
    a.max_pages = b->max_pages;
    a.log_ps = __builtin_ctz(kv->page_tokens);
    a.n_tokens = b->n_tokens;
    a.window = b->window;
    a.scale = sm_scale;
    a.softcap = b->softcap;
    const dim3 grid(b->n_tokens, b->Hq);
    if (kv->D == 64) attn_paged_row_kernel<64><<<grid, 64, 0, s>>>(a, kv->v);
    else attn_paged_row_kernel<128><<<grid, 64, 0, s>>>(a, kv->v);
    return launch_status();
}

}  // namespace vq
