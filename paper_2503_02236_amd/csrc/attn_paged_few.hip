// Attention over the pages for requests of few rows (decode steps): tiles of 16 rows and 64 keys.
//
// As attn_paged.hip, with v_mfma_f32_16x16x32_f16: a score costs a lane what it costs there, but of 32 columns of one
// or a few rows half would be computed for nothing, and what a tile costs beside its scores (maximum, statistics, codes, branches) is paid once for 64 keys.
//   S^T, four products of 16 keys: key 16 a + 4 b + t is row 4 a + b of product t, so lane group g (of 16 lanes) ends with the scores of
//                 the 16 keys of block g, score (t, i) that of key 16 g + 4 i + t.  Group g takes channels 32 g .. 32 g + 31.
//   O^T, step s over the keys whose last two bits are 2 s and 2 s + 1: slot 8 g + 4 j + e of the operands is key 16 g + 4 e + 2 s + j, the lane's own
//                 score; lane 4 e + c of a group asks for the entries of its four keys 16 g + 4 e + (0 .. 3) -- one dword of codes -- and position block c, part f, and
//                 the transposing read hands them out by channel.
// D = 128, v = 4 or 8.  A round of 8 tiles takes 1.6 us, of twice the keys that the wider tiles take 1.3 us for.  What is left is what a tile costs whatever its
// rows: a gather and its address for every 8 bytes of entries (64 of each in 115 vector instructions), and the time until all wavefronts are done with a
// request (2 - 4 us, its sums 1 us).  16 requests of up to 4096 tokens, 32 heads: 48.2 us, where their 103 MB of codes would take 15 from HBM.
#include "attn_paged.h"

namespace vq {

using namespace paged;

namespace {

template <int V, bool COPIES, int MODS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_paged_few_kernel(PagedArgs a) {
    constexpr int D = 128, P = D / V, ES = 2 * V, ROWS = 16, KEYS = 64;
    constexpr int KW = P / 16;                   // dwords of a lane's K codes of a key: its 32 channels
    constexpr int CPS = 8 / V;                   // codes of a step of 8 channels
    constexpr int F = D / 16;                    // products of 16 channels
    constexpr int NR = F * 4 / V;                // positions of a lane's V codes
    constexpr int NB = 3;                        // tiles of codes in flight
    constexpr int KN = 4 * 4 * CPS, VN = 2 * F;  // gathers of a lane: of a tile's keys, of a step's values
    extern __shared__ __align__(16) unsigned char smem[];   // (from LDS address 0: kernel_setup checks that)
    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int nwg = gridDim.x, id = (nwg & 7) == 0 ? (int)(blockIdx.x & 7) * (nwg >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
    const int h = id / a.workers, w = id - h * a.workers;

    Tables<D, V, COPIES, false> k_books, v_books;
    const size_t books = (size_t)h * a.G * a.E * ES;
    k_books.load(a, reinterpret_cast<const unsigned char *>(a.k_cb) + books, tid);
    v_books.load(a, reinterpret_cast<const unsigned char *>(a.v_cb) + books, tid);
    Share sh;
    if (!find_share<kThreads>(a, w, reinterpret_cast<long long *>(smem + kScanOff), &sh)) return;
    k_books.store(a, smem, tid);
    v_books.store(a, smem + kSide, tid);

    const int ps_mask = (1 << a.log_ps) - 1;
    const int c0 = lane & 3, e0 = (lane >> 2) & 3;
    const unsigned copy = (unsigned)((V == 4 ? lane & 31 : lane & 15) * ES);
    const unsigned k_const = COPIES ? copy : (unsigned)(g * (P / 4) * 256 * ES);
    const unsigned v_const = (unsigned)kSide + (COPIES ? copy : (unsigned)(c0 * NR * 256 * ES));
    const uint8_t *const k_lane = a.k_codes + (4 * (col & 3) * P + g * (P / 4));     // key 16 (col / 4) + 4 (col % 4) + t
    const uint8_t *const v_lane = a.v_codes + (c0 * NR * 16 + 4 * e0);
    size_t *const bases = reinterpret_cast<size_t *>(smem + kBaseOff) + wave * 64;
    const size_t *const k_bases = bases + (col >> 2), *const v_bases = bases + g;
    float4_t *const xs = reinterpret_cast<float4_t *>(smem + kJoinOff);
    float *xm = reinterpret_cast<float *>(smem + kStatOff), *xl = xm + kWaves * 32;
    int *starts = reinterpret_cast<int *>(smem + kListOff);
    Piece *list = reinterpret_cast<Piece *>(smem + kListOff + 256);

    auto gather_address = [&](uint32_t word, int byte, unsigned lane_const) {
        if constexpr (COPIES)
            return byte == 0 ? row_address<0>(word, lane_const) : byte == 1 ? row_address<1>(word, lane_const)
                   : byte == 2 ? row_address<2>(word, lane_const) : row_address<3>(word, lane_const);
        else return ((word >> (8 * byte)) & 0xFFu) * ES + lane_const;
    };

    long long left = sh.u1 - sh.u0, x = sh.x;
    int b = sh.b;
    while (left > 0) {
        int rounds_in_list;
        __syncthreads();   // (the list before is done with)
        const int pieces = list_pieces<NB>(a, &b, &x, &left, wave == 0, starts, list, &rounds_in_list);
        __syncthreads();
        if (pieces == 0) continue;

        // Pages of 16 rounds of this wavefront at a time: lane 4 s + k finds the first byte of the codes of block k of round s.
        int next_id, next_off;
        auto page_ids = [&](int step) {
            const int t = min(step + (lane >> 2), rounds_in_list - 1);
            int p = 0;
#pragma unroll
            for (int d = 32; d; d >>= 1)
                if (p + d < pieces && starts[p + d] <= t) p += d;
            const Piece &pc = list[p];
            const int idx = max(min(((pc.r0 + t - starts[p]) << 3) + wave, pc.count - 1), 0);
            const int at = (idx < pc.front ? idx : pc.lo + idx - pc.front) * KEYS + 16 * (lane & 3);
            next_id = a.table[(size_t)pc.b * a.max_pages + (max(min(at, pc.len - 1), 0) >> a.log_ps)];
            next_off = (at & ps_mask) * P;
        };
        auto write_bases = [&]() { bases[lane] = (((size_t)min(max(next_id, 0), a.n_pages - 1) * a.H + h) << a.log_ps) * P + (size_t)next_off; };
        page_ids(0);
        write_bases();
        page_ids(16);
        size_t k_base = k_bases[0], v_base = v_bases[0];
        struct Codes {
            uint32_t k[4][KW], v[NR];
        } ring[NB];
        auto fetch = [&](int step, Codes &c) {
            const uint8_t *kp = k_lane + k_base, *vp = v_lane + v_base;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const typename Raw<4 * KW>::type u = global_read<4 * KW>(kp + t * P);
                __builtin_memcpy(c.k[t], &u, 4 * KW);
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) c.v[n] = global_read<4>(vp + 16 * n);
            if (((step + 1) & 15) == 0) {
                write_bases();
                page_ids(step + 17);
            }
            k_base = k_bases[4 * ((step + 1) & 15)];
            v_base = v_bases[4 * ((step + 1) & 15)];
        };
#pragma unroll
        for (int u = 0; u < NB; ++u) fetch(u, ring[u]);
        // K entries of a tile as operands, product t and step c of the channels: gather `at` of a lane, the steps ascending
        V16 kop[4][4];
        auto gather_k = [&](const Codes &codes, int at) {
            const int c = at / (4 * CPS), t = at / CPS % 4, n = at % CPS, code = c * CPS + n;
            lds_read<ES>(gather_address(codes.k[t][code / 4], code & 3, k_const) + (unsigned)(COPIES ? 0 : code * 256 * ES), &kop[t][c].w[n * (ES / 4)]);
        };

        int step = 0;
        for (int piece = 0; piece < pieces; ++piece) {
            const Piece pc = uniform_piece(list[piece]);
            const int rows = min(pc.rows - pc.row0, ROWS);
            const bool valid = col < rows;
            const int row = pc.row0 + min(col, rows - 1), i = token_of(a, row), hq = h * a.group + (row - i * a.group);
            const int pos = pc.pos0 + i;
            half8_t qf[4];
            {
                const half_t *qp = a.q + (size_t)(pc.first + i) * a.q_stride + (size_t)hq * D + g * 32;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    V16 u = ld16(qp + 8 * c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u.w[e] ^= a.q_sign;
                    qf[c] = u.h8;
                }
            }
            float4_t o[F];
#pragma unroll
            for (int f = 0; f < F; ++f) o[f] = float4_t{0.f, 0.f, 0.f, 0.f};
            float m_ref = -FLT_MAX, lsum = 0.f;
            bool far = false;   // a reference of the wavefront is
            // this wavefront's tiles: idx0, idx0 + 8, ...
            const int pos_f = pc.pos0 + token_of(a, pc.row0), pos_l = pc.pos0 + token_of(a, pc.row0 + rows - 1);
            const int idx0 = (pc.r0 << 3) + wave, rounds = pc.r1 - pc.r0;
            const int tiles = min(max((pc.count - idx0 + 7) >> 3, 0), rounds);
            int all_from = a.window > 0 ? max(pos_l - a.window + 1, 0) : 0;   // first keys of tiles that all rows attend whole: from here on,
            const int all_to = min(pos_f, pc.len - 1) - (KEYS - 1);           // up to here
            const unsigned all_span = (unsigned)max(all_to - all_from, 0);
            if (all_to < all_from) all_from = -1;   // (none)
            const float slope2 = MODS && a.slopes ? a.slopes[hq] * kLog2e : 0.f;
            const int see_to = min(pos, pc.len - 1), see_from = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
            float4_t s[4], next[4];   // scores (t, i) of a tile, of the next one
            float scale2 = a.scale2;
            asm("" : "+v"(scale2));   // (a product and sum with a scalar operand takes twice as long)
            if (tiles > 0) {
#pragma unroll
                for (int n = 0; n < KN; ++n) gather_k(ring[0], n);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    s[t] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < 4; ++c) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kop[t][c].h8, qf[c], s[t], 0, 0, 0);
                }
#pragma unroll
                for (int n = 0; n < KN / 2; ++n) gather_k(ring[1], n);
            }
            auto body = [&](int tile, Codes &codes, const Codes &after, const Codes &second) {
                const int idx = idx0 + (tile << 3), t0 = (idx < pc.front ? idx : pc.lo + idx - pc.front) * KEYS;
                if constexpr (MODS) {
                    if constexpr (MODS == kLargelyCapped) {
                        if (__builtin_expect((unsigned)(t0 - all_from) > all_span, 0)) {
                            const int see = attended_keys(t0 + 16 * g, see_from, see_to, pc.prefix);
#pragma unroll
                            for (int e = 0; e < 16; ++e) s[e / 4][e % 4] = attended_or_zero(s[e / 4][e % 4], see, 4 * (e % 4) + e / 4);
                        }
                        cap_scores(a, scale2, [&](int e) { return s[e / 4][e % 4]; }, [&](int e, float x) { s[e / 4][e % 4] = x; });
                    } else if (a.cap_in > 0.f) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            s[e / 4][e % 4] = a.cap_out - 2.f * a.cap_out * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[e / 4][e % 4] * a.cap_in) + 1.f);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[e / 4][e % 4] *= scale2;
                    }
                    if (a.slopes) {
                        const float back = (float)(pos - t0 - 16 * g);
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[e / 4][e % 4] -= slope2 * fabsf(back - (float)(4 * (e % 4) + e / 4));
                    }
                }
                if (__builtin_expect((unsigned)(t0 - all_from) > all_span, 0)) {
                    const int see = attended_keys(t0 + 16 * g, see_from, see_to, pc.prefix);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e / 4][e % 4] = attended(s[e / 4][e % 4], see, 4 * (e % 4) + e / 4);
                    // Codes behind the request's end may name anything, and a weight of zero times an infinity is none: they become the
                    // tile's first token's.
                    if (t0 + KEYS > pc.len) {
                        const int live = min(max(pc.len - (t0 + 16 * g + 4 * e0), 0), 4);   // bytes that stay
                        const uint32_t mask = live == 4 ? 0xFFFFFFFFu : (1u << (8 * live)) - 1u;
#pragma unroll
                        for (int n = 0; n < NR; ++n) {
                            const uint32_t good = (__shfl((int)codes.v[n], lane & 3, 64) & 0xFF) * 0x01010101u;
                            codes.v[n] = (codes.v[n] & mask) | (good & ~mask);
                        }
                    }
                }
                // running maximum (a NaN raises nothing: its row's weights are NaN by themselves)
                float mt = s[0][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mt = __builtin_elementwise_maximum(mt, s[e / 4][e % 4]);
                {
                    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
                    mt = __builtin_elementwise_maximum(__uint_as_float(y[0]), __uint_as_float(y[1]));
                    const auto z = __builtin_amdgcn_permlane16_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
                    mt = __builtin_elementwise_maximum(__uint_as_float(z[0]), __uint_as_float(z[1]));
                }
                if (!MODS) mt *= scale2;
                if (__builtin_expect(__ballot(mt - m_ref > kRise) != 0, 0)) {
                    const float m_new = mt - m_ref > kRise ? mt : m_ref, f = __builtin_amdgcn_exp2f(m_ref - m_new);
                    m_ref = m_new;
                    if (!MODS) far = __ballot(is_far(m_ref)) != 0;
                    lsum *= f;
#pragma unroll
                    for (int k = 0; k < F; ++k) o[k] *= f;
                }
                float sub = kHeadroom - m_ref;
                if (__builtin_expect(!MODS && far, 0)) {
                    const bool mine = is_far(m_ref);
                    const float back = __builtin_amdgcn_rcpf(scale2);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x = s[e / 4][e % 4] * scale2;
                        asm("" : "+v"(x));   // (rounded, as the maximum is)
                        s[e / 4][e % 4] = mine ? (x - m_ref) * back : s[e / 4][e % 4];
                    }
                    sub = mine ? kHeadroom : sub;
                }
                V16 vop[2][F];
                auto gather_v = [&](int k, int at) {   // step k, part f of the position block, half j of the four keys
                    const int f = at / 2, j = at % 2, n = f * 4 / V;
                    lds_read_transposed(gather_address(codes.v[n], 2 * k + j, v_const) + (unsigned)((COPIES ? 0 : n * 256 * ES) + (f * 4 % V) * 2), &vop[k][f].w[2 * j]);
                };
                // Four matrix instructions at a time with the vector instructions beside them, gathers ahead of their use (attn_paged.hip)
                __builtin_amdgcn_sched_barrier(0);
                V16 pf[2];
#pragma unroll
                for (int t = 0; t < 4; ++t) next[t] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 4; ++c) {   // scores of the next tile; weights of this one
#pragma unroll
                    for (int t = 0; t < 4; ++t) next[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kop[t][c].h8, qf[c], next[t], 0, 0, 0);
                    if (c == 0) {
#pragma unroll
                        for (int n = 0; n < KN / 2; ++n) gather_k(after, KN / 2 + n);
                    } else if (c < 3) {
#pragma unroll
                        for (int n = 0; n < VN / 2; ++n) gather_v(0, (c - 1) * (VN / 2) + n);
                    } else {
#pragma unroll
                        for (int n = 0; n < VN / 2; ++n) gather_v(1, n);
                    }
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {   // product c's scores: half c % 2 of step c / 2
                        const float p0 = __builtin_amdgcn_exp2f(MODS ? s[c][e] + sub : __builtin_fmaf(s[c][e], scale2, sub));
                        const float p1 = __builtin_amdgcn_exp2f(MODS ? s[c][e + 1] + sub : __builtin_fmaf(s[c][e + 1], scale2, sub));
                        const half2_t p2 = {(half_t)p0, (half_t)p1}, one = {(half_t)1.f, (half_t)1.f};
                        pf[c / 2].h2[2 * (c % 2) + e / 2] = p2;
                        lsum = dot2(p2, one, lsum);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) {   // O^T += V^T P^T
#pragma unroll
                    for (int n = 0; n < F / 2; ++n) {
                        const int k = m / 2, f = m % 2 * (F / 2) + n;
                        o[f] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vop[k][f].h8, pf[k].h8, o[f], 0, 0, 0);
                    }
                    if (m == 0) {
#pragma unroll
                        for (int n = 0; n < VN / 2; ++n) gather_v(1, VN / 2 + n);
                    } else if (m < 3) {
#pragma unroll
                        for (int n = 0; n < KN / 4; ++n) gather_k(second, (m - 1) * (KN / 4) + n);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) s[t] = next[t];
            };
            for (int tile = 0; tile < rounds; tile += NB)
#pragma unroll
                for (int u = 0; u < NB; ++u, ++step) {
                    if (__builtin_expect(tile + u < tiles, 1)) body(tile + u, ring[u], ring[(u + 1) % NB], ring[(u + 2) % NB]);
                    fetch(step + NB, ring[u]);
                }
            lsum += __shfl_xor(lsum, 16, 64);
            lsum += __shfl_xor(lsum, 32, 64);

            // join the eight wavefronts, in order; four channels of a lane, f, end with wavefront f
            if (g == 0) {
                xm[wave * ROWS + col] = m_ref;
                xl[wave * ROWS + col] = lsum;
            }
            __syncthreads();
            float M = m_ref, L = 0.f, ms[kWaves], ls[kWaves];
#pragma unroll
            for (int k = 0; k < kWaves; ++k) {
                ms[k] = xm[k * ROWS + col];
                ls[k] = xl[k * ROWS + col];
            }
#pragma unroll
            for (int k = 0; k < kWaves; ++k) M = fmaxf(M, ms[k]);
#pragma unroll
            for (int k = 0; k < kWaves; ++k) L += ls[k] * __builtin_amdgcn_exp2f(ms[k] - M);
            {
                const float f = __builtin_amdgcn_exp2f(m_ref - M);
#pragma unroll
                for (int k = 0; k < F; ++k) o[k] *= f;
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const size_t part = part_of(a, h, w, pc.r0 > 0 ? 0 : 1);
            if (!pc.whole && valid && g == 0 && wave == 0) {
                float *st = part_stats<D>(a, part) + col * 2;
                st[0] = M;
                st[1] = L;
            }
            // AT: parts f that the buffer holds at once, of the rows' lanes alone (32 / AT rows at most)
            auto join = [&](auto at_once) {
                constexpr int AT = decltype(at_once)::value, RJ = 32 / AT;
                const int slot = g * RJ + (col & (RJ - 1));   // of 4 RJ
                const bool mine = col < RJ;
                auto cell = [&](int w_, int f) { return xs + (w_ * AT + f % AT) * 4 * RJ + slot; };
#pragma unroll
                for (int f0 = 0; f0 < F; f0 += AT) {
#pragma unroll
                    for (int f = f0; f < f0 + AT; ++f)
                        if (mine) *cell(wave, f) = o[f];
                    __syncthreads();
                    if (mine && wave >= f0 && wave < f0 + AT) {
                        float4_t y[kWaves], t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < kWaves; ++k) y[k] = *cell(k, wave);
#pragma unroll
                        for (int k = 0; k < kWaves; ++k) t += y[k];
                        if (valid) {
                            const int ch = 32 * g + 4 * wave;
                            if (pc.whole) {
                                V8 z;
#pragma unroll
                                for (int e = 0; e < 4; ++e) z.h4[e] = (half_t)(t[e] * inv);
                                *reinterpret_cast<uint2 *>(a.out + (size_t)(pc.first + i) * a.out_stride + (size_t)hq * D + ch) = z.u;
                            } else {
                                *reinterpret_cast<float4_t *>(part_sums<D>(a, part) + (size_t)col * D + ch) = t;
                            }
                        }
                    }
                    __syncthreads();   // (the buffer is the next parts', or the next piece's)
                }
            };
            if (rows <= 4) join(std::integral_constant<int, 8>());
            else join(std::integral_constant<int, 2>());
        }
    }
}

template <int V, bool COPIES, int MODS>
int run_few(const PagedArgs &a, hipStream_t s) {
    static KernelSetup setup;
    if (int st = kernel_setup(reinterpret_cast<const void *>(&attn_paged_few_kernel<V, COPIES, MODS>), kLds, true, setup)) return st;
    attn_paged_few_kernel<V, COPIES, MODS><<<a.H * a.workers, kThreads, kLds, s>>>(a);
    return merge<128>(a, s);
}
template <int V, bool COPIES>
int run_few_with(const PagedArgs &a, hipStream_t s) {
    if (a.mods == kPlain) return run_few<V, COPIES, kPlain>(a, s);
    return a.mods == kModified ? run_few<V, COPIES, kModified>(a, s) : run_few<V, COPIES, kLargelyCapped>(a, s);
}
template <int V>
int run_few_as(const PagedArgs &a, hipStream_t s) { return a.G == 1 ? run_few_with<V, true>(a, s) : run_few_with<V, false>(a, s); }

}  // namespace

namespace paged {

bool few_supported(int D, int V) { return D == 128 && V >= 4; }

int launch_few(const PagedArgs &a, int V, hipStream_t s) { return V == 8 ? run_few_as<8>(a, s) : run_few_as<4>(a, s); }

}  // namespace paged

}  // namespace vq
