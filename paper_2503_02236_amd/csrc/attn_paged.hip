// Attention of the new tokens of a batch of requests over a paged cache of VQ codes (vq_attn_paged).
//
// Mathematics.  For a cache head h the rows are (new token, query head of the group).  A wavefront takes 32 rows and walks over
// tiles of 32 cached tokens with the running maximum m, sum l and accumulators of a softmax:
//   S^T = K Q^T   v_mfma_f32_32x32x16_f16, operand A = K: lane (key, half) takes 8 channels of its key, gathered by code from the
//                 codebook in LDS straight into the operand.  Which key a row of the operand is, and which channel a step, is free: row
//                 8 a + 4 b + c is key 16 b + 4 c + a, and half l takes the channels of its half of the head, so that a lane's codes are
//                 consecutive bytes, and its 16 scores are those of the 16 consecutive keys of block l, score e that of key 4 (e % 4) + e / 4;
//   O^T = V^T P^T with P^T as operand B: exactly those scores, after exp2, as halves: no shuffle, no LDS.  Operand A = V^T: for v = 4 and 8 a
//                 lane asks for the entries of four consecutive tokens (a dword of codes: the layout of the value pages) at its positions, and
//                 the transposing LDS read hands them out by channel; for v = 2 a lane reads its channels' pairs for the block's
//                 tokens and permutes them into operands.
// A weight is 2^(s - m + 6) rounded to a half (relative error 2^-11, what the matrix instruction takes; the sum l adds the rounded ones, so
// that weights add up to one): m follows the row's own maximum, and only when that has grown by more than 6, so weights lie below 2^12 and those
// that fall below a half's range are below 2^-31 of the largest.  Sums, statistics and outputs before the last rounding are fp32.
//
// Codebooks in LDS (64 KiB a side).  One codebook per head: every entry 256 / (2 v) times in a row of 256 bytes, lane l reads copy l, and no
// two lanes of a pass meet in a bank (1.6 ns a gather of 8 bytes on a compute unit, 2.2 from a single copy).  More: a table per
// sub-vector.  Values for v = 2: row e holds entry e for all 32 positions of the operand.
//
// Work.  A workgroup of 8 wavefronts (one per compute unit, for its LDS) belongs to a cache head and takes an equal share of the head's
// work.  A request's rows are cut into blocks of 256 / ways rows; in a block `ways` wavefronts share 32 rows and take every ways-th tile of keys
// (a round: one tile per wavefront), so that few rows fill the workgroup and many are not joined at the end.  Blocks of a request go in pairs (the last with the
// first, ...), whose rounds add up to nearly the same number C: the work before a block is a product, not a sum, and every workgroup finds its share
// with one scan over the requests.  A block cut by a share's border leaves its sums in ws, and attn_paged_merge_kernel joins them in order.
// The rounds of a share are one sequence over all its blocks: codes are requested NB tiles ahead (pages 32 rounds ahead), across blocks too.
//
// What bounds it.  Not memory: codes that lie in L2 take as long as codes from HBM (57 and 61 us where both were timed).  Two wavefronts a SIMD, each
// with a tile's 16 matrix instructions (18 ns each) and 125 vector instructions (1.9 ns: addresses of the gathers, weights), in order: a chunk of 2048 tokens
// by counters has the matrix units busy for 46 % of the time and issues vector instructions for 45 %, little of it together, at 1.9 GHz; no bank conflicts.
// A round of 8 tiles takes 1.25 - 1.4 us, and before the first one lie 5 - 6 us: lengths, pages, codebooks, codes, each a trip to memory.
// 240 GFLOP of a prompt's chunk 0.27 - 0.29 ms by machine (823 - 900 TFLOP/s; a register loop of the same instruction reaches 1645 with such operands, fed by
// LDS gathers 1458).  One wavefront a SIMD with 64 rows, where every gather is used twice, took 318 - 365 us: a wavefront alone issues at
// most one instruction in 4.7 clocks.
#include <algorithm>

#include "attn_paged.h"

namespace vq {

using namespace paged;

namespace {

template <int D, int V, bool COPIES, int MODS>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_paged_kernel(PagedArgs a) {
    constexpr int P = D / V, ES = 2 * V;
    constexpr int CH = D / 32;                   // channels per lane of an operand V^T
    constexpr int NC = D / 16;                   // steps of the product with K
    constexpr int KW = P / 8;                    // dwords of a lane's K codes: half a token's
    constexpr int CPS = 8 / V;                   // K codes of a step
    constexpr bool TR = V >= 4;                  // V by transposing reads
    constexpr int NR = TR ? CH * 4 / V : CH / V; // positions of a lane's V codes
    constexpr int VW = TR ? NR : NR * 4;         // dwords of them: four or sixteen keys each
    constexpr int NB = V == 2 ? 3 : 4;           // tiles of codes in flight
    constexpr int NG = D / 16;                   // groups of eight accumulators
    constexpr int KN = NC * CPS, VN = TR ? 2 * CH : 8 * NR;   // gathers of a lane: of a tile's keys, of 16 keys' values
    extern __shared__ __align__(16) unsigned char smem[];   // (from LDS address 0: kernel_setup checks that)
    const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // consecutive workers of a head on one die: its codebooks and codes in one L2
    const int nwg = gridDim.x, id = (nwg & 7) == 0 ? (int)(blockIdx.x & 7) * (nwg >> 3) + (int)(blockIdx.x >> 3) : (int)blockIdx.x;
    const int h = id / a.workers, w = id - h * a.workers;

    // The codebooks first (they arrive while the share is looked for), the codes next (they arrive while the codebooks are written).
    Tables<D, V, COPIES, false> k_books;
    Tables<D, V, COPIES, !TR> v_books;
    const size_t books = (size_t)h * a.G * a.E * ES;
    k_books.load(a, reinterpret_cast<const unsigned char *>(a.k_cb) + books, tid);
    v_books.load(a, reinterpret_cast<const unsigned char *>(a.v_cb) + books, tid);
    Share sh;
    if (!find_share<kThreads>(a, w, reinterpret_cast<long long *>(smem + kScanOff), &sh)) return;
    k_books.store(a, smem, tid);
    v_books.store(a, smem + kSide, tid);

    const int ps_mask = (1 << a.log_ps) - 1;
    // TR: the position block of a lane's V codes and its keys among the 16 of its half
    const int c0 = 4 * ((lane >> 4) & 1) + (lane & 3), e0 = (lane >> 2) & 3;
    // lane constants of the gathers
    const unsigned copy = (unsigned)((V == 2 ? lane : V == 4 ? ln : ln & 15) * ES);
    const unsigned k_const = COPIES ? copy : (unsigned)(lh * (P / 2) * 256 * ES);
    const unsigned v_const = (unsigned)kSide + (!TR ? (unsigned)(ln * CH * 2) : COPIES ? copy : (unsigned)(c0 * NR * 256 * ES));
    // where the lane's codes lie in a block of 16 tokens
    const uint8_t *const k_lane = a.k_codes + ((4 * (ln & 3) + (ln >> 3)) * P + lh * (P / 2));
    const uint8_t *const v_lane = a.v_codes + (TR ? c0 * NR * 16 + 4 * e0 : ln * NR * 16);
    size_t *const bases = reinterpret_cast<size_t *>(smem + kBaseOff) + wave * 64;
    const size_t *const k_bases = bases + ((ln >> 2) & 1), *const v_bases = bases + lh;
    float *xs = reinterpret_cast<float *>(smem + kJoinOff), *xm = reinterpret_cast<float *>(smem + kStatOff), *xl = xm + kWaves * 32;
    int *starts = reinterpret_cast<int *>(smem + kListOff);
    Piece *list = reinterpret_cast<Piece *>(smem + kListOff + 256);

    long long left = sh.u1 - sh.u0, x = sh.x;
    int b = sh.b;
    while (left > 0) {
        int rounds_in_list;
        __syncthreads();   // (the list before is done with)
        const int pieces = list_pieces<NB>(a, &b, &x, &left, wave == 0, starts, list, &rounds_in_list);
        __syncthreads();
        if (pieces == 0) continue;

        // Pages of 32 rounds of this wavefront at a time: lane 2 s + k finds the first byte of the codes of block k (16 tokens) of
        // round s.  The list is one sequence of rounds, so codes are requested across its pieces' borders.
        int next_id, next_off;
        auto page_ids = [&](int step) {
            const int t = min(step + (lane >> 1), rounds_in_list - 1);
            int p = 0;
#pragma unroll
            for (int d = 32; d; d >>= 1)
                if (p + d < pieces && starts[p + d] <= t) p += d;
            const Piece &pc = list[p];
            const int idx = max(min(((pc.r0 + t - starts[p]) << pc.log_ways) + (wave & ((1 << pc.log_ways) - 1)), pc.count - 1), 0);
            const int at = (idx < pc.front ? idx : pc.lo + idx - pc.front) * 32 + 16 * (lane & 1);
            next_id = a.table[(size_t)pc.b * a.max_pages + (max(min(at, pc.len - 1), 0) >> a.log_ps)];
            next_off = (at & ps_mask) * P;
        };
        auto write_bases = [&]() { bases[lane] = (((size_t)min(max(next_id, 0), a.n_pages - 1) * a.H + h) << a.log_ps) * P + (size_t)next_off; };
        page_ids(0);
        write_bases();
        page_ids(32);
        size_t k_base = k_bases[0], v_base = v_bases[0];
        struct Codes {
            uint32_t k[KW], v[VW];
        } ring[NB];
        auto fetch = [&](int step, Codes &c) {
            constexpr int KB = KW >= 4 ? 16 : KW * 4, VB = TR ? 4 : 16;
            const uint8_t *kp = k_lane + k_base, *vp = v_lane + v_base;
#pragma unroll
            for (int n = 0; n < KW; n += KB / 4) {
                const typename Raw<KB>::type u = global_read<KB>(kp + 4 * n);
                __builtin_memcpy(&c.k[n], &u, KB);
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const typename Raw<VB>::type u = global_read<VB>(vp + 16 * n);
                __builtin_memcpy(&c.v[n * (VB / 4)], &u, VB);
            }
            if (((step + 1) & 31) == 0) {
                write_bases();
                page_ids(step + 33);
            }
            k_base = k_bases[2 * ((step + 1) & 31)];
            v_base = v_bases[2 * ((step + 1) & 31)];
        };
#pragma unroll
        for (int u = 0; u < NB; ++u) fetch(u, ring[u]);
        // K entries of a tile as operands: one gather
        V16 kop[NC];
        auto gather_k = [&](const Codes &codes, int at) {
            const uint32_t word = codes.k[at / 4];
            unsigned addr;
            if constexpr (COPIES) {
                addr = (at & 3) == 0 ? row_address<0>(word, k_const) : (at & 3) == 1 ? row_address<1>(word, k_const)
                       : (at & 3) == 2 ? row_address<2>(word, k_const) : row_address<3>(word, k_const);
            } else {
                addr = ((word >> (8 * (at & 3))) & 0xFFu) * ES + k_const + (unsigned)(at * 256 * ES);
            }
            lds_read<ES>(addr, &kop[at / CPS].w[at % CPS * (ES / 4)]);
        };

        int step = 0;
        for (int piece = 0; piece < pieces; ++piece) {
            const Piece pc = uniform_piece(list[piece]);
            const int ways = 1 << pc.log_ways, rt = wave >> pc.log_ways, kw = wave & (ways - 1);
            const int row0 = pc.row0 + rt * 32, tile_rows = min(pc.rows - row0, 32);
            const bool valid = ln < tile_rows;
            const int row = valid ? row0 + ln : min(row0, pc.rows - 1), i = token_of(a, row), hq = h * a.group + (row - i * a.group);
            const int pos = pc.pos0 + i;
            half8_t qf[NC];
            {
                const half_t *qp = a.q + (size_t)(pc.first + i) * a.q_stride + (size_t)hq * D + lh * (D / 2);
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    V16 u = ld16(qp + 8 * c);
#pragma unroll
                    for (int e = 0; e < 4; ++e) u.w[e] ^= a.q_sign;
                    qf[c] = u.h8;
                }
            }
            float16_t o[CH];
#pragma unroll
            for (int f = 0; f < CH; ++f)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[f][e] = 0.f;
            float m_ref = -FLT_MAX, lsum = 0.f;
            bool far = false;   // a reference of the wavefront is
            // tiles of this wavefront's rows, of those of the block
            const int pos_f = pc.pos0 + token_of(a, max(row0, 0)), pos_l = pc.pos0 + token_of(a, max(row0 + tile_rows - 1, 0));
            const int count = tile_rows > 0 ? min(pc.front + max(((max(pos_l + 1, pc.prefix) + 31) >> 5) - pc.lo, 0), pc.count) : 0;
            const float slope2 = MODS && a.slopes ? a.slopes[hq] * kLog2e : 0.f;
            const int see_to = min(pos, pc.len - 1), see_from = a.window > 0 ? max(pos - a.window + 1, 0) : 0;

            // This wavefront's tiles: idx0, idx0 + ways, ...
            const int idx0 = (pc.r0 << pc.log_ways) + kw, rounds = pc.r1 - pc.r0;
            const int tiles = min(max((count - idx0 + ways - 1) >> pc.log_ways, 0), rounds);
            // The scores of a tile are formed while the weights of the tile before it are: s holds a tile's, next the following one's.
            float16_t scores[2];
            const float scale2 = [&] {
                float x = a.scale2;
                asm("" : "+v"(x));   // (a product and sum with a scalar operand takes twice as long)
                return x;
            }();
            if (tiles > 0) {
                float16_t &s = scores[0];
#pragma unroll
                for (int n = 0; n < KN; ++n) gather_k(ring[0], n);
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(kop[c].h8, qf[c], s, 0, 0, 0);
#pragma unroll
                for (int n = 0; n < KN / 2; ++n) gather_k(ring[1], n);
            }
            auto body = [&](int tile, float16_t &s, float16_t &next, Codes &codes, const Codes &after, const Codes &second) {
                const int idx = idx0 + (tile << pc.log_ways), t0 = (idx < pc.front ? idx : pc.lo + idx - pc.front) * 32;
                if (t0 + 32 > pc.len) {
                    // Codes behind the request's end may name anything, and a weight of zero times an infinity is none: they become the
                    // tile's first token's.
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        const uint32_t good = (__shfl((int)codes.v[TR ? n : 4 * n], TR ? lane & 19 : ln, 64) & 0xFF) * 0x01010101u;
#pragma unroll
                        for (int d = 0; d < VW / NR; ++d) {
                            const int live = min(max(pc.len - (t0 + 16 * lh + 4 * (TR ? e0 : d)), 0), 4);   // bytes that stay
                            const uint32_t mask = live == 4 ? 0xFFFFFFFFu : (1u << (8 * live)) - 1u;
                            uint32_t &word = codes.v[n * (VW / NR) + d];
                            word = (word & mask) | (good & ~mask);
                        }
                    }
                }
                if constexpr (MODS) {   // (uniform branches: a choice per score would compute both sides)
                    if constexpr (MODS == kLargelyCapped) {
                        if (!((t0 + 31 <= pos_f && t0 + 31 < pc.len && (a.window == 0 || pos_l - t0 < a.window)) || t0 + 32 <= pc.prefix)) {
                            const int see = attended_keys(t0 + 16 * lh, see_from, see_to, pc.prefix);
#pragma unroll
                            for (int e = 0; e < 16; ++e) s[e] = attended_or_zero(s[e], see, 4 * (e & 3) + (e >> 2));
                        }
                        cap_scores(a, scale2, [&](int e) { return s[e]; }, [&](int e, float x) { s[e] = x; });
                    } else if (a.cap_in > 0.f) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            s[e] = a.cap_out - 2.f * a.cap_out * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[e] * a.cap_in) + 1.f);
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[e] *= scale2;
                    }
                    if (a.slopes) {
                        const float back = (float)(pos - t0 - 16 * lh);
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[e] -= slope2 * fabsf(back - (float)(4 * (e & 3) + (e >> 2)));
                    }
                }
                if (!((t0 + 31 <= pos_f && t0 + 31 < pc.len && (a.window == 0 || pos_l - t0 < a.window)) || t0 + 32 <= pc.prefix)) {
                    const int see = attended_keys(t0 + 16 * lh, see_from, see_to, pc.prefix);
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[e] = attended(s[e], see, 4 * (e & 3) + (e >> 2));
                }
                // running maximum (a NaN raises nothing: its row's weights are NaN by themselves)
                float mt = s[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mt = __builtin_elementwise_maximum(mt, s[e]);
                {
                    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
                    mt = __builtin_elementwise_maximum(__uint_as_float(y[0]), __uint_as_float(y[1]));
                }
                if (!MODS) mt *= scale2;
                if (__ballot(mt - m_ref > kRise)) {
                    const float m_new = mt - m_ref > kRise ? mt : m_ref, f = __builtin_amdgcn_exp2f(m_ref - m_new);
                    m_ref = m_new;
                    if (!MODS) far = __ballot(is_far(m_ref)) != 0;
                    lsum *= f;
#pragma unroll
                    for (int k = 0; k < CH; ++k)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[k][e] *= f;
                }
                float sub = kHeadroom - m_ref;
                if (__builtin_expect(!MODS && far, 0)) {
                    const bool mine = is_far(m_ref);
                    const float back = __builtin_amdgcn_rcpf(scale2);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float x = s[e] * scale2;
                        asm("" : "+v"(x));   // (rounded, as the maximum is)
                        s[e] = mine ? (x - m_ref) * back : s[e];
                    }
                    sub = mine ? kHeadroom : sub;
                }

                // Values of 16 keys, k of the two steps: operands as they come (TR), or channel pairs of the lane's eight keys.
                // TR: lane 4 e + c of a group of 16 asks for the entry of key 16 lh + 4 e + 2 k + j and position block c, part f; the
                // transposing read gives lane l the four keys e of channel l % 4 of block l / 4.
                V16 vop[2][TR ? CH : 1];
                uint32_t g[2][8][TR ? 1 : CH / 2];
                auto gather_v = [&](int k, int at) {
                    auto address = [&](uint32_t word, int byte) {
                        if constexpr (!TR || COPIES)
                            return byte == 0 ? row_address<0>(word, v_const) : byte == 1 ? row_address<1>(word, v_const)
                                   : byte == 2 ? row_address<2>(word, v_const) : row_address<3>(word, v_const);
                        else return ((word >> (8 * byte)) & 0xFFu) * ES + v_const;
                    };
                    if constexpr (TR) {
                        const int f = at / 2, j = at % 2, n = f * 4 / V;
                        lds_read_transposed(address(codes.v[n], 2 * k + j) + (unsigned)((COPIES ? 0 : n * 256 * ES) + (f * 4 % V) * 2), &vop[k][f].w[2 * j]);
                    } else {   // slot 4 j + e of the eight is key 4 e + 2 k + j of the 16
                        const int i = at / NR, n = at % NR;
                        lds_read<2 * V>(address(codes.v[4 * n + (i & 3)], 2 * k + (i >> 2)) + (unsigned)(n * 2 * V), &g[k][i][n * (V / 2)]);
                    }
                };
                // A matrix instruction at a time with the vector instructions of its 32 clocks, and the gathers some 130 clocks ahead of
                // their use: in bursts they overrun the counter of outstanding reads (15), and a wait for an old one waits for new ones.
                __builtin_amdgcn_sched_barrier(0);
                V16 pf[2];
#pragma unroll
                for (int e = 0; e < 16; ++e) next[e] = 0.f;
                constexpr int EW = 16 / NC, Q = NC / 4;   // weights per step, steps of a quarter
#pragma unroll
                for (int c = 0; c < NC; ++c) {   // scores of the next tile; weights of this one
                    next = __builtin_amdgcn_mfma_f32_32x32x16_f16(kop[c].h8, qf[c], next, 0, 0, 0);
                    if (c < Q) {
#pragma unroll
                        for (int n = 0; n < KN / 2 / Q; ++n) gather_k(after, KN / 2 + c * (KN / 2 / Q) + n);
                    } else if (c < 3 * Q) {
#pragma unroll
                        for (int n = 0; n < VN / (2 * Q); ++n) gather_v(0, (c - Q) * (VN / (2 * Q)) + n);
                    } else {
#pragma unroll
                        for (int n = 0; n < VN / (2 * Q); ++n) gather_v(1, (c - 3 * Q) * (VN / (2 * Q)) + n);
                    }
#pragma unroll
                    for (int e = c * EW; e < (c + 1) * EW; e += 2) {
                        const float p0 = __builtin_amdgcn_exp2f(MODS ? s[e] + sub : __builtin_fmaf(s[e], scale2, sub));
                        const float p1 = __builtin_amdgcn_exp2f(MODS ? s[e + 1] + sub : __builtin_fmaf(s[e + 1], scale2, sub));
                        const half2_t p2 = {(half_t)p0, (half_t)p1}, one = {(half_t)1.f, (half_t)1.f};
                        pf[e / 8].h2[e % 8 / 2] = p2;
                        lsum = dot2(p2, one, lsum);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                constexpr int R = CH / 2;                 // steps of a quarter of the product with V
#pragma unroll
                for (int m = 0; m < 2 * CH; ++m) {
                    const int k = m / CH, f = m % CH;
                    V16 op;
                    if constexpr (TR) {
                        op = vop[k][f];
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) op.w[e] = __builtin_amdgcn_perm(g[k][2 * e + 1][f / 2], g[k][2 * e][f / 2], f & 1 ? 0x07060302u : 0x05040100u);
                    }
                    o[f] = __builtin_amdgcn_mfma_f32_32x32x16_f16(op.h8, pf[k].h8, o[f], 0, 0, 0);
                    if (m < R) {
#pragma unroll
                        for (int n = 0; n < VN / 2 / R; ++n) gather_v(1, VN / 2 + m * (VN / 2 / R) + n);
                    } else if (m < 3 * R) {
#pragma unroll
                        for (int n = 0; n < KN / 2 / (2 * R); ++n) gather_k(second, (m - R) * (KN / 2 / (2 * R)) + n);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            for (int tile = 0; tile < rounds; tile += NB)
#pragma unroll
                for (int u = 0; u < NB; ++u, ++step) {
                    if (tile + u < tiles) {
                        body(tile + u, scores[NB % 2 ? 0 : u % 2], scores[NB % 2 ? 1 : 1 - u % 2], ring[u], ring[(u + 1) % NB], ring[(u + 2) % NB]);
                        if (NB % 2) scores[0] = scores[1];
                    }
                    fetch(step + NB, ring[u]);
                }
            {
                const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(lsum), __float_as_uint(lsum), false, false);
                lsum = __uint_as_float(y[0]) + __uint_as_float(y[1]);
            }

            // join the wavefronts that share rows, in order of kw; group g of eight accumulators ends with wavefront g % ways
            float L = lsum, M = m_ref;
            if (ways > 1) {
                if (lh == 0) {
                    xm[wave * 32 + ln] = m_ref;
                    xl[wave * 32 + ln] = lsum;
                }
                __syncthreads();
                float ms[kWaves], ls[kWaves];
#pragma unroll
                for (int k = 0; k < kWaves; ++k) {   // (past the rows' wavefronts: their first once more, without weight)
                    const int from = (wave - kw + (k < ways ? k : 0)) * 32 + ln;
                    ms[k] = xm[from];
                    ls[k] = k < ways ? xl[from] : 0.f;
                }
                L = 0.f;
#pragma unroll
                for (int k = 0; k < kWaves; ++k) M = fmaxf(M, ms[k]);
#pragma unroll
                for (int k = 0; k < kWaves; ++k) L += ls[k] * __builtin_amdgcn_exp2f(ms[k] - M);
                const float f = __builtin_amdgcn_exp2f(m_ref - M);
#pragma unroll
                for (int k = 0; k < CH; ++k)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[k][e] *= f;
            }
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const size_t part = part_of(a, h, w, pc.r0 > 0 ? 0 : 1);
            const int prow = rt * 32 + ln;
            if (!pc.whole && valid && lh == 0 && kw == 0) {
                float *st = part_stats<D>(a, part) + prow * 2;
                st[0] = M;
                st[1] = L;
            }
            auto group = [&](int g, float (&y)[8]) {   // eight consecutive channels
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    y[e] = TR ? o[CH == 4 ? 2 * (g & 1) + e / 4 : e / 4][4 * (CH == 4 ? g >> 1 : g) + e % 4]
                              : o[e % CH][CH == 4 ? 4 * (g >> 1) + 2 * (g & 1) + e / 4 : 4 * g + e / 2];
            };
            auto store = [&](int g, const float (&y)[8]) {
                if (!valid) return;
                const int ch = CH == 4 ? 32 * (g >> 1) + 16 * lh + 8 * (g & 1) : 16 * g + 8 * lh;
                if (pc.whole) {
                    half8_t z;
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = (half_t)(y[e] * inv);
                    *reinterpret_cast<half8_t *>(a.out + (size_t)(pc.first + i) * a.out_stride + (size_t)hq * D + ch) = z;
                } else {
                    float4_t *to = reinterpret_cast<float4_t *>(part_sums<D>(a, part) + (size_t)prow * D + ch);
                    to[0] = float4_t{y[0], y[1], y[2], y[3]};
                    to[1] = float4_t{y[4], y[5], y[6], y[7]};
                }
            };
            // AT: groups that the buffer holds at once, of the rows' lanes alone (32 / AT rows at most)
            auto join = [&](auto at_once) {
                constexpr int AT = decltype(at_once)::value, ROWS = 32 / AT;
                float4_t *buf = reinterpret_cast<float4_t *>(xs);
                const int slot = lh * ROWS + (ln & (ROWS - 1));   // of 2 ROWS
                auto cell = [&](int w_, int g, int half) { return buf + ((w_ * AT + g % AT) * 2 + half) * 2 * ROWS + slot; };
                const bool mine = ln < ROWS;
#pragma unroll
                for (int g0 = 0; g0 < NG; g0 += AT) {
#pragma unroll
                    for (int g = g0; g < g0 + AT && g < NG; ++g) {
                        float y[8];
                        group(g, y);
                        if (mine && (g & (ways - 1)) != kw) {
                            *cell(wave, g, 0) = float4_t{y[0], y[1], y[2], y[3]};
                            *cell(wave, g, 1) = float4_t{y[4], y[5], y[6], y[7]};
                        }
                    }
                    __syncthreads();
#pragma unroll
                    for (int g = g0; g < g0 + AT && g < NG; ++g) {
                        if (!mine || (g & (ways - 1)) != kw) continue;
                        float y[8];
                        group(g, y);
                        float t[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                        for (int k0 = 0; k0 < ways; k0 += 2) {   // (ways is even)
                            float4_t z[2][2];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                z[k][0] = *cell(wave - kw + k0 + k, g, 0);
                                z[k][1] = *cell(wave - kw + k0 + k, g, 1);
                            }
#pragma unroll
                            for (int k = 0; k < 2; ++k)
#pragma unroll
                                for (int e = 0; e < 8; ++e) t[e] += k0 + k == kw ? y[e] : z[k][e / 4][e % 4];
                        }
                        store(g, t);
                    }
                    if (g0 + AT < NG) __syncthreads();
                }
                __syncthreads();   // (the buffers are the next piece's)
            };
            if (ways == 1) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    float y[8];
                    group(g, y);
                    store(g, y);
                }
            } else if (pc.rows - pc.row0 <= 4) {
                join(std::integral_constant<int, 8>());
            } else {
                join(std::integral_constant<int, 1>());
            }
        }
    }
}

// How a call is cut, from its sizes alone.
struct PagedPlan {
    int few, workers, min_log_ways, cut;
    size_t ws;
};
PagedPlan paged_plan(const vq_kv_pages_t *kv, const vq_paged_batch_t *b) {
    PagedPlan p;
    p.workers = kv->H >= 256 ? 1 : 256 / kv->H;
    const long long rows = (long long)b->n_tokens * (b->Hq / kv->H) * kv->H;
    // Tiles of 16 rows and 64 keys for requests of 16 rows on average at most, where there is enough to read: a tile takes about as long as
    // one of 32 rows and 32 keys, so long caches take less (us of both, few rows first; H = 32, a row a request: 16 requests of 16384 tokens
    // 132 and 150, 64 of 4096 154 and 165; H = 8, 16 rows a request: 64 of 16384 125 and 163, 64 of 1024 32 and 44), but a
    // wavefront alone with a larger tile is later with it (one of 300 tokens 17 and 13, H = 32; 16 of 2048 42 and 38).  The wider
    // tiles take longer per row beyond four (their sums join in more steps), so there it pays earlier.  The average is all that the host knows: a
    // chunk among many single tokens runs in such tiles too.  D = 64 and v = 2 have no such tile, built or timed.
    const long long keys = (long long)b->B * kv->H * b->max_pages * kv->page_tokens, few_rows = (long long)b->n_tokens * (b->Hq / kv->H);
    p.few = few_supported(kv->D, kv->v) && few_rows <= 16ll * b->B && keys >= (few_rows > 4ll * b->B ? 1ll << 18 : 1ll << 21);
    // Wavefronts that share rows read other tiles of keys and join their sums; wavefronts with rows of their own gather the same keys each, and few
    // rows are few blocks to deal out.  Rows of all heads, us with 1 / 2 / 4 wavefronts a 32 rows: 32768 98 / 99 / 87, 65536 296 / 274 / 283 (2048 new tokens of 8192),
    // 102400 225 / 238 / 245, 268800 329 / 370 / 474.
    p.min_log_ways = p.few ? 3 : rows >= 96 * 1024 ? 0 : rows >= 40 * 1024 ? 1 : 2;
    // Blocks of short requests stay whole: a share's border inside one costs the joining launch, 2 - 5 us, more than the shares' evenness gains.  Whole and
    // cut, us: 8 requests of 1000 tokens, a new one each, 16.6 and 23.2; 4 of 900 new tokens of 1000, 96 and 108; of 1500 60 and 63.  At 2000 chunks gain by the
    // cut (16 of 500 new ones 268 and 260) and a few single tokens lose (8 of them 19.8 and 24.0): the line looks at lengths alone and takes the chunks' side.
    p.cut = p.workers > 1 && (long long)b->max_pages * kv->page_tokens > 1536;
    p.ws = p.cut ? (size_t)kv->H * p.workers * 2 * ((kWaves * (p.few ? 16 : 32)) >> p.min_log_ways) * (kv->D + 2) * sizeof(float) : 0;
    return p;
}

template <int D, int V, bool COPIES, int MODS>
int run_wide(const PagedArgs &a, hipStream_t s) {
    static KernelSetup setup;
    if (int st = kernel_setup(reinterpret_cast<const void *>(&attn_paged_kernel<D, V, COPIES, MODS>), kLds, true, setup)) return st;
    attn_paged_kernel<D, V, COPIES, MODS><<<a.H * a.workers, kThreads, kLds, s>>>(a);
    return merge<D>(a, s);
}
template <int D, int V, bool COPIES>
int run_wide_with(const PagedArgs &a, hipStream_t s) {
    if (a.mods == kPlain) return run_wide<D, V, COPIES, kPlain>(a, s);
    return a.mods == kModified ? run_wide<D, V, COPIES, kModified>(a, s) : run_wide<D, V, COPIES, kLargelyCapped>(a, s);
}
template <int D, int V>
int run_paged_as(const PagedArgs &a, hipStream_t s) { return a.G == 1 ? run_wide_with<D, V, true>(a, s) : run_wide_with<D, V, false>(a, s); }

}  // namespace

bool attn_paged_supported(const vq_kv_pages_t *kv) {
    const int PG = kv->D / kv->v / kv->cb_groups;
    return (kv->D == 64 || kv->D == 128) && (PG & (PG - 1)) == 0;
}

size_t attn_paged_workspace(const vq_kv_pages_t *kv, const vq_paged_batch_t *b) { return paged_plan(kv, b).ws; }

int launch_attn_paged(const vq_kv_pages_t *kv, const vq_paged_batch_t *b, const void *q, size_t q_stride, float sm_scale, void *out,
                      size_t out_stride, void *ws, hipStream_t s) {
    const PagedPlan p = paged_plan(kv, b);
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
    a.ws = (float *)ws;
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.B = b->B;
    a.H = kv->H;
    a.group = b->Hq / kv->H;
    a.group_shift = 31;
    while ((1ll << (a.group_shift - 31)) < a.group) ++a.group_shift;
    a.group_inverse = (unsigned)(((1ull << a.group_shift) + a.group - 1) / a.group);
    a.E = kv->n_entries;
    a.G = kv->cb_groups;
    a.pg_shift = __builtin_ctz(kv->D / kv->v / kv->cb_groups);
    a.n_pages = kv->n_pages;
    a.max_pages = b->max_pages;
    a.log_ps = __builtin_ctz(kv->page_tokens);
    a.n_tokens = b->n_tokens;
    a.window = b->window < b->max_pages * kv->page_tokens ? b->window : 0;   // (one that reaches every token is none)
    a.workers = p.workers;
    a.tile_rows = p.few ? 16 : 32;
    a.log_keys = p.few ? 6 : 5;
    a.min_log_ways = p.min_log_ways;
    a.cut = p.cut;
    a.min_share = 2;   // (4 requests of 4096 tokens, 8 heads, us with 1 / 2 / 4 rounds: 21.2 / 20.9 / 25.0; one: 22.8 / 20.8 / 21.2)
    const float scale = sm_scale < 0.f ? -sm_scale : sm_scale;
    a.scale2 = scale * kLog2e > FLT_MIN ? scale * kLog2e : FLT_MIN;   // (above zero: minus infinity times it has to stay)
    a.q_sign = sm_scale < 0.f ? 0x80008000u : 0u;
    // (finite: a zero score times the first stays zero, and a cap that the second shortens is beyond any score)
    a.cap_in = b->softcap > 0.f ? std::min(2.f * a.scale2 / b->softcap, FLT_MAX) : 0.f;
    a.cap_out = std::min(b->softcap * kLog2e, FLT_MAX / 4);
    for (int i = 0; i < 3; ++i) a.cap_poly[i] = kCapPoly[i] * a.scale2;
    a.mods = a.cap_in > 0.f && b->softcap > kLargeCap ? kLargelyCapped : a.cap_in > 0.f || b->slopes ? kModified : kPlain;
    if (p.few) return launch_few(a, kv->v, s);
    if (kv->D == 64) return kv->v == 8 ? run_paged_as<64, 8>(a, s) : kv->v == 4 ? run_paged_as<64, 4>(a, s) : run_paged_as<64, 2>(a, s);
    return kv->v == 8 ? run_paged_as<128, 8>(a, s) : kv->v == 4 ? run_paged_as<128, 4>(a, s) : run_paged_as<128, 2>(a, s);
}

}  // namespace vq
