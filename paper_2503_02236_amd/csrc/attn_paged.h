// What the kernels of vq_attn_paged share: a request in numbers, the cut of the work into shares and pieces, the codebooks' way into LDS, and
// the launch that joins cut blocks (attn_paged.hip has the whole picture).
#pragma once
#include <cfloat>
#include <climits>
#include <type_traits>

#include "vq_common.h"

namespace vq {

namespace paged {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 8, kThreads = kWaves * 64;
constexpr int kSide = 65536;                  // LDS of a side's codebooks
constexpr int kJoinOff = 2 * kSide;           // sums of wavefronts that share rows, 16 KiB
constexpr int kStatOff = kJoinOff + 16384;    // their maxima and sums of weights, [wave][32] each
constexpr int kScanOff = kStatOff + 2048;
constexpr int kListOff = kScanOff + 256;      // pieces of the share, 64 at a time: their first rounds, and a Piece each
constexpr int kBaseOff = kListOff + 256 + 64 * 64;   // where the codes of the next rounds lie, [wave][64]
constexpr int kLds = kBaseOff + kWaves * 64 * 8;
// Weights are 2^(s - m + 6), s up to 6 above m.  6 - m is a float: off by 2 at most upwards (where m's last bit is worth 4 or 8, from 2^25 on; beyond, it is
// -m), so a weight is 2^14 at most, a half, whatever the scores.
constexpr float kHeadroom = 6.f, kRise = 6.f; // (log2)
// Where the scale is applied in the weight's fused multiply-add, s is a product that this does not round, and the maximum does: beyond this they may differ by a
// sixteenth and more (from 2^25 on weights would be no halves), so such rows' scores are rounded and taken less m first.
constexpr float kFar = 1048576.f;
__device__ __forceinline__ bool is_far(float m) { return fabsf(m) > kFar && m != -FLT_MAX; }

struct PagedArgs {
    const uint8_t *k_codes, *v_codes;
    const half_t *k_cb, *v_cb;
    const int *table, *cu_new, *seq_lens, *prefix_lens;
    const float *slopes;
    const half_t *q;
    half_t *out;
    float *ws;
    size_t q_stride, out_stride;
    int B, H, group, E, G, pg_shift, n_pages, max_pages, log_ps, n_tokens, window;
    unsigned group_inverse;   // row / group = row * group_inverse >> group_shift, for rows below 2^31
    int group_shift;
    int workers;        // workgroups of a cache head
    int tile_rows, log_keys;   // of a tile: 32 rows and 32 keys, or 16 and 64
    int min_log_ways;   // fewest wavefronts that share a tile's rows
    int cut;            // 0: blocks are not cut
    int min_share;      // rounds
    float scale2;       // |sm_scale| log2(e)
    unsigned q_sign;    // sign of sm_scale, in both halves
    float cap_in, cap_out, cap_poly[3];   // softcap: cap_out - 2 cap_out / (2^(s cap_in) + 1), or cap_scores; cap_in 0: none
    int mods;           // kPlain ...
};

__device__ __forceinline__ int token_of(const PagedArgs &a, int row) { return (int)(((unsigned long long)(unsigned)row * a.group_inverse) >> a.group_shift); }

// A request, in numbers that fit no memory access out of bounds.
struct Request {
    int first, n, len, prefix, rows, log_ways, blocks, items, C;
};
// Tiles of keys that some of the tokens [i0, i1] attends: [0, front) and [lo, hi).
struct Tiles {
    int front, lo, hi;
    __device__ int count() const { return front + max(hi - lo, 0); }
};
__device__ __forceinline__ Tiles tiles_of(const PagedArgs &a, const Request &r, int i0, int i1) {
    const int p0 = r.len - r.n + i0, p1 = r.len - r.n + i1;
    Tiles t;
    t.lo = (a.window > 0 && p0 >= a.window ? p0 - a.window + 1 : 0) >> a.log_keys;
    t.hi = (max(p1 + 1, r.prefix) + (1 << a.log_keys) - 1) >> a.log_keys;
    t.front = min((r.prefix + (1 << a.log_keys) - 1) >> a.log_keys, t.lo);
    return t;
}
__device__ __forceinline__ int block_rows(const PagedArgs &a, const Request &r) { return (kWaves * a.tile_rows) >> r.log_ways; }
__device__ __forceinline__ Tiles block_tiles(const PagedArgs &a, const Request &r, int j) {
    const int row = j * block_rows(a, r);
    return tiles_of(a, r, token_of(a, row), token_of(a, min(row + block_rows(a, r), r.rows) - 1));
}
__device__ __forceinline__ int block_rounds(const PagedArgs &a, const Request &r, int j) {   // (a block that attends nothing writes zeros)
    return max((block_tiles(a, r, j).count() + (1 << r.log_ways) - 1) >> r.log_ways, 1);
}
__device__ __forceinline__ Request request_of(const PagedArgs &a, int b) {
    Request r;
    const int c0 = min(max(a.cu_new[b], 0), a.n_tokens), c1 = min(max(a.cu_new[b + 1], 0), a.n_tokens);
    r.first = c0;
    r.n = max(c1 - c0, 0);
    r.len = min(max(a.seq_lens[b], 0), a.max_pages << a.log_ps);
    r.prefix = a.prefix_lens ? min(max(a.prefix_lens[b], 0), r.len) : 0;
    r.rows = r.n * a.group;
    r.log_ways = max(r.rows <= 32 ? 3 : r.rows <= 64 ? 2 : r.rows <= 128 ? 1 : 0, a.min_log_ways);
    r.blocks = (r.rows + block_rows(a, r) - 1) / block_rows(a, r);
    r.items = (r.blocks + 1) / 2;
    r.C = r.blocks == 0 ? 0 : block_rounds(a, r, 0);
    if (r.blocks > 1) r.C = max(r.C + block_rounds(a, r, r.blocks - 1), 2 * block_rounds(a, r, r.blocks / 2)) + 1;
    return r;
}

__device__ __forceinline__ long long shfl_ll(long long v, int from) {
    return ((long long)__builtin_amdgcn_readlane((int)(v >> 32), from) << 32) | (unsigned)__builtin_amdgcn_readlane((int)v, from);
}

// The share of worker w: rounds [u0, u1) of the head's, the first of them round x of request b.  False: none.  All threads of the
// workgroup call it; xs: LDS, threads / 64 + 2 values.
struct Share {
    long long u0, u1, share, x;
    int b;
};
template <int THREADS>
__device__ __forceinline__ bool find_share(const PagedArgs &a, int w, long long *xs, Share *out) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int NW = THREADS / 64;
    auto share_of = [&](long long total) {
        out->share = max((total + a.workers - 1) / a.workers, (long long)a.min_share);
        out->u0 = w * out->share;
        out->u1 = min(out->u0 + out->share, total);
        return out->u0 < total;
    };
    if (a.B <= 64) {   // every wavefront for itself
        long long own = 0;
        if (lane < a.B) {
            const Request r = request_of(a, lane);
            own = (long long)r.items * r.C;
        }
        long long upto = own;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const long long y = __shfl_up(upto, d, 64);
            if (lane >= d) upto += y;
        }
        if (!share_of(shfl_ll(upto, 63))) return false;
        out->b = __ffsll((long long)__ballot(out->u0 < upto)) - 1;
        out->x = out->u0 - shfl_ll(upto - own, out->b);
        return true;
    }
    long long mine = 0, total = 0, own = 0;
    for (int b = tid; b < a.B; b += THREADS) {
        const Request r = request_of(a, b);
        own = (long long)r.items * r.C;
        mine += own;
    }
    long long incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const long long y = __shfl_up(incl, d, 64);
        if (lane >= d) incl += y;
    }
    if (lane == 63) xs[wave] = incl;
    __syncthreads();
    long long before = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
        if (i < wave) before += xs[i];
        total += xs[i];
    }
    incl += before;
    if (!share_of(total)) return false;
    __syncthreads();
    if (a.B <= THREADS) {
        if (incl - mine <= out->u0 && out->u0 < incl) {
            xs[NW] = tid;
            xs[NW + 1] = out->u0 - (incl - mine);
        }
    } else {
        long long carry = 0;
        for (int b0 = 0; b0 < a.B; b0 += THREADS) {
            const int b = b0 + tid;
            long long u = 0;
            if (b < a.B) {
                const Request r = request_of(a, b);
                u = (long long)r.items * r.C;
            }
            long long in = u, chunk = 0, lower = 0;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const long long y = __shfl_up(in, d, 64);
                if (lane >= d) in += y;
            }
            if (lane == 63) xs[wave] = in;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                if (i < wave) lower += xs[i];
                chunk += xs[i];
            }
            __syncthreads();
            const long long from = carry + lower + in - u;
            if (from <= out->u0 && out->u0 < from + u) {
                xs[NW] = b;
                xs[NW + 1] = out->u0 - from;
            }
            carry += chunk;
        }
    }
    __syncthreads();
    const long long b = xs[NW], x = xs[NW + 1];
    out->b = __builtin_amdgcn_readfirstlane((int)b);
    out->x = ((long long)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)x);
    return true;
}

// Rounds [r0, r1) of a block of a request.
struct alignas(16) Piece {
    int first, pos0, len, prefix;       // of the request: its first row of q, length before its new tokens, length, prefix
    int rows, log_ways, row0, b;        // rows of the request, first row of the block
    int front, lo, count, whole;        // tiles of the block: [0, front) and [lo, ...), count in all; r0 .. r1 is all of it
    int r0, r1, pad0, pad1;
};
__device__ __forceinline__ Piece uniform_piece(const Piece &p) {
    Piece u;
    constexpr int N = sizeof(Piece) / 4;
    int t[N];
    __builtin_memcpy(t, &p, sizeof(Piece));
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = __builtin_amdgcn_readfirstlane(t[i]);
    __builtin_memcpy(&u, t, sizeof(Piece));
    return u;
}

// The next pieces of a share, 64 at most: from round *x of request *b on, *left rounds; all three step behind them.  A lane makes a piece:
// of one request (as many as have a single block), or of one block of a larger request.  Every wavefront of the workgroup makes the same list,
// one writes it.  Returns the pieces; *rounds: theirs, each piece's rounded up to PAD.
template <int PAD>
__device__ __forceinline__ int list_pieces(const PagedArgs &a, int *b, long long *x, long long *left, bool write, int *starts, Piece *list, int *rounds) {
    const int lane = threadIdx.x & 63;
    Request r = {};
    if (*b + lane < a.B) r = request_of(a, *b + lane);
    Piece pc = {};
    int from, to, j = 0, off = 0, n = 0;   // rounds [from, to) of the item; the block's first in it, the block's number of them
    bool there;
    const unsigned long long large = __ballot(r.blocks > 1);
    if (large & 1) {
        Request u;
        constexpr int N = sizeof(Request) / 4;
        int t[N];
        __builtin_memcpy(t, &r, sizeof(Request));
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = __builtin_amdgcn_readfirstlane(t[i]);
        __builtin_memcpy(&u, t, sizeof(Request));
        r = u;
        const int k0 = (int)(*x / r.C), from0 = (int)(*x - (long long)k0 * r.C), ahead = lane >> 1, k = k0 + ahead;
        const long long before = ahead == 0 ? 0 : (long long)ahead * r.C - from0;
        from = ahead == 0 ? from0 : 0;
        to = from + (int)min(max(*left - before, 0ll), (long long)(r.C - from));
        there = k < r.items && to > from;
        if (there) {
            const int jl = r.blocks - 1 - k, nl = block_rounds(a, r, jl);
            j = (lane & 1) ? k : jl;
            off = (lane & 1) ? nl : 0;
            n = (lane & 1) ? block_rounds(a, r, k) : nl;
            there = !((lane & 1) && k == jl);
        }
        const long long taken = min(*left, (long long)(min(k0 + 32, r.items) - k0) * r.C - from0);
        *left -= taken;
        *x += taken;
        pc.b = *b;
        if (*x == (long long)r.items * r.C) {
            *x = 0;
            *b += 1;
        }
    } else {
        const int simple = large ? __ffsll((long long)large) - 1 : 64;
        from = lane == 0 ? (int)*x : 0;
        const int avail = lane < simple ? r.items * r.C - from : 0;
        long long upto = avail;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const long long y = __shfl_up(upto, d, 64);
            if (lane >= d) upto += y;
        }
        to = from + (int)min(max(*left - (upto - avail), 0ll), (long long)avail);
        there = to > from;
        n = there ? block_rounds(a, r, 0) : 0;
        *left -= min(*left, shfl_ll(upto, 63));
        pc.b = *b + lane;
        *x = 0;
        *b += simple;
    }
    if (a.cut) {
        pc.r0 = max(from - off, 0);
        pc.r1 = to == r.C ? n : min(to - off, n);
    } else {   // whole blocks, with the share that they begin in
        pc.r0 = 0;
        pc.r1 = off >= from && (off < to || to == r.C) ? n : 0;
    }
    there = there && pc.r0 < pc.r1;
    pc.whole = pc.r0 == 0 && pc.r1 == n;
    const int mine = there ? (pc.r1 - pc.r0 + PAD - 1) / PAD * PAD : 0;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(upto, d, 64);
        if (lane >= d) upto += y;
    }
    *rounds = __builtin_amdgcn_readlane(upto, 63);
    const unsigned long long all = __ballot(there);
    if (write && there) {
        const Tiles t = block_tiles(a, r, j);
        pc.first = r.first;
        pc.pos0 = r.len - r.n;
        pc.len = r.len;
        pc.prefix = r.prefix;
        pc.rows = r.rows;
        pc.log_ways = r.log_ways;
        pc.row0 = j * block_rows(a, r);
        pc.front = t.front;
        pc.lo = t.lo;
        pc.count = t.count();
        pc.pad0 = pc.pad1 = 0;
        const int at = __popcll(all & ((1ull << lane) - 1ull));
        starts[at] = upto - mine;
        list[at] = pc;
    }
    return __popcll(all);
}

// Sums of cut blocks: two per worker (the block that its share begins inside, the one that it ends inside), [rows][D] and [rows][2].
__device__ __forceinline__ size_t part_of(const PagedArgs &a, int h, int w, int which) { return ((size_t)h * a.workers + w) * 2 + which; }
__host__ __device__ __forceinline__ int part_rows(const PagedArgs &a) { return (kWaves * a.tile_rows) >> a.min_log_ways; }
template <int D>
__device__ __forceinline__ float *part_sums(const PagedArgs &a, size_t part) { return a.ws + part * part_rows(a) * D; }
template <int D>
__device__ __forceinline__ float *part_stats(const PagedArgs &a, size_t part) {
    return a.ws + (size_t)a.H * a.workers * 2 * part_rows(a) * D + part * part_rows(a) * 2;
}

template <int BYTES>
struct Raw;
template <>
struct Raw<16> { typedef unsigned type __attribute__((ext_vector_type(4))); };
template <>
struct Raw<8> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <>
struct Raw<4> { typedef unsigned type; };

// BYTES from an LDS byte address to dwords
template <int BYTES>
__device__ __forceinline__ void lds_read(unsigned addr, uint32_t *to) {
    typedef typename Raw<BYTES>::type raw_t;
    const raw_t r = *reinterpret_cast<const __attribute__((address_space(3))) raw_t *>((uintptr_t)addr);
    __builtin_memcpy(to, &r, BYTES);
}
// ds_read_b64_tr_b16: of each group of 16 lanes, lane l gets half l % 4 of what lanes l / 4, 4 + l / 4, 8 + l / 4 and 12 + l / 4 ask for
__device__ __forceinline__ void lds_read_transposed(unsigned addr, uint32_t *to) {
    typedef short raw_t __attribute__((ext_vector_type(4)));
    const raw_t r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<raw_t __attribute__((address_space(3))) *>((uintptr_t)addr));
    __builtin_memcpy(to, &r, 8);
}
template <int BYTES>
__device__ __forceinline__ typename Raw<BYTES>::type global_read(const void *p) {
    return *reinterpret_cast<const typename Raw<BYTES>::type *>(p);
}

// byte B of w in bits 8 .. 15, the lane's constant around it
template <int B>
__device__ __forceinline__ unsigned row_address(uint32_t w, unsigned lane_const) {
    return __builtin_amdgcn_perm(w, lane_const, 0x0c020000u | ((4u + B) << 8));
}

// Bits of 16 keys from `key` on that a row attends: [from, to] and the prefix.  A word per lane, where 16 conditions would take 32 scalar
// registers and spill others (a masked tile costs 100 instructions, not 280: a third of the time of a step of one short request).
__device__ __forceinline__ int attended_keys(int key, int from, int to, int prefix) {
    auto below = [&](int end) { return (1 << min(max(end - key, 0), 16)) - 1; };
    return (below(to + 1) & ~below(from)) | below(prefix);
}
__device__ __forceinline__ float attended(float s, int keys, int bit) {   // s, or minus infinity
    const unsigned keep = (unsigned)((int)((unsigned)keys << (31 - bit)) >> 31);
    return __uint_as_float((__float_as_uint(s) & keep) | (0xFF800000u & ~keep));
}
__device__ __forceinline__ float attended_or_zero(float s, int keys, int bit) {
    return __uint_as_float(__float_as_uint(s) & (unsigned)((int)((unsigned)keys << (31 - bit)) >> 31));
}

// What a kernel does to scores: nothing, a cap of up to kLargeCap and a bias, or a larger cap and a bias.
enum { kPlain, kModified, kLargelyCapped };
// cap tanh(s / cap) is cap - 2 cap / (2^x + 1), x = 2 log2(e) s / cap: a difference of numbers of the cap's size, off by 14 2^-24 caps at most (the
// roundings of x, 2^x, the sum, its reciprocal, the product and the difference).  Up to this cap that is 2^-12, half a weight's rounding, whatever the score.
constexpr float kLargeCap = 256.f;
// A lane's 16 scores q . k under a larger cap, in units of log2: the same where the lane's largest has |x| > 1, the cap being below three times that
// score.  Otherwise tanh(y) = y (1 + ...), a polynomial in x^2 (least maximum of the relative error on |x| <= 1, 2^-24.6) times the scale, whose error is relative
// to the score: a cap far above the scores is none.  A lane has keys of one row, those that it does not attend are zero here, and lanes choose for
// themselves: what a row gets follows from what it attends alone.  A mixed step takes 96.2 us with the first form alone, 94.4 with the polynomial, and up to 111 with both
// in a wavefront (a cap near three times the largest scores), so smaller caps have the first form only.
constexpr float kCapPoly[3] = {-4.00369909e-02f, 1.91897040e-03f, -8.53218143e-05f};
template <typename Get, typename Set>
__device__ __forceinline__ void cap_scores(const PagedArgs &a, float scale2, Get get, Set set) {
    float top = fabsf(get(0));
#pragma unroll
    for (int e = 1; e < 16; ++e) top = __builtin_elementwise_maximum(top, fabsf(get(e)));
    if (top * a.cap_in <= 1.f) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float x = get(e) * a.cap_in, w = x * x;
            const float q = __builtin_fmaf(w, __builtin_fmaf(w, a.cap_poly[2], a.cap_poly[1]), a.cap_poly[0]);
            set(e, get(e) * __builtin_fmaf(w, q, scale2));
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) set(e, a.cap_out - 2.f * a.cap_out * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(get(e) * a.cap_in) + 1.f));
    }
}

// One side's codebooks of a head (cb) for LDS: load() requests them, store() writes them.  By entry: every entry 256 / (2 v) times in a row of
// 256 bytes, or a table per sub-vector.  By position (v = 2, values): row e holds entry e for all 32 positions of the operand.  Rows of
// entries that do not exist are zero.
template <int D, int V, bool COPIES, bool POSITIONS>
struct Tables {
    static constexpr int ES = 2 * V, P = D / V, CH = D / 32;
    static constexpr int US = POSITIONS ? 2 * (V < CH ? V : CH) : ES;      // bytes of a unit of memory
    static constexpr int UNITS = 2 * D / US;                               // POSITIONS: units of a row
    static constexpr int N = (POSITIONS ? 256 * UNITS : COPIES ? 256 * 16 : P * 256) / kThreads;
    typedef typename Raw<US>::type unit_t;
    unit_t u[N];

    static __device__ __forceinline__ void place(int at, int *row, int *unit) {
        if (!POSITIONS) {
            *row = COPIES ? at >> 4 : at & 255;
            *unit = COPIES ? 0 : at >> 8;
        } else if (COPIES) {   // neighbours read one entry
            *row = at / UNITS;
            *unit = at % UNITS;
        } else {               // eight entries of eight positions: 64-byte pieces from memory, eight columns of LDS
            *row = (at >> 3) / UNITS * 8 + (at & 7);
            *unit = (at >> 3) % UNITS;
        }
    }
    __device__ __forceinline__ void load(const PagedArgs &a, const unsigned char *cb, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int row, unit;
            place(tid + i * kThreads, &row, &unit);
            const int ch = POSITIONS ? unit * (US / 2) : unit * V, p = COPIES ? 0 : (ch / V) >> a.pg_shift;
            u[i] = global_read<US>(cb + (unsigned)((p * a.E + min(row, a.E - 1)) * ES + (POSITIONS ? ch % V * 2 : 0)));
        }
    }
    __device__ __forceinline__ void store(const PagedArgs &a, unsigned char *to, int tid) const {
        const unit_t none = {};
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = tid + i * kThreads;
            int row, unit;
            place(at, &row, &unit);
            const unit_t x = row < a.E ? u[i] : none;
            if (POSITIONS) {
                *reinterpret_cast<unit_t *>(to + row * 256 + unit * US) = x;
            } else if (COPIES) {
                unit_t r[16 / US];
#pragma unroll
                for (int k = 0; k < 16 / US; ++k) r[k] = x;
                uint4 q;
                __builtin_memcpy(&q, r, 16);
                reinterpret_cast<uint4 *>(to)[at] = q;
            } else {
                reinterpret_cast<unit_t *>(to)[at] = x;
            }
        }
    }
};

constexpr int kMergeRows = 32;   // of a workgroup
// Joins the sums of the block that worker w's share begins inside, if no worker before it began there too.
template <int D>
static __global__ __launch_bounds__(256) void attn_paged_merge_kernel(PagedArgs a) {
    __shared__ long long xs[256 / 64 + 2];
    const int w = blockIdx.x + 1, h = blockIdx.y, tid = threadIdx.x;
    Share sh;
    if (!find_share<256>(a, w, xs, &sh)) return;
    const Request r = request_of(a, sh.b);
    const int k = (int)(sh.x / r.C), from = (int)(sh.x - (long long)k * r.C);
    const int jl = r.blocks - 1 - k, nl = block_rounds(a, r, jl);
    int j = jl, off = 0, rounds = nl;
    if (from >= nl) {
        if (k == jl) return;
        j = k;
        off = nl;
        rounds = block_rounds(a, r, k);
    }
    if ((int)blockIdx.z * kMergeRows >= block_rows(a, r) || from <= off || from >= off + rounds || from - sh.share > off) return;
    // pieces: the end of worker w - 1's share, then the beginnings of w's and of those behind it that begin inside the block
    const long long end = sh.u0 - from + min(off + rounds, r.C);
    const int pieces = 1 + (int)((end - sh.u0 + sh.share - 1) / sh.share);
    const int row0 = j * block_rows(a, r), rows = min(block_rows(a, r), r.rows - row0);
    constexpr int PER = D / 8;   // threads of a row
    for (int t = tid; t < kMergeRows * PER; t += 256) {
        const int lr = blockIdx.z * kMergeRows + t / PER, ch = t % PER * 8, row = row0 + lr;
        if (lr >= rows) break;
        // (four pieces at a time are requested at once: each is a trip to memory, or two)
        constexpr int N = 4;
        auto part = [&](int p) { return part_of(a, h, w - 1 + p, p == 0 ? 1 : 0); };
        float M = -FLT_MAX, L = 0.f, x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int p0 = 0; p0 < pieces; p0 += N) {
            float m[N], l[N];
            float4_t y[N][2];
#pragma unroll
            for (int p = 0; p < N; ++p) {   // (past the end: the last one once more, without weight)
                const size_t from = part(min(p0 + p, pieces - 1));
                const float *st = part_stats<D>(a, from) + lr * 2;
                m[p] = st[0];
                l[p] = st[1];
                const float4_t *sums = reinterpret_cast<const float4_t *>(part_sums<D>(a, from) + (size_t)lr * D + ch);
                y[p][0] = sums[0];
                y[p][1] = sums[1];
            }
            float top = M;
#pragma unroll
            for (int p = 0; p < N; ++p) top = fmaxf(top, m[p]);
            const float keep = __builtin_amdgcn_exp2f(M - top);
            M = top;
            L *= keep;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= keep;
#pragma unroll
            for (int p = 0; p < N; ++p) {
                if (p0 + p >= pieces) break;
                const float f = __builtin_amdgcn_exp2f(m[p] - M);
                L += l[p] * f;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += y[p][e / 4][e % 4] * f;
            }
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        half8_t y;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = (half_t)(x[e] * inv);
        const int i = token_of(a, row), hq = h * a.group + (row - i * a.group);
        *reinterpret_cast<half8_t *>(a.out + (size_t)(r.first + i) * a.out_stride + (size_t)hq * D + ch) = y;
    }
}

template <int D>
static inline int merge(const PagedArgs &a, hipStream_t s) {
    if (a.cut) attn_paged_merge_kernel<D><<<dim3(a.workers - 1, a.H, (part_rows(a) + kMergeRows - 1) / kMergeRows), 256, 0, s>>>(a);
    return launch_status();
}

// Requests of few rows: tiles of 16 rows and 64 keys (attn_paged_few.hip).
bool few_supported(int D, int V);
int launch_few(const PagedArgs &a, int V, hipStream_t s);

}  // namespace paged

}  // namespace vq
