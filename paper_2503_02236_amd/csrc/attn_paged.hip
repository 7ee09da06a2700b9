// Attention of the new tokens of a batch of requests over a paged cache of VQ codes (vq_attn_paged).
//
// Mathematics.  For a cache head h the rows are (new token, query head of the group).  A wavefront takes 32 rows and walks over
// tiles of 32 cached tokens with the running maximum m, sum l and accumulators of a softmax:
//   S^T = K Q^T   v_mfma_f32_32x32x16_f16, operand A = K: lane (key, half) takes 8 channels of its key, gathered by code from the
//                 codebook in LDS straight into the operand.  Which key a row of the operand is, and which channel a step, is free: row
//                 16 s + 8 a + 4 l + j is key 16 s + 8 l + 4 a + j, and half l takes the channels of its half of the head, so that a lane's codes are
//                 consecutive bytes and its scores are those of the keys 16 s + 8 l + (0 .. 7) of one row;
//   O^T = V^T P^T with P^T as operand B: exactly those scores, after exp2, as halves: no shuffle, no LDS.  Operand A = V^T: the lane
//                 takes the channels of one position for its 8 keys (8 consecutive bytes of codes: the layout of the value pages), and
//                 permutes the gathered pairs into D / 32 operands.
// A weight is 2^(s - m + 6) rounded to a half (relative error 2^-11; the sum l takes it unrounded): m follows the maximum only when
// that has grown by more than 8, so weights lie below 2^14 and those that fall below a half's range are below 2^-31 of the largest.
// Sums, statistics and outputs before the last rounding are fp32.
//
// Codebooks in LDS (64 KiB a side).  V: row e holds entry e for all 32 channel positions of the operand, so the 32 lanes of a pass
// read 32 different columns: no bank conflicts, whatever the codebook groups.  K: one codebook per head: every entry
// 256 / (2 v) times in a row of 256 bytes, lane l reads copy l, again without conflicts; more: a table per sub-vector.
//
// Work.  A workgroup of 8 wavefronts (one per compute unit, for its LDS) belongs to a cache head and takes an equal share of the head's
// work.  A request's rows are cut into blocks of 256 / ways rows; in a block `ways` wavefronts share 32 rows and take every ways-th tile of keys
// (a round: one tile per wavefront), so that few rows fill the workgroup and many are not joined at the end.  Blocks of a request go in pairs (the last with the
// first, ...), whose rounds add up to nearly the same number C: the work before a block is a product, not a sum, and every workgroup finds its share
// with one scan over the requests.  A block cut by a share's border leaves its sums in ws, and attn_paged_merge_kernel joins them in order.
#include <cfloat>
#include <climits>
#include <type_traits>

#include "vq_common.h"

namespace vq {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 8, kThreads = kWaves * 64;
constexpr int kSide = 65536;                  // LDS of a side's codebooks
constexpr int kJoinOff = 2 * kSide;           // sums of wavefronts that share rows, 2 KiB each
constexpr int kStatOff = kJoinOff + 16384;    // their maxima and sums of weights, [wave][32] each
constexpr int kScanOff = kStatOff + 2048;
constexpr int kListOff = kScanOff + 256;      // pieces of the share, 64 at a time: their first rounds, and a Piece each
constexpr int kBaseOff = kListOff + 256 + 64 * 64;   // where the codes of the next rounds lie, [wave][64]
constexpr int kLds = kBaseOff + kWaves * 64 * 8;
constexpr float kHeadroom = 6.f, kRise = 8.f; // (log2)

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
    int min_log_ways;   // fewest wavefronts that share 32 rows
    int cut;            // 0: blocks are not cut
    int min_share;      // rounds
    float scale2;       // |sm_scale| log2(e)
    unsigned q_sign;    // sign of sm_scale, in both halves
    float cap_in, cap_out;   // softcap: cap_out - 2 cap_out / (2^(s cap_in) + 1), 0: none
};

__device__ __forceinline__ int token_of(const PagedArgs &a, int row) { return (int)(((unsigned long long)(unsigned)row * a.group_inverse) >> a.group_shift); }

// A request, in numbers that fit no memory access out of bounds.
struct Request {
    int first, n, len, prefix, rows, log_ways, blocks, items, C;
};
// Tiles of 32 keys that some of the tokens [i0, i1] attends: [0, front) and [lo, hi).
struct Tiles {
    int front, lo, hi;
    __device__ int count() const { return front + max(hi - lo, 0); }
};
__device__ __forceinline__ Tiles tiles_of(const PagedArgs &a, const Request &r, int i0, int i1) {
    const int p0 = r.len - r.n + i0, p1 = r.len - r.n + i1;
    Tiles t;
    t.lo = (a.window > 0 && p0 >= a.window ? p0 - a.window + 1 : 0) >> 5;
    t.hi = (max(p1 + 1, r.prefix) + 31) >> 5;
    t.front = min((r.prefix + 31) >> 5, t.lo);
    return t;
}
__device__ __forceinline__ int block_rows(const Request &r) { return (kWaves * 32) >> r.log_ways; }
__device__ __forceinline__ Tiles block_tiles(const PagedArgs &a, const Request &r, int j) {
    const int row = j * block_rows(r);
    return tiles_of(a, r, token_of(a, row), token_of(a, min(row + block_rows(r), r.rows) - 1));
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
    r.blocks = (r.rows + block_rows(r) - 1) / block_rows(r);
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
        pc.row0 = j * block_rows(r);
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
__host__ __device__ __forceinline__ int part_rows(const PagedArgs &a) { return (kWaves * 32) >> a.min_log_ways; }
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

template <int D, int V, bool COPIES, bool MODS>
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
            // tiles of this wavefront's rows, of those of the block
            const int pos_f = pc.pos0 + token_of(a, max(row0, 0)), pos_l = pc.pos0 + token_of(a, max(row0 + tile_rows - 1, 0));
            const int count = tile_rows > 0 ? min(pc.front + max(((max(pos_l + 1, pc.prefix) + 31) >> 5) - pc.lo, 0), pc.count) : 0;
            const float slope2 = MODS && a.slopes ? a.slopes[hq] * kLog2e : 0.f;
            const int see_to = min(pos, pc.len - 1), see_from = a.window > 0 ? pos - a.window + 1 : INT_MIN;

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
                if constexpr (MODS) {   // (two uniform branches: a choice per score would compute both sides)
                    if (a.cap_out > 0.f) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) s[e] = a.cap_out - 2.f * a.cap_out * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[e] * a.cap_in) + 1.f);
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
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int key = t0 + 16 * lh + 4 * (e & 3) + (e >> 2);
                        const bool see = (key <= see_to && key >= see_from) || key < pc.prefix;
                        s[e] = see ? s[e] : -INFINITY;
                    }
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
                if (__ballot(mt > m_ref + kRise)) {
                    const float m_new = mt > m_ref ? mt : m_ref, f = __builtin_amdgcn_exp2f(m_ref - m_new);
                    m_ref = m_new;
                    lsum *= f;
#pragma unroll
                    for (int k = 0; k < CH; ++k)
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[k][e] *= f;
                }
                const float sub = kHeadroom - m_ref;

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

constexpr int kMergeRows = 32;   // of a workgroup
// Joins the sums of the block that worker w's share begins inside, if no worker before it began there too.
template <int D>
__global__ __launch_bounds__(256) void attn_paged_merge_kernel(PagedArgs a) {
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
    if ((int)blockIdx.z * kMergeRows >= block_rows(r) || from <= off || from >= off + rounds || from - sh.share > off) return;
    // pieces: the end of worker w - 1's share, then the beginnings of w's and of those behind it that begin inside the block
    const long long end = sh.u0 - from + min(off + rounds, r.C);
    const int pieces = 1 + (int)((end - sh.u0 + sh.share - 1) / sh.share);
    const int row0 = j * block_rows(r), rows = min(block_rows(r), r.rows - row0);
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

// How a call is cut, from its sizes alone.
struct PagedPlan {
    int workers, min_log_ways, cut;
    size_t ws;
};
PagedPlan paged_plan(const vq_kv_pages_t *kv, const vq_paged_batch_t *b) {
    PagedPlan p;
    p.workers = kv->H >= 256 ? 1 : 256 / kv->H;
    const long long rows = (long long)b->n_tokens * (b->Hq / kv->H) * kv->H;
    p.min_log_ways = rows >= 256 * 1024 ? 0 : rows >= 128 * 1024 ? 1 : 2;
    p.cut = p.workers > 1 && (long long)b->max_pages * kv->page_tokens > 512;
    p.ws = p.cut ? (size_t)kv->H * p.workers * 2 * ((kWaves * 32) >> p.min_log_ways) * (kv->D + 2) * sizeof(float) : 0;
    return p;
}

template <int D, int V, bool COPIES, bool MODS>
int run_paged(const PagedArgs &a, hipStream_t s) {
    static KernelSetup setup;
    if (int st = kernel_setup(reinterpret_cast<const void *>(&attn_paged_kernel<D, V, COPIES, MODS>), kLds, true, setup)) return st;
    attn_paged_kernel<D, V, COPIES, MODS><<<a.H * a.workers, kThreads, kLds, s>>>(a);
    if (a.cut) attn_paged_merge_kernel<D><<<dim3(a.workers - 1, a.H, part_rows(a) / kMergeRows), 256, 0, s>>>(a);
    return launch_status();
}
template <int D, int V>
int run_paged_as(const PagedArgs &a, hipStream_t s) {
    const bool mods = a.cap_out > 0.f || a.slopes;
    if (a.G == 1) return mods ? run_paged<D, V, true, true>(a, s) : run_paged<D, V, true, false>(a, s);
    return mods ? run_paged<D, V, false, true>(a, s) : run_paged<D, V, false, false>(a, s);
}

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
    a.min_log_ways = p.min_log_ways;
    a.cut = p.cut;
    a.min_share = 2;
    const float scale = sm_scale < 0.f ? -sm_scale : sm_scale;
    a.scale2 = scale * kLog2e > FLT_MIN ? scale * kLog2e : FLT_MIN;   // (above zero: minus infinity times it has to stay)
    a.q_sign = sm_scale < 0.f ? 0x80008000u : 0u;
    a.cap_out = b->softcap * kLog2e;
    a.cap_in = b->softcap > 0.f ? 2.f * a.scale2 / b->softcap : 0.f;
    if (kv->D == 64) return kv->v == 8 ? run_paged_as<64, 8>(a, s) : kv->v == 4 ? run_paged_as<64, 4>(a, s) : run_paged_as<64, 2>(a, s);
    return kv->v == 8 ? run_paged_as<128, 8>(a, s) : kv->v == 4 ? run_paged_as<128, 4>(a, s) : run_paged_as<128, 2>(a, s);
}

}  // namespace vq
