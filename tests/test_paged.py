"""The paged VQ cache (vq_kv_pages_assign, vq_kv_quantize_paged, vq_attn_paged): refusals on the CPU, results on the GPU.

Definitions, written out once more and slowly: pages by a walk over the requests, codes by the oracle of vq_kv_quantize, attention
by a dense softmax in 64 bits whose hidden tokens are left out (not weighted with zero)."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2503_02236_amd as vq
from paper_2503_02236_amd.binding import vq_kv_pages_t, vq_page_step_t, vq_paged_batch_t

VQ_ERR_NULL, VQ_ERR_SHAPE, VQ_ERR_UNSUPPORTED, VQ_ERR_ALIGN, VQ_ERR_WORKSPACE = -1, -2, -3, -4, -5
P16 = 0x10000   # an aligned fake device address, never dereferenced on the error paths
gpu = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ refusals (no GPU)

def pages(**kw):
    d = dict(H=2, D=128, v=4, n_entries=256, cb_groups=1, n_pages=8, page_tokens=16, k_codes=P16, v_codes=P16, k_codebooks=P16, v_codebooks=P16)
    d.update(kw)
    return vq_kv_pages_t(**d)


def step(**kw):
    d = dict(B=2, max_pages=4, page_tokens=16, n_pages=8, n_tokens=5, new_lens=P16, lens=P16, block_table=P16, free_pages=P16, n_free=P16, seq_lens=P16,
             n_free_out=P16, cu_new=P16, slots=P16, positions=P16, status=P16)
    d.update(kw)
    return vq_page_step_t(**d)


def batch(**kw):
    d = dict(B=2, max_pages=4, n_tokens=5, Hq=4, block_table=P16, cu_new=P16, seq_lens=P16, prefix_lens=None, slopes=None, window=0, softcap=0.0)
    d.update(kw)
    return vq_paged_batch_t(**d)


BAD_PAGES = [
    (dict(k_codes=None), VQ_ERR_NULL), (dict(v_codebooks=None), VQ_ERR_NULL), (dict(H=-1), VQ_ERR_SHAPE), (dict(D=0), VQ_ERR_SHAPE),
    (dict(v=3), VQ_ERR_UNSUPPORTED), (dict(n_entries=257), VQ_ERR_UNSUPPORTED), (dict(n_entries=0), VQ_ERR_UNSUPPORTED), (dict(cb_groups=3), VQ_ERR_SHAPE),
    (dict(D=512), VQ_ERR_UNSUPPORTED), (dict(n_pages=-1), VQ_ERR_SHAPE), (dict(page_tokens=8), VQ_ERR_SHAPE), (dict(page_tokens=24), VQ_ERR_SHAPE),
    (dict(page_tokens=512), VQ_ERR_SHAPE), (dict(page_tokens=0), VQ_ERR_SHAPE), (dict(page_tokens=-16), VQ_ERR_SHAPE),
    (dict(n_pages=1 << 27, page_tokens=16), VQ_ERR_SHAPE), (dict(v_codes=P16 + 8), VQ_ERR_ALIGN)]


@pytest.mark.parametrize("kw,want", BAD_PAGES)
def test_page_descriptor_validation(kw, want):
    lib, kv = vq.lib(), pages(**kw)
    assert lib.vq_kv_quantize_paged(ctypes.byref(kv), P16, 256, P16, 256, P16, 1, None) == want
    assert lib.vq_attn_paged(ctypes.byref(kv), ctypes.byref(batch()), P16, 512, 1.0, P16, 512, P16, 1 << 30, None) == want
    assert lib.vq_attn_paged_workspace(ctypes.byref(kv), ctypes.byref(batch())) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(B=-1), VQ_ERR_SHAPE), (dict(B=65537), VQ_ERR_SHAPE), (dict(max_pages=0), VQ_ERR_SHAPE), (dict(B=65536, max_pages=32768), VQ_ERR_SHAPE),
    (dict(max_pages=1 << 27), VQ_ERR_SHAPE), (dict(n_tokens=-1), VQ_ERR_SHAPE), (dict(n_tokens=(1 << 20) + 1), VQ_ERR_SHAPE),
    (dict(page_tokens=17), VQ_ERR_SHAPE), (dict(n_pages=-1), VQ_ERR_SHAPE), (dict(n_pages=1 << 27), VQ_ERR_SHAPE)]
    + [({k: None}, VQ_ERR_NULL) for k in ("new_lens", "lens", "block_table", "free_pages", "n_free", "seq_lens", "n_free_out", "cu_new", "slots", "status")]
    + [({k: P16 + 2}, VQ_ERR_ALIGN) for k in ("new_lens", "lens", "block_table", "free_pages", "n_free", "seq_lens", "n_free_out", "cu_new", "slots",
                                              "positions", "status")])
def test_assign_validation(kw, want):
    assert vq.lib().vq_kv_pages_assign(ctypes.byref(step(**kw)), None) == want


def test_assign_without_a_descriptor():
    assert vq.lib().vq_kv_pages_assign(None, None) == VQ_ERR_NULL


def test_quantize_paged_validation():
    lib, kv = vq.lib(), pages()
    call = lambda k=P16, ks=256, v=P16, vs=256, slots=P16, n=3, kv=kv: lib.vq_kv_quantize_paged(ctypes.byref(kv), k, ks, v, vs, slots, n, None)  # noqa: E731
    assert lib.vq_kv_quantize_paged(None, P16, 256, P16, 256, P16, 1, None) == VQ_ERR_NULL
    assert call(k=None) == VQ_ERR_NULL and call(v=None) == VQ_ERR_NULL and call(slots=None) == VQ_ERR_NULL
    assert call(n=-1) == VQ_ERR_SHAPE and call(n=(1 << 20) + 1) == VQ_ERR_SHAPE
    assert call(ks=248) == VQ_ERR_SHAPE and call(vs=0) == VQ_ERR_SHAPE and call(ks=(1 << 23) + 8) == VQ_ERR_SHAPE
    assert call(ks=260) == VQ_ERR_ALIGN and call(vs=257) == VQ_ERR_ALIGN
    assert call(k=P16 + 2) == VQ_ERR_ALIGN and call(v=P16 + 8) == VQ_ERR_ALIGN and call(slots=P16 + 1) == VQ_ERR_ALIGN
    assert call(kv=pages(cb_groups=32, n_entries=256, D=256, v=8), ks=512, vs=512) == VQ_ERR_UNSUPPORTED     # 128 KiB of codebooks
    assert call(kv=pages(v=2, n_entries=3)) == VQ_ERR_UNSUPPORTED                             # 12 bytes of codebook
    assert call(n=0) == 0 and call(n=0, k=None, v=None, slots=None) == 0


def test_attn_paged_validation():
    lib = vq.lib()
    kv = pages()
    size = lambda kv=kv, **kw: lib.vq_attn_paged_workspace(ctypes.byref(kv), ctypes.byref(batch(**kw)))  # noqa: E731

    def call(kv=kv, q=P16, qs=512, out=P16, os_=512, ws=P16, n=1 << 40, **kw):
        return lib.vq_attn_paged(ctypes.byref(kv), ctypes.byref(batch(**kw)), q, qs, 0.1, out, os_, ws, n, None)

    assert lib.vq_attn_paged(ctypes.byref(kv), None, P16, 512, 1.0, P16, 512, None, 0, None) == VQ_ERR_NULL
    for k in ("block_table", "cu_new", "seq_lens"):
        assert call(**{k: None}) == VQ_ERR_NULL
        assert call(**{k: P16 + 2}) == VQ_ERR_ALIGN
    assert call(q=None) == VQ_ERR_NULL and call(out=None) == VQ_ERR_NULL
    for k in ("prefix_lens", "slopes"):
        assert call(**{k: P16 + 1}) == VQ_ERR_ALIGN
    for kw in (dict(B=-1), dict(B=65537), dict(max_pages=0), dict(max_pages=1 << 27), dict(n_tokens=-1), dict(n_tokens=(1 << 20) + 1), dict(Hq=0), dict(Hq=3),
               dict(window=-1), dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=float("inf"))):
        assert call(**kw) == VQ_ERR_SHAPE, kw
        assert size(**kw) == 0
    assert call(qs=504) == VQ_ERR_SHAPE and call(os_=0) == VQ_ERR_SHAPE
    assert call(qs=516) == VQ_ERR_ALIGN and call(os_=513) == VQ_ERR_ALIGN
    assert call(q=P16 + 8) == VQ_ERR_ALIGN and call(out=P16 + 2) == VQ_ERR_ALIGN
    assert call(kv=pages(D=256), qs=1024, os_=1024) == VQ_ERR_UNSUPPORTED
    assert call(kv=pages(D=96), qs=512) == VQ_ERR_UNSUPPORTED
    assert call(kv=pages(H=0)) == VQ_ERR_SHAPE
    need = size()
    if need:
        assert call(ws=None) == VQ_ERR_WORKSPACE and call(n=need - 1) == VQ_ERR_WORKSPACE and call(ws=P16 + 8) == VQ_ERR_ALIGN
    assert call(B=0) == 0 and call(n_tokens=0, q=None, out=None) == 0      # nothing to attend for


def test_binding_refuses_what_does_not_fit():
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        vq.vq_kv_pages_assign(i32(2), i32(2), i32(2, 3), i32(8), i32(1), 16, n_tokens=4, plan=vq.VQPagePlan(2, 4, "cpu"))
    with pytest.raises(ValueError, match="n_tokens or a plan"):
        vq.vq_kv_pages_assign(i32(2), i32(2), i32(2, 3), i32(8), i32(1), 16)
    kv = vq.VQKVPagesDev(2, 128, 4, 16, torch.zeros(8, 2, 16, 32, dtype=torch.uint8), torch.zeros(8, 2, 1, 32, 16, dtype=torch.uint8),
                         torch.zeros(2, 1, 256, 4, dtype=torch.float16), torch.zeros(2, 1, 256, 4, dtype=torch.float16))
    with pytest.raises(ValueError, match="GPU"):
        vq.vq_kv_quantize_paged(kv, torch.zeros(3, 2, 128, dtype=torch.float16), torch.zeros(3, 2, 128, dtype=torch.float16), i32(3))
    with pytest.raises(ValueError, match="GPU"):
        vq.vq_attn_paged(kv, torch.zeros(3, 4, 128, dtype=torch.float16), 1.0, i32(2, 3), i32(3), i32(2))
    bad = vq.VQKVPagesDev(2, 128, 4, 16, kv.k_codes, torch.zeros(8, 2, 16, 32, dtype=torch.uint8), kv.k_codebooks, kv.v_codebooks)
    with pytest.raises(ValueError, match="v_codes must have the shape"):
        bad.desc()


# ------------------------------------------------------------------------------------------------ definitions

def assign_oracle(new, lens, table, free, n_free, ps, cap):
    new, lens, table, free = [int(x) for x in new], [int(x) for x in lens], table.copy(), free.copy()
    B, W = table.shape
    status, seq, cu, slots, positions = [0] * B, list(lens), [0], [], []
    for b in range(B):
        if new[b] < 0:
            for j in range(-(-lens[b] // ps)):
                free[n_free] = table[b, j]
                n_free += 1
            seq[b] = 0
    asked = needed = 0
    top = n_free
    for b in range(B):
        n = max(new[b], 0)
        if n:
            have, want = -(-seq[b] // ps), -(-(seq[b] + n) // ps)
            if want > W:
                status[b] = 1
            else:
                asked += n
                if asked > cap:
                    status[b] = 1
                elif want > have:
                    needed += want - have
                    if needed > top:
                        status[b] = 1
            if status[b]:
                n = 0
            else:
                for j in range(have, want):
                    n_free -= 1
                    table[b, j] = free[n_free]
        for t in range(seq[b], seq[b] + n):
            slots.append(int(table[b, t // ps]) * ps + t % ps)
            positions.append(t)
        seq[b] += n
        cu.append(cu[-1] + n)
    pad = [-1] * (cap - len(slots))
    return dict(cu_new=cu, seq_lens=seq, slots=slots + pad, positions=positions + pad, status=status, table=table, free=free, n_free=n_free)


class Case:
    """A pool and a batch on the host.  reqs: (tokens in the cache, new tokens) of every request; codes behind a request's length, and in pages
    of nobody, are any bytes."""

    def __init__(self, reqs, H=2, group=1, D=128, v=4, G=1, E=256, ps=16, seed=0, spare=3, extra_rows=0, window=0, softcap=0.0, slopes=None, prefix=None,
                 sm_scale=None, sigma=1.0):
        g = np.random.Generator(np.random.PCG64(seed + 77))
        self.reqs, self.H, self.group, self.D, self.v, self.G, self.E, self.ps = reqs, H, group, D, v, G, E, ps
        self.window, self.softcap, self.prefix = window, softcap, prefix
        self.sm_scale = D ** -0.5 if sm_scale is None else sm_scale
        P, B, Hq = D // v, len(reqs), H * group
        counts = [-(-ln // ps) for ln, _ in reqs]
        self.n_pages = sum(counts) + spare
        perm = g.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((B, max(counts + [1]) + 1), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = perm[at:at + c]
            at += c
        self.k_codes = g.integers(0, 256, (self.n_pages, H, ps, P), dtype=np.uint8)
        self.v_codes = g.integers(0, 256, (self.n_pages, H, ps // 16, P, 16), dtype=np.uint8)
        self.K_codes, self.V_codes = [], []     # [T][H][P] per request
        for b, (ln, _) in enumerate(reqs):
            t = np.arange(ln)
            pg, off = self.table[b, t // ps], t % ps
            kc, vc = g.integers(0, E, (ln, H, P), dtype=np.uint8), g.integers(0, E, (ln, H, P), dtype=np.uint8)
            self.k_codes[pg, :, off] = kc
            self.v_codes[pg, :, off // 16, :, off % 16] = vc
            self.K_codes.append(kc)
            self.V_codes.append(vc)
        f16 = lambda *s: (g.normal(0, sigma, s)).astype(np.float16)  # noqa: E731
        self.k_cb, self.v_cb = f16(H, G, E, v), f16(H, G, E, v)
        self.cu = np.concatenate([[0], np.cumsum([n for _, n in reqs])]).astype(np.int32)
        self.seq = np.array([ln for ln, _ in reqs], np.int32)
        self.rows = int(self.cu[-1])
        self.q = g.normal(0, 1, (self.rows + extra_rows, Hq, D)).astype(np.float16)
        self.slopes = None if slopes is None else np.asarray(slopes, np.float32)
        self.prefix_lens = None if prefix is None else np.asarray(prefix, np.int32)

    def dev(self, device, layout="plain"):
        t = lambda a: None if a is None else torch.from_numpy(a).to(device)  # noqa: E731
        kv = vq.VQKVPagesDev(self.H, self.D, self.v, self.ps, t(self.k_codes), t(self.v_codes), t(self.k_cb), t(self.v_cb))
        q = t(self.q)
        if layout == "strided":
            wide = torch.full((q.shape[0], q.shape[1] + 3, self.D), float("nan"), dtype=torch.float16, device=device)
            wide[:, 1:1 + q.shape[1]] = q
            q = wide[:, 1:1 + q.shape[1]]
        return kv, q, t(self.table), t(self.cu), t(self.seq), dict(window=self.window, softcap=self.softcap, slopes=t(self.slopes), prefix_lens=t(self.prefix_lens))

    def values(self, codes, cb):
        P = self.D // self.v
        g = np.arange(P) // (P // self.G)
        h = np.arange(self.H)[None, :, None]
        return cb.astype(np.float64)[h, g[None, None], codes].reshape(codes.shape[0], self.H, self.D)

    def attend(self):
        """(out, bound on the error of an fp32 computation with fp16 weights) [rows][Hq][D], 64 bits.

        Bound: the output's rounding, half a step 2^-11 of it; every weight rounded to a half (2^-11) and wrong by its score's error s,
        a factor of e^s - 1 in the weight and in the sum of weights.  A score is a sum of D exact products in fp32 in some order, D + 2
        roundings of 2^-24 of sum |q k|, scaled; a capped one is off by 8 roundings of the cap more, a biased one by 4 of the
        bias; 2^x and the difference to the maximum by 4 of the score itself.  Weights below 2^-31 of the largest may vanish."""
        Hq = self.H * self.group
        out, bound = np.zeros((self.rows, Hq, self.D)), np.zeros((self.rows, Hq, self.D))
        for b, (ln, n) in enumerate(self.reqs):
            K, V = self.values(self.K_codes[b], self.k_cb), self.values(self.V_codes[b], self.v_cb)
            t = np.arange(ln)
            for i in range(n):
                pos = ln - n + i
                see = t <= pos
                if self.window:
                    see &= t > pos - self.window
                if self.prefix is not None:
                    see |= t < self.prefix[b]
                if not see.any():
                    continue
                for hq in range(Hq):
                    h = hq // self.group
                    qv, k, val = self.q[self.cu[b] + i, hq].astype(np.float64), K[see, h], V[see, h]
                    s = self.sm_scale * (k @ qv)
                    ds = abs(self.sm_scale) * (self.D + 2) * 2.0 ** -24 * (np.abs(k) @ np.abs(qv))
                    if self.softcap:
                        s = self.softcap * np.tanh(s / self.softcap)
                        ds = ds + 8 * 2.0 ** -24 * self.softcap
                    if self.slopes is not None:
                        s = s - float(self.slopes[hq]) * np.abs(pos - t[see])
                        ds = ds + 4 * 2.0 ** -24 * abs(float(self.slopes[hq])) * np.abs(pos - t[see])
                    ds = ds + 4 * 2.0 ** -24 * (np.abs(s) + np.abs(s).max())
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    o = p @ val
                    r = self.cu[b] + i
                    out[r, hq] = o
                    e = np.expm1(ds)
                    bound[r, hq] = (2.0 ** -11 * np.abs(o) + (p * (2.0 ** -11 + e)) @ np.abs(val) + (p @ (2.0 ** -11 + e)) * np.abs(o)
                                    + len(s) * 2.0 ** -31 * np.abs(val).max() + 2.0 ** -25)
        return out, bound * 1.01      # (products of the small terms)


def check(case, got):
    want, bound = case.attend()
    got = got.float().cpu().numpy().astype(np.float64)[:case.rows]
    assert np.isfinite(got).all()
    worst = np.abs(got - want) / np.maximum(bound, 1e-30)
    at = np.unravel_index(np.argmax(worst), worst.shape) if worst.size else None
    assert worst.size == 0 or worst[at] <= 1.0, (at, worst[at], got[at], want[at])


def attend(case, device, layout="plain"):
    kv, q, table, cu, seq, mods = case.dev(device, layout)
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device=device)
    got = vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, out=out, **mods)
    torch.cuda.synchronize()
    assert got is out and bool((out[case.rows:] == 7.0).all())     # rows behind the last request stay
    return out


# ------------------------------------------------------------------------------------------------ pages

def run_assign(device, new, lens, table, free, n_free, ps, cap, in_place=False):
    t = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=device)  # noqa: E731
    new, lens, table, free, n_free = t(new), t(lens), t(table), t(free), t([n_free])
    plan = vq.VQPagePlan(new.shape[0], cap, device, seq_lens=lens if in_place else None)
    out = None if in_place else torch.full_like(n_free, 99)
    vq.vq_kv_pages_assign(new, lens, table, free, n_free, ps, plan=plan, n_free_out=out)
    torch.cuda.synchronize()
    n = lambda x: x.cpu().numpy()  # noqa: E731
    return dict(cu_new=n(plan.cu_new), seq_lens=n(plan.seq_lens), slots=n(plan.slots), positions=n(plan.positions), status=n(plan.status), table=n(table),
                free=n(free), n_free=int((n_free if in_place else out).item()))


def check_assign(got, want):
    for k in want:
        assert np.array_equal(np.asarray(got[k]), np.asarray(want[k])), k


def pool(rng, lens, ps, W, spare):
    """A table whose rows hold the pages of these lengths, the free list and the number of free pages."""
    counts = [-(-ln // ps) for ln in lens]
    n_pages = sum(counts) + spare
    perm = rng.permutation(n_pages)
    table, at = np.full((len(lens), W), -5, np.int32), 0
    for b, c in enumerate(counts):
        table[b, :c] = perm[at:at + c]
        at += c
    free = np.full(n_pages, -7, np.int32)
    free[:spare] = perm[at:]
    return table, free, spare


@gpu
@pytest.mark.parametrize("B,ps,longest,chunk,gone,spare,cap,in_place", [
    (1, 16, 40, 1, 0.0, 2, 1, False), (1, 16, 1, 16, 0.0, 1, 16, True), (5, 16, 64, 17, 0.3, 9, 64, True), (64, 32, 300, 3, 0.2, 40, 200, False),
    (257, 16, 90, 40, 0.1, 500, 4000, False), (300, 64, 500, 200, 0.5, 30, 9000, True),      # the pool runs out
    (100, 16, 50, 30, 0.1, 4000, 500, False),                                                 # more tokens than the step takes
    (1024, 16, 100, 9, 0.2, 900, 6000, True), (1025, 128, 400, 60, 0.1, 700, 30000, False), (2600, 16, 40, 5, 0.3, 600, 9000, True)])
def test_assign_matches_a_walk_over_the_requests(gpu_device, B, ps, longest, chunk, gone, spare, cap, in_place):
    rng = np.random.Generator(np.random.PCG64(B * 31 + ps))
    lens = rng.integers(0, longest + 1, B)
    lens[rng.random(B) < 0.2] //= ps
    new = rng.integers(0, chunk + 1, B)
    new[rng.random(B) < gone] = -1
    W = -(-longest // ps) + chunk // ps // 2 + 1          # some rows are too short
    table, free, n_free = pool(rng, lens, ps, W, spare)
    want = assign_oracle(new, lens, table, free, n_free, ps, cap)
    check_assign(run_assign(gpu_device, new, lens, table, free, n_free, ps, cap, in_place), want)


@gpu
@pytest.mark.parametrize("new,lens,W,spare,cap", [
    ([], [], 1, 3, 4), ([0, 0], [0, 5], 2, 1, 4), ([-1, -1], [33, 0], 3, 0, 0), ([16, 1], [0, 16], 2, 2, 17), ([16, 1], [0, 16], 2, 1, 17),
    ([3, 3, 3], [14, 14, 14], 2, 2, 9), ([3, 0, 3], [14, 14, 12], 2, 0, 9), ([40, 1], [0, 3], 2, 9, 50), ([2, 2, 1], [0, 0, 0], 1, 9, 3),
    ([2 ** 31 - 1, 1, 2 ** 31 - 1], [5, 5, 0], 4, 9, 8), ([5], [0], 1, 0, 5), ([0, -1], [17, 31], 4, 0, 0)])
def test_assign_small_and_refused(gpu_device, new, lens, W, spare, cap):
    rng = np.random.Generator(np.random.PCG64(5))
    table, free, n_free = pool(rng, lens, 16, W, spare)
    table = table.reshape(len(lens), W)
    want = assign_oracle(new, lens, table, free, n_free, 16, cap)
    check_assign(run_assign(gpu_device, new, lens, table, free, n_free, 16, cap), want)


@gpu
def test_assign_bounds_values_that_no_step_produces(gpu_device):
    """Lengths beyond the row, a free count beyond the pool, page ids out of range: nothing is read or written out of bounds."""
    got = run_assign(gpu_device, [1, 0, 2, -3], [-4, 100, 15, 10 ** 9], np.array([[50, 3], [0, 1], [-9, 2], [7, 7]], np.int32),
                     np.array([4, 5, 6, 9, 9, 9], np.int32), 77, 16, 6)
    # n_free is 6, and two more pages do not fit the list; lens are 0, 32, 15, gone
    assert got["status"].tolist() == [0, 0, 0, 0] and got["cu_new"].tolist() == [0, 1, 1, 3, 3]
    assert got["seq_lens"].tolist() == [1, 32, 17, 0] and got["n_free"] == 4
    assert got["table"].tolist()[0][0] == 9 and got["slots"].tolist()[0] == -1      # page 9 of 6
    assert got["slots"].tolist()[1] == -1 and got["table"].tolist()[2] == [-9, 9]   # page -9


# ------------------------------------------------------------------------------------------------ codes into pages

def run_quantize(device, H, D, v, G, E, ps, n, slots, n_pages, seed, stride_rows=0, cb=None, x=None):
    g = np.random.Generator(np.random.PCG64(seed))
    P = D // v
    k_cb, v_cb = (g.normal(0, 1, (H, G, E, v)).astype(np.float16) for _ in range(2)) if cb is None else cb
    k, val = (g.normal(0, 1, (n, H, D)).astype(np.float16) for _ in range(2)) if x is None else x
    k_codes, v_codes = g.integers(0, 256, (n_pages, H, ps, P), dtype=np.uint8), g.integers(0, 256, (n_pages, H, ps // 16, P, 16), dtype=np.uint8)
    want_k, want_v = k_codes.copy(), v_codes.copy()
    kc = oracle.kv_quantize(np.ascontiguousarray(k.transpose(1, 0, 2))[None], k_cb)[0]      # [H][n][P]
    vc = oracle.kv_quantize(np.ascontiguousarray(val.transpose(1, 0, 2))[None], v_cb)[0]
    for i, s in enumerate(slots):
        if 0 <= s < n_pages * ps:
            want_k[s // ps, :, s % ps] = kc[:, i]
            want_v[s // ps, :, s % ps // 16, :, s % 16] = vc[:, i]
    t = lambda a: torch.from_numpy(a).to(device)  # noqa: E731
    kd, vd = t(k), t(val)
    if stride_rows:
        wide = torch.full((n, 2 * H + stride_rows, D), float("nan"), dtype=torch.float16, device=device)
        wide[:, :H], wide[:, H + stride_rows:] = kd, vd
        kd, vd = wide[:, :H], wide[:, H + stride_rows:]
    kv = vq.VQKVPagesDev(H, D, v, ps, t(k_codes), t(v_codes), t(k_cb), t(v_cb))
    vq.vq_kv_quantize_paged(kv, kd, vd, torch.tensor(np.asarray(slots), dtype=torch.int32, device=device))
    torch.cuda.synchronize()
    assert np.array_equal(kv.k_codes.cpu().numpy(), want_k)
    assert np.array_equal(kv.v_codes.cpu().numpy(), want_v)


@gpu
@pytest.mark.parametrize("H,D,v,G,E,ps,n,stride_rows", [
    (1, 128, 4, 1, 256, 16, 1, 0), (32, 128, 4, 1, 256, 16, 1, 2), (8, 128, 4, 32, 256, 16, 64, 0), (3, 128, 4, 4, 100, 32, 33, 1), (2, 64, 8, 1, 256, 64, 257, 0),
    (5, 64, 2, 32, 256, 128, 65, 3), (2, 128, 2, 64, 256, 16, 150, 0), (4, 128, 8, 16, 32, 16, 100, 1), (2, 128, 4, 1, 8, 16, 700, 0), (2, 128, 8, 1, 6, 256, 300, 5),
    (16, 128, 4, 1, 256, 16, 1500, 1), (1, 256, 8, 2, 64, 32, 40, 0), (2, 40, 2, 4, 16, 16, 50, 1), (2, 72, 8, 3, 256, 16, 600, 0)])
def test_quantize_paged_codes(gpu_device, H, D, v, G, E, ps, n, stride_rows):
    rng = np.random.Generator(np.random.PCG64(n))
    n_pages = -(-n // ps) + 4
    # a run of consecutive slots from an odd one on, then any order, with padding among it
    slots = np.concatenate([np.arange(3, 3 + n // 2), rng.permutation(np.arange(3 + n // 2, n_pages * ps))[:n - n // 2]]).astype(np.int64)
    if n > 3:
        slots[n // 3] = -1
        slots[n - 1] = n_pages * ps       # also out of range
    run_quantize(gpu_device, H, D, v, G, E, ps, n, slots, n_pages, seed=n + D, stride_rows=stride_rows)


@gpu
@pytest.mark.parametrize("v,G,n", [(4, 1, 3), (4, 32, 40), (8, 1, 300), (2, 1, 300)])
def test_quantize_paged_hard_values(gpu_device, v, G, n):
    """Infinities, NaN, zeros and ties take the definition's answers: the lowest index of the smallest distance, entry 0 where there is none."""
    g = np.random.Generator(np.random.PCG64(n + v))
    H, D, E = 2, 128, 256
    x = [g.normal(0, 1, (n, H, D)).astype(np.float16) for _ in range(2)]
    for a in x:
        flat = a.reshape(-1)
        at = g.permutation(flat.size)[:max(8, flat.size // 50)]
        flat[at] = g.choice(np.array([np.nan, np.inf, -np.inf, 0.0, 65504.0, 6e-8], np.float16), at.size)
    cb = [np.round(g.normal(0, 1, (H, G, E, v)) * 2).astype(np.float16) / 2 for _ in range(2)]     # many equal entries
    run_quantize(gpu_device, H, D, v, G, E, 16, n, np.arange(n) + 5, -(-(n + 5) // 16), seed=1, x=x, cb=cb)


@gpu
@pytest.mark.parametrize("D,v,G,E", [(64, 8, 8, 100), (64, 8, 1, 256), (64, 8, 1, 16)])
def test_quantize_paged_most_tokens(gpu_device, D, v, G, E):
    """2^20 tokens, of which all but a few are padding; each of the kernels."""
    n, at = 1 << 20, [0, 17, 65535, 65536, 777777, (1 << 20) - 1]
    rng = np.random.Generator(np.random.PCG64(3))
    cb = [torch.from_numpy(rng.normal(0, 1, (1, G, E, v)).astype(np.float16)).to(gpu_device) for _ in range(2)]
    x = torch.zeros((n, 1, D), dtype=torch.float16, device=gpu_device)
    x[at] = torch.from_numpy(rng.normal(0, 1, (len(at), 1, D)).astype(np.float16)).to(gpu_device)
    slots = torch.full((n,), -1, dtype=torch.int32, device=gpu_device)
    slots[at] = torch.arange(20, 20 + len(at), dtype=torch.int32, device=gpu_device)
    got = []
    for xs, sl in ((x, slots), (x[at], slots[at])):
        k = torch.full((4, 1, 16, D // v), 201, dtype=torch.uint8, device=gpu_device)
        val = torch.full((4, 1, 1, D // v, 16), 201, dtype=torch.uint8, device=gpu_device)
        vq.vq_kv_quantize_paged(vq.VQKVPagesDev(1, D, v, 16, k, val, *cb), xs, xs, sl)
        got.append((k, val))
    torch.cuda.synchronize()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert int((got[0][0] != 201).any(-1).sum()) == len(at)


# ------------------------------------------------------------------------------------------------ attention

@gpu
@pytest.mark.parametrize("lens", [[1], [2, 15, 16, 17], [31, 32, 33, 63, 64, 65], [255, 256, 257, 300], [1000, 1, 511]])
@pytest.mark.parametrize("D,v,G,group", [(128, 4, 1, 1), (128, 4, 32, 4), (64, 8, 1, 3), (128, 2, 64, 1), (128, 8, 16, 8), (64, 2, 32, 5), (64, 4, 4, 1), (128, 8, 1, 1), (128, 2, 1, 2)])
def test_attend_single_tokens(gpu_device, lens, D, v, G, group):
    case = Case([(ln, 1) for ln in lens], D=D, v=v, G=G, group=group, seed=len(lens) + D + v)
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("reqs,kw", [
    ([(7, 7)], {}), ([(33, 33), (64, 31)], dict(group=1)), ([(70, 32)], dict(group=3, H=1)), ([(300, 65)], dict(H=1, group=1)), ([(200, 200)], dict(H=1, group=2)),
    ([(513, 130)], dict(H=1, group=1, G=32)), ([(140, 5), (3, 3), (90, 33), (1, 1), (260, 1)], dict(group=4, ps=32)),
    ([(400, 300)], dict(H=1, D=64, v=4, G=16)), ([(150, 70), (40, 40)], dict(D=64, v=8, group=2)), ([(150, 70), (40, 40)], dict(v=2, G=64, ps=64)),
    ([(150, 70), (40, 40)], dict(v=8, G=4, E=100, ps=128)), ([(333, 77)], dict(H=3, E=17, v=8, G=2, ps=256))])
def test_attend_chunks(gpu_device, reqs, kw):
    case = Case(reqs, seed=len(reqs), extra_rows=2, **kw)
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=16), dict(window=33), dict(window=100000), dict(window=20, prefix=[5, 0, 300, 40]), dict(prefix=[70, 1, 33, 1000]),
                                dict(softcap=5.0), dict(softcap=30.0, window=40), dict(slopes=True), dict(slopes=True, prefix=[90, 9, 2, 64], window=17, softcap=2.0),
                                dict(sm_scale=-0.3), dict(sm_scale=0.0), dict(sm_scale=1.5), dict(sm_scale=0.0, window=3, prefix=[1, 2, 3, 4])])
@pytest.mark.parametrize("G", [1, 32])
def test_attend_masks_and_scores(gpu_device, kw, G):
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = [0.5, 0.01, 2.0, -0.02]
    case = Case([(120, 70), (17, 17), (200, 1), (64, 3)], H=2, group=2, G=G, seed=3, **kw)
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("window", [0, 5])
def test_attend_rows_that_see_nothing_are_zero(gpu_device, window):
    """An empty request, one without new tokens, and one whose length is below its number of new tokens (rows before its first token)."""
    case = Case([(0, 0), (20, 0), (3, 8), (0, 4), (40, 2)], window=window, group=2, seed=9, extra_rows=3)
    out = attend(case, gpu_device)
    check(case, out)
    assert bool((out[:5] == 0).all()) and bool((out[8:12] == 0).all()) and bool((out[5] != 0).any())


@gpu
@pytest.mark.parametrize("reqs,kw", [
    ([(9000, 1)], dict(H=1, group=1)), ([(5000, 3), (12000, 1), (40, 1)], dict(H=2, group=2, G=32)), ([(3000, 40)], dict(H=1, group=4, ps=64)),
    ([(4000, 1)] * 5 + [(100, 1)] * 3, dict(H=1, group=8, v=8)), ([(2500, 70)], dict(H=1, D=64, v=2, G=1, softcap=20.0, slopes=[0.001])),
    ([(6000, 5)], dict(H=1, group=1, window=2500, prefix=[100], v=2, G=64))])
def test_attend_long_requests(gpu_device, reqs, kw):
    case = Case(reqs, seed=11, **kw)
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("H,group", [(5, 1), (40, 1), (300, 1), (7, 3), (1, 40)])
def test_attend_head_counts(gpu_device, H, group):
    case = Case([(50, 3), (200, 1)], H=H, group=group, D=64, v=8, seed=H)
    check(case, attend(case, gpu_device))


# Requests of few rows on tables that may name many pages take narrower tiles: B H max_pages page_tokens of 2^21 and more.
def on_a_wide_table(case):
    W = -(-(1 << 21) // (len(case.reqs) * case.H * case.ps))
    assert case.rows * case.group <= 16 * len(case.reqs) and W >= case.table.shape[1]
    wide = np.full((len(case.reqs), W), -1, np.int32)
    wide[:, :case.table.shape[1]] = case.table
    case.table = wide
    workers = max(256 // case.H, 1)
    kv, q, table = case.dev("cuda")[:3]
    assert vq.vq_attn_paged_workspace(kv, q, table) == case.H * workers * 2 * 16 * (case.D + 2) * 4
    return case


@gpu
@pytest.mark.parametrize("lens", [[1], [2, 15, 16, 17], [31, 32, 33, 63, 64, 65], [127, 128, 129, 511, 512, 513], [1000, 1, 1537]])
@pytest.mark.parametrize("v,G,group,ps", [(4, 1, 1, 16), (4, 32, 3, 16), (8, 1, 16, 64), (8, 16, 5, 32), (4, 8, 9, 128), (8, 2, 2, 16)])
def test_attend_few_rows_single_tokens(gpu_device, lens, v, G, group, ps):
    case = on_a_wide_table(Case([(ln, 1) for ln in lens], v=v, G=G, group=group, ps=ps, seed=len(lens) + v))
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("kw", [dict(window=1), dict(window=63), dict(window=64), dict(window=200), dict(window=20, prefix=[5, 0, 300, 40, 0, 1]),
                                dict(prefix=[70, 1, 33, 1000, 0, 7]), dict(softcap=5.0), dict(softcap=30.0, window=40), dict(slopes=True),
                                dict(slopes=True, prefix=[90, 9, 2, 64, 0, 65], window=17, softcap=2.0), dict(sm_scale=-0.3), dict(sm_scale=0.0), dict(sm_scale=1.5)])
@pytest.mark.parametrize("v,G", [(4, 1), (4, 32), (8, 1), (8, 8)])
def test_attend_few_rows_masks_and_scores(gpu_device, kw, v, G):
    """One of the requests has more rows than a tile, one no new tokens, one rows before its first token."""
    kw = dict(kw)
    if kw.get("slopes"):
        kw["slopes"] = [0.5, 0.01, 2.0, -0.02]
    case = on_a_wide_table(Case([(120, 23), (17, 0), (700, 1), (64, 3), (3, 8), (0, 0)], H=2, group=2, v=v, G=G, seed=3, extra_rows=2, **kw))
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("reqs,kw", [
    ([(9000, 1)], dict(H=1, group=1)), ([(5000, 3), (12000, 1), (40, 1)], dict(H=2, group=2, G=32)), ([(3000, 1), (1, 1)], dict(H=3, group=15, v=8, ps=64)),
    ([(4000, 1)] * 5 + [(100, 1)] * 3, dict(H=1, group=8, v=8)), ([(6000, 5)], dict(H=1, group=1, window=2500, prefix=[100], v=8, G=16)),
    ([(300, 1)] * 70, dict(H=1, group=2)), ([(4000, 40)] + [(50, 1)] * 20, dict(H=1, group=1, v=8)), ([(900, 1)], dict(H=300, group=5, v=8))])
def test_attend_few_rows_long_and_many_requests(gpu_device, reqs, kw):
    case = Case(reqs, seed=11, **kw)
    check(case, attend(on_a_wide_table(case) if case.H < 256 else case, gpu_device))     # (a head per workgroup: five rows are enough)


@gpu
@pytest.mark.parametrize("n", [1, 3])
def test_attend_few_rows_in_whole_blocks(gpu_device, n):
    """Short requests on a short table: no block is cut, and many workgroups of a head have one or none to begin with."""
    case = Case([(5 + 3 * b, n) for b in range(100)] + [(9, 0)], H=16, group=5, v=8, seed=n)
    kv, q, table = case.dev(gpu_device)[:3]
    assert vq.vq_attn_paged_workspace(kv, q, table) == 0 and table.numel() * case.ps * case.H >= 1 << 18
    check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("v,G", [(4, 1), (8, 16)])
def test_attend_few_rows_growing_scores_and_values_that_are_none(gpu_device, v, G):
    """The largest score comes last; codes behind the end name entries that are infinite or NaN; a NaN in a query stays in its row."""
    case = Case([(1501, 2), (90, 1)], H=1, group=2, v=v, G=G, E=200, seed=6, sm_scale=2.0)
    order = np.argsort(case.values(case.K_codes[0], case.k_cb)[:, 0] @ case.q[0, 0].astype(np.float64))
    case.K_codes[0] = case.K_codes[0][order]
    t = np.arange(1501)
    case.k_codes[case.table[0, t // 16], :, t % 16] = case.K_codes[0]
    want = attend(on_a_wide_table(case), gpu_device)
    check(case, want)
    wider = [np.concatenate([cb, np.full((1, G, 56, v), x, np.float16)], 2) for cb, x in ((case.k_cb, np.nan), (case.v_cb, np.inf))]
    case.k_cb, case.v_cb = wider
    assert torch.equal(attend(case, gpu_device), want)     # (256 entries: any byte behind the end is one)
    case.q[1, 1, 3] = np.nan
    got = attend(case, gpu_device)
    assert bool(torch.isnan(got[1, 1]).all())
    got[1, 1] = want[1, 1]
    assert torch.equal(got, want)


@gpu
def test_attend_many_requests(gpu_device):
    rng = np.random.Generator(np.random.PCG64(4))
    case = Case([(int(rng.integers(0, 60)), int(rng.integers(0, 3))) for _ in range(1100)], H=1, group=2, D=64, v=8, seed=4)
    check(case, attend(case, gpu_device))


@gpu
def test_attend_sharp_and_equal_scores(gpu_device):
    """Scores of hundreds (a weight of one and the rest nothing), and a codebook of one entry (all scores equal)."""
    case = Case([(300, 40)], H=1, sigma=8.0, sm_scale=1.0, seed=2)
    check(case, attend(case, gpu_device))
    case = Case([(300, 40)], H=1, E=1, v=8, seed=2)
    check(case, attend(case, gpu_device))


@gpu
def test_attend_growing_scores(gpu_device):
    """The largest score comes last, and every few tiles a larger one: the running maximum rises again and again."""
    case = Case([(1500, 33)], H=1, v=8, G=1, seed=6)
    order = np.argsort(case.values(case.K_codes[0], case.k_cb)[:, 0] @ case.q[0, 0].astype(np.float64))
    case.K_codes[0] = case.K_codes[0][order]
    t = np.arange(1500)
    case.k_codes[case.table[0, t // 16], :, t % 16] = case.K_codes[0]
    case.sm_scale = 2.0
    check(case, attend(case, gpu_device))


@gpu
def test_attend_strided_queries_and_outputs(gpu_device):
    case = Case([(100, 9), (33, 33)], group=2, seed=8)
    a = attend(case, gpu_device)
    b = attend(case, gpu_device, layout="strided")
    assert torch.equal(a, b)
    kv, q, table, cu, seq, mods = case.dev(gpu_device)
    wide = torch.full((q.shape[0], q.shape[1] + 1, case.D), 5.0, dtype=torch.float16, device=gpu_device)
    vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, out=wide[:, 1:], **mods)
    assert torch.equal(wide[:, 1:], a) and bool((wide[:, 0] == 5.0).all())


@gpu
def test_attend_is_repeatable_and_rows_are_independent_of_their_neighbours(gpu_device):
    case = Case([(700, 3), (90, 33), (2000, 1)], group=2, seed=12)
    first = attend(case, gpu_device)
    for _ in range(3):
        assert torch.equal(attend(case, gpu_device), first)
    # NaN and infinity in one query: its own row only
    kv, q, table, cu, seq, mods = case.dev(gpu_device)
    q[1, 1, 5], q[4, 0, 7] = float("nan"), float("inf")
    out = vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, **mods)
    torch.cuda.synchronize()
    hit = torch.zeros(out.shape[:2], dtype=torch.bool, device=gpu_device)
    hit[1, 1], hit[4, 0] = True, True
    assert torch.equal(out[~hit], first[~hit]) and bool(torch.isnan(out[1, 1]).all())


@gpu
@pytest.mark.parametrize("kw", [dict(), dict(G=32), dict(v=2), dict(v=8, G=16), dict(D=64), dict(slopes=[0.1] * 4, prefix=[9, 200, 3, 0])])
def test_attend_ignores_what_it_does_not_attend(gpu_device, kw):
    """Codes and table entries behind a request's length, pages of others; among those codes an entry that is infinite, and codes beyond the codebook."""
    case = Case([(37, 5), (100, 1), (16, 2), (31, 31)], E=199, group=2, seed=13, **kw)
    base = attend(case, gpu_device)
    kv, q, table, cu, seq, mods = case.dev(gpu_device)
    inf = torch.full_like(kv.k_codebooks[:, :, :1], float("inf"))
    kv.k_codebooks, kv.v_codebooks = torch.cat([kv.k_codebooks, inf], 2).contiguous(), torch.cat([kv.v_codebooks, -inf], 2).contiguous()
    used = torch.zeros(kv.k_codes.shape[0], case.ps, dtype=torch.bool)
    for b, (ln, _) in enumerate(case.reqs):
        for t in range(ln):
            used[case.table[b, t // 16], t % 16] = True
    used = used.to(gpu_device)
    table[table < 0] = 2 ** 30
    for junk in (199, 255):
        kv.k_codes.copy_(torch.where(used[:, None, :, None], kv.k_codes, junk))
        kv.v_codes.copy_(torch.where(used.view(-1, 1, 1, 1, 16), kv.v_codes, junk))
        out = vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, **mods)
        assert torch.equal(out, base), junk


@gpu
def test_offsets_beyond_32_bits(gpu_device):
    """Pages whose codes lie more than 4 GiB into the pool, written and attended."""
    H, D, v, ps = 32, 128, 2, 256
    n_pages = 8400                                     # 4.4 GB a side
    case = Case([(300, 2), (600, 1)], H=H, D=D, v=v, ps=ps, G=1, seed=14)
    small, q, table, cu, seq, mods = case.dev(gpu_device)
    kv = vq.VQKVPagesDev(H, D, v, ps, torch.empty((n_pages, H, ps, D // v), dtype=torch.uint8, device=gpu_device),
                         torch.empty((n_pages, H, ps // 16, D // v, 16), dtype=torch.uint8, device=gpu_device), small.k_codebooks, small.v_codebooks)
    shift = n_pages - case.n_pages
    kv.k_codes[shift:] = small.k_codes
    kv.v_codes[shift:] = small.v_codes
    far = torch.where(table >= 0, table + shift, table)
    assert torch.equal(vq.vq_attn_paged(kv, q, case.sm_scale, far, cu, seq), vq.vq_attn_paged(small, q, case.sm_scale, table, cu, seq))
    g = torch.Generator(device=gpu_device)
    g.manual_seed(1)
    x = torch.randn((40, H, D), generator=g, device=gpu_device).half()
    slots = torch.arange(40, dtype=torch.int32, device=gpu_device) + 5
    vq.vq_kv_quantize_paged(small, x, -x, slots)
    vq.vq_kv_quantize_paged(kv, x, -x, slots + shift * ps)
    assert torch.equal(kv.k_codes[shift:], small.k_codes) and torch.equal(kv.v_codes[shift:], small.v_codes)


# ------------------------------------------------------------------------------------------------ together

class Server:
    """Requests over a pool, on the GPU with the three calls, and on the host token by token."""

    def __init__(self, device, B=4, H=2, group=2, D=128, v=4, G=1, E=256, ps=16, n_pages=60, W=12, seed=0, cap=70):
        g = np.random.Generator(np.random.PCG64(seed))
        self.g, self.device, self.B, self.H, self.group, self.D, self.v, self.ps, self.cap = g, device, B, H, group, D, v, ps, cap
        self.k_cb, self.v_cb = (g.normal(0, 1, (H, G, E, v)).astype(np.float16) for _ in range(2))
        t = lambda a: torch.from_numpy(a).to(device)  # noqa: E731
        P = D // v
        self.kv = vq.VQKVPagesDev(H, D, v, ps, torch.zeros((n_pages, H, ps, P), dtype=torch.uint8, device=device),
                                  torch.zeros((n_pages, H, ps // 16, P, 16), dtype=torch.uint8, device=device), t(self.k_cb), t(self.v_cb))
        self.table = torch.full((B, W), -1, dtype=torch.int32, device=device)
        self.free = torch.arange(n_pages, dtype=torch.int32, device=device)
        self.n_free = torch.tensor([n_pages], dtype=torch.int32, device=device)
        self.lens = torch.zeros(B, dtype=torch.int32, device=device)
        self.plan = vq.VQPagePlan(B, cap, device, seq_lens=self.lens)
        self.new = torch.zeros(B, dtype=torch.int32, device=device)
        self.qkv = torch.zeros((cap, H * group + 2 * H, D), dtype=torch.float16, device=device)
        self.out = torch.zeros((cap, H * group, D), dtype=torch.float16, device=device)
        q = self.qkv[:, :H * group]
        need = vq.vq_attn_paged_workspace(self.kv, q, self.table)
        self.ws = vq.new_workspace(need, device)
        self.keys, self.vals = [[] for _ in range(B)], [[] for _ in range(B)]      # codes [H][P] of every token

    def run(self):
        Hq, H = self.H * self.group, self.H
        vq.vq_kv_pages_assign(self.new, self.lens, self.table, self.free, self.n_free, self.ps, plan=self.plan)
        vq.vq_kv_quantize_paged(self.kv, self.qkv[:, Hq:Hq + H], self.qkv[:, Hq + H:], self.plan.slots)
        vq.vq_attn_paged(self.kv, self.qkv[:, :Hq], self.D ** -0.5, self.table, self.plan.cu_new, self.lens, out=self.out, ws=self.ws)

    def inputs(self, new):
        self.new.copy_(torch.tensor(new, dtype=torch.int32))
        self.x = self.g.normal(0, 1, tuple(self.qkv.shape)).astype(np.float16)
        self.qkv.copy_(torch.from_numpy(self.x))
        self.out.fill_(9.0)

    def check(self, new):
        torch.cuda.synchronize()
        Hq, H, P = self.H * self.group, self.H, self.D // self.v
        assert self.plan.status.sum().item() == 0
        k = oracle.kv_quantize(np.ascontiguousarray(self.x[:, Hq:Hq + H].transpose(1, 0, 2))[None], self.k_cb)[0]
        val = oracle.kv_quantize(np.ascontiguousarray(self.x[:, Hq + H:].transpose(1, 0, 2))[None], self.v_cb)[0]
        at, reqs = 0, []
        for b, n in enumerate(new):
            if n < 0:
                self.keys[b], self.vals[b] = [], []
            for i in range(max(n, 0)):
                self.keys[b].append(k[:, at + i])
                self.vals[b].append(val[:, at + i])
            at += max(n, 0)
            reqs.append((len(self.keys[b]), max(n, 0)))
        case = Case(reqs, H=H, group=self.group, D=self.D, v=self.v, G=self.k_cb.shape[1], E=self.k_cb.shape[2], ps=self.ps)
        case.k_cb, case.v_cb, case.q = self.k_cb, self.v_cb, self.x[:, :Hq]
        case.K_codes = [np.array(x, np.uint8).reshape(-1, H, P) for x in self.keys]
        case.V_codes = [np.array(x, np.uint8).reshape(-1, H, P) for x in self.vals]
        assert self.lens.tolist() == [len(x) for x in self.keys]
        check(case, self.out)
        assert bool((self.out[case.rows:] == 9.0).all())
        held = sum(-(-len(x) // self.ps) for x in self.keys)
        assert self.n_free.item() == self.free.shape[0] - held


STEPS = [[20, 0, 1, 33], [1, 40, 1, 1], [1, 1, 1, -1], [5, 1, -1, 17], [1, 1, 30, 1], [-1, 1, 1, 1], [64, 1, 1, 1]]


@gpu
@pytest.mark.parametrize("kw", [dict(), dict(G=32, ps=32), dict(D=64, v=2, group=4), dict(v=8, H=3)])
def test_steps_of_continuous_batching(gpu_device, kw):
    s = Server(gpu_device, **kw)
    for new in STEPS:
        s.inputs(new)
        s.run()
        s.check(new)


@gpu
def test_a_step_is_captured_and_replayed(gpu_device):
    """One graph of a step, replayed with other lengths and inputs, with eager work between the replays."""
    s = Server(gpu_device, seed=3)
    s.inputs(STEPS[0])
    s.run()
    s.check(STEPS[0])
    keep = [t.clone() for t in (s.table, s.free, s.n_free, s.lens, s.kv.k_codes, s.kv.v_codes)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.run()
    for t, old in zip((s.table, s.free, s.n_free, s.lens, s.kv.k_codes, s.kv.v_codes), keep):
        t.copy_(old)
    for new in STEPS[1:]:
        s.inputs(new)
        graph.replay()
        s.check(new)
        torch.ones(1000, device=gpu_device).cumsum(0).sum().item()


@gpu
def test_two_graphs_share_a_workspace(gpu_device):
    a, b = Case([(3000, 2), (50, 1)], H=1, group=2, seed=21), Case([(40, 3), (5000, 1)], H=1, group=2, seed=22)
    dev = [c.dev(gpu_device) for c in (a, b)]
    ws = vq.new_workspace(max(vq.vq_attn_paged_workspace(d[0], d[1], d[2]) for d in dev), gpu_device)
    outs, graphs = [], []
    for c, (kv, q, table, cu, seq, mods) in zip((a, b), dev):
        want = vq.vq_attn_paged(kv, q, c.sm_scale, table, cu, seq, ws=ws, **mods)
        out = torch.empty_like(want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            vq.vq_attn_paged(kv, q, c.sm_scale, table, cu, seq, out=out, ws=ws, **mods)
        graphs.append(g)
        outs.append((out, want))
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for out, want in outs:
            assert torch.equal(out, want)
            out.zero_()


@gpu
def test_calls_follow_the_current_stream(gpu_device):
    case = Case([(500, 3), (70, 1)], seed=15)
    want = attend(case, gpu_device)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        kv, q, table, cu, seq, mods = case.dev(gpu_device)
        q2 = torch.zeros_like(q)
        big = torch.ones(1 << 26, device=gpu_device)
        for _ in range(20):
            big = big * 1.0000001
        q2.copy_(q)                                    # behind the work above, on this stream
        out = vq.vq_attn_paged(kv, q2, case.sm_scale, table, cu, seq, **mods)
    st.synchronize()
    assert torch.equal(out[:case.rows], want[:case.rows])


@gpu
def test_one_request_in_pages_is_the_contiguous_cache(gpu_device):
    """vq_attn_decode over the same codes: within both calls' rounding of the same sums."""
    case = Case([(2000, 1), (700, 1)], H=4, seed=16)
    got = attend(case, gpu_device).float()
    T, P = 2000, 32
    k = np.zeros((2, 4, T, P), np.uint8)
    val = np.zeros_like(k)
    for b in range(2):
        k[b, :, :case.seq[b]], val[b, :, :case.seq[b]] = case.K_codes[b].transpose(1, 0, 2), case.V_codes[b].transpose(1, 0, 2)
    t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(gpu_device)  # noqa: E731
    kd = vq.VQKVDev(2, 4, 128, T, 4, t(k), t(val), t(case.k_cb), t(case.v_cb), t(case.seq))
    want = vq.vq_attn_decode(kd, t(case.q), case.sm_scale).float()
    _, bound = case.attend()
    assert bool(((got - want).abs() <= 2 * torch.from_numpy(bound).to(gpu_device)).all())


@gpu
def test_native_marshalling_does_what_ctypes_does(gpu_device, monkeypatch):
    """The three calls through the native part of the binding and without it: the same results, and the same errors for what does not fit."""
    from paper_2503_02236_amd import binding
    native = binding._marshal
    assert native is not None, "the native part of the binding is not built"
    case = Case([(300, 20), (40, 1)], group=2, seed=31, window=90, softcap=9.0, slopes=[0.01, 0.0, 0.3, 0.02], prefix=[5, 0])
    kv, q, table, cu, seq, mods = case.dev(gpu_device, "strided")
    results = []
    for which in (native, None):
        monkeypatch.setattr(binding, "_marshal", which)
        out = torch.zeros(q.shape, dtype=torch.float16, device=gpu_device)
        assert vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, out=out, **mods) is out
        fresh = vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, **mods)
        codes = vq.VQKVPagesDev(kv.H, kv.D, kv.v, kv.page_tokens, kv.k_codes.clone(), kv.v_codes.clone(), kv.k_codebooks, kv.v_codebooks)
        vq.vq_kv_quantize_paged(codes, q[:, :2], q[:, 2:], torch.arange(21, dtype=torch.int32, device=gpu_device) + 3)
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=gpu_device)  # noqa: E731
        lens, new, tab, free, n_free = i32([3, 40]), i32([20, -1]), i32([[5, -1, -1], [1, 2, 3]]), i32([0, 4, -9, -9, -9, -9]), i32([2])
        plan = vq.VQPagePlan(2, 30, gpu_device)
        assert vq.vq_kv_pages_assign(new, lens, tab, free, n_free, 16, plan=plan) is plan
        results.append([out, fresh, codes.k_codes, codes.v_codes, tab, free, n_free, plan.cu_new, plan.seq_lens, plan.slots, plan.positions, plan.status])
        for bad in (dict(slopes=torch.zeros(3, device=gpu_device)), dict(prefix_lens=cu), dict(out=out[:, :3]), dict(softcap=-1.0), dict(window=-4)):
            with pytest.raises((ValueError, TypeError, vq.VQError)):
                vq.vq_attn_paged(kv, q, case.sm_scale, table, cu, seq, **bad)
        with pytest.raises(ValueError):
            vq.vq_kv_quantize_paged(codes, q[:, :2], q[:, 2:], torch.arange(20, dtype=torch.int32, device=gpu_device))
        with pytest.raises(ValueError):
            vq.vq_kv_quantize_paged(codes, q[:, :3], q[:, :3], torch.arange(21, dtype=torch.int32, device=gpu_device))
        with pytest.raises(TypeError):
            vq.vq_kv_pages_assign(new.long(), lens, tab, free, n_free, 16, plan=plan)
        with pytest.raises(vq.VQError):
            vq.vq_kv_pages_assign(new, lens, tab, free, n_free, 15, plan=plan)
        torch.cuda.synchronize()
    for x, y in zip(*results):
        assert torch.equal(x, y)
