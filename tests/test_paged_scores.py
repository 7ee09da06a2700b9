"""Scores of vq_attn_paged where they are hard on the arithmetic: caps of any size, rows beside others, scores of millions, very many small weights."""
import numpy as np
import pytest
import torch

import paged_reference
from test_paged import Case, attend, on_a_wide_table

gpu = pytest.mark.gpu
KERNELS = [dict(v=4), dict(v=2, G=64), dict(v=8, D=64), dict(v=4, G=1, wide=True), dict(v=8, G=8, wide=True)]     # wide: tiles of few rows
REQS = [(120, 23), (17, 0), (700, 1), (64, 3), (3, 8), (0, 0)]


def make(reqs, wide=False, **kw):
    case = Case(reqs, **{**dict(H=2, group=2), **kw})
    return on_a_wide_table(case) if wide else case


# ------------------------------------------------------------------------------------------------ caps

def test_the_capped_reference_is_the_cap_itself():
    """The bound of a capped score by an fp32 emulation of the two forms, and against caps that are none."""
    rng = np.random.Generator(np.random.PCG64(1))
    case = Case([(40, 40)], H=1, softcap=1e30, seed=1)
    free = Case([(40, 40)], H=1, seed=1)
    a, ba = paged_reference.attend(case)
    b, bb = paged_reference.attend(free)
    assert np.abs(a - b).max() <= 1e-12 and (ba <= bb + 1e-5).all()
    f = np.float32
    for cap in (1e-3, 3.0, 30.0, 256.0, 257.0, 1e4, 1e6, 3e38):
        s = rng.normal(0, 2, 4096).astype(np.float32)
        x = s * f(min(2 * 1.4426950408889634 / cap, np.finfo(np.float32).max))
        w = x * x
        scale = f(0.7)                                     # (of the scores, in the polynomial's coefficients)
        c = [f(k) * scale for k in (-4.00369909e-02, 1.91897040e-03, -8.53218143e-05)]
        small = s * (w * (w * (w * c[2] + c[1]) + c[0]) + scale) / scale
        with np.errstate(over="ignore"):
            large = f(cap) - f(2) * (f(cap) / (np.exp2(x) + f(1)))
        got = (small if cap > 256 and np.abs(x).max() <= 1 else large).astype(np.float64)
        want = cap * np.tanh(s.astype(np.float64) / cap)
        top = np.abs(s).max()
        allowed = 6 * 2.0 ** -24 * np.abs(want) + 14 * 2.0 ** -24 * (cap if cap <= 256 else 0 if 2.885 * top < 0.999 * cap else min(cap, 2.9 * top))
        assert (np.abs(got - want) <= allowed).all(), cap


@gpu
@pytest.mark.parametrize("softcap", [1e-42, 1e-30, 0.01, 3.0, 50.0, 256.0, 257.0, 1e4, 1e6, 1e8, 1.2e38, 3.0e38, float(np.finfo(np.float32).max)])
@pytest.mark.parametrize("kw", KERNELS)
def test_a_cap_of_any_size(gpu_device, softcap, kw):
    """A large cap is none, a small one leaves equal scores; zero scores stay zero under both."""
    case = make(REQS, seed=3, softcap=softcap, sigma=2.0, extra_rows=2, **kw)
    case.q[2] = 0
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("softcap", [2.0, 40.0, 1e5])
@pytest.mark.parametrize("kw", KERNELS)
@pytest.mark.parametrize("mods", [dict(window=20, prefix=[5, 0, 300, 40, 0, 1]), dict(slopes=[0.5, 0.01, 2.0, -0.02], prefix=[90, 9, 2, 64, 0, 65], window=17), dict(sm_scale=-0.6), dict(sm_scale=0.0)])
def test_caps_with_masks_and_biases(gpu_device, softcap, kw, mods):
    case = make(REQS, seed=4, softcap=softcap, sigma=3.0, extra_rows=1, **kw, **mods)
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("softcap", [257.0, 600.0])
@pytest.mark.parametrize("kw", KERNELS)
@pytest.mark.parametrize("mods", [dict(), dict(window=20, prefix=[5, 0, 300, 40, 0, 1]), dict(slopes=[0.5, 0.01, 2.0, -0.02])])
def test_scores_on_both_sides_of_a_large_cap(gpu_device, softcap, kw, mods):
    """Scores of hundreds beside small ones: lanes of a wavefront take either form of the cap."""
    case = make(REQS, seed=5, softcap=softcap, sigma=10.0, sm_scale=0.6, extra_rows=1, **kw, **mods)
    case.q[1::3] *= np.float16(0.125)
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("softcap", [2.0, 40.0, 300.0, 1e5])
@pytest.mark.parametrize("kw", KERNELS)
def test_capped_rows_ignore_what_they_do_not_attend(gpu_device, softcap, kw):
    """Codes behind a request's end that name large or infinite entries: the very same bits."""
    case = make([(37, 5), (100, 1), (16, 2), (31, 3)], E=199, seed=13, softcap=softcap, **kw)
    base = attend(case, gpu_device)
    k_cb, v_cb = case.k_cb, case.v_cb
    for value in (300.0, np.inf, np.nan):
        more = np.full(k_cb.shape[:2] + (57, case.v), value, np.float16)
        case.k_cb, case.v_cb = np.concatenate([k_cb, more], 2), np.concatenate([v_cb, more], 2)
        assert torch.equal(attend(case, gpu_device), base), value


# ------------------------------------------------------------------------------------------------ rows and their neighbours

@gpu
@pytest.mark.parametrize("mods", [dict(), dict(softcap=30.0), dict(softcap=300.0, sm_scale=3.0), dict(slopes=[0.0, 0.01, 0.0, 0.02])])
@pytest.mark.parametrize("kw", KERNELS)
def test_a_row_does_not_depend_on_its_neighbours_queries(gpu_device, kw, mods):
    """Every other row's query changes, to one whose scores grow from tile to tile and to ones of other sizes: the rest keep every bit."""
    case = make([(1501, 13), (90, 3)], v=kw["v"], **{k: x for k, x in kw.items() if k != "v"}, seed=6, **mods)
    order = np.argsort(case.values(case.K_codes[0], case.k_cb)[:, 0] @ case.q[0, 0].astype(np.float64))
    case.K_codes[0] = case.K_codes[0][order]
    t = np.arange(1501)
    case.k_codes[case.table[0, t // 16], :, t % 16] = case.K_codes[0]
    q = case.q.copy()
    base = attend(case, gpu_device)
    paged_reference.check(case, base)
    direction = q[0, 0].astype(np.float32)
    for scale in (0.0, 1.5, 6.0):
        for odd in (0, 1):
            case.q = q.copy()
            rows = case.q[odd::2]
            rows[:] = (direction * scale).astype(np.float16)
            assert torch.equal(attend(case, gpu_device)[1 - odd::2], base[1 - odd::2]), (scale, odd)


# ------------------------------------------------------------------------------------------------ large scores, small weights

def exact_case(kw, n, level, seed):
    """Scores that are whole multiples of `level`: the queries are one in one channel, the entries multiples of level there and zero elsewhere."""
    case = make([(n, 3), (70, 1)], seed=seed, **kw)
    case.q[:] = 0
    case.q[:, :, 0] = 1024
    rng = np.random.Generator(np.random.PCG64(seed))
    case.k_cb[:] = 0
    case.k_cb[..., 0] = rng.integers(-8, 9, case.k_cb.shape[:3]) * level
    case.k_cb[:, :, 0, 0] = 8 * level
    case.sm_scale = 1.0
    return case


@gpu
@pytest.mark.parametrize("kw", KERNELS)
@pytest.mark.parametrize("level", [2.0 ** 7, 2.0 ** 10, 2.0 ** 12])
@pytest.mark.parametrize("sm_scale", [1.0, 0.7, 30.0, -0.7])
@pytest.mark.parametrize("softcap", [0.0, 1e30])
def test_scores_of_millions_and_more(gpu_device, kw, level, sm_scale, softcap):
    """Finite inputs give finite outputs: the keys of the largest score share the weight, the others, far below, have none."""
    case = exact_case(kw, 900, level, 5)
    case.sm_scale, case.softcap = sm_scale, softcap
    got = attend(case, gpu_device).float().cpu().numpy().astype(np.float64)
    for b, (ln, n) in enumerate(case.reqs):
        K, V = case.values(case.K_codes[b], case.k_cb), case.values(case.V_codes[b], case.v_cb)
        for i in range(n):
            for hq in range(case.H * case.group):
                s = sm_scale * K[:ln - n + i + 1, hq // case.group, 0]
                top = s == s.max()
                val = V[:ln - n + i + 1, hq // case.group][top]
                # every weight is the same half, so their rounding cancels: the sum of products, its parts and the output are rounded
                bound = 2.0 ** -11 * np.abs(val.mean(0)) + (len(val) + 8) * 2.0 ** -24 * np.abs(val).mean(0) + 2.0 ** -25
                assert (np.abs(got[case.cu[b] + i, hq] - val.mean(0)) <= bound).all(), (b, i, hq)


@gpu
@pytest.mark.parametrize("kw", KERNELS)
@pytest.mark.parametrize("bits", [19.0, 21.5, 24.25, 27.5])
@pytest.mark.parametrize("first", [True, False])
def test_many_small_weights_beside_a_large_one(gpu_device, kw, bits, first):
    """One key of weight 1 and thousands of 2^-bits: as halves those are subnormal, and together they count."""
    n = 20000
    case = make([(n, 1)], **{**dict(H=1, group=1), **kw}, E=2, seed=8)
    P = case.D // case.v
    case.q[:] = 1
    case.k_cb[:] = 0
    case.k_cb[:, :, 1] = 0.25
    case.v_cb[:] = -30.0
    case.v_cb[:, :, 1] = 1.0
    case.sm_scale = bits * np.log(2) / (0.25 * case.D)
    one = np.zeros((n, 1, P), np.uint8)
    one[0 if first else n - 1] = 1
    case.K_codes = case.V_codes = [one]
    t = np.arange(n)
    case.k_codes[case.table[0, t // 16], :, t % 16] = one
    case.v_codes[case.table[0, t // 16], :, t % 16 // 16, :, t % 16] = one
    paged_reference.check(case, attend(case, gpu_device))
