"""vq_kv_quantize_paged by each of its kernels: what a call takes is asserted, codes are the oracle's."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2503_02236_amd as vq
from paper_2503_02236_amd.binding import vq_kv_pages_t
from test_paged import P16, run_quantize

gpu = pytest.mark.gpu


def plan(H, D, v, G, E, n):
    """(kernel, variant, tokens per workgroup, workgroups that share them) of a call: what the library itself goes by."""
    kv = vq_kv_pages_t(H=H, D=D, v=v, n_entries=E, cb_groups=G, n_pages=4, page_tokens=16, k_codes=P16, v_codes=P16, k_codebooks=P16, v_codebooks=P16)
    out = (ctypes.c_int * 5)()
    vq.lib()._ZN2vq25kv_quantize_paged_plan_ofEPK13vq_kv_pages_tiPi(ctypes.byref(kv), n, out)
    kernel = ("scan", "lane", "matrix")[out[0]]
    return kernel, ("pair", "own", "norms")[out[1]] if kernel == "matrix" else out[1], out[2], out[4]


def slots_of(n, n_pages, ps, rng):
    """A run of consecutive slots from an odd one on, then any order, with padding and slots out of range among it."""
    slots = np.concatenate([np.arange(3, 3 + n // 2), rng.permutation(np.arange(3 + n // 2, n_pages * ps))[:n - n // 2]]).astype(np.int64)
    if n > 3:
        slots[n // 3], slots[n - 1], slots[n // 2] = -1, n_pages * ps, -(1 << 31)
    return slots


CASES = [
    # a lane an item, a lane four items (v 2 and 4), several lanes an item
    (8, 128, 4, 1, 2, 1, "lane", 0), (8, 128, 4, 1, 8, 5, "lane", 0), (8, 128, 4, 1, 4, 31, "lane", 0), (8, 128, 8, 1, 8, 3, "lane", 0), (8, 128, 8, 1, 8, 1999, "lane", 0),
    (8, 128, 4, 1, 8, 2000, "lane", 4), (8, 128, 4, 1, 4, 64, "lane", 4), (8, 128, 4, 1, 2, 201, "lane", 4), (8, 128, 2, 1, 4, 1999, "lane", 4), (8, 128, 2, 8, 8, 64, "lane", 4),
    (8, 128, 2, 8, 8, 2003, "lane", 4),
    # the scan: alone and shared, one to four tokens a workgroup
    (8, 128, 4, 32, 256, 1, "scan", 0), (8, 128, 4, 32, 256, 16, "scan", 0), (8, 128, 4, 32, 256, 65, "scan", 0), (8, 128, 4, 32, 256, 103, "scan", 0), (16, 128, 4, 32, 256, 67, "scan", 0), (8, 128, 4, 4, 256, 48, "scan", 0), (8, 128, 2, 64, 256, 17, "scan", 0), (8, 128, 2, 64, 256, 63, "scan", 0),
    (8, 128, 8, 16, 256, 15, "scan", 0), (32, 128, 4, 1, 256, 1, "scan", 0),
    # the matrix cores, by every way of looking at the best entries
    (8, 128, 4, 32, 256, 301, "matrix", "pair"), (8, 128, 8, 16, 256, 300, "matrix", "pair"), (3, 40, 2, 4, 8, 333, "matrix", "pair"), (2, 72, 8, 3, 8, 700, "matrix", "own"),
    (16, 128, 4, 1, 250, 301, "matrix", "own"), (16, 128, 4, 1, 256, 1501, "matrix", "norms"), (16, 128, 4, 1, 64, 299, "matrix", "norms"), (32, 128, 4, 1, 256, 1100, "matrix", "norms")]


@gpu
@pytest.mark.parametrize("ps,stride_rows", [(16, 0), (64, 3)])
@pytest.mark.parametrize("H,D,v,G,E,n,kernel,variant", CASES)
def test_codes_by_every_kernel(gpu_device, H, D, v, G, E, n, kernel, variant, ps, stride_rows):
    assert plan(H, D, v, G, E, n)[:2] == (kernel, variant)
    n_pages = -(-n // ps) + 4
    run_quantize(gpu_device, H, D, v, G, E, ps, n, slots_of(n, n_pages, ps, np.random.Generator(np.random.PCG64(n + ps))), n_pages, seed=n + D, stride_rows=stride_rows)


def test_the_scan_takes_one_to_several_tokens_alone_and_shared():
    seen = {plan(*c[:6])[2:] for c in CASES if c[6] == "scan"}
    assert {t for t, _ in seen} >= {1, 2, 4} and {s for _, s in seen} >= {1, 2, 4}


@gpu
@pytest.mark.parametrize("v,E,n", [(4, 8, 2000), (2, 4, 1999), (8, 8, 1999), (4, 8, 5)])
def test_lanes_on_hard_values(gpu_device, v, E, n):
    """Infinities, NaN, zeros and ties by the lane kernels: the lowest index of the smallest distance, entry 0 where there is none."""
    H, D = 8, 128
    assert plan(H, D, v, 1, E, n)[:2] == ("lane", 4 if v <= 4 and n > 100 else 0)
    g = np.random.Generator(np.random.PCG64(n + v))
    x = [g.normal(0, 1, (n, H, D)).astype(np.float16) for _ in range(2)]
    for a in x:
        flat = a.reshape(-1)
        at = g.permutation(flat.size)[:max(8, flat.size // 50)]
        flat[at] = g.choice(np.array([np.nan, np.inf, -np.inf, 0.0, 65504.0, 6e-8], np.float16), at.size)
    cb = [np.round(g.normal(0, 1, (H, 1, E, v))).astype(np.float16) for _ in range(2)]
    run_quantize(gpu_device, H, D, v, 1, E, 16, n, np.arange(n) + 5, -(-(n + 5) // 16), seed=1, x=x, cb=cb)


@gpu
@pytest.mark.parametrize("D,v,G,E,kernel,variant", [(64, 8, 1, 8, "lane", 0), (64, 4, 1, 2, "lane", 4), (64, 8, 8, 100, "matrix", "own"), (64, 8, 1, 16, "matrix", "norms")])
def test_the_most_tokens_by_the_oracle(gpu_device, D, v, G, E, kernel, variant):
    """2^20 tokens, of which all but a few are padding."""
    n, at = 1 << 20, [0, 17, 127, 128, 65535, 65536, 777777, (1 << 20) - 1]
    assert plan(1, D, v, G, E, n)[:2] == (kernel, variant)
    rng = np.random.Generator(np.random.PCG64(3))
    cb = [rng.normal(0, 1, (1, G, E, v)).astype(np.float16) for _ in range(2)]
    few = rng.normal(0, 1, (2, len(at), 1, D)).astype(np.float16)
    x = torch.zeros((2, n, 1, D), dtype=torch.float16, device=gpu_device)
    x[:, at] = torch.from_numpy(few).to(gpu_device)
    slots = torch.full((n,), -1, dtype=torch.int32, device=gpu_device)
    slots[at] = torch.arange(20, 20 + len(at), dtype=torch.int32, device=gpu_device)
    k = torch.full((4, 1, 16, D // v), 201, dtype=torch.uint8, device=gpu_device)
    val = torch.full((4, 1, 1, D // v, 16), 201, dtype=torch.uint8, device=gpu_device)
    vq.vq_kv_quantize_paged(vq.VQKVPagesDev(1, D, v, 16, k, val, *(torch.from_numpy(c).to(gpu_device) for c in cb)), x[0], x[1], slots)
    torch.cuda.synchronize()
    want_k, want_v = np.full((64, D // v), 201, np.uint8), np.full((64, D // v), 201, np.uint8)
    for want, xs, c in ((want_k, few[0], cb[0]), (want_v, few[1], cb[1])):
        want[20:20 + len(at)] = oracle.kv_quantize(np.ascontiguousarray(xs.transpose(1, 0, 2))[None], c)[0][0]
    assert np.array_equal(k.cpu().numpy().reshape(64, -1), want_k)
    assert np.array_equal(val.cpu().numpy().transpose(0, 1, 2, 4, 3).reshape(64, -1), want_v)
