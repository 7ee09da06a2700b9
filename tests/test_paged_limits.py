"""The paged calls at their limits: 65536 requests, 2^20 new tokens, a request of 2^25 tokens; rows picked here and there against 64 bits."""
import numpy as np
import pytest
import torch

import paged_reference
import paper_2503_02236_amd as vq
from test_paged import Case, assign_oracle, attend, check_assign, pool, run_assign

gpu = pytest.mark.gpu


def part(case, reqs, rows, codes):
    """A case of these requests (tokens, new tokens), their rows of q and their (request, first token, end) of the whole one's codes."""
    sub = object.__new__(Case)
    sub.__dict__.update(case.__dict__)
    sub.reqs, sub.q = reqs, case.q[rows]
    sub.K_codes, sub.V_codes = [case.K_codes[b][i:j] for b, i, j in codes], [case.V_codes[b][i:j] for b, i, j in codes]
    sub.cu = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    sub.rows = int(sub.cu[-1])
    return sub


@gpu
@pytest.mark.parametrize("kw", [dict(D=64, v=8, H=1, group=1), dict(D=128, v=8, H=2, group=2)])
def test_attend_the_most_requests(gpu_device, kw):
    B, rng = 65536, np.random.Generator(np.random.PCG64(1))
    lens = rng.integers(0, 20, B)
    lens[777] = 3000
    new = np.minimum(lens, rng.integers(0, 3, B))
    new[777] = 5
    case = Case([(int(a), int(b)) for a, b in zip(lens, new)], seed=3, **kw)
    out = attend(case, gpu_device)
    picks = [0, 1, 776, 777, 778, B - 2, B - 1] + rng.integers(0, B, 300).tolist()
    rows = np.concatenate([np.arange(case.cu[b], case.cu[b + 1]) for b in picks])
    paged_reference.check(part(case, [case.reqs[b] for b in picks], rows, [(b, 0, case.reqs[b][0]) for b in picks]), out[torch.from_numpy(rows).to(gpu_device)])


@gpu
@pytest.mark.parametrize("n_free,cap,in_place", [(70000, 1 << 18, True), (3000, 1 << 16, False), (70000, 50000, True)])
def test_assign_the_most_requests(gpu_device, n_free, cap, in_place):
    B, rng = 65536, np.random.Generator(np.random.PCG64(2))
    lens, new = rng.integers(0, 40, B), rng.integers(-1, 4, B)
    table, free, _ = pool(rng, lens, 16, 5, 70000)
    check_assign(run_assign(gpu_device, new, lens, table, free, n_free, 16, cap, in_place), assign_oracle(new, lens, table, free, n_free, 16, cap))


@gpu
@pytest.mark.parametrize("n,kw", [(1 << 20, dict(window=50, group=1, D=64, v=8)), (1 << 18, dict(window=700, group=2, D=128, v=4, softcap=30.0)), (1 << 17, dict(group=1, D=64, v=8))])
def test_attend_the_most_tokens(gpu_device, n, kw):
    """A whole prompt, of up to 2^20 tokens."""
    case = Case([(n, n)], seed=4, ps=256, H=1, **kw)
    out = attend(case, gpu_device)
    for i in [0, 1, 31, 32, 255, 256, 12345, n // 2, n - 2, n - 1] + np.random.Generator(np.random.PCG64(5)).integers(0, n, 20).tolist():
        first = max(0, i + 1 - kw["window"]) if "window" in kw else 0
        paged_reference.check(part(case, [(i + 1 - first, 1)], slice(i, i + 1), [(0, first, i + 1)]), out[i:i + 1])


@gpu
@pytest.mark.parametrize("kw", [dict(D=64, v=8), dict(D=128, v=8), dict(D=64, v=8, slope=1e-6), dict(D=128, v=8, slope=-3e-7, softcap=4.0)])
def test_attend_a_request_of_2_to_25_tokens(gpu_device, kw):
    """One new token behind 2^25 - 4: positions that fp32 does not hold.  The definition in 64 bits by torch, a piece of the keys at a time."""
    D, v, slope, softcap = kw["D"], kw["v"], kw.get("slope"), kw.get("softcap", 0.0)
    T, ps, E, P = (1 << 25) - 3, 256, 256, D // v
    pages = -(-T // ps)
    g = torch.Generator(device=gpu_device).manual_seed(6)
    k_codes = torch.randint(0, E, (pages, 1, ps, P), generator=g, device=gpu_device, dtype=torch.uint8)
    # values follow the position, so that keys left out or weighted wrongly are seen
    rank = (torch.arange(pages * ps, device=gpu_device) * E // (pages * ps)).to(torch.uint8)
    v_codes = rank.view(pages, 1, ps // 16, 1, 16).expand(pages, 1, ps // 16, P, 16).contiguous()
    books = [torch.randn((1, 1, E, v), generator=g, device=gpu_device).half(), (torch.linspace(-1, 1, E, device=gpu_device)[:, None] * torch.tensor([1.0, -0.5] * (v // 2), device=gpu_device)).half()[None, None].contiguous()]
    kv = vq.VQKVPagesDev(1, D, v, ps, k_codes, v_codes, *books)
    table = torch.arange(pages, dtype=torch.int32, device=gpu_device)[None]
    q = torch.randn((1, 1, D), generator=g, device=gpu_device).half()
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=gpu_device)  # noqa: E731
    slopes = None if slope is None else torch.tensor([slope], dtype=torch.float32, device=gpu_device)
    scale = D ** -0.5
    got = vq.vq_attn_paged(kv, q, scale, table, i32([0, 1]), i32([T]), softcap=softcap, slopes=slopes)[0, 0].double()
    qd, book_k, book_v = q[0, 0].double(), books[0][0, 0].double(), books[1][0, 0].double()
    k_codes = k_codes.view(-1, P)
    m, l, acc, size = -np.inf, 0.0, torch.zeros(D, dtype=torch.float64, device=gpu_device), torch.zeros(D, dtype=torch.float64, device=gpu_device)
    for t0 in range(0, T, 1 << 20):
        t1 = min(t0 + (1 << 20), T)
        s = scale * (book_k[k_codes[t0:t1].long()].reshape(t1 - t0, D) @ qd)
        if softcap:
            s = softcap * torch.tanh(s / softcap)
        if slope is not None:
            s = s - float(slopes[0]) * (T - 1 - torch.arange(t0, t1, device=gpu_device)).double().abs()
        top = max(m, s.max().item())
        p, keep = torch.exp(s - top), np.exp(m - top)
        val = book_v[rank[t0:t1].long()].repeat(1, P)
        m, l, acc, size = top, l * keep + p.sum().item(), acc * keep + p @ val, size * keep + p @ val.abs()
    want, size = acc / l, size / l
    # Weights: 2^-11 each in both sums, scores to 6e-5 (D + 2 roundings of sum |q k| < 60, 4 of a bias below 34, 4 of the score, 14 of a cap of 4: less than
    # 2^-24 (130 60 + 136 + 400 + 56) = 5.1e-4); 2048 wavefronts add T / 2048 products each one after the other, 2^-24
    # each in both sums; 2^-31 of the largest weight for every one.
    bound = 2.0 ** -11 * want.abs() + (2 * 2.0 ** -11 + 2 * 5.1e-4 + 2 * 2.0 ** -24 * T / 2048) * size + T * 2.0 ** -31 / l + 2.0 ** -25
    assert bool(torch.isfinite(got).all()) and bool(((got - want).abs() <= bound).all()), ((got - want).abs() / bound).max().item()
