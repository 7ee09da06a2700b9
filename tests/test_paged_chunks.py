"""vq_attn_paged with the row counts of prompts, and with hundreds of requests on tables that blocks are cut on.

How many wavefronts share 32 rows follows the rows of the call, those behind the last request among them, so a padded q of a few
hundred live rows takes the paths of a prompt's chunk: from 40960 rows of all heads on two share, from 98304 on none does."""
import pytest
import torch

import paged_reference
import paper_2503_02236_amd as vq
from test_paged import Case, attend, on_a_wide_table

gpu = pytest.mark.gpu


def padded(reqs, rows, cut=True, **kw):
    """A case of at least `rows` rows of all heads, on a table of more (cut) or less than 1536 tokens; the workspace tells how it is taken."""
    heads = kw.get("H", 2) * kw.get("group", 1)
    live = sum(n for _, n in reqs)
    case = Case(reqs, extra_rows=max(-(-rows // heads) - live, 0), **kw)
    if cut and case.table.shape[1] * case.ps <= 1536:
        wide = torch.full((len(reqs), 1536 // case.ps + 1), -1, dtype=torch.int32).numpy()
        wide[:, :case.table.shape[1]] = case.table
        case.table = wide
    if not cut:
        case.table = case.table[:, :1536 // case.ps].copy()     # (without the column behind the longest request)
    assert (case.table.shape[1] * case.ps > 1536) == cut
    return case


def plan_is(case, device, block):
    """The workspace is that of blocks of `block` rows (0: whole ones)."""
    kv, q, table = case.dev(device)[:3]
    assert vq.vq_attn_paged_workspace(kv, q, table) == case.H * (256 // case.H) * 2 * block * (case.D + 2) * 4


SHARED = {64: 2000, 128: 40960, 256: 98304}       # rows of a cut block: at least this many rows of all heads


@gpu
@pytest.mark.parametrize("rows,block", [(40959, 64), (40960, 128), (98303, 128), (98304, 256)])
def test_the_rows_where_the_sharing_changes(gpu_device, rows, block):
    case = padded([(700, 300), (40, 40), (3, 1)], rows, H=1, D=64, v=8, seed=rows % 7)
    plan_is(case, gpu_device, block)
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("block", [64, 128, 256])
@pytest.mark.parametrize("cut", [True, False])
@pytest.mark.parametrize("kw", [
    dict(H=8, group=4, v=4), dict(H=8, group=3, v=8, G=16), dict(H=4, group=2, v=2, G=64), dict(H=2, group=5, D=64, v=8), dict(H=4, group=1, D=64, v=4, G=16),
    dict(H=2, group=7, D=64, v=2, ps=64), dict(H=32, group=1, v=4, G=32, ps=32), dict(H=3, group=4, v=2, G=1)])
def test_chunks_of_every_sharing(gpu_device, block, cut, kw):
    """Chunks of one to several blocks, whole prompts, and single tokens among them."""
    case = padded([(1500, 290), (129, 129), (33, 33), (700, 1), (257, 65), (1, 1)], SHARED[block], cut, seed=block + kw["v"], **kw)
    plan_is(case, gpu_device, block if cut else 0)
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("block", [128, 256])
@pytest.mark.parametrize("cut", [True, False])
@pytest.mark.parametrize("mods", [dict(window=100), dict(window=33, prefix=[400, 1, 70, 0]), dict(window=300, prefix=[1300, 90, 0, 40]), dict(prefix=[1000, 129, 5, 300]),
                                  dict(slopes=[0.02, 0.3, 0.001, 0.0, -0.01, 0.1], softcap=20.0), dict(softcap=3.0, window=64, prefix=[40, 40, 40, 40])])
@pytest.mark.parametrize("kw", [dict(v=4, group=3), dict(v=2, group=3), dict(v=8, D=64, group=3, G=8)])
def test_chunks_with_masks(gpu_device, block, cut, mods, kw):
    """Windows and prefixes make a block's tiles two ranges, whose number grows, stays or falls from block to block; the group divides no block."""
    case = padded([(1400, 500), (129, 129), (70, 3), (300, 200)], SHARED[block], cut, H=2, seed=block, **kw, **mods)
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("block,v", [(128, 2), (256, 2), (128, 4), (256, 4), (256, 8)])
def test_long_chunks_are_cut_and_joined(gpu_device, block, v):
    """Blocks of many rounds, cut by several shares: sums of 128 and 256 rows in the workspace, joined by more workgroups a block."""
    case = padded([(6000, 300), (2500, 600), (900, 20)], SHARED[block], H=1, group=2, D=64 if v == 8 else 128, v=v, seed=v)
    plan_is(case, gpu_device, block)
    out = attend(case, gpu_device)
    paged_reference.check(case, out)
    assert torch.equal(attend(case, gpu_device), out)


@gpu
@pytest.mark.parametrize("block", [128, 256])
def test_chunks_whose_first_rows_see_nothing(gpu_device, block):
    case = padded([(200, 400), (0, 130), (300, 0), (150, 150)], SHARED[block], H=2, group=2, seed=2, window=50)
    out = attend(case, gpu_device)
    paged_reference.check(case, out)
    assert bool((out[:200] == 0).all()) and bool((out[400:530] == 0).all())


# ------------------------------------------------------------------------------------------------ many requests on a wide table

def lens_of(B, longest):
    return [1 + (37 * b * b + 11 * b) % longest for b in range(B)]


@gpu
@pytest.mark.parametrize("B", [65, 256, 257, 300, 513, 1100])
@pytest.mark.parametrize("kw", [dict(D=64, v=8, group=2), dict(v=2, group=1, G=64), dict(v=4, group=4, G=32)])
def test_many_requests_are_cut_and_joined(gpu_device, B, kw):
    """The joining launch looks for its share among more requests than it has threads."""
    lens = lens_of(B, 120)
    lens[B // 2], lens[B - 1], lens[3] = 1700, 900, 0
    case = padded([(ln, min(ln, 1 + b % 3)) for b, ln in enumerate(lens)], 0, H=1, seed=B, **kw)
    kv, q, table = case.dev(gpu_device)[:3]
    assert vq.vq_attn_paged_workspace(kv, q, table) > 0
    paged_reference.check(case, attend(case, gpu_device))


@gpu
@pytest.mark.parametrize("B", [65, 257, 700, 1100])
@pytest.mark.parametrize("kw", [dict(v=8, group=4, H=2), dict(v=4, group=1, H=4, G=32), dict(v=4, group=5, H=1)])
def test_many_requests_of_few_rows_are_cut_and_joined(gpu_device, B, kw):
    lens = lens_of(B, 150)
    lens[B // 3], lens[B - 2], lens[5] = 2100, 1000, 0
    case = Case([(ln, min(ln, 1)) for ln in lens], seed=B, **kw)
    W = max(case.table.shape[1], -(-(1 << 21) // (B * case.H * case.ps)))
    wide = torch.full((B, W), -1, dtype=torch.int32).numpy()
    wide[:, :case.table.shape[1]] = case.table
    case.table = wide
    plan_is(case, gpu_device, 16)
    paged_reference.check(case, attend(case, gpu_device))


@gpu
def test_a_prompt_among_decoding_requests(gpu_device):
    """A chunk of hundreds of tokens beside a hundred requests of one, in tiles of few rows and in wide ones."""
    reqs = [(50 + 7 * b, 1) for b in range(100)] + [(700, 333)] + [(30, 1)] * 5
    case = Case(reqs, H=2, group=2, seed=4)
    wide = on_a_wide_table(Case(reqs, H=2, group=2, seed=4))
    paged_reference.check(case, attend(case, gpu_device))
    paged_reference.check(wide, attend(wide, gpu_device))
