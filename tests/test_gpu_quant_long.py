"""8-bit prefill and shared prefixes where one work-group walks many key tiles in one go: its page numbers, held for 16
tiles at a time, are exchanged on the way once and more."""
import math

import numpy as np
import pytest
import torch

from paged_cases import attention_bound
from paper_2406_14909_amd import moa as M
from quant_cases import pack

pytestmark = pytest.mark.gpu

TILE, ROWS, GROUPS, TILE_COST = 64, 128, 512, 192      # keys, query rows, work-groups for pieces, a row tile's own cost


def _say(*a):
    print("[case]", *a, flush=True)


def _int(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _pool(pages, page, d, rng, gen):
    k, v = (pack(torch.randn((pages, page, d), generator=gen).bfloat16(), rng) for _ in range(2))
    cache = [torch.from_numpy(x[0]).cuda().view(torch.float8_e4m3fn) for x in (k, v)]
    cache.append(torch.from_numpy(np.stack((k[1], v[1]), -1).astype(np.float32)).cuda())
    return cache, [torch.from_numpy(x[2]).cuda().view(pages * page, d) for x in (k, v)]


def _attend(q, k, v, seen, scale):
    """(o, a, s) in fp64 of rows q [n, d] over keys k, v [m, d] where seen [n, m]."""
    sc = scale * (q @ k.t().contiguous())
    sc = sc.masked_fill(~seen, -math.inf)
    top = sc.amax(1, keepdim=True)
    w = torch.where(seen, (sc - torch.where(top > -math.inf, top, 0.0)).exp(), 0.0)
    total = w.sum(1, keepdim=True)
    w = w / torch.where(total > 0, total, 1.0)
    size = scale * (q.abs() @ k.abs().t().contiguous())
    return w @ v, w @ v.abs(), torch.where(seen, size, 0.0).amax(1)


def _check(got, ref, d, keys):
    o, a, s = (x.cpu().numpy() for x in ref)
    err, bound = np.abs(got.double().cpu().numpy() - o), attention_bound(o, a, s, torch.bfloat16, d, keys)
    worst = float((err / np.maximum(bound, 1e-30)).max())
    assert np.isfinite(err).all() and worst <= 1.0, worst


def _costs(pos, n, windows, s, step, capacity):
    """Cost of each row tile, as the split counts it."""
    out = []
    for w in windows:
        most = min(w + step + s + 64, capacity, pos + n)
        out += [TILE_COST + min(min(pos, capacity) + step * (i + 1), most) for i in range(-(-n // step))]
    return np.array(out)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 64), (128, 16), (64, 256)])
@pytest.mark.parametrize("form,pos,n,windows,s,width", [
    ("short", 600, 1400, (1600, 1920), 5, 2000),             # nothing is cut: no row tile can be longer than these
    ("whole", 2400, 3200, (2300, 2800), 70, 6000),           # nothing is cut: there are enough row tiles
    ("pieces", 6000, 1024, (5800, 6500), 3, 7200),
])
def test_prefill(form, pos, n, windows, s, width, d, page):
    _say("long prefill", form, d, page)
    rng, gen = np.random.default_rng(pos), torch.Generator().manual_seed(pos)
    group, hkv = 8, 2
    many = 3 if form == "short" else 1                 # sequences
    hq, step, cap = group * hkv, ROWS // group, -(-width // page) * page
    costs = np.concatenate([_costs(pos, n, windows, s, step, cap)] * many)
    whole = (costs.max() - (1700 if 4 * len(costs) >= 3 * GROUPS else 1200)) * GROUPS <= costs.sum()
    keys = (costs.max() - TILE_COST) // TILE
    if form == "short":
        most = min(max(windows) + step + s + 64, cap)
        assert many * (n * group // ROWS + 1) * hkv > 400 and TILE_COST + most <= 2200 and keys > 16
    elif form == "whole":
        assert whole and keys > 33
    else:
        assert not whole and costs.sum() // GROUPS // TILE > 16
    plan = M.moa_plan(hq, hkv, d, s, max(windows), "bf16", [float(w) for w in windows], [0.0] * hkv)
    per, held = cap // page, -(-(pos + n) // page)
    pages = many * hkv * held + 3
    cache, (k, v) = _pool(pages, page, d, rng, gen)
    table = rng.choice(np.array([-1, -2 ** 31, 2 ** 31 - 1, pages]), (many, hkv, per))
    table[:, :, :held] = rng.permutation(pages)[:many * hkv * held].reshape(many, hkv, held)
    gone = rng.random((many, hkv, per)) < 0.1                 # absent pages, all along the way
    table = np.where(gone, rng.choice(np.array([-1, pages]), table.shape), table)
    q = torch.randn((many * n, hq, d), generator=gen).bfloat16().cuda()
    at, start = _int([pos] * many), _int(np.arange(many + 1) * n)
    got = M.moa_quant_prefill(plan, q, *cache, _int(table), at, start, M.new_paged_workspace(plan, many, many * n).fill_(0xFF))
    p, j = torch.arange(pos, pos + n, device="cuda")[:, None], torch.arange(pos + n, device="cuda")
    for b in range(many):
        for g, w in enumerate(windows):
            number = torch.from_numpy(table[b, g]).cuda()[j // page]
            there = (number >= 0) & (number < pages)
            row = torch.where(there, number, 0) * page + j % page
            seen = (j <= p) & ((j < s) | (j > p - w)) & there
            for h in range(g * group, (g + 1) * group):
                rows = slice(b * n, (b + 1) * n)
                ref = _attend(q[rows, h].double(), k[row], v[row], seen, 1 / math.sqrt(d))
                _check(got[rows, h], ref, d, pos + n)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_shared_prefix(d, page):
    _say("long shared prefix", d, page)
    rng, gen = np.random.default_rng(d), torch.Generator().manual_seed(d)
    b, group, hkv, s, prefix, windows = 1024, 8, 2, 3, 4200, (4500, 4400)
    hq, tiles = group * hkv, b * group // ROWS
    longest = max(2, -(-2 * -(-prefix // TILE) * tiles // 256))
    assert longest >= 33 and 2 * -(-(-(-prefix // TILE)) // longest) * tiles <= 256        # pieces of 33 key tiles
    plan = M.moa_plan(hq, hkv, d, s, max(windows), "bf16", [float(w) for w in windows], [0.0] * hkv)
    held, per = -(-prefix // page), -(-(prefix + 40) // page) + 1
    own = per - prefix // page
    pages = hkv * held + b * hkv * own
    cache, (k, v) = _pool(pages, page, d, rng, gen)
    order = rng.permutation(pages)
    shared = np.full((hkv, per), -1)
    shared[:, :held] = order[:hkv * held].reshape(hkv, held)
    shared = np.where(rng.random(shared.shape) < 0.1, pages, shared)
    table = np.full((b, hkv, per), -1)
    table[:, :, prefix // page:] = order[hkv * held:].reshape(b, hkv, own)
    at = prefix + rng.integers(0, 40, b)
    at[[5, 700]] = -1
    q = torch.randn((b, hq, d), generator=gen).bfloat16().cuda()
    o = torch.full_like(q, 7.0)
    M.moa_quant_decode_shared(plan, q, *cache, _int(shared), prefix, _int(table), _int(at),
                              M.new_paged_workspace(plan, b, b).fill_(0xFF), o=o)
    assert bool((o[[5, 700]] == 7.0).all())
    live = np.nonzero(at >= 0)[0]
    i, p = torch.from_numpy(live).cuda(), torch.from_numpy(at[live]).cuda()[:, None]
    j = torch.arange(prefix + 40, device="cuda")
    mine = torch.from_numpy(table).cuda()
    for g, w in enumerate(windows):
        number = torch.from_numpy(shared[g]).cuda()[j[:prefix] // page]
        there = (number >= 0) & (number < pages)
        row = torch.where(there, number, 0) * page + j[:prefix] % page
        seen = ((j[:prefix] < s) | (j[:prefix] > p - w)) & there
        behind = mine[i, g][:, j[prefix:] // page] * page + j[prefix:] % page                # [live, 40]
        seen = torch.cat((seen, j[prefix:] <= p), 1)
        for h in range(g * group, (g + 1) * group):
            x = q[i, h].double()
            front = x @ k[row].t().contiguous()
            back = (x[:, None] * k[behind]).sum(-1)
            scale = 1 / math.sqrt(d)
            sc = (scale * torch.cat((front, back), 1)).masked_fill(~seen, -math.inf)
            weight = torch.softmax(sc, 1)
            mean = lambda f: weight[:, :prefix] @ f(v[row]) + (weight[:, prefix:, None] * f(v[behind])).sum(1)
            size = scale * torch.cat((x.abs() @ k[row].abs().t().contiguous(), (x[:, None] * k[behind]).abs().sum(-1)), 1)
            _check(o[i, h], (mean(lambda y: y), mean(torch.abs), torch.where(seen, size, 0.0).amax(1)), d, prefix + 40)


@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_no_numbers_far_into_a_row_tile(d):
    """They reach the rows that see them and no others, also where the tile is taken again behind an exchange."""
    _say("long prefill, NaN", d)
    rng, gen = np.random.default_rng(d), torch.Generator().manual_seed(d)
    page, pos, n, windows, s, group, hkv = 16, 2400, 3200, (2300, 2800), 70, 8, 2
    costs = _costs(pos, n, windows, s, ROWS // group, 6000)
    assert (costs.max() - 1700) * GROUPS <= costs.sum() and 4 * len(costs) >= 3 * GROUPS
    plan = M.moa_plan(hkv * group, hkv, d, s, max(windows), "bf16", [float(w) for w in windows], [0.0] * hkv)
    held = (pos + n) // page
    cache, (k, v) = _pool(hkv * held, page, d, rng, gen)
    table = rng.permutation(hkv * held).reshape(1, hkv, held)
    where = [(0, 40, 3), (0, 1500, 5), (1, 2700, d - 1), (1, 4900, 0)]          # head, position, dimension
    bad = torch.zeros((hkv, pos + n, d), dtype=torch.bool, device="cuda")
    for g, j, e in where:
        row = int(table[0, g, j // page]) * page + j % page
        cache[1].view(torch.uint8).view(-1, d)[row, e] = 0x7F | (0x80 if e else 0)
        v[row, e], bad[g, j, e] = 0.0, True
    q = torch.randn((n, hkv * group, d), generator=gen).bfloat16().cuda()
    got = M.moa_quant_prefill(plan, q, *cache, _int(table), _int([pos]), _int([0, n]), M.new_paged_workspace(plan, 1, n).fill_(0xFF))
    p, j = torch.arange(pos, pos + n, device="cuda")[:, None], torch.arange(pos + n, device="cuda")
    for g, w in enumerate(windows):
        row = torch.from_numpy(table[0, g]).cuda()[j // page] * page + j % page
        seen = (j <= p) & ((j < s) | (j > p - w))
        hit = (seen.float() @ bad[g].float()) > 0                                  # [n, d]
        assert bool(hit.any()) and not bool(hit.all())
        for h in range(g * group, (g + 1) * group):
            same = torch.equal(torch.isnan(got[:, h]), hit)
            assert same, h
            ref = _attend(q[:, h].double(), k[row], v[row], seen, 1 / math.sqrt(d))
            _check(torch.where(hit, ref[0].float().bfloat16(), got[:, h]), ref, d, pos + n)
