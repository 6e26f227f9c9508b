"""A cache held in 4 bits: writes and reads against the definition, bit by bit, and attention over it against 64 bits."""
import math

import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as attention
import kv4_util as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def _normal(size, dtype, seed, sigma=1.0):
    return (torch.randn(size, generator=torch.Generator().manual_seed(seed)) * sigma).to(dtype)


def _stored(k, v, page, pages, slots, seed=0):
    """A cache of random bytes with k and v in `slots`, and its bytes from before."""
    heads, D = k.shape[1:]
    cache = torch.randint(0, 256, (pages, fq.kv4_page_bytes(page, heads, D)), dtype=torch.uint8, generator=torch.Generator().manual_seed(seed))
    device = cache.cuda()
    fq.kv4_write(k, v, device, page, slots.cuda())
    return device, cache


# ------------------------------------------------------------------------------------------------ writes and reads
WRITES = [  # tokens, heads, D, page, how the slots lie
    (1, 1, 128, 16, "one"), (3, 2, 64, 16, "behind"), (4, 8, 128, 16, "aligned"), (5, 8, 128, 64, "behind"), (33, 3, 80, 48, "behind"), (64, 2, 96, 32, "any"),
    (200, 1, 8, 16, "any"), (131, 5, 40, 128, "behind"), (77, 2, 120, 32, "backwards"), (258, 8, 128, 64, "aligned"), (66, 12, 32, 16, "behind"),
]


def _slots(n, page, how, seed):
    pages = n // page + 4
    gen = torch.Generator().manual_seed(seed)
    order = torch.randperm(pages, generator=gen)
    first = {"one": 7, "behind": 5, "aligned": 8, "any": 0, "backwards": 0}[how]
    at = torch.arange(first, first + n)
    slots = order[at // page] * page + at % page
    if how == "any":
        slots = torch.randperm(pages * page, generator=gen)[:n]
        slots[n // 2], slots[n // 3] = -1, pages * page
    return (slots.flip(0) if how == "backwards" else slots), pages


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("tokens,heads,D,page,how", WRITES)
def test_write_and_read(tokens, heads, D, page, how, dtype):
    seed = tokens * 7 + D
    k = _normal((tokens, heads, D), dtype, seed, 3.0)
    v = _normal((tokens, 3 * heads * D + 8), dtype, seed + 1)[:, heads * D:2 * heads * D].view(tokens, heads, D)       # rows within wider ones
    k[0, 0, :8] = 0
    v[tokens // 2, heads - 1] = 0
    slots, pages = _slots(tokens, page, how, seed)
    device, before = _stored(k.cuda(), torch.empty((tokens, 3 * heads * D + 8), dtype=dtype).cuda()[:, :heads * D].view(tokens, heads, D).copy_(v), page, pages, slots)
    got = device.cpu().flatten()
    inside = (slots >= 0) & (slots < pages * page)
    keys, key_second, values, value_second, key_scales, value_scales = ref.places(slots[inside], page, heads, D)
    touched = torch.zeros(got.numel(), dtype=torch.bool)
    for x, codes, second, scales in ((k, keys, key_second, key_scales), (v, values, value_second, value_scales)):
        q, s, _ = ref.quantise(x[inside])
        bits = got[scales].int() | got[scales + 1].int() << 8
        assert torch.equal((bits - ((bits >> 15) << 16)).to(torch.int16).view(dtype).double(), s), "scales"
        b = got[codes].int()
        found = torch.where(second, (b >> 3 & 7) * (1 - 2 * (b >> 6 & 1)), (b & 7) * (1 - 2 * (b >> 7)))
        assert torch.equal(found.double(), q), "codes"
        touched[codes.flatten()] = True
        touched[scales.flatten()] = True
        touched[scales.flatten() + 1] = True
    # codes and scales behind a head's last value share the record's room: whole groups of 32 are written
    S = (D + 31) // 32
    keys, _, values, _, _, _ = ref.places(slots[inside], page, heads, 32 * S)
    touched[keys.flatten()] = True
    touched[values.flatten()] = True
    assert torch.equal(got[~touched], before.flatten()[~touched]), "written outside the slots"
    k_back, v_back = fq.kv4_read(device, page, heads, D, slots.cuda(), dtype)
    for back, x in ((k_back, k), (v_back, v)):
        want = torch.zeros(x.shape, dtype=torch.float64)
        want[inside] = ref.quantise(x[inside])[2]
        assert torch.equal(back.cpu().double(), want)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_large_small_and_broken_values(dtype):
    top = torch.finfo(dtype).max
    least = 2.0 ** ref.SCALES[dtype][1]
    k = torch.zeros((9, 1, 64), dtype=dtype)
    k[0, 0, :3] = torch.tensor([top, -top, top / 3], dtype=dtype)
    k[1, 0, 5], k[1, 0, 40] = least, 3 * least
    k[2, 0, :8] = torch.arange(8).to(dtype) * least * 11
    k[3, 0, 9] = math.inf
    k[4, 0, 60] = -math.inf
    k[5, 0, 33] = math.nan
    k[6, 0] = _normal((64,), dtype, 4, 1e-6 if dtype == F16 else 1e-30)
    k[7, 0, :32] = 7.5        # halves: 7.5 scales
    k[8, 0, :5] = torch.tensor([7.5, 0.5, 1.5, 2.5, -2.5], dtype=dtype)
    slots = torch.arange(9) + 3
    device, _ = _stored(k.cuda(), (-k).cuda(), 16, 1, slots)
    back, minus = fq.kv4_read(device, 16, 1, 64, slots.cuda(), dtype)
    want = ref.quantise(k)[2]
    assert torch.equal(back.cpu().double().nan_to_num(9e300), want.nan_to_num(9e300))
    assert torch.equal(-minus.cpu().double().nan_to_num(-9e300), want.nan_to_num(9e300))
    assert int(want.isnan().sum()) == 3 * 32


def test_read_takes_slots_twice_and_outside():
    k, v = _normal((4, 2, 64), F16, 1), _normal((4, 2, 64), F16, 2)
    device, _ = _stored(k.cuda(), v.cuda(), 16, 3, torch.tensor([0, 17, 18, 40]))
    back, _ = fq.kv4_read(device, 16, 2, 64, torch.tensor([17, 17, -5, 48, 0, 17]).cuda(), F16)
    want = ref.quantise(k)[2]
    assert torch.equal(back.cpu().double(), torch.stack([want[1], want[1], want[0] * 0, want[0] * 0, want[0], want[1]]))


# ------------------------------------------------------------------------------------------------ attention
def _context(lens, nodes, hk, D, page, dtype, seed, spread=1.0):
    """A cache with random keys and values in every slot of the sequences, garbage in all others; (device, table, keys and values [pages, page, hk, D])."""
    gen = torch.Generator().manual_seed(seed)
    used = [max(1, (max(0, n) + nodes + page - 1) // page) for n in lens]
    width, pages = max(used) + 1, sum(used) + 3
    order = torch.randperm(pages, generator=gen)
    table = torch.full((len(lens), width), 1 << 30, dtype=torch.int32)       # (entries that no token lies in are not read)
    at = 0
    k, v = torch.zeros((pages, page, hk, D), dtype=dtype), torch.zeros((pages, page, hk, D), dtype=dtype)
    slots = []
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
        count = max(0, lens[b]) + nodes
        j = torch.arange(count)
        slots.append(table[b].long()[j // page] * page + j % page)
    slots = torch.cat(slots)
    scale = torch.exp(torch.randn((len(slots), hk, 1), generator=gen) * math.log(spread)) if spread != 1.0 else 1.0
    for x in (k, v):
        x.view(-1, hk, D)[slots] = (torch.randn((len(slots), hk, D), generator=gen) * scale).to(dtype)
    device, _ = _stored(k.view(-1, hk, D)[slots].cuda(), v.view(-1, hk, D)[slots].cuda(), page, pages, slots, seed)
    for x in (k, v):
        x.view(-1, hk, D)[slots] = ref.quantise(x.view(-1, hk, D)[slots])[2].to(dtype)
    return device, table, k, v


def _check(lens, nodes, hq, hk, D, page, dtype, seed, sees=None, mask=None, scale=None, sigma=1.5, spread=1.0, workspace=None):
    device, table, k, v = _context(lens, nodes, hk, D, page, dtype, seed, spread)
    q = _normal((len(lens), nodes, hq, D), dtype, seed + 1, sigma)
    got = fq.attention_tree_kv4(q.cuda(), device, page, hk, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), mask=mask, scale=scale,
                                workspace=workspace)
    want, tol = attention.tree(q, k, v, table.clamp_max(k.shape[0] - 1), lens, attention.chain(len(lens), nodes) if sees is None else sees, scale)
    attention.compare(got, want, tol, f"{lens} {nodes} {hq}/{hk}/{D} page {page} {dtype}")
    return got, (device, table, q)


CASES = [  # lengths, nodes, heads, key heads, D, page
    ([0], 1, 4, 4, 128, 16), ([1], 1, 32, 8, 128, 16), ([15, 16, 17], 1, 8, 2, 64, 16), ([31, 32, 33, 500], 1, 8, 8, 80, 32), ([777], 1, 4, 4, 128, 64),
    ([5, -1, 1300, 64], 1, 12, 4, 96, 48), ([700, 2, 90], 5, 8, 2, 128, 16), ([260], 17, 2, 2, 32, 32), ([129, 900], 8, 8, 4, 40, 64), ([3000], 2, 16, 1, 64, 128),
    ([100, 1000], 24, 8, 4, 128, 32), ([350, 0, 47], 40, 4, 2, 96, 16), ([64, 65], 33, 3, 3, 128, 64), ([1024], 48, 16, 4, 128, 32), ([500], 70, 4, 2, 80, 64),
    ([10, 333], 130, 2, 1, 24, 16), ([2000], 100, 8, 4, 64, 128), ([0, 7], 200, 4, 4, 128, 16),
]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lens,nodes,hq,hk,D,page", CASES)
def test_attention(lens, nodes, hq, hk, D, page, dtype):
    _check(lens, nodes, hq, hk, D, page, dtype, len(lens) + nodes + D)
