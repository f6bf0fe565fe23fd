"""Appends with the position rotation, page bounds, and the 4-bit cache's
rounding, against float64 on the CPU (tests/paged4_util.py)."""
import math

import pytest
import torch

from .paged4_util import LEVELS, Case4, exponents, quantise, rotate, rounding, values
from .paged_util import Case
from .test_gpu_paged import nan_like, run_decode, run_evict, run_prefill

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32


def frequencies(rot, base=10000.0):
    return None if rot == 0 else (base ** (-torch.arange(0, rot, 2).double() / rot)).float()


def cu_of(new):
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return cu


def where(case, new):
    """(sequence, position in the cache, token) of every new token; lens as the device has them."""
    cap = case.g.max_pages * case.g.page_size
    for b, n in enumerate(new):
        p0 = min(max(case.lens_host[b], 0), cap) - n
        for i in range(n):
            yield b, p0 + i


def slot(case, b, j):
    p = int(case.table[b, j // case.g.page_size]) if j >= 0 else -1
    return (p, j % case.g.page_size) if 0 <= p < case.g.n_pages else None


def close(got, want, tol, what):
    got = got.cpu().double()
    same = (got == want) | (got.isnan() & want.isnan())
    bad = ~same & ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} off, most {float((got - want)[bad].abs().max()):.3e}"


def run_append(case, new, rot, interleaved=False, far=None, with_q=True, bounds=None, alias=False):
    g, dt = case.g, case.dtype
    cu, T = cu_of(new), sum(new)
    q = case.normal(T, g.n_q_heads, g.head_dim)
    k, v = (case.normal(T, g.n_kv_heads, g.head_dim) for _ in range(2))
    f = frequencies(rot)
    at = list(where(case, new))
    pos = torch.tensor([j for _, j in at], dtype=torch.int32)
    if far is not None:
        pos = torch.randint(0, far, (T,), generator=case.gen, dtype=torch.int32)
    ref = case.ref()
    qd = nan_like(T + 1, g.n_q_heads, g.head_dim, dtype=dt)
    if alias:
        qd[:T] = q.cuda()
    old = None if bounds is None else bounds.cpu().double()
    kw = dict(bounds=bounds) if bounds is not None else {}
    g.append(case.cache, k.cuda(), v.cuda(), cu, q=(qd[:T] if alias else q.cuda()) if with_q else None,
             q_out=qd if with_q and not alias else qd[:T] if with_q else None,
             freqs=None if f is None else f.cuda(), interleaved=interleaved,
             positions=pos.cuda() if far is not None else None, **kw)
    torch.cuda.synchronize()
    if with_q:
        want, tol = rotate(q, pos, f, interleaved, dt)
        close(qd[:T], want, tol + rounding(want, dt), "q")
        assert qd[T:].isnan().all(), "rows behind the last token"
    return at, ref, rotate(k, pos, f, interleaved, dt), v, old


def check_plain(case, new, rot, **kw):
    """An append to a bf16 or fp32 cache, its pools, weights and bounds."""
    bounds = kw.get("bounds")
    at, ref, (k, tol), v, old = run_append(case, new, rot, **kw)
    tol = tol + rounding(k, case.dtype)
    tols = torch.zeros_like(ref.k)
    for t, (b, j) in enumerate(at):
        s = slot(case, b, j)
        if s is not None:
            ref.k[s[0], :, s[1]], ref.v[s[0], :, s[1]] = k[t], v[t].double()
            tols[s[0], :, s[1]] = tol[t]
            if ref.w is not None:
                ref.w[s[0], :, s[1]] = 0.0
    close(case.k, ref.k, tols, "K pool")
    close(case.v, ref.v, 0 * tols, "V pool")
    if case.w is not None:
        case.weights_close(ref)
    if bounds is not None:
        got, P = bounds.cpu().double(), case.g.page_size
        held = case.k.cpu().double()
        for b, n in enumerate(new):
            js = [j for bb, j in at if bb == b and j >= 0]
            for i in sorted({j // P for j in js}):
                s = slot(case, b, i * P)
                if s is None:
                    continue
                mine = [j for j in js if j // P == i]
                x = held[s[0], :, mine[0] % P:mine[-1] % P + 1]
                lo, hi = x.nan_to_num(nan=math.inf, posinf=math.inf, neginf=-math.inf).amin(1), x.amax(1)
                if mine[0] % P:
                    lo, hi = torch.minimum(lo, old[s[0], :, 0]), torch.maximum(hi, old[s[0], :, 1])
                old[s[0], :, 0], old[s[0], :, 1] = lo, hi
        assert torch.equal(got.nan_to_num(nan=7e7), old.nan_to_num(nan=7e7)), "bounds"


SHAPES = [
    # B, Hq, Hkv, d, page, lens, new
    (1, 4, 4, 64, 16, [1], [1]),
    (1, 8, 2, 128, 64, [200], [200]),
    (3, 8, 2, 128, 16, [70, 9, 133], [70, 0, 1]),
    (4, 6, 2, 64, 32, [300, 65, 129, 40], [45, 65, 2, 3]),
    (2, 16, 1, 128, 1, [40, 17], [33, 16]),
    (2, 5, 5, 128, 1024, [1100, 900], [1090, 5]),
    (130, 2, 1, 64, 16, [3 + i % 40 for i in range(130)], [1 + i % 3 for i in range(130)]),   # two launches
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
@pytest.mark.parametrize("bounds", [True, False])
def test_append(dtype, i, bounds):
    B, Hq, Hkv, d, page, lens, new = SHAPES[i]
    case = Case(B, Hq, Hkv, d, page, lens, dtype=dtype, weights=not bounds, seed=300 + i)
    b = None
    if bounds:
        b = nan_like(*case.k.shape[:2], 2, d, dtype=dtype)
        for s, n in enumerate(lens):      # what earlier appends left of pages that go on
            p0 = n - new[s]
            if p0 % page:
                p = int(case.table[s, p0 // page])
                b[p, :, 0], b[p, :, 1] = case.k[p, :, :p0 % page].amin(1), case.k[p, :, :p0 % page].amax(1)
    check_plain(case, new, d, bounds=b)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d,rot", [(64, 0), (64, 16), (64, 48), (128, 32), (128, 64), (128, 112), (128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_of_a_row(dtype, d, rot, interleaved):
    case = Case(2, 6, 2, d, 16, [75, 40], dtype=dtype, seed=310)
    check_plain(case, [60, 7], rot, interleaved=interleaved, alias=rot % 32 == 0)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("far", [1 << 20, (1 << 31) - 1])
def test_far_positions(dtype, far):
    case = Case(2, 8, 2, 128, 16, [200, 40], dtype=dtype, seed=311)
    check_plain(case, [150, 33], 128, far=far, interleaved=far > 1 << 20)


@pytest.mark.parametrize("order", ["nhd", "joined"])
def test_other_strides(order):
    case = Case(2, 8, 2, 128, 16, [75, 40], order=order, weights=True, seed=312)
    check_plain(case, [60, 7], 128, with_q=False)


def test_pages_that_are_not_there():
    """Rows without a page are dropped, their queries rotated all the same;
    lens below the call's tokens, and past the table."""
    case = Case(4, 4, 2, 64, 16, [75, 40, 20, 33], weights=True, seed=313)
    case.table[0, 1] = -1
    case.table[1, 0] = case.g.n_pages
    case.dev_table.copy_(case.table)
    case.lens_host = [75, 40, 5, 1 << 20]
    case.lens.copy_(torch.tensor(case.lens_host, dtype=torch.int32))
    check_plain(case, [75, 33, 20, 9], 64)


def test_nothing_to_append():
    case = Case(2, 4, 2, 64, 16, [75, 40], seed=314)
    check_plain(case, [0, 0], 64)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("page,lens", [(16, [75, 40, 0]), (1, [5, 3]), (256, [700, 256])])
def test_page_bounds(dtype, page, lens):
    """Of all pages; a NaN is left out, an infinity is not."""
    case = Case(len(lens), 4, 2, 128, page, lens, dtype=dtype, seed=315)
    p = int(case.table[0, 0])
    case.k[p, 0, 0, 3], case.k[p, 1, 0, 5] = math.nan, math.inf
    case.table[1, 0] = -1
    case.dev_table.copy_(case.table)
    bounds = nan_like(*case.k.shape[:2], 2, 128, dtype=dtype)
    want = bounds.cpu().double()
    case.g.page_bounds(case.cache, bounds, max_len=1)
    held = case.k.cpu().double()
    for b, n in enumerate(lens):
        for i in range(-(-n // page)):
            s = slot(case, b, i * page)
            if s is not None:
                x = held[s[0], :, :min(page, n - i * page)]
                want[s[0], :, 0] = torch.where(x.isnan(), math.inf, x).amin(1)
                want[s[0], :, 1] = torch.where(x.isnan(), -math.inf, x).amax(1)
    assert torch.equal(bounds.cpu().double().nan_to_num(nan=7e7), want.nan_to_num(nan=7e7))


# -- four bits ---------------------------------------------------------------

def held4(case, s):
    return [(c[s[0], :, s[1]].cpu(), e[s[0], :, s[1]].cpu()) for c, e in (case.k, case.v)]


def check_four(case, new, rot, **kw):
    before = [t.clone() for pool in (case.k, case.v) for t in pool]
    at, _, (k, tol), v, _ = run_append(case, new, rot, **kw)
    rows = []
    for t, (b, j) in enumerate(at):
        s = slot(case, b, j)
        if s is None:
            rows.append((torch.zeros(k.shape[1:]), torch.zeros(k.shape[1:])))
            continue
        (kc, ke), (vc, ve) = held4(case, s)
        c, e = quantise(v[t])
        assert torch.equal(vc, c) and torch.equal(ve, e), f"token {t}: V"
        rows.append((values(kc, ke), values(vc, ve)))
        # K: what the definition gives of the rotated row, or of one within its tolerance
        y, d = k[t].unflatten(-1, (-1, 32)), tol[t].unflatten(-1, (-1, 32))
        lo, hi = exponents((y.abs() - d).amax(-1)), exponents((y.abs() + d).amax(-1))
        got = ke.long() - 127
        assert ((got >= lo) & (got <= hi)).all(), f"token {t}: K scales"
        step = torch.exp2(got.double())[..., None]
        x = rows[-1][0].unflatten(-1, (-1, 32))
        best = (LEVELS * step[..., None] - y.abs()[..., None]).abs().amin(-1)
        assert ((x - y).abs() <= best + 2 * d).all(), f"token {t}: K codes"
        for name, row in zip(("k", "v"), before[::2]):
            row[s[0], :, s[1]] = (kc if name == "k" else vc).cuda()
        for name, row in zip(("k", "v"), before[1::2]):
            row[s[0], :, s[1]] = (ke if name == "k" else ve).cuda()
    for x, y in zip(before, [t for pool in (case.k, case.v) for t in pool]):
        assert torch.equal(x, y), "bytes of other slots"
    T, g = sum(new), case.g
    ko, vo = (nan_like(T + 1, g.n_kv_heads, g.head_dim, dtype=case.dtype) for _ in range(2))
    g.read(case.cache, cu_of(new), ko, vo)
    for t, (x, y) in enumerate(rows):
        assert torch.equal(ko[t].cpu().double(), x.double()) and torch.equal(vo[t].cpu().double(), y.double()), \
            f"token {t} read"
    assert ko[T:].isnan().all() and vo[T:].isnan().all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_append4(dtype, i):
    B, Hq, Hkv, d, page, lens, new = SHAPES[i]
    check_four(Case4(B, Hq, Hkv, d, page, lens, dtype=dtype, seed=i), new, d)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d,rot,interleaved", [(64, 0, False), (128, 64, False), (128, 0, True), (128, 48, True),
                                               (64, 16, True), (128, 128, True)])
def test_part_of_a_row4(dtype, d, rot, interleaved):
    case = Case4(2, 6, 2, d, 16, [75, 40], dtype=dtype, seed=20)
    check_four(case, [60, 7], rot, interleaved=interleaved, far=1 << 20)


def test_pages_that_are_not_there4():
    case = Case4(3, 4, 2, 64, 16, [75, 40, 20], seed=21)
    case.table[0, 1] = -1
    case.table[1, 0] = case.g.n_pages
    case.dev_table.copy_(case.table)
    case.lens_host = [75, 40, 5]
    case.lens.copy_(torch.tensor(case.lens_host, dtype=torch.int32))
    check_four(case, [75, 33, 20], 64)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rounding_to_four_bits(dtype):
    """Every bf16 number beside the largest of its group at which the scale
    moves; ties; groups of zeros, of the smallest and of the largest numbers;
    infinities and NaN."""
    d, Hkv = 64, 2
    rows = []
    for top in (7.0, 7.03125, 6.0, 3.5, 1.75, 1.7578125, 2.0 ** 120, 2.0 ** -100):
        ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]) * top / 7
        near = torch.cat([ties * (1 + s * 2.0 ** -7) for s in (-1, 0, 1)])
        rows.append(torch.cat([torch.tensor([top]), near, -ties[:7], torch.linspace(-top, top, 32)]))
    zero = torch.zeros(64)
    rows += [zero, zero.clone().fill_(1e-40), torch.cat([torch.linspace(0, 2.0 ** -123, 32), torch.full((32,), -0.0)])]
    big = torch.linspace(-3.3e38, 3.3e38, 64)
    odd = torch.randn(64)
    odd[3], odd[40], odd[41] = math.nan, math.inf, -math.inf
    rows += [big, odd, torch.full((64,), math.nan)]
    x = torch.stack(rows).to(dtype)
    T = x.shape[0]
    case = Case4(1, 2, Hkv, d, 16, [T], dtype=dtype, seed=22)
    k = torch.stack([x, -x], 1).contiguous()
    case.g.append(case.cache, k.cuda(), k.flip(1).contiguous().cuda(), [0, T])
    for t in range(T):
        (kc, ke), (vc, ve) = held4(case, slot(case, 0, t))
        for (c, e), r in (((kc, ke), k[t]), ((vc, ve), k[t].flip(0))):
            wc, we = quantise(r)
            assert torch.equal(c, wc) and torch.equal(e, we), f"row {t}"
            assert values(c, e).isfinite().all()


@pytest.mark.parametrize("dtype,interleaved,far", [(BF16, False, 0), (BF16, True, 0), (FP32, False, 900000)])
def test_codes_of_the_rotated_key(dtype, interleaved, far):
    """Each code is that of the key rotated in 64 bits, also where an fp32
    product would be on the other side of a step's middle: 2^22 elements, of
    which a rounding of 2^-24 would move several.  (Both sides' 64-bit errors,
    2^-30 of a number at these positions, would move one in about 1000 runs.)"""
    T, Hkv, d = 4096, 8, 128
    case = Case4(1, Hkv, Hkv, d, 64, [T], dtype=dtype, seed=30)
    gen = torch.Generator().manual_seed(31)
    k = torch.randn((T, Hkv, d), generator=gen).to(dtype)
    f = frequencies(d)
    pos = torch.arange(T, dtype=torch.int32) + far
    case.g.append(case.cache, k.cuda(), k.cuda(), [0, T], freqs=f.cuda(), interleaved=interleaved, positions=pos.cuda())
    codes, scales = quantise(rotate(k, pos, f, interleaved, dtype)[0])
    page, at = case.table[0, torch.arange(T) // 64].long(), torch.arange(T) % 64
    assert torch.equal(case.k[1].cpu()[page, :, at], scales)
    assert torch.equal(case.k[0].cpu()[page, :, at], codes)


def test_scales_out_of_range_read():
    """Bytes that no call writes count as the nearest that one does."""
    case = Case4(1, 2, 1, 64, 16, [20], seed=23)
    case.k[1].copy_(torch.randint(0, 256, case.k[1].shape, generator=case.gen, dtype=torch.uint8))
    case.k[1][:, :, 1] = 255
    case.k[1][:, :, 3] = 0
    ko, vo = (nan_like(20, 1, 64, dtype=FP32) for _ in range(2))
    g = type(case.g)(1, 2, 1, 64, 16, case.g.n_pages, case.g.max_pages, dtype=FP32)
    g.read(case.cache, [0, 20], ko, vo)
    ref = case.ref()
    for j in range(20):
        p, s = slot(case, 0, j)
        assert torch.equal(ko[j].cpu().double(), ref.k[p, :, s]) and torch.equal(vo[j].cpu().double(), ref.v[p, :, s])


# -- together ----------------------------------------------------------------

@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_append_then_attend_then_evict(dtype):
    """A prompt appended rotated, read out by a prefill that takes it from the
    cache; a token more; an eviction, and the bounds after it."""
    case = Case(2, 8, 2, 128, 16, [90, 40], 64, 4, dtype=dtype, weights=True, seed=316)
    bounds = nan_like(*case.k.shape[:2], 2, 128, dtype=dtype)
    check_plain(case, [90, 40], 128, bounds=bounds)
    run_prefill(case, [90, 40], observe=8, append=False)
    run_decode(case, False)
    run_evict(case, 30, 10)
    case.g.page_bounds(case.cache, bounds)


def test_captured():
    """An append captured into a graph and replayed, with eager work between."""
    case = Case(2, 8, 2, 128, 16, [90, 40], seed=317)
    g, f = case.g, frequencies(128).cuda()
    q, k, v = (case.normal(33, h, 128).cuda() for h in (8, 2, 2))
    bounds, qo = g.new_bounds(), torch.empty_like(q)
    bounds.zero_()
    call = lambda: g.append(case.cache, k, v, [0, 20, 33], q=q, q_out=qo, freqs=f, bounds=bounds)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in range(3):
        q.add_(1.0)
        k.add_(0.5)
        bounds.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (qo, case.k, case.v, bounds)]
        qo.fill_(math.nan)
        bounds.zero_()
        call()
        for x, y in zip(got, (qo, case.k, case.v, bounds)):
            assert torch.equal(x.nan_to_num(nan=7e7), y.nan_to_num(nan=7e7)), n


def test_another_stream():
    case = Case(2, 8, 2, 128, 16, [90, 40], seed=318)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        check_plain(case, [33, 40], 128)
