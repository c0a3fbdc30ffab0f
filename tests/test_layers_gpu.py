"""The layer operators (include/layers/lsgd_layers.h) against plain
implementations in binary64, at the sizes, types and values where they can go
wrong. Tolerances count roundings: a half step of a type relative to the value
is finfo(type).eps / 2, and a binary32 sum of n terms in any order is within
n * 2^-24 times the sum of their magnitudes (to first order)."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.device_count() > 0:
    import paper_1906_05936_amd as lsgd
else:  # collected but skipped on machines without a GPU
    lsgd = None

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16
U32 = 2.0 ** -24
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def randn(*shape, seed=0, dtype=F32, scale=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, device=DEV, generator=gen) * scale).to(dtype)


def randint(n, low, high, seed=0, dtype=torch.int64):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(low, high, (n,), device=DEV, generator=gen, dtype=dtype)


def nans(*shape, dtype=F32):
    return torch.full(shape, float("nan"), device=DEV, dtype=dtype)


def assert_close(got, want, bound, what=""):
    """|got - want| <= bound, all in binary64; equal NaNs and infinities."""
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities"
    over = ((got - want).abs() - bound)[fine]
    assert over.numel() == 0 or over.max().item() <= 0, "%s: off by %g over its bound" % (what, over.max().item())


# ---------------------------------------------------------------- lookup

@pytest.mark.parametrize("tdt", [F32, BF16])
@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("rows,dim,n,it", [
    (1, 1, 1, torch.int32), (5, 7, 3, torch.int64), (100, 8, 1000, torch.int32), (333, 129, 257, torch.int64),
    (1000, 1024, 65, torch.int64), (64, 2049, 31, torch.int32), (17, 5000, 9, torch.int64)])
def test_lookup(tdt, odt, rows, dim, n, it):
    table, tokens = randn(rows, dim, seed=1, dtype=tdt), randint(n, -1, rows + 1, seed=2, dtype=it)
    tokens[0] = rows - 1
    out = nans(n + 1, dim, dtype=odt)
    lsgd.embed_lookup(table, tokens, out[:n], scale=1.7)
    t = tokens.long()
    inside = (t >= 0) & (t < rows)
    scale = np.float32(1.7).item()
    want = torch.where(inside[:, None], table.double()[t.clamp(0, rows - 1)] * scale, 0.0)
    # one product rounded to binary32, and once more to odt
    assert_close(out[:n], want, want.abs() * (U32 + (HALF[BF16] * (1 + U32) if odt == BF16 else 0)))
    assert torch.isnan(out[n]).all()


def test_lookup_non_finite_rows_and_extreme_tokens():
    table = randn(4, 16, seed=3)
    table[1, 3], table[2, 5] = float("inf"), float("nan")
    tokens = torch.tensor([1, 2, -2 ** 63, 2 ** 63 - 1, 2 ** 32, 3], device=DEV)
    out = nans(6, 16)
    lsgd.embed_lookup(table, tokens, out)
    assert torch.equal(out[0], table[1]) and torch.isnan(out[1, 5]) and torch.equal(out[5], table[3])
    assert torch.count_nonzero(out[2:5]) == 0


@pytest.mark.parametrize("odt", [F32, BF16])
def test_lookup_outside_the_table_is_zero_whatever_the_scale(odt):
    table, tokens = randn(3, 21, seed=1), torch.tensor([-1, 2, 3], device=DEV)
    for scale in (float("inf"), float("nan"), -2.0):
        out = nans(3, 21, dtype=odt)
        lsgd.embed_lookup(table, tokens, out, scale)
        assert (out[::2] == 0).all()


def test_lookup_empty():
    out = nans(0, 8)
    lsgd.embed_lookup(randn(3, 8), torch.empty(0, dtype=torch.int64, device=DEV), out)
    one = nans(2, 8)
    lsgd.embed_lookup(torch.empty(0, 8, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV), one)
    assert torch.count_nonzero(one) == 0      # a table without rows holds no token


# ---------------------------------------------------------------- gradient

def grad_reference(grads, tokens, rows, scale):
    """(sum, sum of magnitudes, terms of each row) in binary64."""
    t, g = torch.cat([x.reshape(-1) for x in tokens]).long(), torch.cat(grads).double()
    inside = (t >= 0) & (t < rows)
    t, g = t[inside], g[inside]
    total = torch.zeros(rows, g.shape[1], device=DEV, dtype=torch.float64)
    size, n = torch.zeros_like(total), torch.zeros(rows, 1, device=DEV, dtype=torch.float64)
    total.index_add_(0, t, g)
    size.index_add_(0, t, g.abs())
    n.index_add_(0, t, torch.ones(len(t), 1, device=DEV, dtype=torch.float64))
    return total * scale, size * abs(scale), n


def zipf(n, rows, seed, dtype=torch.int64):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    u = torch.rand(n, device=DEV, generator=gen, dtype=torch.float64)
    return (torch.exp(u * math.log(rows + 1)).long() - 1).clamp_(0, rows - 1).to(dtype)


@pytest.mark.parametrize("gdt", [F32, BF16])
@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("rows,dim,n,workers,it,how", [
    (1, 1, 1, 1, torch.int64, "any"), (7, 5, 1, 1, torch.int32, "any"), (50, 33, 64, 1, torch.int64, "any"),
    (50, 33, 65, 1, torch.int32, "same"), (300, 8, 700, 1, torch.int64, "zipf"), (40, 513, 300, 3, torch.int32, "zipf"),
    (1000, 64, 4096, 1, torch.int64, "zipf"), (1000, 64, 4097, 1, torch.int64, "zipf"),
    (511, 24, 1400, 3, torch.int32, "zipf"), (512, 24, 2100, 2, torch.int64, "any"), (3, 520, 5000, 1, torch.int64, "same"),
    (300000, 9, 2500, 2, torch.int64, "zipf"), (70, 16, 9000, 1, torch.int32, "outside"), (2000, 1032, 3000, 4, torch.int64, "zipf"),
    (5, 8, 40000, 1, torch.int32, "any"), (40, 40, 50, 128, torch.int64, "zipf"), (90, 8, 300, 1, torch.int64, "padded"),
    (300, 24, 6000, 2, torch.int32, "padded"), (6000, 520, 30000, 4, torch.int64, "zipf"), (600000, 5, 3000, 1, torch.int64, "zipf"),
    (40, 16, 8192, 1, torch.int32, "zipf"), (40, 16, 8193, 1, torch.int64, "zipf"), (9, 8, 8192, 1, torch.int64, "same"),
    (9, 1100, 50000, 1, torch.int64, "same"), (200, 520, 512, 1, torch.int64, "zipf"), (64, 40, 512, 1, torch.int32, "same"),
    (130, 9, 513, 1, torch.int64, "zipf"), (40000, 600, 500, 1, torch.int64, "zipf"), (65, 24, 170, 3, torch.int64, "any"), (3, 16, 500, 1, torch.int64, "zipf"), (20, 2050, 9000, 2, torch.int32, "zipf"),
    (300000, 9, 9000, 2, torch.int64, "any"), (1000, 4, 1100000, 1, torch.int64, "zipf"), (300000, 12, 600000, 2, torch.int32, "zipf")])
def test_grad(gdt, odt, rows, dim, n, workers, it, how):
    if how == "zipf":
        tokens = [zipf(n, rows, 10 + w, it) for w in range(workers)]
    elif how == "same":
        tokens = [torch.full((n,), rows - 1, device=DEV, dtype=it) for _ in range(workers)]
    elif how == "padded":
        tokens = [torch.where(torch.arange(n, device=DEV) % 3 == 0, zipf(n, rows, 10 + w, it), -1).to(it) for w in range(workers)]
    elif how == "outside":
        tokens = [torch.where(torch.arange(n, device=DEV) % 2 == 0, -5, rows).to(it) for _ in range(workers)]
    else:
        tokens = [randint(n, -1, rows + 1, seed=20 + w, dtype=it) for w in range(workers)]
    grads = [randn(n, dim, seed=30 + w, dtype=gdt) for w in range(workers)]
    scale = np.float32(0.3).item()
    want, size, terms = grad_reference(grads, tokens, rows, scale)
    for accumulate in (False, True):
        buf = randn(rows + 1, dim, seed=5, dtype=odt) if accumulate else nans(rows + 1, dim, dtype=odt)
        before = buf.clone()
        lsgd.embed_grad(grads, tokens, buf[:rows], scale=scale, accumulate=accumulate)
        ref = want + before[:rows].double() if accumulate else want
        # terms - 1 additions, the product, the addition of what was there, the rounding to odt
        bound = size * ((terms + 2) * U32) + ref.abs() * U32
        bound = bound + ref.abs() * HALF[BF16] * 1.01 + bound * 0.01 if odt == BF16 else bound
        if accumulate:
            named = terms[:, 0] > 0
            assert torch.equal(buf[:rows][~named], before[:rows][~named])
        assert_close(buf[:rows], ref, bound, "accumulate=%s" % accumulate)
        assert torch.equal(buf[rows].view(torch.int32 if odt == F32 else torch.int16),
                           before[rows].view(torch.int32 if odt == F32 else torch.int16))
        again = before.clone()
        lsgd.embed_grad(grads, tokens, again[:rows], scale=scale, accumulate=accumulate)
        assert torch.equal(again[:rows], buf[:rows])


@pytest.mark.parametrize("rows", [(1 << 27) + 5, (1 << 31) - 1])
def test_grad_of_a_table_whose_rows_take_every_digit(rows):
    """Tokens that differ in their highest bits, in their lowest, or lie outside (whole
    numbers: exact)."""
    n = 9001
    low, high = randint(n, 0, 6, seed=1), randint(n, 0, 1 + rows // (1 << 27), seed=2) * (1 << 27)
    tokens = torch.where(randint(n, 0, 4, seed=3) > 0, low + high, randint(n, 0, rows + 1, seed=4))
    tokens[::7], tokens[3::7] = -1, rows
    tokens[5], tokens[8] = rows - 1, 0
    g = randint(n, -8, 9, seed=5).float().view(n, 1)
    want = torch.zeros(rows, 1, device=DEV)
    inside = (tokens >= 0) & (tokens < rows)
    want.index_add_(0, tokens[inside], g[inside])
    out = nans(rows, 1)
    lsgd.embed_grad([g], [tokens], out)
    assert torch.equal(out, want)


def test_grad_of_the_most_entries():
    """2^28 of them: four workers that hold the same tensors (whole numbers: exact)."""
    n, rows = 1 << 26, 1003
    tokens, g = zipf(n, rows + 5, 1, torch.int32), randint(n, -3, 4, seed=2).to(BF16).view(n, 1)
    spread = tokens.long() * 512 + torch.arange(n, device=DEV) % 512   # 512 partial sums of a row
    want = torch.zeros((rows + 5) * 512, device=DEV, dtype=torch.float64).index_add_(0, spread, g[:, 0].double())
    want = want.view(rows + 5, 512).sum(1) * 4
    assert want.abs().max() < 1 << 24
    out = nans(rows, 1)
    lsgd.embed_grad([g] * 4, [tokens] * 4, out, scale=0.5)
    assert torch.equal(out[:, 0].double(), want[:rows] * 0.5)


def test_grad_no_tokens():
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    out = nans(5, 9)
    lsgd.embed_grad([torch.empty(0, 9, device=DEV)], [none], out)
    assert torch.count_nonzero(out) == 0
    out = randn(5, 9)
    before = out.clone()
    lsgd.embed_grad([torch.empty(0, 9, device=DEV)], [none], out, accumulate=True)
    assert torch.equal(out, before)


def test_grad_skips_what_padding_holds():
    """NaN and infinities under tokens outside the table touch nothing; under
    one inside, its row only."""
    g = randn(6, 8, seed=1)
    g[1], g[4] = float("nan"), float("inf")
    out = nans(4, 8)
    lsgd.embed_grad([g], [torch.tensor([0, -1, 2, 2, 4, 0], device=DEV)], out)
    assert torch.equal(out[0], g[0] + g[5]) and torch.equal(out[2], g[2] + g[3])
    assert torch.count_nonzero(out[1]) == 0 and torch.count_nonzero(out[3]) == 0
    lsgd.embed_grad([g], [torch.tensor([0, -1, 2, 2, 3, 0], device=DEV)], out)
    assert torch.isinf(out[3]).all() and torch.isfinite(out[:3]).all()


def test_grad_against_differences():
    """The gradient of sum(weights * lookup) in one table entry: lookups of two
    tables that differ there by 1 differ by it (values small whole numbers: exact)."""
    rows, dim, n = 6, 5, 40
    tokens = randint(n, -1, rows, seed=3)
    weights = randint(n * dim, -4, 5, seed=4).view(n, dim).float()
    table = randint(rows * dim, -8, 9, seed=5).view(rows, dim).float()
    out = nans(rows, dim)
    lsgd.embed_grad([weights], [tokens], out, scale=2.0)

    def value(t):
        y = nans(n, dim)
        lsgd.embed_lookup(t, tokens, y, scale=2.0)
        return (y * weights).sum().item()
    base = value(table)
    for r in range(rows):
        for c in range(dim):
            moved = table.clone()
            moved[r, c] += 1
            assert value(moved) - base == out[r, c].item()


def test_mean_gradient_is_the_two_level_mean():
    """All workers at once with scale / N against a gradient buffer per worker
    and the step's two means (whole numbers, N a power of two: exact)."""
    rows, dim, n, N = 37, 24, 90, 8
    tokens = [zipf(n, rows, w) for w in range(N)]
    grads = [randint(n * dim, -64, 65, seed=w).view(n, dim).float() for w in range(N)]
    mean = nans(rows, dim)
    lsgd.embed_grad(grads, tokens, mean, scale=1.0 / N)
    each = [nans(rows, dim) for _ in range(N)]
    for w in range(N):
        lsgd.embed_grad([grads[w]], [tokens[w]], each[w])
    groups = [nans(rows, dim) for _ in range(2)]
    lsgd.group_mean(each, [w // 4 for w in range(N)], 2, groups)
    both = nans(rows, dim)
    lsgd.global_mean(groups, both)
    assert torch.equal(mean, both)


# ---------------------------------------------------------------- 8 bits

def scales_reference(x, block):
    """Scales (as exponents) from the definition, in numpy binary64."""
    rows, cols = x.shape
    sr, kb = -(-rows // block), -(-cols // 128)
    p = np.zeros((sr * block, kb * 128))
    p[:rows, :cols] = np.where(np.isfinite(x), np.abs(x), 0)
    a = p.reshape(sr, block, kb, 128).max(axis=(1, 3))
    e = np.zeros(a.shape, dtype=np.int64)
    for i in np.ndindex(a.shape):
        if a[i] > 0:
            k = max(-126, math.frexp(a[i])[1] - 10)
            while a[i] > 448 * 2.0 ** k:
                k += 1
            e[i] = k
    return e


def codes_reference(v):
    """Nearest e4m3 value of each element of v (|v| <= 448), ties to the even code."""
    table = np.array([(1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6 for e in range(16) for m in range(8)])[:127]
    a = np.abs(v)
    hi = np.clip(np.searchsorted(table, a), 1, 126)
    lo = hi - 1
    dl, dh = a - table[lo], table[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.copysign(table[pick], v)


def check_8bit(x, codes, scales, block):
    x = x.double().cpu().numpy()
    rows, cols = x.shape
    e = scales_reference(x, block)
    s = scales.view(torch.uint8).cpu().numpy().astype(np.int64)
    kb = e.shape[1]
    assert np.array_equal(s[:, :kb], e + 127) and (s[:, kb:] == 127).all()
    q = codes.float().double().cpu().numpy()
    assert (codes.view(torch.uint8)[:, cols:] == 0).all()
    each = np.repeat(np.repeat(e, block, 0)[:rows], 128, 1)[:, :cols]
    fine = np.isfinite(x)
    assert np.array_equal(np.isnan(q[:, :cols]), ~fine)
    want = codes_reference(np.where(fine, np.ldexp(np.where(fine, x, 0), -each), 0))
    assert np.array_equal(np.where(fine, q[:, :cols], 0), want)


def guarded8(rows, cols, block):
    """empty8 with guard rows behind it, and a check that they keep their bytes."""
    q = torch.full((rows + 2, lsgd.pitch8(cols)), 0x55, device=DEV, dtype=torch.uint8)
    s = torch.full((-(-rows // block) + 16, lsgd.scale_pitch8(cols)), 0x55, device=DEV, dtype=torch.uint8)
    codes, scales = q[:rows].view(torch.float8_e4m3fn), s[:-(-rows // block)].view(torch.float8_e8m0fnu)

    def check():
        assert (q[rows:] == 0x55).all() and (s[-(-rows // block):] == 0x55).all()
    return codes, scales, check


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 127), (5, 128), (7, 129), (2, 511), (4, 513), (33, 1999), (1, 8192), (2, 524801), (270000, 3), (5000, 4000)])
def test_quant8(dtype, rows, cols):
    x = randn(rows, cols, seed=rows + cols) * torch.exp(3 * randn(rows, cols, seed=9))
    x = x.to(dtype)
    codes, scales, guard = guarded8(rows, cols, 1)
    lsgd.quant8(x, codes, scales)
    check_8bit(x, codes, scales, 1)
    guard()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quant8_extreme_values(dtype):
    top = torch.finfo(dtype).max
    tiny = 2.0 ** -149 if dtype == F32 else 2.0 ** -133
    rows = [[0.0, -0.0], [448.0, 447.9], [448.0625, 1.0], [tiny, -tiny], [2.0 ** -126, 2.0 ** -127], [top / 2, 1.0],
            [float("inf"), 3.0], [float("nan"), -3.0], [float("-inf"), float("nan")], [1.0, 2.0 ** -9], [1.75, -1.0],
            [1.7578125, 1e-30], [2.0 ** -118, 2.0 ** -127], [17.0, 19.0], [2.0 ** 100, 2.0 ** 90], [256.0, 2.0 ** -10 * 1.5]]
    x = torch.zeros(len(rows), 130, device=DEV)
    x[:, :2] = torch.tensor(rows, device=DEV)
    x[:, 129] = 5.0
    x = x.to(dtype)
    codes, scales, guard = guarded8(len(rows), 130, 1)
    lsgd.quant8(x, codes, scales)
    check_8bit(x, codes, scales, 1)
    guard()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_quant8_passes_over_signalling_nans(dtype):
    """The block's scale is that of its finite elements, wherever the NaN stands."""
    whole = torch.int32 if dtype == F32 else torch.int16
    signalling = torch.tensor(0x7f800001 if dtype == F32 else 0x7f81, dtype=whole, device=DEV).view(dtype)
    for at in (0, 7, 64, 127):
        x = torch.full((2, 128), 3.0, device=DEV, dtype=dtype)
        x.view(whole)[0, at] = signalling.view(whole)
        codes, scales = lsgd.empty8(2, 128)
        lsgd.quant8(x, codes, scales)
        assert torch.equal(scales[0, :1].view(torch.uint8), scales[1, :1].view(torch.uint8))
        assert torch.isnan(codes.float()[0, at]) and torch.isnan(codes.float()).sum() == 1


@pytest.mark.parametrize("rows,cols", [(1, 1), (127, 3), (128, 128), (129, 257), (300, 1000), (1025, 130), (5, 700)])
@pytest.mark.parametrize("n,nt", [(1, 0), (0, 1), (2, 3)])
def test_copy_out8(rows, cols, n, nt):
    p = randn(rows, cols, seed=rows) * 0.02
    if rows > 2:
        p[2, 0] = float("nan")
    reps, ts = [guarded8(rows, cols, 128) for _ in range(n)], [guarded8(cols, rows, 128) for _ in range(nt)]
    lsgd.copy_out8(p, [r[:2] for r in reps], [t[:2] for t in ts])
    for q, s, guard in reps:
        check_8bit(p, q, s, 128)
        guard()
    for q, s, guard in ts:
        check_8bit(p.t().contiguous(), q, s, 128)
        guard()


def test_copy_out8_more_copies_than_a_launch_takes():
    p = randn(130, 140, seed=1)
    reps, ts = [lsgd.empty8(130, 140, 128) for _ in range(70)], [lsgd.empty8(140, 130, 128) for _ in range(33)]
    lsgd.copy_out8(p, reps, ts)
    for copies, ref in ((reps, p), (ts, p.t().contiguous())):
        check_8bit(ref, *copies[0], 128)
        for q, s in copies[1:]:
            assert torch.equal(q.view(torch.uint8), copies[0][0].view(torch.uint8))
            assert torch.equal(s.view(torch.uint8), copies[0][1].view(torch.uint8))


# ---------------------------------------------------------------- products

def values(codes, scales, block, cols):
    rows = codes.shape[0]
    s = scales.float().double().repeat_interleave(128, 1)[:, :codes.shape[1]].repeat_interleave(block, 0)[:rows]
    return (codes.float().double() * s)[:, :cols].contiguous()


def as8(x, block):
    q, s = lsgd.empty8(*x.shape, block)
    if block == 1:
        lsgd.quant8(x, q, s)
    else:
        lsgd.copy_out8(x.float(), [(q, s)])
    return q, s


def check_product(m, n, k, ablock, bblock, odt, seed=0, spread=2.0):
    a = randn(m, k, seed=seed) * torch.exp(spread * randn(m, k, seed=seed + 1))
    b = randn(n, k, seed=seed + 2) * torch.exp(spread * randn(n, k, seed=seed + 3))
    (qa, sa), (qb, sb) = as8(a, ablock), as8(b, bblock)
    buf = nans(m + 1, n, dtype=odt)
    lsgd.matmul8(qa, sa, qb, sb, buf[:m])
    va, vb = values(qa, sa, ablock, k), values(qb, sb, bblock, k)
    want = va @ vb.t().contiguous()
    size = va.abs() @ vb.abs().t().contiguous()
    terms = lsgd.pitch8(k)
    # binary32 sums of `terms` exact products
    bound = size * (terms * U32)
    if odt == BF16:
        # a group of 8 products drops up to 2^-13 of its largest from each of them,
        # and its sum once more: 8 * 2^-13 of the group's magnitudes at most; then the rounding
        bound = bound + size * 2.0 ** -10
        bound = bound * 1.01 + want.abs() * HALF[BF16] * 1.01
    assert_close(buf[:m], want, bound, "%s x %s x %s" % (m, n, k))
    assert torch.isnan(buf[m]).all()


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (1, 16, 128), (2, 17, 129), (16, 128, 512), (17, 130, 640), (33, 1000, 777), (64, 64, 4096),
    (65, 48, 300), (127, 129, 1024), (128, 128, 128), (129, 257, 257), (200, 520, 1537), (256, 256, 256),
    (300, 1025, 520), (513, 700, 640), (1100, 2050, 384), (2100, 4001, 300), (2304, 4100, 1152), (4097, 2090, 200), (2050, 4097, 90),
    (500, 510, 200), (1791, 849, 2100), (1000, 1023, 400), (1024, 1000, 130), (6200, 8200, 300)])
def test_matmul8(odt, m, n, k):
    check_product(m, n, k, 1, 128, odt, seed=m + n + k)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("ablock,bblock", [(1, 1), (128, 1), (128, 128)])
@pytest.mark.parametrize("m,n,k", [(5, 300, 200), (300, 260, 515), (1, 2, 130), (1000, 1300, 260), (2150, 4010, 260)])
def test_matmul8_blocks(odt, ablock, bblock, m, n, k):
    check_product(m, n, k, ablock, bblock, odt, seed=3)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(3, 20, 300), (150, 140, 300), (600, 600, 140), (1200, 2100, 300), (2200, 4003, 300)])
def test_matmul8_whole_numbers_and_their_places(odt, m, n, k):
    """Whole numbers of up to 3: every product and sum is exact in both forms
    (bfloat16 outputs: sums below 256), so each output has one right value."""
    a, b = randint(m * k, -1, 2, seed=1).view(m, k).float(), randint(n * k, -1, 2, seed=2).view(n, k).float()
    a[:, k // 3:] *= (torch.arange(k - k // 3, device=DEV) % 16 == 0)
    (qa, sa), (qb, sb) = as8(a, 1), as8(b, 128)
    out = nans(m, n, dtype=odt)
    lsgd.matmul8(qa, sa, qb, sb, out)
    want = a.double() @ b.double().t().contiguous()
    assert want.abs().max() <= 256 and torch.equal(out.double(), want)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [(3, 20, 300), (150, 140, 300), (600, 600, 140), (1200, 2100, 300), (2200, 4003, 300)])
def test_matmul8_small_terms_beside_large_ones_that_cancel(odt, m, n, k):
    """Pairs of products of 448 * 448 that cancel, among products of 1: all are whole
    numbers and every partial sum stays below 2^24, so that binary32 sums are exact in
    any order, and outputs below 256 are exact in bfloat16 too."""
    a, b = randint(m * k, -1, 2, seed=1).view(m, k).float(), randint(n * k, -1, 2, seed=2).view(n, k).float()
    a *= torch.arange(k, device=DEV) % 2
    places = torch.randperm(k, generator=torch.Generator().manual_seed(3))[:32].to(DEV)
    signs = randint(m * 16, 0, 2, seed=4).view(m, 16) * 2.0 - 1
    a[:, places] = torch.cat([signs, -signs], 1) * 448
    b[:, places] = (randint(n * 16, 0, 2, seed=5).view(n, 16) * 2.0 - 1).repeat(1, 2) * 448
    (qa, sa), (qb, sb) = as8(a, 1), as8(b, 128)
    assert torch.equal(values(qa, sa, 1, k), a.double()) and torch.equal(values(qb, sb, 128, k), b.double())
    out = nans(m, n, dtype=odt)
    lsgd.matmul8(qa, sa, qb, sb, out)
    want = a.double() @ b.double().t().contiguous()
    assert 16 < want.abs().max() < 256 and torch.equal(out.double(), want)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("ablock,bblock", [(1, 128), (1, 1)])
@pytest.mark.parametrize("m,n,k", [(3, 20, 300), (33, 1000, 777), (150, 1400, 2100), (600, 2100, 1300), (1200, 2100, 300), (2200, 4003, 900)])
def test_matmul8_differences_of_large_sums(odt, ablock, bblock, m, n, k):
    """Rows of b that repeat themselves with the other sign but for 2^-6 of their
    size: nearly all of a sum cancels, and its rest has to be right to binary32's
    roundings of the magnitudes, k * 2^-24, and the output's own."""
    a, b = randn(m, k, seed=1), randn(n, k, seed=2)
    half = k // 2
    a[:, half:2 * half] = a[:, :half]
    b[:, half:2 * half] = -b[:, :half] * (1 + 2.0 ** -6 * randn(n, half, seed=3))
    (qa, sa), (qb, sb) = as8(a, ablock), as8(b, bblock)
    va, vb = values(qa, sa, ablock, k), values(qb, sb, bblock, k)
    want, size = va @ vb.t().contiguous(), va.abs() @ vb.abs().t().contiguous()
    out = nans(m, n, dtype=odt)
    lsgd.matmul8(qa, sa, qb, sb, out)
    bound = size * (lsgd.pitch8(k) * U32)
    assert_close(out, want, bound * 1.01 + want.abs() * HALF[BF16] if odt == BF16 else bound)


@pytest.mark.parametrize("odt", [F32, BF16])
def test_matmul8_scales_at_their_ends(odt):
    """Elements near 2^100 against elements near 2^-100: the scales meet in
    binary32's range though neither lies near 1."""
    a, b = randn(20, 200, seed=1) * 2.0 ** 100, randn(40, 200, seed=2) * 2.0 ** -100
    (qa, sa), (qb, sb) = as8(a, 1), as8(b, 128)
    out = nans(20, 40, dtype=odt)
    lsgd.matmul8(qa, sa, qb, sb, out)
    va, vb = values(qa, sa, 1, 200), values(qb, sb, 128, 200)
    size = va.abs() @ vb.abs().t().contiguous()
    want = va @ vb.t().contiguous()
    assert_close(out, want, size * 2.0 ** -10 * 1.01 + want.abs() * HALF[BF16] * 1.01 if odt == BF16 else size * 256 * U32)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("m,n", [(10, 30), (300, 400), (1100, 2000), (2100, 4001)])
def test_matmul8_nan_stays_in_its_row_and_column(odt, m, n):
    a, b = randn(m, 300, seed=1), randn(n, 300, seed=2)
    a[m - 1, 150], b[3, 299] = float("nan"), float("inf")
    (qa, sa), (qb, sb) = as8(a, 1), as8(b, 128)
    out = torch.zeros(m, n, device=DEV, dtype=odt)
    lsgd.matmul8(qa, sa, qb, sb, out)
    want = torch.zeros(m, n, dtype=torch.bool, device=DEV)
    want[m - 1], want[:, 3] = True, True
    assert torch.equal(torch.isnan(out), want) and torch.isfinite(out[~want]).all()


def test_matmul8_empty():
    q, s = lsgd.empty8(3, 0)
    out = nans(3, 3)
    lsgd.matmul8(q, s, q, s, out)
    assert torch.count_nonzero(out) == 0
    q0, s0 = lsgd.empty8(0, 128)
    q1, s1 = as8(randn(4, 128), 1)
    lsgd.matmul8(q0, s0, q1, s1, nans(0, 4))


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("m,n,k", [
    (1, 1, 1), (2, 3, 5), (63, 16, 128), (64, 128, 128), (65, 129, 130), (500, 7, 1000), (1000, 300, 77), (4099, 40, 260),
    (257, 513, 640), (129, 1000, 1025), (3001, 256, 256), (64, 9, 140), (2050, 1021, 2000), (4097, 2047, 1100), (300, 4100, 4300),
    (700, 5001, 4999), (2500, 4096, 4096), (3001, 2051, 4001), (1, 8001, 8000), (8666, 1537, 2900),
    (11999, 2047, 1290)])
def test_weight_grad8(odt, m, n, k):
    x = randn(m, k, seed=m) * torch.exp(randn(m, k, seed=n))
    g = randn(m, n, seed=k, dtype=BF16)
    q, s = as8(x, 1)
    v = values(q, s, 1, k)
    want, size = g.double().t().contiguous() @ v, g.double().abs().t().contiguous() @ v.abs()
    for accumulate in (False, True):
        buf = randn(n + 1, k, seed=7, dtype=odt) if accumulate else nans(n + 1, k, dtype=odt)
        before = buf.clone()
        lsgd.weight_grad8(g, q, s, buf[:n], accumulate=accumulate)
        ref = want + before[:n].double() if accumulate else want
        # m exact products summed in binary32 (padding adds zeros), the addition, the rounding
        bound = size * ((m + 1) * U32) + ref.abs() * U32
        bound = bound * 1.01 + ref.abs() * HALF[BF16] * 1.01 if odt == BF16 else bound
        assert_close(buf[:n], ref, bound, "accumulate=%s" % accumulate)
        kind = torch.int32 if odt == F32 else torch.int16
        assert torch.equal(buf[n].view(kind), before[n].view(kind))
        again = before.clone()
        lsgd.weight_grad8(g, q, s, again[:n], accumulate=accumulate)
        assert torch.equal(again[:n], buf[:n])


def test_weight_grad8_non_finite_rows():
    """An infinity in the gradient meets its column's outputs, a NaN in x its column."""
    m, n, k = 130, 20, 300
    x, g = randn(m, k, seed=1), randn(m, n, seed=2, dtype=BF16)
    g[m - 1, 4], x[7, 200] = float("inf"), float("nan")
    q, s = as8(x, 1)
    out = torch.zeros(n, k, device=DEV)
    lsgd.weight_grad8(g, q, s, out)
    bad = torch.zeros(n, k, dtype=torch.bool, device=DEV)
    bad[4], bad[:, 200] = True, True
    assert not torch.isfinite(out[bad]).any() and torch.isfinite(out[~bad]).all()


def test_weight_grad8_no_rows():
    q, s = lsgd.empty8(0, 40)
    out = nans(3, 40)
    lsgd.weight_grad8(torch.empty(0, 3, dtype=BF16, device=DEV), q, s, out)
    assert torch.count_nonzero(out) == 0
    out = randn(3, 40)
    before = out.clone()
    lsgd.weight_grad8(torch.empty(0, 3, dtype=BF16, device=DEV), q, s, out, accumulate=True)
    assert torch.equal(out, before)


# ---------------------------------------------------------------- together

def test_a_model_s_step():
    """Table -> 8-bit linear layer -> squared error, two workers: forward from
    the copies, gradients into the workers' buffers, one step over both
    parameters, copies again. Gradients against binary64 derivatives of the same
    quantised numbers."""
    rows, dim, wide, n, N = 50, 136, 72, 90, 2
    params = [randn(rows, dim, seed=1) * 0.5, randn(wide, dim, seed=2) * 0.1]
    mom = [torch.zeros_like(p) for p in params]
    replicas = [[torch.empty(rows, dim, device=DEV, dtype=BF16), torch.empty(wide, dim, device=DEV, dtype=BF16)] for _ in range(N)]
    grads = [[nans(rows, dim), nans(wide, dim)] for _ in range(N)]
    plan = lsgd.Plan(params, mom, grads, [0, 1], 2, replicas)
    plan.copy_out()
    w8, w8t = lsgd.empty8(wide, dim, 128), lsgd.empty8(dim, wide, 128)
    want = [torch.zeros_like(p, dtype=torch.float64) for p in params]
    lsgd.copy_out8(params[1], [w8], [w8t])
    for w in range(N):
        tokens = zipf(n, rows, w)
        x, y = nans(n, dim, dtype=BF16), nans(n, wide, dtype=BF16)
        lsgd.embed_lookup(replicas[w][0], tokens, x, scale=3.0)
        x8 = as8(x, 1)
        lsgd.matmul8(*x8, *w8, y)
        dy = (y - randn(n, wide, seed=20 + w, dtype=BF16)) / n
        lsgd.weight_grad8(dy, *x8, grads[w][1])
        dy8 = as8(dy, 1)
        dx = nans(n, dim)
        lsgd.matmul8(*dy8, *w8t, dx)
        lsgd.embed_grad([dx], [tokens], grads[w][0], scale=3.0)
        # the same from the definitions
        dw = dy.double().t().contiguous() @ values(*x8, 1, dim)
        dxr = values(*dy8, 1, wide) @ values(*w8, 128, dim)
        dt = torch.zeros(rows, dim, dtype=torch.float64, device=DEV).index_add_(0, tokens, dxr * 3)
        assert_close(grads[w][1], dw, (n + 1) * U32 * (dy.double().abs().t().contiguous() @ values(*x8, 1, dim).abs()) + dw.abs() * U32)
        each = values(*dy8, 1, wide).abs() @ values(*w8, 128, dim).abs() * 3
        size = torch.zeros_like(dt).index_add_(0, tokens, each)
        assert_close(grads[w][0], dt, size * ((128 + n + 2) * U32) + dt.abs() * U32)
        want[0] += grads[w][0].double() / N
        want[1] += grads[w][1].double() / N
    before = [p.clone() for p in params]
    plan.step(0.5, 0.9, 0.0)
    for p, b, g in zip(params, before, want):
        assert_close(p, b.double() - 0.5 * g, (b.double().abs() + g.abs()) * 4 * U32)
    assert torch.equal(replicas[1][0], params[0].to(BF16))
    plan.close()


def test_captured_and_replayed():
    """All six in one graph, on another stream than the tensors' own, replayed
    on new inputs with eager work between, against eager results."""
    rows, dim, n, wide = 40, 200, 4500, 96

    def inputs(seed):
        return zipf(n, rows, seed), randn(n, dim, seed=seed), randn(wide, dim, seed=seed + 1), randn(n, wide, seed=seed + 2, dtype=BF16)
    tokens, g, p, dy = inputs(1)
    ws1 = torch.empty(lsgd.embed_grad_workspace_size(1, n, rows, dim), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(max(1, lsgd.weight_grad8_workspace_size(n, wide, dim)), dtype=torch.uint8, device=DEV)

    def call(out):
        lsgd.embed_lookup(out["dtable"], tokens, out["x"])
        lsgd.quant8(out["x"], *out["x8"])
        lsgd.copy_out8(p, [out["w8"]])
        lsgd.matmul8(*out["x8"], *out["w8"], out["y"])
        lsgd.weight_grad8(dy, *out["x8"], out["dw"], workspace=ws2)
        lsgd.embed_grad([g], [tokens], out["dtable"], workspace=ws1)

    def room():
        return {"x": nans(n, dim, dtype=BF16), "x8": lsgd.empty8(n, dim), "w8": lsgd.empty8(wide, dim, 128),
                "y": nans(n, wide), "dw": nans(wide, dim), "dtable": torch.zeros(rows, dim, device=DEV)}
    graphed, eager = room(), room()
    call(room())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(graphed)
    graphed["dtable"].zero_()
    for seed in (1, 5, 9, 13):
        for old, new in zip((tokens, g, p, dy), inputs(seed)):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        for key in ("x", "y", "dw", "dtable"):
            assert torch.equal(graphed[key], eager[key]), (seed, key)


def test_two_streams_at_once():
    """The same calls on two streams with workspaces of their own, in flight together."""
    n, rows, dim = 20000, 500, 256
    tokens, g = [zipf(n, rows, s) for s in (1, 2)], [randn(n, dim, seed=s) for s in (3, 4)]
    x, dy = [as8(randn(n, dim, seed=s), 1) for s in (5, 6)], [randn(n, 96, seed=s, dtype=BF16) for s in (7, 8)]
    alone = [(nans(rows, dim), nans(96, dim)) for _ in range(2)]
    for s in range(2):
        lsgd.embed_grad([g[s]], [tokens[s]], alone[s][0])
        lsgd.weight_grad8(dy[s], *x[s], alone[s][1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        both = [(nans(rows, dim), nans(96, dim)) for _ in range(2)]
        torch.cuda.synchronize()
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                lsgd.embed_grad([g[s]], [tokens[s]], both[s][0])
                lsgd.weight_grad8(dy[s], *x[s], both[s][1])
        torch.cuda.synchronize()
        for s in range(2):
            assert torch.equal(both[s][0], alone[s][0]) and torch.equal(both[s][1], alone[s][1])


def test_one_graph_allocates_its_workspaces():
    """Captured without workspaces of the caller's: they live in the graph's own
    memory, so that two graphs replayed in turn keep apart."""
    n, rows, dim = 9000, 300, 64
    tokens, g = [zipf(n, rows, s) for s in (1, 2)], [randn(n, dim, seed=s) for s in (3, 4)]
    want, out, graphs = [nans(rows, dim) for _ in range(2)], [nans(rows, dim) for _ in range(2)], []
    for s in range(2):
        lsgd.embed_grad([g[s]], [tokens[s]], want[s])
    torch.cuda.synchronize()
    for s in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[s]):
            lsgd.embed_grad([g[s]], [tokens[s]], out[s])
    for _ in range(3):
        for s in range(2):
            out[s].fill_(float("nan"))
            graphs[s].replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


def test_lookup_of_more_rows_than_workgroups():
    n, dim = (1 << 24) + 5, 1025
    tokens = randint(n, 0, 3, seed=1, dtype=torch.int32)
    table, out = randn(3, dim, seed=2, dtype=BF16), nans(n, dim, dtype=BF16)
    lsgd.embed_lookup(table, tokens, out)
    for part in (slice(0, 100), slice(n - 100, n), slice(n // 2, n // 2 + 100)):
        assert torch.equal(out[part], table[tokens[part].long()])
    assert torch.equal(out[:, dim - 1], table[tokens.long(), dim - 1])


def test_offsets_past_32_bits():
    """A table and its gradient of more than 2^32 elements."""
    rows, dim = (1 << 22) + 3, 1032
    table = torch.zeros(rows, dim, device=DEV, dtype=BF16)
    tokens = torch.tensor([rows - 1, 0, rows - 2, rows - 1], device=DEV)
    table[rows - 1], table[rows - 2], table[0] = 3.0, 2.0, 1.0
    out = nans(4, dim)
    lsgd.embed_lookup(table, tokens, out)
    assert torch.equal(out[:, 0].cpu(), torch.tensor([3.0, 1.0, 2.0, 3.0])) and torch.equal(out, out[:, :1].expand(-1, dim))
    g = torch.arange(4, device=DEV, dtype=F32).view(4, 1).expand(4, dim).contiguous() + 1
    table.fill_(7.0)
    lsgd.embed_grad([g], [tokens], table)
    assert (table[rows - 1] == 5).all() and (table[0] == 2).all() and (table[rows - 2] == 3).all()
    assert torch.count_nonzero(table[1:rows - 2]) == 0


def test_activations_past_32_bits():
    """8 bits of more than 2^32 elements: the last rows as of themselves alone."""
    rows, cols = (1 << 20) + 77, 4097
    x = torch.zeros(rows, cols, device=DEV, dtype=BF16)
    x[-300:], x[:5] = randn(300, cols, seed=1), randn(5, cols, seed=2)
    codes, scales = as8(x, 1)
    for part in (slice(rows - 300, rows), slice(0, 5)):
        q, s = as8(x[part].clone(), 1)
        assert torch.equal(codes[part].view(torch.uint8), q.view(torch.uint8))
        assert torch.equal(scales[part].view(torch.uint8), s.view(torch.uint8))
    # and products and gradients of them, whose other rows count as 0
    w, last = as8(randn(130, cols, seed=3), 1), (codes[-300:].contiguous(), scales[-300:].contiguous())
    x64, w64 = values(*last, 1, cols), values(*w, 1, cols)
    want, size = x64 @ w64.t().contiguous(), x64.abs() @ w64.abs().t().contiguous()
    for odt in (F32, BF16):
        out = nans(rows, 130, dtype=odt)
        lsgd.matmul8(codes, scales, *w, out)
        bound = size * 2.0 ** -10 * 1.01 + want.abs() * HALF[BF16] * 1.01 if odt == BF16 else size * cols * U32
        assert_close(out[-300:], want, bound)
        assert torch.count_nonzero(out[5:-300]) == 0
    g = torch.zeros(rows, 66, device=DEV, dtype=BF16)
    g[-300:] = randn(300, 66, seed=4)
    out, g64 = nans(66, cols), g[-300:].double().t().contiguous()
    lsgd.weight_grad8(g, codes, scales, out)
    assert_close(out, g64 @ x64, (g64.abs() @ x64.abs()) * (300 * U32))


def test_outputs_past_32_bits():
    """Products and parameter gradients of more than 2^32 elements."""
    m, n, k = 65536 + 130, 65536 + 3, 256
    a, b = as8(randn(m, k, seed=1), 1), as8(randn(n, k, seed=2), 1)
    out = nans(m, n, dtype=BF16)
    lsgd.matmul8(*a, *b, out)
    a64, b64 = values(*a, 1, k), values(*b, 1, k)
    for i in (0, 32768, m - 1):
        want, size = b64 @ a64[i], b64.abs() @ a64[i].abs()
        assert_close(out[i], want, size * 2.0 ** -10 * 1.01 + want.abs() * HALF[BF16] * 1.01)
    assert not torch.isnan(out).any()
    del out, a, b
    g, x = randn(256, m, seed=3, dtype=BF16), as8(randn(256, n, seed=4), 1)
    out = nans(m, n, dtype=BF16)
    lsgd.weight_grad8(g, *x, out)
    x64 = values(*x, 1, n)
    for i in (0, 32768, m - 1):
        gi = g[:, i].double()
        want, size = gi @ x64, gi.abs() @ x64.abs()
        assert_close(out[i], want, size * 256 * U32 + want.abs() * HALF[BF16] * (1 + U32))
    assert not torch.isnan(out).any()


def test_copies_past_32_bits():
    rows, cols = (1 << 22) + 200, 1025
    p = torch.zeros(rows, cols, device=DEV)
    p[-256:] = randn(256, cols, seed=1)
    first = rows // 128 * 128 - 128   # the last whole block of rows, and what is behind it
    copies = [lsgd.empty8(rows, cols, 128), lsgd.empty8(cols, rows, 128)]
    lsgd.copy_out8(p, [copies[0]], [copies[1]])
    q, s = lsgd.empty8(rows - first, cols, 128)
    lsgd.copy_out8(p[first:].contiguous(), [(q, s)])
    assert torch.equal(copies[0][0][first:].view(torch.uint8), q.view(torch.uint8))
    assert torch.equal(copies[0][1][first // 128:].view(torch.uint8), s.view(torch.uint8))
    assert torch.equal(copies[1][0][:, first:rows].view(torch.uint8), q.view(torch.uint8)[:, :cols].T)


def test_copies_of_more_columns_than_a_launch_takes():
    cols = (1 << 29) + 1000
    p, q, s = torch.zeros(2, cols, device=DEV), *lsgd.empty8(2, cols, 128)
    q.view(torch.uint8).fill_(0x55)
    s.view(torch.uint8).fill_(0x55)
    full = (1 << 29) - 128   # columns of the first launch
    parts = [(0, 1024), (full - 512, full + 512), (full, cols)]
    for lo, hi in parts:
        p[:, lo:hi] = randn(2, hi - lo, seed=lo % 7)
    lsgd.copy_out8(p, [(q, s)])
    q, s = q.view(torch.uint8), s.view(torch.uint8)
    for lo, hi in parts:
        want, scales = lsgd.empty8(2, hi - lo, 128)
        lsgd.copy_out8(p[:, lo:hi].contiguous(), [(want, scales)])
        wide = want.shape[1]
        assert torch.equal(q[:, lo:lo + wide], want.view(torch.uint8))
        assert torch.equal(s[:, lo // 128:(lo + wide) // 128], scales.view(torch.uint8)[:, :wide // 128])
    assert torch.count_nonzero(q[:, 1024:full - 512]) == 0 and (s[:, 8:(full - 512) // 128] == 127).all()
    assert torch.count_nonzero(q[:, cols:]) == 0 and (s[:, -(-cols // 128):] == 127).all()


@pytest.mark.parametrize("name", ["gradient", "weights"])
def test_a_workspace_for_another_stream(name):
    """`stream` names a stream that is not the current one: the workspace that the call
    allocates is not memory that work of the current stream still reads."""
    n, rows, dim = 9000, 300, 64
    side = torch.cuda.Stream()
    if name == "gradient":
        size = lsgd.embed_grad_workspace_size(1, n, rows, dim)
        g, t, out = randn(n, dim, seed=1), zipf(n, rows, 2), nans(rows, dim)
        call = lambda **kw: lsgd.embed_grad([g], [t], out, **kw)
    else:
        size = lsgd.weight_grad8_workspace_size(n, 64, 64)
        g, x, out = randn(n, 64, seed=1, dtype=BF16), as8(randn(n, 64, seed=2), 1), nans(64, 64)
        call = lambda **kw: lsgd.weight_grad8(g, *x, out, **kw)
    assert size > 0
    call()
    want = out.clone()
    out.fill_(float("nan"))
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    held = torch.full((size,), 1, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    torch.cuda._sleep(50_000_000)
    seen = held.clone()
    del held
    call(stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert (seen == 1).all() and torch.equal(out, want)


def test_on_a_stream_of_its_own():
    side = torch.cuda.Stream()
    table, tokens = randn(30, 64, seed=1), zipf(6000, 30, 2)
    g = randn(6000, 64, seed=3)
    want = nans(30, 64)
    lsgd.embed_grad([g], [tokens], want)
    torch.cuda.synchronize()
    out, x = nans(30, 64), nans(6000, 64)
    lsgd.embed_grad([g], [tokens], out, stream=side)
    lsgd.embed_lookup(table, tokens, x, stream=side)
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(x, table[tokens])


# ---------------------------------------------------------------- the binding's two paths

def every_call():
    """One call of each, as (name, function of nothing that returns its outputs)."""
    table, tokens, x = randn(30, 72, seed=1), zipf(500, 30, 2), randn(500, 72, seed=3)
    dy, p = randn(500, 40, seed=4, dtype=BF16), randn(40, 72, seed=5)

    def lookup():
        out = nans(500, 72, dtype=BF16)
        lsgd.embed_lookup(table, tokens, out, 2)
        return [out]

    def grad():
        out = nans(30, 72)
        lsgd.embed_grad((x,), [tokens], out, scale=0.5)
        return [out]

    def quant():
        return list(as8(x, 1))

    def copy():
        a, b, t = lsgd.empty8(40, 72, 128), lsgd.empty8(40, 72, 128), lsgd.empty8(72, 40, 128)
        lsgd.copy_out8(p, [a, b], (t,))
        return [*a, *b, *t]

    def product():
        out = nans(500, 40)
        lsgd.matmul8(*as8(x, 1), *as8(p, 128), out)
        return [out]

    def weights():
        out = randn(40, 72, seed=6)
        lsgd.weight_grad8(dy, *as8(x, 1), out, accumulate=True)
        return [out]
    return {f.__name__: f for f in (lookup, grad, quant, copy, product, weights)}


@pytest.mark.parametrize("name", ["lookup", "grad", "quant", "copy", "product", "weights"])
def test_binding_paths_agree(name, monkeypatch):
    from paper_1906_05936_amd import _lib
    assert _lib._marshal is not None
    native = every_call()[name]()
    monkeypatch.setattr(_lib, "_marshal", None)
    for a, b in zip(native, every_call()[name]()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def refused():
    x, t = randn(8, 16, seed=1), torch.zeros(8, dtype=torch.int64, device=DEV)
    (q, s), (w, ws) = lsgd.empty8(8, 16), lsgd.empty8(4, 16, 128)
    g = x[:, :4].bfloat16().contiguous()
    big, many = randn(3000, 16, seed=2), torch.zeros(3000, dtype=torch.int64, device=DEV)
    return [
        (TypeError, lambda: lsgd.embed_lookup(x.half(), t, x)),
        (TypeError, lambda: lsgd.embed_lookup(x, t.short(), x)),
        (ValueError, lambda: lsgd.embed_lookup(x, t, x[:7])),
        (ValueError, lambda: lsgd.embed_lookup(x.t(), t, x)),
        (ValueError, lambda: lsgd.embed_lookup(x, t.cpu(), x)),
        (lsgd.LsgdError, lambda: lsgd.embed_lookup(x, t, x)),
        (ValueError, lambda: lsgd.embed_grad([x], [t, t], x)),
        (ValueError, lambda: lsgd.embed_grad([x, x], [t, t[:7]], x.clone())),
        (TypeError, lambda: lsgd.embed_grad([x, x], [t, t.int()], x.clone())),
        (TypeError, lambda: lsgd.embed_grad([x, x.bfloat16()], [t, t], x.clone())),
        (lsgd.LsgdError, lambda: lsgd.embed_grad([x], [t], x)),
        (lsgd.LsgdError, lambda: lsgd.embed_grad([x] * 150, [t] * 128 + [t] * 22, x.clone())),
        (lsgd.LsgdError, lambda: lsgd.embed_grad([big], [many], x.clone(), workspace=torch.empty(1, dtype=torch.uint8, device=DEV))),
        (ValueError, lambda: lsgd.quant8(x, q[:7], s)),
        (TypeError, lambda: lsgd.quant8(x, q.view(torch.int8), s)),
        (TypeError, lambda: lsgd.quant8(x.double(), q, s)),
        (ValueError, lambda: lsgd.copy_out8(x, [(q, s)])),
        (TypeError, lambda: lsgd.copy_out8(x.bfloat16(), [])),
        (ValueError, lambda: lsgd.matmul8(q, s, w, ws, x)),
        (ValueError, lambda: lsgd.matmul8(q, s[:5], w, ws, x)),
        (ValueError, lambda: lsgd.matmul8(q, s, *lsgd.empty8(4, 300), nans(8, 4))),
        (TypeError, lambda: lsgd.matmul8(x, s, w, ws, nans(8, 4))),
        (TypeError, lambda: lsgd.weight_grad8(x, q, s, nans(16, 16))),
        (ValueError, lambda: lsgd.weight_grad8(g, q, s, nans(5, 16))),
        (ValueError, lambda: lsgd.weight_grad8(g, q, s, nans(4, 200))),
    ]


@pytest.mark.parametrize("k", range(25))
def test_refusals_agree(k, monkeypatch):
    from paper_1906_05936_amd import _lib
    kind, call = refused()[k]
    texts = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(_lib, "_marshal", None)
        with pytest.raises(kind) as e:
            call()
        texts.append(str(e.value))
    assert texts[0] == texts[1]
