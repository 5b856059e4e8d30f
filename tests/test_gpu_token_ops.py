"""The operators of a token policy against their definitions in 64 bits, where they can go wrong: one token to long rows, odd sizes
and strides, masks that leave nothing, lowest values, infinities and NaN in places that do not count, empty sequences, streams and
graphs, results in the memory of the inputs.

Tolerances count roundings (u = half a step: fp32 2^-24, bf16 2^-8, fp16 2^-11).  A sum of n positive terms in several running sums that
are joined in a tree is off by at most (n / 64 + 32) u of its value (64: the smallest number of running sums a row is added up in)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2509_16434_amd import learner as L

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24
torch = pytest.importorskip("torch")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rnd(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def matrix(rows, cols, dtype, seed, pad=0, shift=0, scale=3.0):
    """[rows][cols] with row stride cols + pad, `shift` elements behind an aligned address; the gaps hold NaN."""
    store = torch.full((shift + rows * (cols + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
    m = store[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_((torch.randn(rows, cols, generator=rnd(seed), device="cuda") * scale).to(dtype))
    return m, store


def copy_in_place(x, store):
    """A copy of the matrix x, which lies in `store`, at the same alignment and row stride (a row's sums are added up in an order that
    goes by its alignment)."""
    return store.clone().as_strided(x.shape, x.stride(), x.storage_offset())


# ------------------------------------------------------------------------------------------------------------ rows of logits

def row_definition(x, target, temperature):
    """(active, z - m, p, logp, H) in 64 bits; H and products with p = 0 count 0."""
    z = x.double() / temperature
    ok = (target >= 0) & (target < x.shape[1])
    z = torch.where(ok[:, None], z, 0.0)
    m = z.amax(1, keepdim=True)
    active = ok & (m[:, 0] != -math.inf)
    d = torch.where(active[:, None], z - torch.where(m == -math.inf, 0.0, m), 0.0)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    at = torch.where(ok, target, 0).long()[:, None]
    logp = (d.gather(1, at) - s.log())[:, 0]
    ent = s.log()[:, 0] - torch.where(e > 0, e * d, 0.0).sum(1) / s[:, 0]
    return active, at, d, e / s, torch.where(active, logp, 0.0), torch.where(active, ent, 0.0)


def row_tolerance(d, p, at, V):
    """What fp32 may lose in logp and H of a row: roundings of z_t - m (difference, 1/T, product), of every exponent (three roundings of
    |d| and two steps of exp2 each, weighted by p), of the sums, the logarithm and the last differences."""
    spread = torch.where(p > 0, p * d.abs(), 0.0).sum(1)
    zt = d.gather(1, at)[:, 0].abs()
    zt = torch.where(torch.isinf(zt), 0.0, zt)
    logs = math.log(V)
    tol = U32 * (4 * zt + 8 * spread + V / 64 + 48 + 4 * logs)
    square = torch.where(p > 0, p * d * d, 0.0).sum(1)
    return tol, U32 * (8 * square + (V / 64 + 56) * (1 + spread) + 4 * logs)


SHAPES = [(1, 1), (3, 2), (5, 63), (7, 64), (129, 65), (64, 256), (17, 1000), (2, 4097), (33, 8192), (9, 16385), (4, 50257), (1, 131075), (700, 33), (2, 262147),
          (300, 12289), (40, 70001), (9001, 24), (3, 160001), (50, 300), (50, 700), (2, 204803)]
HARD = {"plain": 0, "banned": 1, "lowest": 2}


def logits_case(rows, vocab, dtype, seed, pad=0, shift=0, kind="plain"):
    x, store = matrix(rows, vocab, dtype, seed, pad, shift)
    target = torch.randint(0, vocab, (rows,), generator=rnd(seed + 1), device="cuda").to(torch.int32)
    if kind != "plain":
        low = -math.inf if kind == "banned" else torch.finfo(dtype).min
        ban = torch.rand(rows, vocab, generator=rnd(seed + 2), device="cuda") < 0.5
        ban.scatter_(1, target.long()[:, None], False)
        x.masked_fill_(ban, low)
        if rows > 3:
            x[1] = low                      # a row whose mask leaves nothing
            x[2] = low
            x[2, vocab - 1] = 1.0           # a row that it leaves one token of
            target[2] = vocab - 1
            target[3] = -1                  # an idle row, with NaN among its logits
            x[3, 0] = float("nan")
    if rows > 6:
        target[5], target[6] = vocab, -100
        x[6] = float("nan")
    return x, store, target


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_token_logp(rows, vocab, dtype):
    for k, (temperature, pad, shift, kind) in enumerate(((1.0, 0, 0, "plain"), (0.7, 3, 1, "banned"), (1.3, 1, 5, "lowest"))):
        x, _, target = logits_case(rows, vocab, TYPES[dtype], 100 * k + rows, pad, shift, kind)
        active, at, d, p, logp, ent = row_definition(x, target, temperature)
        tol, tol_ent = row_tolerance(d, p, at, vocab)
        for want in (False, True):
            got, got_ent, stat = L.token_logp(x, target, temperature=temperature, want_entropy=want)
            assert bool(((got.double() - logp).abs() <= tol).all()), (kind, float((got.double() - logp).abs().max()))
            assert bool((got[~active] == 0).all()) and (got_ent is None) == (not want)
            if want:
                assert bool(((got_ent.double() - ent).abs() <= tol_ent).all()), (kind, float((got_ent.double() - ent).abs().max()))
        assert torch.equal(stat, L.token_logp(x, target, temperature=temperature)[2]), "twice the same"


def gradient_definition(active, at, d, p, g, h, ent, temperature):
    logq = torch.where(p > 0, p.log(), 0.0)
    grad = -p * (g[:, None] + h[:, None] * (logq + ent[:, None]))
    grad.scatter_add_(1, at, g[:, None])
    size = p * (g.abs()[:, None] + h.abs()[:, None] * (logq.abs() + ent.abs()[:, None] + 1))
    size.scatter_add_(1, at, g.abs()[:, None])
    zero = ~active[:, None]
    return grad.masked_fill(zero, 0.0) / temperature, size.masked_fill(zero, 0.0) / temperature


def gradient_tolerance(grad, size, d, tol, V, dtype):
    """Half a step of the type, and of the fp32 value before it: p is off by its exponent's roundings (|d|) and by those of the row's sums
    (tol, of the logarithm; the roundings of adding up again), everything else by a few."""
    far = torch.where(torch.isinf(d), 0.0, d.abs())
    rel = U32 * (8 * far + V / 64 + 64) + 2 * tol[:, None]
    return half_step(dtype) * grad.abs() * 1.001 + rel * size + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_token_logp_backward(rows, vocab, dtype):
    dt = TYPES[dtype]
    for k, (temperature, pad, shift, kind) in enumerate(((1.0, 0, 0, "plain"), (0.7, 3, 1, "banned"), (1.3, 1, 5, "lowest"))):
        x, store, target = logits_case(rows, vocab, dt, 100 * k + rows, pad, shift, kind)
        active, at, d, p, _, ent = row_definition(x, target, temperature)
        tol, tol_ent = row_tolerance(d, p, at, vocab)
        g, h = (torch.randn(rows, generator=rnd(7 + q), device="cuda") for q in range(2))
        logp, got_ent, stat = L.token_logp(x, target, temperature=temperature, want_entropy=True)
        for with_ent in (False, True):
            out, _ = matrix(rows, vocab, dt, 1, 2 * pad, 3)
            frame = out.new_empty(0).set_(out.untyped_storage()).clone()
            got = L.token_logp_backward(x, target, stat, g, temperature=temperature, entropy=got_ent, dentropy=h if with_ent else None, out=out)
            assert got.data_ptr() == out.data_ptr()
            want, size = gradient_definition(active, at, d, p, g.double(), h.double() * with_ent, ent, temperature)
            bound = gradient_tolerance(want, size, d, tol + with_ent * (tol_ent + tol) * h.abs().double() / (g.abs().double() + h.abs().double()), vocab, dt)
            off = (got.double() - want).abs()
            assert bool((off <= bound).all()), (kind, with_ent, float((off / bound).max()))
            # what lies between the rows stays
            now = out.new_empty(0).set_(out.untyped_storage()).clone()
            inside = torch.zeros_like(now, dtype=torch.bool)
            inside[3:3 + rows * (vocab + 2 * pad)].view(rows, -1)[:, :vocab] = True
            assert torch.equal(now[~inside].view(torch.uint8), frame[~inside].view(torch.uint8))
        there = copy_in_place(x, store)
        here = L.token_logp_backward(there, target, stat, g, temperature=temperature, out=there)
        assert here.data_ptr() == there.data_ptr()
        assert torch.equal(there, L.token_logp_backward(x, target, stat, g, temperature=temperature)), "in the logits' own memory"


def loss_definition(x, target, old, adv, ref, weight, scale, temperature, lo, hi, kl_coef, ent_coef):
    active, at, d, p, logp, ent = row_definition(x, target, temperature)
    old, adv = (torch.where(active, v.double(), 0.0) for v in (old, adv))
    lr = torch.where(active, logp - old, 0.0)
    rho = lr.exp()
    s1, s2 = rho * adv, rho.clamp(1 - lo, 1 + hi) * adv
    w = torch.where(active, (weight.double() if weight is not None else torch.ones_like(adv)) * scale, 0.0)
    g = torch.where(s1 <= s2, -s1, 0.0)
    kl = torch.zeros_like(g)
    if ref is not None:
        far = torch.where(active, ref.double() - logp, 0.0)
        kl = far.exp() - far - 1
        g = g + kl_coef * (1 - far.exp())
    pi = -torch.minimum(s1, s2)
    n = max(int(active.sum()), 1)
    parts = [(w * v).sum().item() for v in (pi, kl, ent)]
    clipped = ((rho < 1 - lo) | (rho > 1 + hi)) & active
    stats = [parts[0] + kl_coef * parts[1] - ent_coef * parts[2], parts[0], parts[1], parts[2] * (ent_coef != 0),
             (torch.where(active, rho - 1 - lr, 0.0)).sum().item() / n, clipped.sum().item() / n, int(active.sum()), 0.0]
    return active, at, d, p, logp, ent, w, g, rho, stats


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_token_loss(rows, vocab, dtype):
    dt = TYPES[dtype]
    for k, (temperature, pad, shift, kind, kl_coef, ent_coef, weighted) in enumerate((
            (1.0, 0, 0, "plain", 0.0, 0.0, False), (0.7, 3, 1, "banned", 0.1, 0.02, True), (1.3, 1, 5, "lowest", 0.05, 0.0, True), (1.0, 0, 0, "banned", 0.0, 0.3, False))):
        x, store, target = logits_case(rows, vocab, dt, 100 * k + rows, pad, shift, kind)
        base = row_definition(x, target, temperature)[4]
        noise = lambda q, a: (a * torch.randn(rows, generator=rnd(q), device="cuda"))  # noqa: E731
        old, ref, adv = (base + noise(11, 0.2)).float(), (base + noise(12, 0.4)).float(), noise(13, 1.0)
        idle = ~((target >= 0) & (target < vocab))
        old[idle], adv[idle], ref[idle] = float("nan"), float("nan"), float("nan")   # not read
        # ratios inside 1e-4 of a border may be taken either way by 32 and 64 bits: they are moved off it
        for border in (0.8, 1.3):
            near = ((base - old.double()).exp() / border - 1).abs() < 1e-3
            old = torch.where(near, old + 0.01, old)
        weight = torch.rand(rows, generator=rnd(14), device="cuda") if weighted else None
        hp = dict(scale=16.0 / rows, temperature=temperature, clip_lo=0.2, clip_hi=0.3, kl_coef=kl_coef, ent_coef=ent_coef)
        use_ref = ref if kl_coef else None
        active, at, d, p, logp, ent, w, g, rho, stats = loss_definition(x, target, old, adv, use_ref, weight, hp["scale"], temperature, 0.2, 0.3, kl_coef, ent_coef)
        got, got_stats, got_logp = L.token_loss(x, target, old, adv, logp_ref=use_ref, weight=weight, **hp)
        tol, tol_ent = row_tolerance(d, p, at, vocab)
        assert bool(((got_logp.double() - logp).abs() <= tol).all())
        want, size = gradient_definition(active, at, d, p, torch.where(active, w * g, 0.0), torch.where(active, -ent_coef * w, 0.0), ent, temperature)
        # the coefficients: exp of a difference off by tol (and the roundings of logp - old), of x by as much
        move = (tol + U32 * (logp.abs() * 4 + 8)) * torch.where(active, w.abs() * (rho * adv.double().abs().nan_to_num() + kl_coef * 4 + ent_coef), 0.0)
        ref_rho = torch.where(active, (ref.double() - logp).exp(), 0.0) if kl_coef else torch.zeros_like(logp)
        move = move + (tol + U32 * (logp.abs() * 4 + 8)) * w.abs() * kl_coef * ref_rho
        onehot = torch.zeros_like(p).scatter_(1, at, 1.0)
        bound = gradient_tolerance(want, size, d, tol + tol_ent * (ent_coef > 0), vocab, dt) + (move[:, None] * (p + onehot)) / temperature * 1.01
        off = (got.double() - want).abs()
        assert bool((off <= bound).all()), (kind, float((off / bound).max()))
        # sums over rows in 64 bits of terms that are off by the rows' tolerances, rounded once
        term = (w.abs() * (rho * adv.double().abs().nan_to_num() + 1)).sum().item()
        slack = float((tol + tol_ent + U32 * 8 * (logp.abs() + 1)).max()) * 4
        for q, (a, b) in enumerate(zip(got_stats.tolist(), stats)):
            size_q = term + abs(b) if q < 4 else 1 + abs(b)
            assert abs(a - b) <= slack * (size_q + (w.abs() * (ref_rho + ent)).sum().item()) + 4 * U32 * abs(b), (q, a, b)
        assert got_stats[6].item() == stats[6]
        there = copy_in_place(x, store)
        assert torch.equal(L.token_loss(there, target, old, adv, logp_ref=use_ref, weight=weight, out=there, **hp)[0], got), "in the logits' own memory, and twice the same"
        whole = there.new_empty(0).set_(there.untyped_storage()).clone()
        for m in (whole, store):   # what lies between the rows stays
            m.as_strided(x.shape, x.stride(), x.storage_offset()).zero_()
        assert torch.equal(whole.view(torch.uint8), store.view(torch.uint8))


def test_token_loss_directional_differences():
    """The gradient against differences of the loss itself along random directions (step 2^-6 of logits of order 1; the second
    differences that remain are of order step^2 = 2.4e-4, the loss's own roundings 2^-24 * 10 / 2^-6 = 4e-5)."""
    rows, V = 6, 11
    g = rnd(3)
    x = torch.randn(rows, V, generator=g, device="cuda")
    target = torch.tensor([0, 10, 3, 4, -1, 7], dtype=torch.int32, device="cuda")
    logp = L.token_logp(x, target)[0]
    # ratios well inside the clip range, or well outside on the side that carries no gradient
    old = logp + torch.tensor([0.05, -0.05, 0.6, -0.6, 0.0, 0.02], device="cuda")
    adv = torch.tensor([1.0, -1.0, -1.0, 1.0, 1.0, 0.5], device="cuda")
    ref = logp + 0.3
    call = lambda x: L.token_loss(x, target, old, adv, logp_ref=ref, kl_coef=0.2, ent_coef=0.1, clip_lo=0.2, clip_hi=0.2)  # noqa: E731
    grad = call(x)[0]
    for q in range(4):
        v = torch.randn(rows, V, generator=g, device="cuda")
        eps = 2.0 ** -6
        diff = (call(x + eps * v)[1][0] - call(x - eps * v)[1][0]).item() / (2 * eps)
        assert abs(diff - (grad * v).sum().item()) <= 5e-3, q
    assert bool((grad[4] == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [40, 300, 3000, 9000, 40000, 70000, 140000, 210000])
def test_rows_that_are_not_numbers_are_reported(vocab, dtype):
    x = torch.randn(5, vocab, device="cuda", generator=rnd(1)).to(TYPES[dtype])
    x[1, 7], x[2, vocab - 1] = float("nan"), float("inf")
    x[3] = -math.inf
    x[3, 5] = float("nan")
    x[4] = -math.inf
    t = torch.zeros(5, dtype=torch.int32, device="cuda")
    logp, ent, stat = L.token_logp(x, t, want_entropy=True)
    assert torch.isnan(logp).tolist() == [False, True, True, True, False] == torch.isnan(ent).tolist()
    z = torch.zeros(5, device="cuda")
    for ent_coef in (0.0, 0.1):
        d, stats, _ = L.token_loss(x, t, z, z + 1, ent_coef=ent_coef)
        back = L.token_logp_backward(x, t, stat, z + 1, entropy=ent, dentropy=z + ent_coef)
        assert stats[7].item() == 1.0 and math.isnan(stats[0].item()) and stats[6].item() == 4
        for grad in (d, back):
            assert bool(torch.isfinite(grad[0]).all()) and all(bool(torch.isnan(grad[k]).any()) for k in (1, 2, 3)) and not bool(grad[4].any())


def test_targets_that_a_mask_forbids():
    # a target that its mask forbids: log-probability -infinity, no NaN elsewhere
    y = torch.zeros(2, 8, device="cuda")
    y[0, 3] = -math.inf
    t = torch.tensor([3, 3], dtype=torch.int32, device="cuda")
    logp, ent, stat = L.token_logp(y, t, want_entropy=True)
    assert logp[0].item() == -math.inf and abs(ent[0].item() - math.log(7)) < 1e-5
    back = L.token_logp_backward(y, t, stat, torch.ones(2, device="cuda"), entropy=ent, dentropy=torch.ones(2, device="cuda"))
    assert bool(torch.isfinite(back).all()) and abs(back[0, 3].item() - 1) < 1e-6   # -p + 1 with p = 0


def test_a_reference_that_is_only_reported():
    """kl_coef 0 with a reference, and a target that its mask forbids: the estimate is infinite, the loss and the gradient are not."""
    x = torch.randn(3, 40, device="cuda", generator=rnd(2))
    x[1, 4] = -math.inf
    t, z = torch.full((3,), 4, dtype=torch.int32, device="cuda"), torch.full((3,), -4.0, device="cuda")
    d, stats, logp = L.token_loss(x, t, z, z, logp_ref=z)
    assert bool(torch.isfinite(d).all()) and math.isfinite(stats[0].item()) and stats[2].item() == math.inf and stats[7].item() == 0 and logp[1].item() == -math.inf
    assert torch.equal(d, L.token_loss(x, t, z, z)[0])


def test_many_rows():
    """More rows than a grid's second dimension holds: every row is that of a call on the last rows alone."""
    rows, V, first = 66001, 1100, 65000
    x = torch.randn(rows, V, device="cuda", generator=rnd(6))
    t = torch.randint(0, V, (rows,), device="cuda", generator=rnd(7)).to(torch.int32)
    g = torch.randn(rows, device="cuda", generator=rnd(8))
    part = slice(first, None)
    logp, _, stat = L.token_logp(x, t)
    d, dd = L.token_logp_backward(x, t, stat, g), L.dropout(x, 0.5, 4)
    again, _, stat_again = L.token_logp(x[part], t[part])
    assert torch.equal(logp[part], again) and torch.equal(d[part], L.token_logp_backward(x[part], t[part], stat_again, g[part]))
    ids = torch.arange(rows, device="cuda")
    assert torch.equal(dd[part], L.dropout(x[part], 0.5, 4, row_ids=ids[part]))
    assert float((d.double().sum(1)).abs().max()) < 1e-4   # a gradient by logits adds up to 0
    for q in (0, 65534, 65535, 65536, rows - 1):
        want = g[q].double() * ((torch.arange(V, device="cuda") == t[q]).double() - torch.softmax(x[q].double(), 0))
        assert float((d[q].double() - want).abs().max()) < 1e-5


def test_rows_far_apart():
    """Row offsets beyond 2^31 elements."""
    V, ld = 1001, (1 << 30) + 8
    store = torch.empty(2 * ld + V, dtype=torch.bfloat16, device="cuda")
    x = store.as_strided((3, V), (ld, 1))
    x.copy_(torch.randn(3, V, device="cuda", generator=rnd(5)))
    t = torch.tensor([1, 2, 1000], dtype=torch.int32, device="cuda")
    near = torch.empty(3, 1008, dtype=torch.bfloat16, device="cuda")[:, :V]   # rows at 16-byte boundaries, as x has them
    near.copy_(x)
    z = torch.zeros(3, device="cuda")
    for a, b in zip(L.token_logp(x, t, want_entropy=True), L.token_logp(near, t, want_entropy=True)):
        assert torch.equal(a, b)
    want = L.token_loss(near, t, z, z + 1, ent_coef=0.1)[0]
    assert torch.equal(L.token_loss(x, t, z, z + 1, ent_coef=0.1, out=x)[0], want)
    y = L.dropout(x, 0.5, 3)
    assert torch.equal(y, L.dropout(want, 0.5, 3))


def test_no_rows():
    x, t, z = torch.empty(0, 5, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    logp, ent, stat = L.token_logp(x, t, want_entropy=True)
    assert logp.shape == ent.shape == (0,) and stat.shape == (0, 2)
    d, stats, _ = L.token_loss(x, t, z, z)
    assert d.shape == (0, 5) and stats.tolist() == [0.0] * 8
    assert L.token_logp_backward(x, t, stat, z).shape == (0, 5)
    assert L.dropout(x, 0.5, 1).shape == (0, 5) and L.dropout(torch.empty(5, 0, device="cuda"), 0.5, 1).shape == (5, 0)
    off = torch.zeros(1, dtype=torch.int64, device="cuda")
    assert L.token_gae(z, z, off, 0.9, 0.9)[0].shape == (0,)
    dlogp, margin, stats = L.pair_loss(z, off)
    assert dlogp.shape == margin.shape == (0,) and stats.tolist() == [0.0] * 7
    hp = L.PairHParams(0, 0, 0.1, 0.0, 1.0)   # through the C call: nothing but the statistics is there
    stats.fill_(7.0)
    torch.cuda.synchronize()
    assert L._lib.ppo_pair_loss(0, 0, None, None, None, None, C.byref(hp), None, None, stats.data_ptr(), None, 0, None) == 0
    torch.cuda.synchronize()
    assert stats.tolist() == [0.0] * 7
    dlogp, margin, stats = L.pair_loss(torch.full((700,), 3.0, device="cuda"), off)   # tokens, but no pair
    assert dlogp.tolist() == [0.0] * 700 and stats.tolist() == [0.0] * 7
    dlogp, margin, stats = L.pair_loss(z, torch.zeros(9, dtype=torch.int64, device="cuda"))   # pairs, but no token
    assert dlogp.shape == (0,) and margin.tolist() == [0.0] * 4 and stats.tolist() == [0.0] * 7
    for a in L.token_gae(torch.ones(5000, device="cuda"), torch.ones(5000, device="cuda"), off, 0.9, 0.9):   # tokens, but no sequence
        assert not bool(a.any())
    # only idle rows
    x, t = torch.randn(3, 5, device="cuda"), torch.full((3,), -1, dtype=torch.int32, device="cuda")
    d, stats, logp = L.token_loss(x, t, x[:, 0].contiguous(), x[:, 1].contiguous(), ent_coef=0.5)
    assert not bool(d.any()) and stats.tolist() == [0.0] * 8 and not bool(logp.any())


# --------------------------------------------------------------------------------------------------------------- sequences

def cuts(lengths, before=0, behind=0):
    o = before + np.concatenate([[0], np.cumsum(lengths)])
    return torch.tensor(o, dtype=torch.int64, device="cuda"), int(o[-1]) + behind


PAIR_LENGTHS = [([1], [1]), ([0], [5]), ([3, 0, 64, 1], [2, 0, 65, 1]), ([5000], [1]), ([257, 1000, 31], [513, 2, 4099]), ([1] * 300, [2] * 300), ([100003, 7], [50001, 9]),
                ([0, 0], [0, 0]), (list(range(40)), list(range(40, 0, -1))), ([5] * 256, [3] * 256), ([5] * 257, [3] * 257), ([700] * 130, [90] * 130), ([6000] * 20, [9000] * 20), ([2] * 5000, [1] * 5000), ([150] * 2100, [90] * 2100)]


def pair_definition(logp, ref, keep, off, pairs, kind, beta, ls, mean, scale):
    x = logp.double().cpu().numpy() - (0 if ref is None else ref.double().cpu().numpy())
    off, grad, margin, rows = off.cpu().numpy(), np.zeros(x.size), np.zeros(pairs), []
    for k in range(pairs):
        spans = [np.arange(off[s], off[s + 1]) for s in (k, k + pairs)]
        spans = [i[keep[i]] for i in spans]
        if min(map(len, spans)) == 0:
            continue
        f = [1 / len(i) if mean else 1.0 for i in spans]
        S = [math.fsum(x[i]) * q for i, q in zip(spans, f)]
        D = S[0] - S[1]
        if kind == "sigmoid":
            soft = lambda v: math.log1p(math.exp(-abs(v))) + max(-v, 0.0)  # noqa: E731
            l = (1 - ls) * soft(beta * D) + ls * soft(-beta * D)
            sig = 1 / (1 + math.exp(-beta * D)) if beta * D > -700 else 0.0
            slope = -beta * ((1 - ls) * (1 - sig) - ls * sig)
        else:
            l, slope = (D - 0.5 / beta) ** 2, 2 * (D - 0.5 / beta)
        for i, q, sign in zip(spans, f, (1, -1)):
            grad[i] = sign * slope * q * scale
        margin[k] = beta * D
        rows.append((l, float(D > 0), beta * D, beta * S[0], beta * S[1]))
    m = np.sum(rows, 0) if rows else np.zeros(5)
    n = len(rows)
    return grad, margin, [m[0] * scale] + [v / max(n, 1) for v in m[1:]] + [n, 0.0]


@pytest.mark.parametrize("case", range(len(PAIR_LENGTHS)))
def test_pair_loss(case):
    chosen, rejected = PAIR_LENGTHS[case]
    pairs = len(chosen)
    for k, (kind, ls, mean, with_ref, masked, before, behind) in enumerate((
            ("sigmoid", 0.0, False, True, False, 0, 0), ("sigmoid", 0.1, True, False, True, 5, 3), ("squared", 0.0, False, True, True, 1, 0),
            ("squared", 0.0, True, True, False, 0, 700), ("sigmoid", 1.0, False, False, False, 3, 0))):
        off, T = cuts(chosen + rejected, before, behind)
        g = rnd(case * 10 + k)
        logp = -torch.empty(T, device="cuda").exponential_(1.0, generator=g)
        ref = (logp + 0.2 * torch.randn(T, generator=g, device="cuda")) if with_ref else None
        mask = (torch.rand(T, generator=g, device="cuda") < 0.6).to(torch.uint8) if masked else None
        keep = np.ones(T, bool) if mask is None else mask.cpu().numpy() != 0
        beta, scale = 0.125, 0.5 / pairs
        if masked:
            hide = torch.from_numpy(~keep).cuda()
            logp[hide] = float("nan")
            if ref is not None:
                ref[hide] = float("inf")
        grad, margin, stats = pair_definition(torch.nan_to_num(logp), None if ref is None else torch.nan_to_num(ref, posinf=0.0), keep, off, pairs, kind, beta, ls, mean, scale)
        got, got_margin, got_stats = L.pair_loss(logp, off, logp_ref=ref, mask=mask, kind=kind, beta=beta, label_smoothing=ls, length_mean=mean, scale=scale)
        # everything is held in 64 bits and rounded once; label_smoothing and scale are fp32 arguments (2 u of relative error in the sigmoid's
        # slope, which is a difference of two numbers of at most beta)
        near = lambda a, b, size: np.abs(a - b) <= 2 * U32 * np.abs(b) + 4 * U32 * size + 1e-30  # noqa: E731
        assert near(got.double().cpu().numpy(), grad, beta * scale * (kind == "sigmoid") + np.abs(grad)).all()
        assert near(got_margin.double().cpu().numpy(), margin, 0).all()
        assert all(near(a, b, abs(b)) for a, b in zip(got_stats.tolist(), stats)), (got_stats.tolist(), stats)
        again = L.pair_loss(logp, off, logp_ref=ref, mask=mask, kind=kind, beta=beta, label_smoothing=ls, length_mean=mean, scale=scale)
        assert torch.equal(got, again[0]) and torch.equal(got_stats, again[2])


def test_pair_loss_extremes():
    """Margins that saturate the sigmoid, and sums that cancel: 20000 tokens of -30 against 20000 that differ in one by 2^-10."""
    off, T = cuts([20000, 1, 1] + [20000, 1, 1])
    logp = torch.full((T,), -30.0, device="cuda")
    logp[20002] = -30.0 + 2.0 ** -10        # the first rejected token
    logp[20000], logp[40002] = 1e5, -1e5    # a pair far on the right side
    logp[20001], logp[40003] = -1e5, 1e5    # and one far on the wrong side
    grad, margin, stats = L.pair_loss(logp, off, beta=1.0)
    assert margin.tolist() == [-(2.0 ** -10), 2e5, -2e5]
    assert grad[20000].item() == 0.0 and grad[20001].item() == -1.0 and abs(grad[0].item() + 0.5 + 2.0 ** -12) < 1e-6
    assert abs(stats[0].item() / 2e5 - 1) < 1e-5 and stats[6].item() == 0


def test_offsets_outside_the_arrays_reach_no_memory():
    """Offsets that are wrong are held inside [0, tokens]; the other arrays keep their guards."""
    T = 100
    store = torch.full((T + 64,), 7.0, device="cuda")
    logp = store[32:32 + T]
    off = torch.tensor([-(1 << 40), 50, 1 << 50], dtype=torch.int64, device="cuda")
    want = torch.tensor([0, 50, 100], dtype=torch.int64, device="cuda")
    for a, b in zip(L.pair_loss(logp, off), L.pair_loss(logp, want)):
        assert torch.equal(a, b)
    for a, b in zip(L.token_gae(logp, logp, off, 0.9, 0.8), L.token_gae(logp, logp, want, 0.9, 0.8)):
        assert torch.equal(a, b)
    down = torch.tensor([60, 20, 90], dtype=torch.int64, device="cuda")   # decreasing: results unspecified, but finite and inside
    assert bool(torch.isfinite(L.pair_loss(logp, down)[0]).all()) and bool(torch.isfinite(L.token_gae(logp, logp, down, 0.9, 0.8)[0]).all())


def gae_definition(r, v, off, last, keep, gamma, lam):
    adv, ret = np.zeros(r.size), np.zeros(r.size)
    for s in range(off.size - 1):
        A, V = 0.0, 0.0 if last is None else float(last[s])
        for i in range(off[s + 1] - 1, off[s] - 1, -1):
            if keep[i]:
                A = r[i] + gamma * V - v[i] + gamma * lam * A
                V = v[i]
                adv[i], ret[i] = A, A + V
    return adv, ret


GAE_LENGTHS = [[1], [0, 1, 0, 0, 2], [63, 64, 65], [2047, 2048, 2049, 1], [1] * 5000, [0] * 7 + [3] + [0] * 9, [70001], list(range(100)), [4096] * 3, [30000, 5, 9000, 0, 1]]


@pytest.mark.parametrize("case", range(len(GAE_LENGTHS)))
def test_token_gae(case):
    for k, (gamma, lam, masked, boot, before, behind) in enumerate(((0.99, 0.95, 0.0, False, 0, 0), (0.999, 1.0, 0.4, True, 3, 5), (1.0, 1.0, 0.0, True, 0, 2000),
                                                                    (0.9, 0.0, 0.97, True, 2, 0), (0.0, 0.5, 0.3, False, 0, 0), (0.97, 0.9, 1.0, True, 1, 1))):
        off, T = cuts(GAE_LENGTHS[case], before, behind)
        g = rnd(case * 10 + k)
        r, v = 0.1 * torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
        last = torch.randn(off.numel() - 1, generator=g, device="cuda") if boot else None
        mask = (torch.rand(T, generator=g, device="cuda") >= masked).to(torch.uint8) if masked else None
        keep = np.ones(T, bool) if mask is None else mask.cpu().numpy() != 0
        if masked:
            hide = torch.from_numpy(~keep).cuda()
            r[hide], v[hide] = float("nan"), float("inf")
        rr, vv = (np.nan_to_num(x.double().cpu().numpy(), posinf=0.0) for x in (r, v))
        adv, ret = gae_definition(rr, vv, off.cpu().numpy(), None if last is None else last.double().cpu().numpy(), keep, gamma, lam)
        got, got_ret = L.token_gae(r, v, off, gamma, lam, last_value=last, mask=mask)
        # 64 bits inside, rounded once; what 64 bits lose over 70001 tokens is far below a rounding to 32
        for a, b in ((got, adv), (got_ret, ret)):
            off_by = np.abs(a.double().cpu().numpy() - b)
            assert (off_by <= U32 * np.abs(b) * 1.01 + 1e-10).all(), (k, off_by.max())
        assert torch.equal(got, L.token_gae(r, v, off, gamma, lam, last_value=last, mask=mask)[0])


@pytest.mark.parametrize("lengths", [[3000001], [100000, 2800000, 0, 7], [9000000], [8500000, 400001], [4096] * 2200])
def test_token_gae_over_many_tiles(lengths):
    """Long batches, by the recurrence itself: every advantage and its successor's, each rounded once, satisfy it to their roundings; the last
    tokens give the boundary values."""
    off, T = cuts(lengths)
    g = rnd(len(lengths))
    r, v = 0.1 * torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    last = torch.randn(len(lengths), generator=g, device="cuda")
    for gamma, lam in ((0.9999, 1.0), (0.99, 0.95)):
        adv, ret = (x.double() for x in L.token_gae(r, v, off, gamma, lam, last_value=last))
        nonempty = off[1:] > off[:-1]
        tails = (off[1:] - 1)[nonempty]
        after, v_after = torch.cat([adv[1:], adv[:1]]), torch.cat([v[1:], v[:1]]).double()
        after[tails], v_after[tails] = 0.0, last.double()[nonempty]
        rest = adv - (r.double() + gamma * v_after - v.double() + gamma * lam * after)
        assert bool((rest.abs() <= 1.01 * U32 * (adv.abs() + after.abs()) + 1e-10).all())
        assert bool(((ret - adv - v.double()).abs() <= 1.01 * U32 * (ret.abs() + adv.abs()) + 1e-10).all())


def test_token_gae_is_ppo_gae_on_full_sequences():
    """Sequences of one length without masks and dones: the learner's own advantages, to its tolerance."""
    from oracle import ppo_oracle as orc
    T, N = 16, 37
    g = rnd(8)
    r, v, last = torch.randn(N, T, generator=g, device="cuda"), torch.randn(N, T, generator=g, device="cuda"), torch.randn(N, generator=g, device="cuda")
    off = torch.arange(N + 1, device="cuda") * T
    adv, ret = L.token_gae(r.view(-1), v.view(-1), off, 0.99, 0.95, last_value=last)
    t = lambda x: np.ascontiguousarray(x.cpu().numpy().T)  # noqa: E731
    oadv, oret = orc.gae(t(r), np.zeros((T, N), np.uint8), t(v), last.cpu().numpy(), 0.99, 0.95)
    np.testing.assert_allclose(adv.view(N, T).cpu().numpy().T, oadv, rtol=1e-5, atol=1e-5)
    np.testing.assert_allclose(ret.view(N, T).cpu().numpy().T, oret, rtol=1e-5, atol=1e-5)


# ------------------------------------------------------------------------------------------------------------------ dropout

def mask_definition(seed, layer, ids, cols, border):
    u, G = np.uint64, 0x9E3779B97F4A7C15

    def mix(z):
        z = (z ^ (z >> u(30))) * u(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> u(27))) * u(0x94D049BB133111EB)
        return z ^ (z >> u(31))

    wrap = lambda x: u(x % (1 << 64))  # noqa: E731
    with np.errstate(over="ignore"):
        s = mix(wrap(seed + G))
        s = mix(s ^ wrap(layer + G))
        s = mix(s ^ (np.asarray(ids, np.int64).astype(np.uint64) + u(G)))
        c = np.arange(cols)
        z = mix(s[:, None] + (c // 4 + 1).astype(np.uint64) * u(G))
        return ((z >> (c % 4 * 16).astype(np.uint64)) & u(0xFFFF)) >= u(border)


DROP_SHAPES = [(1, 1), (1, 5), (3, 2), (64, 1024), (5, 63), (129, 65), (1000, 3), (7, 4097), (300, 2048), (2, 70001), (4100, 8)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", DROP_SHAPES)
def test_dropout(rows, cols, dtype):
    dt = TYPES[dtype]
    for k, (p, seed, layer, ids, pad, shift, residual) in enumerate(((0.1, 1, 0, False, 0, 0, False), (0.5, (1 << 64) - 1, 7, True, 1, 3, True), (0.9, 1 << 40, (1 << 64) - 1, True, 8, 0, False),
                                                                     (0.25, 5, 2, False, 0, 8, True), (0.0, 1, 1, False, 3, 0, True), (1.0, 1, 1, True, 0, 1, True))):
        x, _ = matrix(rows, cols, dt, k, pad, shift)
        res = matrix(rows, cols, dt, 50 + k, 2 * pad, shift + 1)[0] if residual else None
        row_ids = torch.randint(-(1 << 62), 1 << 62, (rows,), generator=rnd(k), device="cuda") if ids else None
        if ids and rows > 2:
            row_ids[rows - 1] = row_ids[0]   # one sample twice
        border = int(p * 65536 + 0.5)
        keep = torch.from_numpy(mask_definition(seed, layer, range(rows) if row_ids is None else row_ids.cpu().numpy(), cols, border)).cuda()
        if p == 0.5:
            x[~keep] = float("nan")          # dropped: not looked at
        out, _ = matrix(rows, cols, dt, 3, pad + 1, 2)
        y = L.dropout(x, p, seed, layer=layer, row_ids=row_ids, residual=res, out=out)
        scale = 65536 / (65536 - border) if border < 65536 else 0.0
        want = torch.where(keep, x.double() * scale, 0.0)
        size = want.abs()
        if res is not None:
            want, size = want + res.double(), size + res.double().abs()
        # the factor, the product and the sum in fp32 (3 u), the result's type once
        assert bool(((y.double() - want).abs() <= half_step(dt) * 1.001 * want.abs() + 3.01 * U32 * size + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps).all())
        if res is None:
            assert bool((y[~keep] == 0).all())
        there = x.clone()
        alone = L.dropout(x.contiguous(), p, seed, layer=layer, row_ids=row_ids, residual=None if res is None else res.contiguous())
        assert torch.equal(alone, y)
        assert torch.equal(L.dropout(there, p, seed, layer=layer, row_ids=row_ids, residual=res, out=there), y)
        if res is not None:
            r2 = res.clone()
            assert torch.equal(L.dropout(x, p, seed, layer=layer, row_ids=row_ids, residual=r2, out=r2), y)


def test_dropout_drops_the_share_it_should():
    """2^22 units: the share of dropped ones is p to within five standard deviations; neighbouring rows, columns and layers agree no
    more often than independent masks do."""
    ones = torch.ones(2048, 2048, device="cuda")
    for p in (0.1, 0.5):
        m = [(L.dropout(ones, p, 9, layer=layer) == 0) for layer in (0, 1)]
        n, q = ones.numel(), int(p * 65536 + 0.5) / 65536
        assert abs(m[0].float().mean().item() - q) <= 5 * math.sqrt(q * (1 - q) / n)
        both = q * q
        for a, b in ((m[0][1:], m[0][:-1]), (m[0][:, 1:], m[0][:, :-1]), (m[0][:, 4:], m[0][:, :-4]), (m[0], m[1])):
            assert abs((a & b).float().mean().item() - both) <= 5 * math.sqrt(both * (1 - both) / a.numel()) + 1e-7


# ------------------------------------------------------------------------------------------- streams, graphs, refusals, the whole

def everything(x, target, old, ref, adv, off, mask, hidden, ids, stream=None):
    """One call of every operator; the results."""
    logp, ent, stat = L.token_logp(x, target, want_entropy=True, stream=stream)
    out = [logp, ent, stat, L.token_logp_backward(x, target, stat, adv, entropy=ent, dentropy=old, stream=stream)]
    out += L.token_loss(x, target, old, adv, logp_ref=ref, kl_coef=0.1, ent_coef=0.01, stream=stream)
    out += L.pair_loss(logp, off, logp_ref=ref, mask=mask, stream=stream)
    out += L.token_gae(adv, old, off, 0.99, 0.95, mask=mask, stream=stream)
    out.append(L.dropout(hidden, 0.3, 5, row_ids=ids, residual=hidden, stream=stream))
    return out


def everything_inputs(seed, rows, vocab):
    g = rnd(seed)
    x = torch.randn(rows, vocab, generator=g, device="cuda").to(torch.bfloat16)
    target = torch.randint(-1, vocab, (rows,), generator=g, device="cuda").to(torch.int32)
    old, ref, adv = (torch.randn(rows, generator=g, device="cuda") - c for c in (5, 5, 0))
    off = torch.cat([torch.tensor([0, rows], device="cuda"), torch.randint(0, rows, (3,), generator=g, device="cuda")]).sort()[0]
    mask = (torch.rand(rows, generator=g, device="cuda") < 0.8).to(torch.uint8)
    return x, target, old, ref, adv, off, mask, torch.randn(rows, 500, generator=g, device="cuda"), torch.randperm(rows, generator=g, device="cuda")


@pytest.mark.parametrize("rows,vocab", [(30, 200), (40, 1000), (6, 50000), (600, 9000)])
def test_on_a_side_stream_and_in_graphs(rows, vocab):
    args = everything_inputs(1, rows, vocab)
    want = everything(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = everything(*args, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(side):
        got = everything(*args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # two graphs on their own inputs, replayed in turns with new inputs between, against the eager results
    held = [[a.clone() for a in everything_inputs(2 + k, rows, vocab)] for k in range(2)]
    graphs, outs = [], []
    for h in held:
        everything(*h)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(everything(*h))
        graphs.append(graph)
    for turn in range(3):
        fresh = [everything_inputs(10 + 2 * turn + k, rows, vocab) for k in range(2)]
        for h, f in zip(held, fresh):
            for a, b in zip(h, f):
                a.copy_(b)
        for graph in graphs:
            graph.replay()
        eager = [everything(*f) for f in fresh]
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            assert all(torch.equal(a, b) for a, b in zip(o, e)), turn


def test_the_binding_refuses():
    x, t, z = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int64, device="cuda")
    wide = torch.randn(4, 20, device="cuda")   # side by side in the same rows is not an overlap
    want = L.dropout(wide[:, :8], 0.5, 1)
    assert torch.equal(L.dropout(wide[:, :8], 0.5, 1, out=wide[:, 8:16]), want) and torch.equal(wide[:, 8:16], want)
    wrong = [
        lambda: L.dropout(wide[:, :8], 0.5, 1, out=wide[:, 7:15]), lambda: L.dropout(wide[:3, :8], 0.5, 1, out=wide[1:, 4:12]),
        lambda: L.token_logp(x.double(), t), lambda: L.token_logp(x[0], t), lambda: L.token_logp(x.t(), t), lambda: L.token_logp(x, t.long()), lambda: L.token_logp(x, t[:3]),
        lambda: L.token_logp(x[:, ::2], t), lambda: L.token_logp(x, t.cpu()), lambda: L.token_loss(x, t, z, z[:2]), lambda: L.token_loss(x, t, z.half(), z),
        lambda: L.token_loss(x, t, z, z, out=x.half()), lambda: L.token_loss(x, t, z, z, out=x[:3]), lambda: L.token_logp_backward(x, t, z, z),
        lambda: L.token_logp(x[:1].expand(4, 8), t), lambda: L.dropout(x, 0.1, 1, row_ids=t), lambda: L.dropout(x, 0.1, 1, residual=x.half()),
        lambda: L.dropout(x[1:], 0.1, 1, out=x[:3]), lambda: L.token_loss(x[:, 1:], t, z, z, out=x[:, :-1]), lambda: L.pair_loss(z, off[:2]), lambda: L.pair_loss(z, off, mask=t),
        lambda: L.pair_loss(z, off.int()), lambda: L.token_gae(z, z, off, 0.9, 0.9, last_value=z), lambda: L.token_gae(z, z[:2], off, 0.9, 0.9), lambda: L.token_gae(z, z, off[:0], 0.9, 0.9),
        lambda: L.dropout(x.unsqueeze(0), 0.1, 1),
    ]
    for k, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was taken")
    for call in (lambda: L.token_logp(x, None), lambda: L.token_logp(x, [0]), lambda: L.dropout(x, "a", 1), lambda: L.dropout(x, 0.1, 1.5), lambda: L.token_logp_backward(x, t, None, z),
                 lambda: L.token_logp_backward(x, t, torch.zeros(4, 2, device="cuda"), z, dentropy=z)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(OverflowError):
        L.dropout(x, 0.1, 1 << 64)
    for call in (lambda: L.dropout(x, 1.5, 1), lambda: L.token_logp(x, t, temperature=0.0), lambda: L.token_loss(x, t, z, z, kl_coef=0.1), lambda: L.token_gae(z, z, off, 1.5, 0.9),
                 lambda: L.pair_loss(z, off, beta=-1.0), lambda: L.token_logp(torch.zeros(4, 0, device="cuda"), t)):
        with pytest.raises(L.LearnerError):
            call()


def test_one_step_of_a_token_policy():
    """The operators as a training program uses them: rollout with dropout, log-probabilities, advantages, then a shuffled minibatch:
    the same units are dropped, so every ratio is 1 and nothing is clipped; the gradient of the head's weights and of the hidden layer is
    that of the whole loss, differentiated in 64 bits."""
    g = rnd(4)
    S, H, V, p, seed = 60, 32, 130, 0.25, 77
    hidden, W = torch.randn(S, H, generator=g, device="cuda"), 0.3 * torch.randn(V, H, generator=g, device="cuda")
    off = torch.tensor([0, 13, 13, 40, 60], dtype=torch.int64, device="cuda")
    action = torch.randint(0, V, (S,), generator=g, device="cuda").to(torch.int32)
    head = lambda h: h @ W.t()  # noqa: E731
    old = L.token_logp(head(L.dropout(hidden, p, seed)), action)[0]
    adv, ret = L.token_gae(torch.randn(S, generator=g, device="cuda"), torch.randn(S, generator=g, device="cuda"), off, 0.99, 0.95)
    assert bool(torch.isfinite(adv).all())
    perm = torch.randperm(S, generator=g, device="cuda")[:41]
    mb = hidden[perm].contiguous()
    dropped = L.dropout(mb, p, seed, row_ids=perm)
    dlogits, stats, _ = L.token_loss(head(dropped), action[perm], old[perm], adv[perm], scale=1.0 / perm.numel(), ent_coef=0.01)
    # a product of 32 terms may be added up in another order in a batch of another size: logp to a few u of its size
    assert stats[5].item() == 0.0 and abs(stats[4].item()) < 1e-9 and stats[6].item() == perm.numel()
    dW, dh = dlogits.t() @ dropped, L.dropout(dlogits @ W, p, seed, row_ids=perm)
    keep = torch.from_numpy(mask_definition(seed, 0, perm.cpu().numpy(), H, int(p * 65536 + 0.5))).cuda().double() * (65536 / (65536 - int(p * 65536 + 0.5)))
    h64, W64 = mb.double().requires_grad_(), W.double().requires_grad_()
    logq = torch.log_softmax((h64 * keep) @ W64.t(), 1)
    lp = logq.gather(1, action[perm].long()[:, None])[:, 0]
    rho = (lp - old[perm].double()).exp()
    loss = -(rho * adv[perm].double()).mean() - 0.01 * -(logq.exp() * logq).sum(1).mean()
    loss.backward()
    # fp32 products of 130 and 41 terms: 200 u of the norm
    for a, b in ((dW, W64.grad), (dh, h64.grad)):
        assert float((a.double() - b).norm() / b.norm()) <= 200 * U32 * 4
    assert abs(stats[0].item() - loss.item()) <= 1e-5
    # the same answers as preference pairs: sequences 0, 1 against 2, 3 (the second chosen one is empty: one pair counts)
    logits = head(dropped := L.dropout(hidden, p, seed))
    logp, _, stat = L.token_logp(logits, action)
    dlogp, margin, pstats = L.pair_loss(logp, off, logp_ref=old + 0.1, beta=0.2)
    dW = L.token_logp_backward(logits, action, stat, dlogp).t() @ dropped
    W64 = W.double().requires_grad_()
    lp = torch.log_softmax(dropped.double() @ W64.t(), 1).gather(1, action.long()[:, None])[:, 0] - (old.double() + 0.1)
    D = lp[0:13].sum() - lp[13:40].sum()
    (-torch.nn.functional.logsigmoid(0.2 * D)).backward()
    assert pstats[5].item() == 1 and abs(margin[0].item() - 0.2 * D.item()) <= 1e-4 and margin[1].item() == 0
    assert float((dW.double() - W64.grad).norm() / W64.grad.norm()) <= 200 * U32 * 4


def test_nothing_is_allocated_and_nothing_synchronises():
    """The library's calls into the caller's arrays while a graph is being recorded, where an allocation or a synchronisation by the
    library would end the recording."""
    x, target, old, ref, adv, off, mask, hidden, ids = everything_inputs(3, 24, 3000)
    everything(x, target, old, ref, adv, off, mask, hidden, ids)
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        everything(x, target, old, ref, adv, off, mask, hidden, ids)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] >= free - (64 << 20)
