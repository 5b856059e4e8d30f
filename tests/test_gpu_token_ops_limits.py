"""The operators of a token policy at the ends of their ranges: temperatures and coefficients whose products leave fp32, infinite
log-probabilities, log-ratios next to 0, masks over whole tiles, offsets that are wrong, calls recorded into a graph.

Definitions, and tolerances that count roundings, are those of test_gpu_token_ops."""
import ctypes as C
import math

import pytest

from paper_2509_16434_amd import learner as L

from test_gpu_token_ops import test_token_logp_backward as check_token_logp_backward
from test_gpu_token_ops import test_token_loss as check_token_loss
from test_gpu_token_ops import TYPES, U32, everything_inputs, gradient_definition, gradient_tolerance, rnd, row_definition, row_tolerance

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def rows_at(temperature, rows, vocab, dtype, seed, low):
    """Logits that differ by a few temperatures, about half of them banned with `low`; a row that the mask leaves nothing of, one that it
    leaves one token of, an idle one."""
    x = (torch.randn(rows, vocab, generator=rnd(seed), device="cuda") * (3 * min(temperature, 1.0))).to(dtype)
    target = torch.randint(0, vocab, (rows,), generator=rnd(seed + 1), device="cuda").to(torch.int32)
    ban = torch.rand(rows, vocab, generator=rnd(seed + 2), device="cuda") < 0.5
    ban.scatter_(1, target.long()[:, None], False)
    x.masked_fill_(ban, low)
    x[1], x[2] = low, low
    x[2, vocab // 2], target[2], target[3] = 0.0, vocab // 2, -1
    return x, target


# every width of the kernels' groups, rows in slices, rows read twice
WIDTHS = [(5, 40), (5, 400), (5, 700), (5, 3000), (5, 9000), (5, 20000), (5, 70000), (100, 45000), (100, 210000)]
# temperature, coefficient of the entropy, what a banned logit is: 1 / T and its square beyond fp32, e of the lowest value above 0, coefficients
# whose product with a large negative number is infinite
SETTINGS = [(1e-6, 1.0, "banned"), (1e-6, 1.0, "lowest"), (1e-25, 1.0, "banned"), (1e-38, 0.1, "banned"), (3e37, 1.0, "lowest"), (1.0, 1e10, "banned"), (1.0, 1e36, "lowest")]


def vanishing(size, h, ent, temperature):
    """exp2 gives 0 below 2^-126: what a probability below that would have added to an element."""
    return 4 * 2.0 ** -126 * (size + h * (200 + ent.abs())[:, None]) / temperature


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("temperature,h,kind", SETTINGS)
@pytest.mark.parametrize("rows,vocab", WIDTHS)
def test_entropy_and_its_gradient_at_any_temperature(rows, vocab, temperature, h, kind, dtype):
    dt = TYPES[dtype]
    x, target = rows_at(temperature, rows, vocab, dt, vocab, -math.inf if kind == "banned" else torch.finfo(dt).min)
    active, at, d, p, logp, ent = row_definition(x, target, temperature)
    tol, tol_ent = row_tolerance(d, p, at, vocab)
    got, got_ent, stat = L.token_logp(x, target, temperature=temperature, want_entropy=True)
    assert bool(((got.double() - logp).abs() <= tol).all()) and bool(((got_ent.double() - ent).abs() <= tol_ent).all())
    g = 0.3 * torch.randn(rows, generator=rnd(5), device="cuda")
    for dlogp, dent in ((g, None), (g, h * torch.randn(rows, generator=rnd(6), device="cuda"))):
        back = L.token_logp_backward(x, target, stat, dlogp, temperature=temperature, entropy=got_ent if dent is not None else None, dentropy=dent).double()
        e = torch.zeros_like(ent) if dent is None else dent.double()
        want, size = gradient_definition(active, at, d, p, dlogp.double(), e, ent, temperature)
        bound = gradient_tolerance(want, size, d, tol + (dent is not None) * (tol_ent + tol), vocab, dt) + vanishing(dlogp.double().abs()[:, None], e.abs()[:, None], ent, temperature)
        off = (back - want).abs()
        assert bool((off <= bound).all()), (dent is not None, float((off / bound).nan_to_num(nan=math.inf).max()))
    # the loss: nothing is clipped, so that dL/dlogp = -rho A
    old, adv = (logp + 0.1 * torch.randn(rows, generator=rnd(7), device="cuda")).float(), 0.3 * torch.randn(rows, generator=rnd(8), device="cuda")
    for ent_coef in (0.0, h):
        grad, stats, _ = L.token_loss(x, target, old, adv, temperature=temperature, clip_lo=0.9, clip_hi=9.0, ent_coef=ent_coef)
        rho = torch.where(active, (logp - old.double()).exp(), 0.0)
        minus_h = torch.where(active, -ent_coef * torch.ones_like(ent), 0.0)
        want, size = gradient_definition(active, at, d, p, -rho * adv.double(), minus_h, ent, temperature)
        move = (tol + U32 * (4 * logp.abs() + 8)) * rho * adv.double().abs()
        bound = gradient_tolerance(want, size, d, tol + (ent_coef > 0) * tol_ent, vocab, dt) + 1.01 * move[:, None] * (p + torch.zeros_like(p).scatter_(1, at, 1.0)) / temperature
        bound = bound + vanishing((rho * adv.double().abs())[:, None], ent_coef, ent, temperature)
        off = (grad.double() - want).abs()
        assert bool((off <= bound).all()), (ent_coef, float((off / bound).nan_to_num(nan=math.inf).max()))
        # a hundred entropies of 10 times 1e36 are beyond fp32: L is infinite then, and says so
        assert stats[7].item() == (ent_coef * ent.sum().item() > torch.finfo(torch.float32).max) and (ent_coef == 0 or abs(stats[3].item() - ent.sum().item()) <= float(tol_ent.sum()) + 4 * U32 * ent.sum().item())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", WIDTHS)
def test_rows_of_one_token_have_no_gradient(rows, vocab, dtype):
    """One token left: p = 1, so that every gradient is 0 whatever the coefficients and the temperature."""
    x = torch.full((rows, vocab), -math.inf, dtype=TYPES[dtype], device="cuda")
    target = torch.randint(0, vocab, (rows,), generator=rnd(vocab), device="cuda").to(torch.int32)
    x.scatter_(1, target.long()[:, None], 2.5)
    old = torch.zeros(rows, device="cuda")
    for temperature, size in ((1.0, 1e6), (1e-3, 1e30), (6e-39, 1e9)):
        logp, ent, stat = L.token_logp(x, target, temperature=temperature, want_entropy=True)
        assert not bool(logp.any()) and not bool(ent.any())
        for dent in (None, old + size):
            assert not bool(L.token_logp_backward(x, target, stat, old + size, temperature=temperature, entropy=ent if dent is not None else None, dentropy=dent).any())
        for ent_coef in (0.0, size):
            if ent_coef * size > torch.finfo(torch.float32).max:   # dL/dH itself is beyond fp32: refused
                with pytest.raises(L.LearnerError):
                    L.token_loss(x, target, old, old + 1, scale=size, temperature=temperature, ent_coef=ent_coef)
                continue
            grad, stats, _ = L.token_loss(x, target, old, old + 1, scale=size, temperature=temperature, ent_coef=ent_coef)
            assert not bool(grad.any()) and stats[7].item() == 0


@pytest.mark.parametrize("pairs", [2, 300, 2500])
def test_pairs_of_infinite_difference(pairs):
    """A token that its mask forbids (or the reference's does) makes a difference infinite: the loss of such a pair is 0 on the right side,
    infinite on the wrong one, and with smoothing infinite on both; its gradient is finite, and 0 on the right side."""
    n, beta = 3, 0.5
    off = torch.arange(2 * pairs + 1, device="cuda") * n
    base = -torch.rand(2 * pairs * n, generator=rnd(1), device="cuda")
    at = pairs // 2   # the pair; its sequences begin at n * at and n * (pairs + at)
    D = (base[:pairs * n] - base[pairs * n:]).double().view(pairs, n).sum(1)
    others = torch.ones(pairs, dtype=torch.bool, device="cuda")
    others[at] = False
    for place, value, with_ref, sign in ((pairs + at, -math.inf, False, 1), (at, -math.inf, True, 1), (at, -math.inf, False, -1)):
        logp, ref = base.clone(), torch.zeros_like(base) if with_ref else None
        (ref if with_ref else logp)[n * place + 1] = value
        for ls in (0.0, 1.0, 0.25):
            grad, margin, stats = L.pair_loss(logp, off, logp_ref=ref, beta=beta, label_smoothing=ls, scale=1.0 / pairs)
            soft = torch.nn.functional.softplus
            rest = ((1 - ls) * soft(-beta * D) + ls * soft(beta * D))[others].sum().item() / pairs
            finite = (sign > 0 and ls == 0) or (sign < 0 and ls == 1)
            assert margin[at].item() == sign * math.inf and stats[6].item() == (not finite)
            # 64 bits inside; scale and the result are rounded once each
            assert abs(stats[0].item() - rest) <= 4 * U32 * rest if finite else stats[0].item() == math.inf
            slope = beta * (ls - (sign < 0)) / pairs
            mine = torch.cat([grad[n * at:n * (at + 1)], -grad[n * (pairs + at):n * (pairs + at + 1)]])
            assert bool(torch.isfinite(grad).all()) and bool(((mine - slope).abs() <= 4 * U32 * abs(slope)).all())


def test_a_forbidden_token_in_a_rejected_answer():
    """The whole chain: log-probability -infinity, a pair on its right side, and a gradient of the logits without NaN."""
    x = torch.randn(6, 50, generator=rnd(3), device="cuda")
    x[4, 7] = -math.inf
    target = torch.tensor([1, 2, 3, 4, 7, 6], dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 2, 3, 4, 6], dtype=torch.int64, device="cuda")   # chosen 0, 1; rejected 2, 3 (of two tokens)
    logp, _, stat = L.token_logp(x, target)
    dlogp, margin, stats = L.pair_loss(logp, off, beta=0.3)
    D = (logp[0] + logp[1] - logp[3]).item()
    assert stats[6].item() == 0 and margin[1].item() == math.inf and abs(stats[0].item() - math.log1p(math.exp(-0.3 * D))) <= 1e-6
    d = L.token_logp_backward(x, target, stat, dlogp)
    assert bool(torch.isfinite(d).all()) and not bool(d[2].any()) and not bool(d[4:].any()) and bool(d[0].any())


@pytest.mark.parametrize("size", [0.0, 2.0 ** -20, 2.0 ** -12, 2.0 ** -7, 0.1, 0.6, 3.0, 20.0])
@pytest.mark.parametrize("rows,vocab", [(1, 30), (100, 300), (300, 3000), (5, 70000)])
def test_estimates_from_log_ratios_next_to_0(rows, vocab, size):
    """exp x - 1 - x is positive for every x but 0, and keeps its digits: 12 roundings of fp32 of every term.  (exp x - 1 and x are off by one
    and a half and no roundings of about |x|, the result is about x^2 / 2; so the difference of the two is not enough below |x| = 1/2, and has
    lost a factor of 10 there.)"""
    x = torch.randn(rows, vocab, generator=rnd(1), device="cuda")
    target = torch.randint(0, vocab, (rows,), generator=rnd(2), device="cuda").to(torch.int32)
    zero = torch.zeros(rows, device="cuda")
    logp = L.token_loss(x, target, zero, zero)[2]
    far = size * torch.randn(rows, generator=rnd(3), device="cuda")
    old, ref = logp - far, logp + far
    weight = torch.rand(rows, generator=rnd(4), device="cuda") + 0.5
    stats, again = L.token_loss(x, target, old, zero, logp_ref=ref, weight=weight)[1:]
    assert torch.equal(again, logp)

    def estimate(d):
        """In 64 bits: the series where the difference loses digits."""
        term, total = d * d / 2, torch.zeros_like(d)
        for k in range(3, 20):
            total, term = total + term, term * d / k
        return torch.where(d.abs() < 0.5, total, torch.expm1(d) - d)

    # the differences that are taken, as fp32 has them (exact where the two are within a factor of two of one another)
    lr, d = (logp - old).double(), (ref - logp).double()
    want_kl, want_old = (weight.double() * estimate(d)).sum().item(), estimate(lr).mean().item()
    for got, want in ((stats[2].item(), want_kl), (stats[4].item(), want_old)):
        assert abs(got - want) <= 13 * U32 * want and (got > 0) == (want > 0), (got, want)


def test_a_result_in_the_memory_of_a_saved_tensor_is_noticed():
    """`out` is a change of its tensor that autograd sees: a backward pass that needs what it held fails instead of using the gradient in its
    place."""
    t, z = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    for call in (lambda x: L.dropout(x, 0.5, 1, out=x), lambda x: L.token_loss(x, t, z, z + 1, out=x)[0], lambda x: L.token_logp_backward(x, t, L.token_logp(x, t)[2], z + 1, out=x)):
        leaf = torch.randn(4, 8, device="cuda", requires_grad=True)
        x = leaf.exp()   # its backward pass multiplies by x
        before = x._version
        out = call(x)
        assert out is x and x._version > before
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            x.sum().backward()
    # results of their own: nothing of the inputs' history changes, and none is theirs
    leaf = torch.randn(4, 8, device="cuda", requires_grad=True)
    x = leaf.exp()
    d = L.token_loss(x, t, z, z + 1)[0]
    assert not d.requires_grad
    x.backward(d)
    assert torch.equal(leaf.grad, d * x.detach())
    with torch.inference_mode():   # no versions there
        x = torch.randn(4, 8, device="cuda")
        assert L.dropout(x, 0.5, 1, out=x) is x
    assert L.dropout(x, 0.5, 1, out=torch.empty(4, 8, device="cuda")).shape == (4, 8)


def test_no_memory_is_torchs_error():
    """A result that does not fit is torch's own OutOfMemoryError, as a caller who retries with less expects."""
    torch.cuda.empty_cache()
    x = torch.zeros((torch.cuda.memory_reserved() >> 8) + (1 << 20), 64, device="cuda")   # larger than all that may be free inside what others hold
    torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (64 << 20)) / torch.cuda.get_device_properties(0).total_memory)
    try:
        with pytest.raises(torch.OutOfMemoryError):
            L.dropout(x, 0.5, 1)
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert L.dropout(x, 0.5, 1).shape == x.shape


# ------------------------------------------------------------------------------------------ the C calls, on the caller's arrays

class Guarded:
    """An array between two others that nobody may write: everything holds the byte 0x5A first."""

    def __init__(self, n, dtype=torch.float32):
        size = n * torch.empty(0, dtype=dtype).element_size()
        self.whole = torch.full((4096 + -(-size // 256) * 256 + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
        self.size, self.inner = size, self.whole[4096:4096 + size].view(dtype)

    def ptr(self):
        return self.inner.data_ptr()

    def intact(self):
        return bool((self.whole[:4096] == 0x5A).all()) and bool((self.whole[4096 + self.size:] == 0x5A).all())


def ptr(t):
    return None if t is None else t.data_ptr()


def c_calls(x, target, old, ref, adv, off, mask, hidden, ids, stream, made):
    """One call of every operator into arrays made before (the first time: into `made`); the results."""
    rows, V = x.shape
    cols, ld, seqs, lib = hidden.shape[1], x.stride(0), off.numel() - 1, L._lib
    sizes = dict(logp=rows, ent=rows, stat=2 * rows, d=rows * V, dl=rows * V, loss_stats=8, loss_logp=rows, dlogp=rows, margin=seqs // 2, pair_stats=7, adv=rows, ret=rows, y=rows * cols)
    ws = dict(ws_logp=lib.ppo_token_logp_ws_bytes(rows, V), ws_loss=lib.ppo_token_loss_ws_bytes(rows, V), ws_pair=lib.ppo_pair_ws_bytes(seqs // 2, rows),
              ws_gae=lib.ppo_token_gae_ws_bytes(seqs, rows))
    if not made:
        made.update({k: Guarded(n, x.dtype if k in ("d", "dl") else hidden.dtype if k == "y" else torch.float32) for k, n in sizes.items()})
        made.update({k: Guarded(n, torch.uint8) for k, n in ws.items()})
    o = {k: g.ptr() for k, g in made.items()}
    code, thp, php = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}, L.TokenHParams(1.0, 0.2, 0.2, 0.1, 0.01, 1.0), L.PairHParams(0, 0, 0.1, 0.0, 1.0)
    for rc in (
            lib.ppo_token_logp(code[x.dtype], rows, V, ptr(x), ld, ptr(target), 1.0, o["logp"], o["ent"], o["stat"], o["ws_logp"], ws["ws_logp"], stream),
            lib.ppo_token_logp_backward(code[x.dtype], rows, V, ptr(x), ld, ptr(target), 1.0, o["stat"], ptr(adv), o["ent"], ptr(old), o["d"], V, stream),
            lib.ppo_token_loss(code[x.dtype], rows, V, ptr(x), ld, ptr(target), ptr(old), ptr(ref), ptr(adv), None, C.byref(thp), o["dl"], V, o["loss_logp"], o["loss_stats"],
                               o["ws_loss"], ws["ws_loss"], stream),
            lib.ppo_pair_loss(seqs // 2, rows, o["logp"], ptr(ref), ptr(mask), ptr(off), C.byref(php), o["dlogp"], o["margin"], o["pair_stats"], o["ws_pair"], ws["ws_pair"], stream),
            lib.ppo_token_gae(seqs, rows, ptr(adv), ptr(old), ptr(mask), ptr(off), None, 0.99, 0.95, o["adv"], o["ret"], o["ws_gae"], ws["ws_gae"], stream),
            lib.ppo_dropout(code[hidden.dtype], rows, cols, ptr(hidden), cols, ptr(ids), ptr(hidden), cols, 0.3, 5, 0, o["y"], cols, stream)):
        assert rc == 0, lib.ppo_last_error(None)
    return [made[k].inner for k in sizes]


@pytest.mark.parametrize("rows,vocab", [(30, 200), (128, 512), (300, 3000), (6, 50000), (9000, 40)])
def test_the_c_calls_while_a_graph_is_recorded(rows, vocab):
    """The library's calls alone between the beginning and the end of a recording, which an allocation or a synchronisation ends with an
    error; every replay, with new inputs and eager work between, gives what an eager call gives; nothing beside the results and workspaces,
    which are of the sizes asked for, is written."""
    held = [a.clone() for a in everything_inputs(20, rows, vocab)]
    made, side, graph = {}, torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c_calls(*held, side.cuda_stream, made)   # the results are allocated here, not in the recording
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        outs = c_calls(*held, side.cuda_stream, made)
    for turn in range(3):
        fresh, eager = everything_inputs(30 + turn, rows, vocab), {}
        want = c_calls(*fresh, torch.cuda.current_stream().cuda_stream, eager)
        for a, b in zip(held, fresh):
            a.copy_(b)
        for o in outs:
            o.view(torch.uint8).fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(outs, want)), turn
        assert all(g.intact() for d in (made, eager) for g in d.values())


# offsets as a program error leaves them: outside the tokens, decreasing, all at one end
WRONG = {"outside": lambda T, n: [-(1 << 40)] + [T // 2] * (n - 1) + [1 << 50], "decreasing": lambda T, n: [T - k * T // (n + 1) for k in range(n + 1)],
         "to and fro": lambda T, n: [(k * 7919) % (T + 1) for k in range(n + 1)], "behind": lambda T, n: [T + 1 + k for k in range(n + 1)],
         "before": lambda T, n: [k - n - 1 for k in range(n + 1)], "ends swapped": lambda T, n: [T] + [k * T // n for k in range(1, n)] + [0]}


@pytest.mark.parametrize("kind", WRONG)
@pytest.mark.parametrize("T,seqs", [(1, 2), (100, 2), (5003, 8), (70001, 600), (70001, 5000)])
def test_wrong_offsets_write_nothing_beside_the_results(kind, T, seqs):
    logp, last = torch.randn(T, generator=rnd(1), device="cuda"), torch.randn(seqs, generator=rnd(2), device="cuda")
    off, lib = torch.tensor(WRONG[kind](T, seqs), dtype=torch.int64, device="cuda"), L._lib
    stream, hp = torch.cuda.current_stream().cuda_stream, L.PairHParams(0, 1, 0.1, 0.0, 1.0)
    g = {k: Guarded(n) for k, n in dict(dlogp=T, margin=seqs // 2, stats=7, adv=T, ret=T).items()}
    sizes = lib.ppo_pair_ws_bytes(seqs // 2, T), lib.ppo_token_gae_ws_bytes(seqs, T)
    g["ws"], g["ws2"] = (Guarded(n, torch.uint8) for n in sizes)
    assert lib.ppo_pair_loss(seqs // 2, T, ptr(logp), None, None, ptr(off), C.byref(hp), g["dlogp"].ptr(), g["margin"].ptr(), g["stats"].ptr(), g["ws"].ptr(), sizes[0], stream) == 0
    assert lib.ppo_token_gae(seqs, T, ptr(logp), ptr(logp), None, ptr(off), ptr(last), 0.9, 0.8, g["adv"].ptr(), g["ret"].ptr(), g["ws2"].ptr(), sizes[1], stream) == 0
    torch.cuda.synchronize()
    assert all(a.intact() for a in g.values())
    assert all(bool(torch.isfinite(g[k].inner).all()) for k in ("margin", "stats", "adv", "ret"))


# ------------------------------------------------------------------------------------------------ masks over whole tiles

TILE = 2048   # tokens that a block of the advantages takes


def tile_masks(T, longest):
    """What a mask may leave of the tiles: runs of wholly masked tiles (the longest of `longest`), stretches with one token a tile, a stretch
    without a mask, and between them two tokens in five."""
    g = rnd(T)
    keep = torch.rand(T, generator=g, device="cuda") < 0.4
    keep[:700], keep[2 * TILE:5 * TILE + 17] = True, False
    single = torch.arange(7 * TILE + 1033, min(T, 20 * TILE), TILE, device="cuda")
    keep[7 * TILE:20 * TILE] = False
    keep[single] = True
    keep[22 * TILE:24 * TILE] = True
    keep[25 * TILE + 5:(25 + longest) * TILE + 9] = False
    return keep


@pytest.mark.parametrize("lengths,longest", [([60000], 3), ([5 * TILE + 20, 1, 25 * TILE, 0, 7 * TILE], 4), ([900001], 300), ([300000, 0, 700000, 5], 257), ([9000001], 1100),
                                             ([70000, 8600000, 400000], 2500)])
def test_advantages_across_masked_tiles(lengths, longest):
    """Values and advantages pass through tiles that the mask leaves nothing or one token of: the recurrence between one unmasked token and
    the next, each advantage rounded once, and the boundary values behind the last ones."""
    off = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    T, g = int(off[-1]), rnd(len(lengths))
    keep = tile_masks(T, longest)
    r, v = 0.1 * torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    r[~keep], v[~keep] = math.nan, math.inf
    last = torch.randn(len(lengths), generator=g, device="cuda")
    at = torch.cat([off.new_zeros(1), keep.cumsum(0)])[off]   # the sequences' bounds among the unmasked tokens
    rk, vk = r[keep].double(), v[keep].double()
    nonempty = at[1:] > at[:-1]
    tails = (at[1:] - 1)[nonempty]
    v_after = torch.cat([vk[1:], vk[:1]])
    v_after[tails] = last.double()[nonempty]
    for gamma, lam in ((0.9999, 1.0), (0.99, 0.95), (0.9, 0.0), (1.0, 1.0), (0.0, 0.7)):
        adv, ret = L.token_gae(r, v, off, gamma, lam, last_value=last, mask=keep.to(torch.uint8))
        assert not bool(adv[~keep].any()) and not bool(ret[~keep].any())
        a, b = adv[keep].double(), ret[keep].double()
        after = torch.cat([a[1:], a[:1]])
        after[tails] = 0.0
        rest = a - (rk + gamma * v_after - vk + gamma * lam * after)
        assert bool((rest.abs() <= 1.01 * U32 * (a.abs() + after.abs()) + 1e-10).all()), (gamma, lam, float(rest.abs().max()))
        assert bool(((b - a - vk).abs() <= 1.01 * U32 * (b.abs() + a.abs()) + 1e-10).all())


# ------------------------------------------------------------------------------------------- both sides of the rules' borders

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(32, 512), (33, 512), (64, 256), (65, 256), (128, 128), (128, 129), (129, 128), (128, 512), (64, 512)])
def test_loss_in_one_launch_and_in_two(rows, vocab, dtype):
    """At most 16384 logits in at most 128 rows are one launch."""
    assert (L._lib.ppo_token_loss_ws_bytes(rows, vocab) == 0) == (rows <= 128 and rows * vocab <= 16384)
    check_token_loss(rows, vocab, dtype)


@pytest.mark.parametrize("rows,vocab,dtype", [(1098, 65536, "bf16"), (1099, 65536, "fp16"), (2197, 16384, "fp32"), (2198, 16384, "fp32"), (140000, 513, "bf16"), (140800, 512, "bf16")])
def test_gradients_into_and_past_the_caches(rows, vocab, dtype):
    """Gradients of 144 MB and a little less and more."""
    assert abs(rows * vocab * torch.empty(0, dtype=TYPES[dtype]).element_size() / 144e6 - 1) < 3e-3
    check_token_logp_backward(rows, vocab, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [72, 73, 96, 97])
def test_loss_of_rows_in_slices_and_whole(rows, dtype):
    """72 rows of 32 bits and 96 of 16 are the most that are cut into slices."""
    check_token_loss(rows, 41001, dtype)


# the widest rows that a group's registers hold, and the first that they do not: pieces of 16 bytes of 8 (fp32: 4) logits
@pytest.mark.parametrize("rows,vocab,dtype", [(97, 65536, "bf16"), (97, 65537, "fp16"), (97, 131071, "fp16"), (97, 131079, "bf16"), (97, 204799, "bf16"), (97, 204801, "fp16"), (97, 210001, "bf16"),
                                              (97, 32767, "fp32"), (97, 32773, "fp32"), (97, 65535, "fp32"), (97, 65541, "fp32"), (97, 102400, "fp32"), (97, 102405, "fp32")])
def test_loss_of_long_rows_that_are_whole(rows, vocab, dtype):
    check_token_loss(rows, vocab, dtype)


@pytest.mark.parametrize("vocab,dtype", [(180001, "bf16"), (210001, "bf16"), (90001, "fp32"), (120001, "fp32")])
def test_long_whole_rows_that_are_not_numbers(vocab, dtype):
    x = torch.randn(100, vocab, device="cuda", generator=rnd(1)).to(TYPES[dtype])
    x[1, 7], x[2, vocab - 1] = math.nan, math.inf
    x[3] = -math.inf
    x[3, 5] = math.nan
    x[4] = -math.inf
    t, z = torch.zeros(100, dtype=torch.int32, device="cuda"), torch.zeros(100, device="cuda")
    t[5] = vocab
    x[5] = math.nan
    for ent_coef in (0.0, 0.1):
        d, stats, logp = L.token_loss(x, t, z, z + 1, ent_coef=ent_coef)
        assert stats[7].item() == 1.0 and stats[6].item() == 98
        bad = torch.zeros(100, dtype=torch.bool, device="cuda")
        bad[1:4] = True
        assert torch.equal(torch.isnan(d).any(1), bad) and torch.equal(torch.isnan(logp), bad) and not bool(d[4:6].any())


@pytest.mark.parametrize("rows", [0, 1])
@pytest.mark.parametrize("vocab", [1, 600, 50000, 1 << 24])
def test_the_smallest_and_the_widest_rows(rows, vocab):
    x = torch.randn(rows, vocab, device="cuda", generator=rnd(2))
    t = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda")
    z = torch.zeros(rows, device="cuda")
    logp, ent, stat = L.token_logp(x, t, want_entropy=True)
    d, stats, again = L.token_loss(x, t, logp, z + 1, ent_coef=0.5)
    back = L.token_logp_backward(x, t, stat, -(z + 1), entropy=ent, dentropy=z - 0.5)
    assert stats[6].item() == rows and d.shape == back.shape == x.shape
    if rows:
        q = torch.log_softmax(x.double(), 1)
        H = -(q.exp() * q).sum()
        want = q.exp() * (1 + 0.5 * (q + H))
        want[0, -1] -= 1
        # sums of V terms in 64 V / V .. running sums: V / 64 + 32 roundings, of which the random ones cancel; the entropy's coefficient is off by
        # as much of H = 17
        tol = U32 * (vocab / 64 + 64)
        assert abs(logp.item() - q[0, -1].item()) <= tol + 4 * U32 * 17 and abs(ent.item() - H.item()) <= 20 * tol
        for got in (d, back):
            assert bool(((got.double() - want).abs() <= q.exp() * 20 * tol + U32 * 64 * want.abs() + 1e-30).all())


def test_the_most_rows():
    rows = (1 << 24) - 1
    x = torch.randn(rows, 2, device="cuda", generator=rnd(3))
    t = torch.randint(-1, 2, (rows,), device="cuda", generator=rnd(4)).to(torch.int32)
    z = torch.ones(rows, device="cuda")
    active = t >= 0
    want = torch.where(active, torch.nn.functional.logsigmoid(torch.where(t == 1, -1, 1) * (x[:, 0] - x[:, 1]).double()), 0.0)
    logp, _, stat = L.token_logp(x, t)
    assert float((logp.double() - want).abs().max()) <= U32 * 80
    back = L.token_logp_backward(x, t, stat, z)
    d, stats, again = L.token_loss(x, t, logp, -z)
    p = torch.where(active, -torch.expm1(want), 0.0)   # 1 - p_t
    grad = torch.stack([torch.where(t == 0, p, -p), torch.where(t == 1, p, -p)], 1)
    assert float((back.double() - grad).abs().max()) <= U32 * 200 and float((d.double() - grad).abs().max()) <= U32 * 200
    assert stats[6].item() == int(active.sum()) and abs(stats[0].item() / int(active.sum()) - 1) <= 1e-5
    y = L.dropout(x, 0.5, 9)
    part = torch.arange(rows - 1000, rows, device="cuda")
    assert torch.equal(y[-1000:], L.dropout(x[-1000:], 0.5, 9, row_ids=part))


def test_the_longest_dropout_row():
    from test_gpu_token_ops import mask_definition
    cols, q = 1 << 30, 32768
    x = torch.ones(1, cols, dtype=torch.bfloat16, device="cuda")
    y = L.dropout(x, 0.5, 7, out=x)
    step = 1 << 22   # 2^22 columns at every one of 7 places, by the definition
    import numpy as np
    for at in (0, 1 << 28, (1 << 29) - step // 2, 1 << 29, 3 << 28, cols - step):
        with np.errstate(over="ignore"):
            keep = _mask_of_columns(7, 0, 0, at, step, q)
        assert np.array_equal((y[0, at:at + step] != 0).cpu().numpy(), keep), at
    assert np.array_equal((y[:, :4096] != 0).cpu().numpy(), mask_definition(7, 0, [0], 4096, q))


def _mask_of_columns(seed, layer, row, first, n, border):
    """mask_definition for the columns from `first` on (a multiple of 4)."""
    import numpy as np
    u, G = np.uint64, 0x9E3779B97F4A7C15

    def mix(z):
        z = (z ^ (z >> u(30))) * u(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> u(27))) * u(0x94D049BB133111EB)
        return z ^ (z >> u(31))

    s = mix(np.array([(seed + G) % (1 << 64)], np.uint64))
    s = mix(s ^ u((layer + G) % (1 << 64)))
    s = mix(s ^ u((row + G) % (1 << 64)))
    c = first + np.arange(n)
    z = mix(s[0] + (c // 4 + 1).astype(np.uint64) * u(G))
    return ((z >> (c % 4 * 16).astype(np.uint64)) & u(0xFFFF)) >= u(border)


def test_the_most_pairs():
    """2^23 - 1 pairs of one token each: every margin by itself, the statistics over all."""
    pairs = (1 << 23) - 1
    logp = -torch.rand(2 * pairs, device="cuda", generator=rnd(5))
    off = torch.arange(2 * pairs + 1, device="cuda")
    grad, margin, stats = L.pair_loss(logp, off, beta=0.5, scale=1.0 / pairs)
    D = 0.5 * (logp[:pairs].double() - logp[pairs:].double())
    assert bool(((margin.double() - D).abs() <= 2 * U32 * D.abs()).all())
    slope = -0.5 * torch.sigmoid(-D) / pairs
    assert bool(((grad[:pairs].double() - slope).abs() <= 4 * U32 * slope.abs()).all()) and torch.equal(grad[pairs:], -grad[:pairs])
    loss = torch.nn.functional.softplus(-D).sum().item() / pairs
    assert abs(stats[0].item() - loss) <= 4 * U32 * loss and stats[5].item() == pairs and abs(stats[1].item() - (D > 0).double().mean().item()) <= 2 * U32


def test_many_empty_sequences():
    """More empty sequences than tokens, in front of, between and behind those that have some."""
    T, n = 5000, 300000
    cut = torch.randint(0, T + 1, (n - 1,), device="cuda", generator=rnd(6)).sort()[0]
    cut[cut < 60] = 0
    cut[(cut > 2000) & (cut < 4000)] = 2000
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), cut, torch.full((1,), T, device="cuda")])
    r, v, last = torch.randn(T, device="cuda"), torch.randn(T, device="cuda"), torch.randn(n, device="cuda")
    adv, ret = L.token_gae(r, v, off, 0.99, 0.95, last_value=last)
    full = torch.nonzero(off[1:] > off[:-1])[:, 0]
    few = torch.cat([off[full], off[-1:]])
    again = L.token_gae(r, v, few, 0.99, 0.95, last_value=last[full])
    assert torch.equal(adv, again[0]) and torch.equal(ret, again[1])


def test_inputs_dropped_while_another_stream_reads_them():
    """Inputs that the caller drops behind a call on another stream keep their memory until that stream has read them."""
    side, n = torch.cuda.Stream(), 1 << 22
    ids, t = torch.arange(n // 64, device="cuda"), torch.zeros(n // 64, dtype=torch.int32, device="cuda")
    calls = (lambda x, s: L.dropout(x, 0.5, 3, row_ids=ids, stream=s), lambda x, s: L.token_logp(x, t, stream=s)[0],
             lambda x, s: L.token_gae(x.view(-1), x.view(-1), ids * 64, 0.9, 0.9, stream=s)[0])
    for call in calls:
        torch.cuda.empty_cache()
        x = torch.randn(n // 64, 64, device="cuda", generator=rnd(1))
        want, place = call(x.clone(), None), x.data_ptr()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)   # the call waits behind this
        got = call(x, side)
        del x
        other = [torch.full((n // 64, 64), math.nan, device="cuda") for _ in range(4)]
        assert all(o.data_ptr() != place for o in other)
        side.synchronize()
        assert torch.equal(got, want)


def test_a_recording_on_the_stream_that_is_given():
    """stream= inside a recording on that stream, replayed with new inputs."""
    x, t = torch.randn(300, 700, device="cuda"), torch.randint(0, 700, (300,), device="cuda").to(torch.int32)
    z, side, graph = torch.zeros(300, device="cuda"), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    L.token_loss(x, t, z, z + 1)
    torch.cuda.synchronize()
    old, adv = z - 6, z + 1
    with torch.cuda.graph(graph, stream=side):
        out = L.token_loss(x, t, old, adv, ent_coef=0.1, stream=side)
    for turn in range(3):
        x.copy_(torch.randn(300, 700, device="cuda", generator=rnd(turn)))
        graph.replay()
        want = L.token_loss(x, t, old, adv, ent_coef=0.1)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_what_is_not_a_number_stays_in_its_sequence():
    """NaN and infinities among a sequence's tokens reach its earlier tokens and nothing else, within a tile and across tiles."""
    lengths = [5, 3000, 1, 0, 7000, 2, 4100]
    off = torch.tensor([0] + lengths, device="cuda").cumsum(0)
    T = int(off[-1])
    r, v, last = torch.randn(T, generator=rnd(1), device="cuda"), torch.randn(T, generator=rnd(2), device="cuda"), torch.randn(len(lengths), generator=rnd(3), device="cuda")
    clean = L.token_gae(r, v, off, 0.99, 0.95, last_value=last)
    for seq, at, place, value in ((1, 2500, r, math.nan), (4, 6000, v, math.inf), (4, 0, r, -math.inf), (6, 4099, v, math.nan), (5, None, last, math.nan), (0, 4, r, math.inf)):
        a, b, c = r.clone(), v.clone(), last.clone()
        (a if place is r else b if place is v else c)[seq if place is last else int(off[seq]) + at] = value
        adv, ret = L.token_gae(a, b, off, 0.99, 0.95, last_value=c)
        end = int(off[seq + 1]) if at is None else int(off[seq]) + at + 1
        bad = torch.zeros(T, dtype=torch.bool, device="cuda")
        bad[int(off[seq]):end] = True
        assert torch.equal(~torch.isfinite(adv), bad)
        assert all(torch.equal(x[~bad], y[~bad]) for x, y in zip((adv, ret), clean))
    # pairs: the other pairs' gradients and margins stay
    off = torch.tensor([0, 5, 3005, 3006, 10006, 10008, 14108], device="cuda")
    clean = L.pair_loss(r[:14108], off)
    x = r[:14108].clone()
    x[3005] = math.nan   # the third chosen one's
    grad, margin, stats = L.pair_loss(x, off)
    bad = torch.zeros(14108, dtype=torch.bool, device="cuda")
    bad[3005:3006], bad[10008:] = True, True
    assert torch.equal(torch.isnan(grad), bad) and torch.equal(grad[~bad], clean[0][~bad]) and torch.equal(margin[:2], clean[1][:2]) and stats[6].item() == 1


def test_tokens_beyond_32_bits():
    """2^32 tokens and some, in sequences that cross 2^31 and 2^32: constant rewards give geometric sums, constant log-probabilities known ones."""
    T, gl = (1 << 32) + 12293, 0.96875 * 0.5
    bounds = [0, 7, (1 << 31) - 5000, (1 << 31) + 3, (1 << 32) - 3, (1 << 32) + 5000, T]
    off = torch.tensor(bounds, device="cuda")
    r = torch.ones(T, device="cuda")
    v = torch.zeros(T, device="cuda")
    adv, ret = L.token_gae(r, v, off, 0.96875, 0.5)
    for lo, hi in zip(bounds, bounds[1:]):
        for at in (lo, lo + 1, (lo + hi) // 2, hi - 3, hi - 2, hi - 1):
            want = (1 - gl ** (hi - at)) / (1 - gl)
            assert abs(adv[at].item() - want) <= 2 * U32 * want and ret[at].item() == adv[at].item(), at
    assert float(adv.amin()) >= 1 and float(adv.amax()) < 1 / (1 - gl) * (1 + 2 * U32)
    del v, ret
    # 0.5 each: differences of the sequences' lengths, halved; exact in 64 bits
    r.fill_(0.5)
    grad, margin, stats = L.pair_loss(r, off, kind="squared", beta=0.5)
    n = [b - a for a, b in zip(bounds, bounds[1:])]
    for k in range(3):
        D = 0.5 * (n[k] - n[k + 3])
        assert abs(margin[k].item() - 0.5 * D) <= 2 * U32 * abs(0.5 * D)
        slope = 2 * (D - 1)
        for s, sign in ((k, 1), (k + 3, -1)):
            for at in (bounds[s], bounds[s + 1] - 1, (bounds[s] + bounds[s + 1]) // 2):
                assert abs(grad[at].item() - sign * slope) <= 2 * U32 * abs(slope)
    del r, adv, grad
    torch.cuda.empty_cache()
