"""The operators without a context (dropout, token log-probabilities, clipped token loss, preference loss, packed advantages)
on a host without a GPU: what they refuse, before any HIP call, and what the binding makes of it."""
import ctypes as C
import os
import re

import pytest

from paper_2509_16434_amd import learner as L

lib = L._lib
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ppo_learner.h")
P, ODD, NUL = 1 << 20, (1 << 20) + 1, None   # an address that is aligned to every type, one that is not; never followed
INF, NAN = float("inf"), float("nan")
BIG = 1 << 40


def _struct(name, before):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    body = text[:text.index("} " + name + ";")]
    return re.findall(r"(\w+)\s*[,;]", body[body.rindex("typedef struct {"):])


def test_structs_match_the_header():
    assert _struct("ppo_token_hparams", None) == [f for f, _ in L.TokenHParams._fields_] and C.sizeof(L.TokenHParams) == 24
    assert _struct("ppo_pair_hparams", None) == [f for f, _ in L.PairHParams._fields_] and C.sizeof(L.PairHParams) == 20
    assert "#define PPO_TOKEN_MAX_VOCAB (1 << 24)" in open(HEADER).read() and "#define PPO_TOKEN_MAX_ROWS ((1 << 24) - 1)" in open(HEADER).read()


def test_kernels_keep_their_rows_in_registers():
    """No kernel of the operators spills (the widest loss with spilled registers ran at a quarter of its speed)."""
    import struct

    import msgpack
    lib_bytes, magic, at, found = open(L.LIB_PATH, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__", 0, {}
    while (at := lib_bytes.find(magic, at)) >= 0:
        entries, p = struct.unpack_from("<Q", lib_bytes, at + 24)[0], at + 32
        for _ in range(entries if entries < 16 else 0):
            off, size, n = struct.unpack_from("<QQQ", lib_bytes, p)
            target = lib_bytes[p + 24:p + 24 + n]
            p += 24 + n
            if not target.endswith(b"gfx950"):
                continue
            elf = lib_bytes[at + off:at + off + size]
            headers, count = struct.unpack_from("<Q", elf, 32)[0], struct.unpack_from("<H", elf, 56)[0]
            for k in range(count):
                kind, _, note = struct.unpack_from("<IIQ", elf, headers + 56 * k)
                nn, nd, ty = struct.unpack_from("<III", elf, note) if kind == 4 else (0, 0, 0)
                if ty == 32:   # the notes of the kernels
                    start = note + 12 + (nn + 3 & ~3)
                    found.update({m[".name"]: m for m in msgpack.unpackb(elf[start:start + nd])["amdhsa.kernels"]})
        at += len(magic)
    ours = {n: m for n, m in found.items() if re.match(r"_Z\d+k_(token|pair|gae|dropout)", n)}
    assert len(ours) > 100 and any("k_token_loss" in n for n in ours) and any("k_gae_part" in n for n in ours)
    for n, m in ours.items():
        assert m[".vgpr_spill_count"] == 0 and m[".private_segment_fixed_size"] == 0, n


def test_workspace_sizes():
    for rows, vocab in ((0, 1), (1, 1), (16, 131072), (1 << 20, 256), ((1 << 24) - 1, 2)):
        for size in (lib.ppo_token_logp_ws_bytes, lib.ppo_token_loss_ws_bytes):
            assert 0 <= size(rows, vocab) <= 4096 * rows + (1 << 20)
            assert size(-1, 8) == size(8, 0) == size(8, (1 << 24) + 1) == L.PPO_ESHAPE
    assert lib.ppo_pair_ws_bytes(4, 100) >= 0 and lib.ppo_pair_ws_bytes(-1, 100) == lib.ppo_pair_ws_bytes(1, -1) == L.PPO_ESHAPE
    assert lib.ppo_token_gae_ws_bytes(4, 100) >= 0 and lib.ppo_token_gae_ws_bytes(1, -1) == lib.ppo_token_gae_ws_bytes(-1, 1) == L.PPO_ESHAPE


DROPOUT = dict(dtype=1, rows=4, cols=8, x=P, ldx=8, ids=NUL, res=NUL, ldr=8, p=0.1, seed=1, layer=0, y=P, ldy=8, st=NUL)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), L.PPO_EINVAL), (dict(dtype=-1), L.PPO_EINVAL), (dict(rows=-1), L.PPO_ESHAPE), (dict(cols=-1), L.PPO_ESHAPE), (dict(rows=BIG), L.PPO_ESHAPE), (dict(rows=1 << 24), L.PPO_ESHAPE), (dict(cols=BIG, ldx=BIG, ldy=BIG), L.PPO_ESHAPE),
    (dict(p=-0.1), L.PPO_EINVAL), (dict(p=1.1), L.PPO_EINVAL), (dict(p=NAN), L.PPO_EINVAL), (dict(x=NUL), L.PPO_EINVAL), (dict(y=NUL), L.PPO_EINVAL),
    (dict(x=ODD), L.PPO_EINVAL), (dict(ldx=7), L.PPO_ESHAPE), (dict(ldy=7), L.PPO_ESHAPE), (dict(res=P, ldr=7), L.PPO_ESHAPE), (dict(ids=P + 4), L.PPO_EINVAL),
    (dict(rows=0, x=NUL, y=NUL), 0), (dict(cols=0, x=NUL, y=NUL), 0),
])
def test_dropout_refuses(change, code):
    a = dict(DROPOUT, **change)
    assert lib.ppo_dropout(*a.values()) == code
    if code:
        assert len(lib.ppo_last_error(None)) > 5


LOGP = dict(dtype=1, rows=4, vocab=8, x=P, ld=8, target=P, temperature=1.0, logp=P, entropy=NUL, stat=NUL, ws=P, wsb=1 << 20, st=NUL)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=5), L.PPO_EINVAL), (dict(rows=-1), L.PPO_ESHAPE), (dict(rows=1 << 24), L.PPO_ESHAPE), (dict(vocab=0), L.PPO_ESHAPE), (dict(vocab=(1 << 24) + 1, ld=1 << 25), L.PPO_ESHAPE),
    (dict(temperature=0.0), L.PPO_EINVAL), (dict(temperature=-1.0), L.PPO_EINVAL), (dict(temperature=INF), L.PPO_EINVAL), (dict(temperature=NAN), L.PPO_EINVAL),
    (dict(temperature=1e-45), L.PPO_EINVAL), (dict(temperature=3.5e-39), L.PPO_EINVAL), (dict(x=NUL), L.PPO_EINVAL), (dict(x=ODD), L.PPO_EINVAL), (dict(ld=7), L.PPO_ESHAPE), (dict(target=NUL), L.PPO_EINVAL),
    (dict(logp=NUL), L.PPO_EINVAL), (dict(stat=P + 2), L.PPO_EINVAL), (dict(rows=0, x=NUL, target=NUL, logp=NUL, ws=NUL, wsb=0), 0),
])
def test_token_logp_refuses(change, code):
    assert lib.ppo_token_logp(*dict(LOGP, **change).values()) == code


BACK = dict(dtype=0, rows=4, vocab=8, x=P, ld=8, target=P, temperature=1.0, stat=P, dlogp=P, entropy=NUL, dentropy=NUL, d=P, ldd=8, st=NUL)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=-2), L.PPO_EINVAL), (dict(vocab=-3), L.PPO_ESHAPE), (dict(temperature=0.0), L.PPO_EINVAL), (dict(d=NUL), L.PPO_EINVAL), (dict(ldd=3), L.PPO_ESHAPE),
    (dict(stat=NUL), L.PPO_EINVAL), (dict(dlogp=NUL), L.PPO_EINVAL), (dict(dentropy=P), L.PPO_EINVAL),   # an entropy gradient without the entropies
    (dict(target=NUL), L.PPO_EINVAL), (dict(d=P + 2), L.PPO_EINVAL), (dict(rows=0, x=NUL, target=NUL, stat=NUL, dlogp=NUL, d=NUL), 0),
])
def test_token_logp_backward_refuses(change, code):
    assert lib.ppo_token_logp_backward(*dict(BACK, **change).values()) == code


LOSS = dict(dtype=1, rows=4, vocab=600, x=P, ld=600, target=P, old=P, ref=NUL, adv=P, weight=NUL, hp=None, d=P, ldd=600, logp=P, stats=P, ws=P, wsb=1 << 20, st=NUL)
HP = dict(temperature=1.0, clip_lo=0.2, clip_hi=0.2, kl_coef=0.0, ent_coef=0.0, scale=1.0)


@pytest.mark.parametrize("change,hp,code", [
    (dict(dtype=9), {}, L.PPO_EINVAL), (dict(rows=BIG), {}, L.PPO_ESHAPE), (dict(vocab=0), {}, L.PPO_ESHAPE), (dict(hp=0), {}, L.PPO_EINVAL),
    ({}, dict(temperature=0.0), L.PPO_EINVAL), ({}, dict(clip_lo=1.5), L.PPO_EINVAL), ({}, dict(clip_lo=-0.1), L.PPO_EINVAL), ({}, dict(clip_hi=-1.0), L.PPO_EINVAL),
    ({}, dict(clip_hi=INF), L.PPO_EINVAL), ({}, dict(kl_coef=-0.1), L.PPO_EINVAL), ({}, dict(kl_coef=0.1), L.PPO_EINVAL),   # the last: no reference
    ({}, dict(ent_coef=NAN), L.PPO_EINVAL), ({}, dict(scale=INF), L.PPO_EINVAL), (dict(old=NUL), {}, L.PPO_EINVAL), (dict(adv=NUL), {}, L.PPO_EINVAL),
    (dict(stats=NUL), {}, L.PPO_EINVAL), (dict(d=NUL), {}, L.PPO_EINVAL), (dict(ldd=599), {}, L.PPO_ESHAPE), (dict(ws=NUL), {}, L.PPO_EINVAL), (dict(wsb=8), {}, L.PPO_EINVAL),
    (dict(ws=P + 8), {}, L.PPO_EINVAL), (dict(weight=P + 1), {}, L.PPO_EINVAL),
])
def test_token_loss_refuses(change, hp, code):
    a = dict(LOSS, **change)
    h = L.TokenHParams(**dict(HP, **hp))
    a["hp"] = C.byref(h) if a["hp"] is None else None
    assert lib.ppo_token_loss(*a.values()) == code


PAIR = dict(pairs=2, tokens=10, logp=P, ref=NUL, mask=NUL, offsets=P, hp=None, dlogp=P, margin=P, stats=P, ws=P, wsb=1 << 20, st=NUL)
PHP = dict(kind=0, length_mean=0, beta=0.1, label_smoothing=0.0, scale=1.0)


@pytest.mark.parametrize("change,hp,code", [
    (dict(pairs=-1), {}, L.PPO_ESHAPE), (dict(pairs=1 << 23), {}, L.PPO_ESHAPE), (dict(tokens=-1), {}, L.PPO_ESHAPE), (dict(hp=0), {}, L.PPO_EINVAL), ({}, dict(kind=2), L.PPO_EINVAL), ({}, dict(kind=-1), L.PPO_EINVAL),
    ({}, dict(beta=0.0), L.PPO_EINVAL), ({}, dict(beta=INF), L.PPO_EINVAL), ({}, dict(label_smoothing=1.5), L.PPO_EINVAL), ({}, dict(label_smoothing=NAN), L.PPO_EINVAL),
    ({}, dict(scale=NAN), L.PPO_EINVAL), (dict(logp=NUL), {}, L.PPO_EINVAL), (dict(dlogp=NUL), {}, L.PPO_EINVAL), (dict(offsets=NUL), {}, L.PPO_EINVAL),
    (dict(offsets=P + 4), {}, L.PPO_EINVAL), (dict(stats=NUL), {}, L.PPO_EINVAL), (dict(ws=NUL), {}, L.PPO_EINVAL), (dict(wsb=4), {}, L.PPO_EINVAL), (dict(ref=P + 1), {}, L.PPO_EINVAL),
])
def test_pair_loss_refuses(change, hp, code):
    a = dict(PAIR, **change)
    h = L.PairHParams(**dict(PHP, **hp))
    a["hp"] = C.byref(h) if a["hp"] is None else None
    assert lib.ppo_pair_loss(*a.values()) == code


GAE = dict(sequences=2, tokens=10, reward=P, value=P, mask=NUL, offsets=P, last=NUL, gamma=0.99, lam=0.95, adv=P, ret=P, ws=P, wsb=1 << 20, st=NUL)


@pytest.mark.parametrize("change,code", [
    (dict(sequences=-1), L.PPO_ESHAPE), (dict(tokens=-1), L.PPO_ESHAPE), (dict(tokens=1 << 50), L.PPO_ESHAPE), (dict(gamma=1.1), L.PPO_EINVAL), (dict(gamma=NAN), L.PPO_EINVAL),
    (dict(lam=-0.1), L.PPO_EINVAL), (dict(reward=NUL), L.PPO_EINVAL), (dict(value=NUL), L.PPO_EINVAL), (dict(offsets=NUL), L.PPO_EINVAL), (dict(adv=NUL), L.PPO_EINVAL),
    (dict(ret=NUL), L.PPO_EINVAL), (dict(adv=P + 2), L.PPO_EINVAL), (dict(tokens=0, reward=NUL, value=NUL, offsets=NUL, adv=NUL, ret=NUL, ws=NUL, wsb=0), 0),
])
def test_token_gae_refuses(change, code):
    assert lib.ppo_token_gae(*dict(GAE, **change).values()) == code


def test_the_binding_takes_cuda_tensors_only():
    import torch
    x, t = torch.zeros(2, 4), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: L.dropout(x, 0.1, 1), lambda: L.token_logp(x, t), lambda: L.token_logp_backward(x, t, x, x), lambda: L.token_loss(x, t, x, x),
                 lambda: L.pair_loss(x, t), lambda: L.token_gae(x, x, t, 0.9, 0.9), lambda: L.dropout(None, 0.1, 1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        L.pair_loss(x, t, kind="other")
    n = L._native
    with pytest.raises(TypeError):
        n.dropout(0, 1, 2)
    with pytest.raises(TypeError):
        n.dropout(0, 3.0, 0.1, 1, 0, None, None, None)
    with pytest.raises(ValueError):
        n.token_logp(0, x, t, 1.0, False)
