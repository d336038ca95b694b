"""The paged 4-bit cache: append with rotation, read-back, attention over it, and the table of rotations, against
plain implementations in 64 bits written from the formulas of include/symar.h.

Every page that a test does not write holds 0xFF bytes (scales that are NaN), and so does the rest of a sequence's last
page: whatever a kernel takes from there shows."""
import math

import numpy as np
import pytest
import torch

from paper_2607_16100_b200 import symar

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def kv():
    c = symar.KVContext.on_torch()
    yield c
    assert c.status()[0] == symar.OK
    c.destroy()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(*shape, seed, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=gen(seed), device="cuda").to(dtype)


class Setup:
    """A pool of poisoned pages and a shuffled page table for sequences of (new tokens, all tokens)."""

    def __init__(self, seqs, kv_heads, dim, page, seed=0, single=None):
        self.seqs, self.dim, self.page, self.heads = seqs, dim, page, kv_heads
        width = max(1, max(-(-t // page) for _, t in seqs))
        pool = len(seqs) * width + 2
        self.cache = symar.PagedKV.zeros(pool, kv_heads, dim, page)
        self.cache.pages.fill_(255)
        order = torch.randperm(pool, generator=gen(seed), device="cuda")[:len(seqs) * width]
        self.table = order.view(len(seqs), width).to(torch.int32).contiguous()
        for b, (_, t) in enumerate(seqs):                 # columns beyond a sequence's tokens are never looked at
            self.table[b, -(-t // page):] = -1
        self.lengths = torch.tensor([t for _, t in seqs], dtype=torch.int32, device="cuda")
        new = [n for n, _ in seqs]
        one = all(n == 1 for n in new) if single is None else single
        self.start = None if one else torch.tensor(np.cumsum([0] + new), dtype=torch.int32, device="cuda")
        self.tokens = sum(new)
        self.batch = symar.KVBatch(self.lengths, self.table, self.start)
        self.place = [(b, t - n + i) for b, (n, t) in enumerate(seqs) for i in range(n)]   # (sequence, position) per row

    def whole(self):
        """The same sequences with all their tokens as new ones."""
        s = object.__new__(Setup)
        s.__dict__.update(self.__dict__)
        s.seqs = [(t, t) for _, t in self.seqs]
        s.start = torch.tensor(np.cumsum([0] + [t for _, t in self.seqs]), dtype=torch.int32, device="cuda")
        s.tokens = int(s.start[-1])
        s.batch = symar.KVBatch(s.lengths, s.table, s.start)
        return s

    def fill(self, kv, seed, scale=1.0):
        """Random keys and values in all tokens of all sequences; gives the values that the cache then holds (float64)."""
        s = self.whole()
        if s.tokens == 0:
            return []
        k = normal(s.tokens, self.heads, self.dim, seed=seed, dtype=torch.float32) * scale
        v = normal(s.tokens, self.heads, self.dim, seed=seed + 1, dtype=torch.float32) * scale
        kv.append(self.cache, s.batch, k, v)
        k, v = kv.read(self.cache, s.batch, s.tokens, dtype=torch.float32)
        cut = [t for _, t in self.seqs]
        return list(zip(k.double().split(cut), v.double().split(cut)))


def rotate64(x, table, positions, interleaved):
    rot = 2 * table.shape[1]
    y = x.double().clone()
    for row, pos in enumerate(positions):
        if pos < 0:
            continue
        c, s = table[pos, :, 0].double(), table[pos, :, 1].double()
        if interleaved:
            a, b = y[row, :, 0:rot:2].clone(), y[row, :, 1:rot:2].clone()
            y[row, :, 0:rot:2], y[row, :, 1:rot:2] = a * c - b * s, b * c + a * s
        else:
            h = rot // 2
            a, b = y[row, :, :h].clone(), y[row, :, h:rot].clone()
            y[row, :, :h], y[row, :, h:rot] = a * c - b * s, b * c + a * s
    return y


def stored_is_near(got, x, slack):
    """`got` is what the cache holds for x: within half a step of the group's scale.  The step is (hi - lo) / 15 with its four
    lowest bits cleared (2^-19 of it at most); the ends, at codes that the clamp may have moved by one rounding of the zero
    point, are up to a whole step off.  `slack`: absolute difference that x itself may have."""
    g, y = x.unflatten(-1, (-1, 64)), got.double().unflatten(-1, (-1, 64))
    step = (g.amax(-1, keepdim=True).clamp(min=0) - g.amin(-1, keepdim=True).clamp(max=0)) / 15
    err = (y - g).abs()
    assert (err <= step * (1 + 2.0 ** -16) + 4 * slack).all()
    inner = (g - g.amin(-1, keepdim=True).clamp(max=0) >= step) & (g.amax(-1, keepdim=True).clamp(min=0) - g >= step)
    assert (err <= torch.where(inner, 0.5 * step * (1 + 2.0 ** -15), step * 1.001) + 4 * slack).all()


APPEND = [
    # seqs (new, total), q_heads, kv_heads, dim, page, rot, interleaved
    ([(1, 1)], 8, 1, 128, 64, 128, False),
    ([(1, 17), (1, 0), (1, 64), (1, 65)], 4, 2, 64, 16, 64, True),
    ([(1, 300), (1, 16)], 16, 8, 256, 32, 128, False),
    ([(3, 3), (0, 5), (17, 40), (1, 1), (0, 0)], 6, 3, 128, 16, 64, True),
    ([(64, 64), (65, 130), (2, 1)], 2, 2, 64, 64, 16, False),
    ([(700, 700)], 5, 1, 128, 128, 128, False),
    ([(33, 290)], 4, 1, 256, 256, 100, False),          # halves of 50 channels: pairs cross every vector
    ([(9, 20)], 3, 1, 64, 16, 6, True),
    ([(5, 9), (4, 31)], 2, 1, 128, 16, 0, False),       # no rotation
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,hq,hkv,dim,page,rot,interleaved", APPEND)
def test_append_and_read(kv, seqs, hq, hkv, dim, page, rot, interleaved, dtype):
    s = Setup(seqs, hkv, dim, page, seed=1)
    q, k, v = (normal(s.tokens, h, dim, seed=i, dtype=DT[dtype]) for i, h in enumerate((hq, hkv, hkv)))
    table = symar.rope_table(max(1, max(t for _, t in seqs)), rot, base=1000.0) if rot else None
    before = s.cache.pages.clone()
    qo = kv.append(s.cache, s.batch, k, v, q=q, rotations=table, interleaved=interleaved)
    positions = [p for _, p in s.place]
    # two products and a sum in binary32, then one rounding to the type
    want_q = rotate64(q, table, positions, interleaved) if rot else q.double()
    size = q.double().abs().amax().item() * 2
    u = 2.0 ** -24 * 3 * size
    assert ((qo.double() - want_q).abs() <= u + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * want_q.abs()).all()
    rk, rv = kv.read(s.cache, s.batch, s.tokens, dtype=torch.float32)
    live = torch.tensor([p >= 0 for p in positions], device="cuda")
    want_k = rotate64(k, table, positions, interleaved) if rot else k.double()
    stored_is_near(rk[live], want_k[live], u)
    stored_is_near(rv[live], v[live].double(), 0.0)
    assert (rk[~live] == 0).all() and (rv[~live] == 0).all()
    # in bfloat16 the same values, rounded once
    bk, bv = kv.read(s.cache, s.batch, s.tokens, dtype=torch.bfloat16)
    assert torch.equal(bk, rk.bfloat16()) and torch.equal(bv, rv.bfloat16())
    # nothing but the new tokens' entries was written
    touched = torch.zeros_like(before, dtype=torch.bool)
    grp = dim // 64
    for b, pos in s.place:
        if pos < 0:
            continue
        page_no, slot = int(s.table[b, pos // page]), pos % page
        for side in (0, page):
            touched[page_no, :, (side + slot) * dim // 2:(side + slot + 1) * dim // 2] = True
            w = page * dim + 4 * (side + slot) * grp
            touched[page_no, :, w:w + 4 * grp] = True
    assert torch.equal(s.cache.pages[~touched], before[~touched])
    assert kv.status()[0] == symar.OK


def quantise_numpy(x):
    """The storing rule in numpy's binary32 arithmetic: codes and words of x [..., 64]."""
    x = x.astype(np.float32)
    f = np.float32
    lo, hi = np.minimum(x.min(-1), f(0)), np.maximum(x.max(-1), f(0))
    fifteenth = f(1.0 / 15.0)
    bits = (hi * fifteenth - lo * fifteenth).astype(f).view(np.uint32) & ~np.uint32(15)
    s = bits.view(f)
    some = s >= f(2.0 ** -126)
    with np.errstate(all="ignore"):
        r = np.where(some, f(1) / s, f(0)).astype(f)
        z = np.rint(-lo * r).astype(f)
        n = np.clip(np.rint((x * r[..., None]).astype(f)) + z[..., None], 0, 15).astype(np.int64)
    return n, np.where(some, bits | z.astype(np.uint32), 0).astype(np.uint32)


@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
def test_stored_bytes_are_those_of_the_rule(kv, dim, page):
    rng = np.random.default_rng(3)
    tokens, heads = 40, 2
    x = rng.standard_normal((2, tokens, heads, dim)).astype(np.float32)
    x[:, 1] = 0.0                                        # nothing to scale
    x[:, 2] = np.abs(x[:, 2]) + 100.0                    # one sign: zero stays the lower end
    x[:, 3] = -np.abs(x[:, 3])
    x[:, 4] *= 1e38 / 4
    x[:, 5] *= 1e-38                                     # the scale is near the smallest normal number
    x[:, 6] *= 1e-42                                     # and below it: stored as zeros
    x[:, 7, :, ::2] = 3.4028235e38
    x[:, 7, :, 1::2] = -3.4028235e38
    x[:, 8] = np.round(x[:, 8] * 4)                      # ties
    s = Setup([(tokens, tokens)], heads, dim, page)
    kv.append(s.cache, s.batch, torch.from_numpy(x[0]).cuda(), torch.from_numpy(x[1]).cuda())
    n, words = quantise_numpy(x.reshape(2, tokens, heads, dim // 64, 64))
    pages = s.cache.pages.cpu().numpy()
    table = s.table.cpu().numpy()
    for side in range(2):
        for t in range(tokens):
            for h in range(heads):
                block, row = pages[table[0, t // page], h], side * page + t % page
                codes = block[row * dim // 2:(row + 1) * dim // 2]
                got = np.stack([codes & 15, codes >> 4], -1).reshape(dim // 64, 64)
                at = page * dim + 4 * row * (dim // 64)
                assert np.array_equal(block[at:at + dim // 16].view(np.uint32), words[side, t, h]), (side, t, h)
                assert np.array_equal(got, n[side, t, h]), (side, t, h)


def test_groups_with_values_that_are_not_finite_read_back_as_nan(kv):
    s = Setup([(4, 4)], 1, 128, 16)
    k, v = normal(4, 1, 128, seed=1), normal(4, 1, 128, seed=2)
    k[0, 0, 3], k[1, 0, 70], v[2, 0, 0] = math.nan, math.inf, -math.inf
    kv.append(s.cache, s.batch, k, v)
    rk, rv = kv.read(s.cache, s.batch, 4, dtype=torch.float32)
    odd = torch.isnan(torch.stack([rk, rv])).view(2, 4, 2, 64)
    assert (odd.all(-1) == odd.any(-1)).all()
    want = torch.zeros(2, 4, 2, dtype=torch.bool)
    want[0, 0, 0] = want[0, 1, 1] = want[1, 2, 0] = True
    assert torch.equal(odd.any(-1).cpu(), want)


@pytest.mark.parametrize("offset", [0, 1, 4])
def test_append_takes_any_strides_and_q_in_place(kv, offset):
    """q, k and v as slices of one projection's rows, heads last to first, at any alignment; q rotated in place."""
    hq, hkv, dim, tokens = 4, 2, 128, 21
    table = symar.rope_table(64, dim)
    row = (hq + 2 * hkv) * dim + offset
    for dtype in (torch.bfloat16, torch.float32):
        for interleaved in (False, True):
            qkv = normal(tokens, row, seed=7, dtype=dtype)
            q, k, v = qkv[:, offset:].unflatten(1, (-1, dim)).split([hq, hkv, hkv], 1)
            s, t = Setup([(tokens, 50)], hkv, dim, 16), Setup([(tokens, 50)], hkv, dim, 16)
            want = kv.append(s.cache, s.batch, k.contiguous(), v.contiguous(), q=q.contiguous(), rotations=table,
                             interleaved=interleaved)
            kept = qkv[:, :offset].clone(), k.clone(), v.clone()
            got = kv.append(t.cache, t.batch, k, v, q=q, q_out=q, rotations=table, interleaved=interleaved)
            assert got is q and torch.equal(q, want) and torch.equal(s.cache.pages, t.cache.pages)
            assert torch.equal(qkv[:, :offset], kept[0]) and torch.equal(k, kept[1]) and torch.equal(v, kept[2])
            # a layout of [heads][tokens][channels]
            u = Setup([(tokens, 50)], hkv, dim, 16)
            kt, vt = kept[1].transpose(0, 1).contiguous().transpose(0, 1), kept[2].transpose(0, 1).contiguous().transpose(0, 1)
            kv.append(u.cache, u.batch, kt, vt, rotations=table, interleaved=interleaved)
            assert torch.equal(u.cache.pages, s.cache.pages)


def table64(rows, rot, base, kind, factor, original, low, high, magnitude):
    i = np.arange(rot // 2, dtype=np.float64)
    f = float(base) ** (-2 * i / rot)
    if kind == "linear":
        f = f / factor
    elif kind == "base":
        f = (base * factor ** (rot / (rot - 2))) ** (-2 * i / rot)
    elif kind == "by_parts":
        g = np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = (1 - g) * f / factor + g * f
    a = np.arange(rows, dtype=np.float64)[:, None] * f
    return np.stack([np.cos(a), np.sin(a)], -1) * magnitude


@pytest.mark.parametrize("kind,factor", [("plain", 1.0), ("linear", 4.0), ("base", 8.0), ("by_parts", 32.0)])
@pytest.mark.parametrize("rot,rows", [(128, 513), (64, 70001), (6, 40)])
def test_rope_table(kind, factor, rot, rows):
    got = symar.rope_table(rows, rot, base=500000.0, kind=kind, factor=factor, original=8192.0, low=1.0, high=4.0, magnitude=1.25)
    want = table64(rows, rot, 500000.0, kind, factor, 8192.0, 1.0, 4.0, 1.25)
    # one rounding to binary32; the angle in binary64 is off by a few 2^-53 of itself
    tol = 2.0 ** -24 * 1.25 + rows * 32 * 2.0 ** -53
    assert np.abs(got.double().cpu().numpy() - want).max() <= tol


# ---- attention ----

def attention64(s, filled, q, scale, window):
    """(out, bound per element) in 64 bits.

    Bound.  The tensor cores' sums truncate, 2^-23 of the running sum of |products| for each of D additions: a score is off by
    at most e = D 2^-23 scale sum |q k| (+ the same again for the roundings of scaling and of 2^x), which changes every
    probability by a factor within 1 +- 2.5 e.  A probability times its group's scale is rounded to bf16 (2^-8), the sums over
    tokens truncate again (2^-23 each), and the result is rounded to bf16 once (2^-8)."""
    share = q.shape[1] // s.heads
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    for row, (b, pos) in enumerate(s.place):
        lo = max(0, pos - window + 1) if window else 0
        if pos < 0 or lo > pos:
            continue
        k, v = (t[lo:pos + 1] for t in filled[b])
        for h in range(q.shape[1]):
            kk, vv, qq = k[:, h // share], v[:, h // share], q[row, h].double()
            p = torch.softmax(kk @ qq * scale, 0)
            e = 2 * q.shape[2] * 2.0 ** -23 * scale * (kk.abs() @ qq.abs()).max() + 1e-6
            out[row, h] = p @ vv
            tol[row, h] = (p @ vv.abs()) * (2.5 * e + 2.0 ** -8 + (pos + 1 - lo) * 2.0 ** -23) + 2.0 ** -8 * out[row, h].abs()
    return out, tol * 1.01 + 1e-37


ATTENTION = [
    # seqs (new, total), q_heads, kv_heads, dim, page, window
    ([(1, 1)], 1, 1, 64, 16, 0),
    ([(1, 15), (1, 16), (1, 17), (1, 0), (1, 63), (1, 64), (1, 65)], 8, 1, 128, 16, 0),
    ([(1, 513)], 8, 1, 128, 64, 0),
    ([(1, 1000), (1, 3), (1, 129)], 8, 8, 64, 32, 0),
    ([(1, 777), (1, 260)], 16, 2, 256, 64, 0),
    ([(1, 700), (1, 1)], 10, 2, 128, 128, 0),
    ([(1, 300), (1, 64)], 32, 2, 128, 256, 0),
    ([(1, 400), (1, 20), (1, 129)], 8, 2, 128, 32, 100),
    ([(1, 200)], 4, 4, 128, 16, 1),
    ([(4, 130), (1, 9), (3, 3), (0, 50), (5, 2)], 4, 2, 128, 16, 0),     # the last one's first tokens see nothing
    ([(33, 33), (17, 100)], 6, 2, 64, 16, 0),
    ([(70, 300)], 8, 1, 128, 64, 0),
    ([(70, 300), (2, 400)], 8, 2, 128, 64, 50),
    ([(40, 90)], 5, 1, 256, 32, 0),
    ([(130, 257), (1, 600), (64, 64)], 2, 1, 128, 128, 0),
    ([(20, 20), (0, 0), (1, 1)], 24, 8, 64, 16, 7),
]


@pytest.mark.parametrize("seqs,hq,hkv,dim,page,window", ATTENTION)
def test_attention(kv, seqs, hq, hkv, dim, page, window):
    s = Setup(seqs, hkv, dim, page, seed=2)
    filled = s.fill(kv, seed=11)
    q = normal(s.tokens, hq, dim, seed=5)
    got = kv.attention(s.cache, s.batch, q, window=window)
    want, tol = attention64(s, filled, q, dim ** -0.5, window)
    assert torch.isfinite(got).all()
    err = (got.double() - want).abs()
    assert (err <= tol).all(), (err / tol).max().item()
    # rows that see nothing are zeros, and two calls give the same bits
    for row, (_, pos) in enumerate(s.place):
        if pos < 0:
            assert (got[row] == 0).all()
    assert torch.equal(got, kv.attention(s.cache, s.batch, q, window=window))
    assert kv.status()[0] == symar.OK


@pytest.mark.parametrize("count,longest,hq,hkv,dim,page", [(1, 20011, 8, 1, 128, 64), (1, 9000, 64, 8, 128, 16), (150, 700, 8, 2, 128, 16),
                                                            (3, 5000, 4, 1, 256, 32), (40, 300, 32, 8, 64, 64)])
def test_work_shared_between_blocks(kv, count, longest, hq, hkv, dim, page):
    """Long sequences and many unequal ones: partial results of several blocks, joined."""
    seqs = [(1, 1 + (i * 7919 + longest - 1) % longest) for i in range(count)]
    s = Setup(seqs, hkv, dim, page, seed=2)
    filled = s.fill(kv, seed=21)
    q = normal(s.tokens, hq, dim, seed=5)
    got = kv.attention(s.cache, s.batch, q)
    want, tol = attention64(s, filled, q, dim ** -0.5, 0)
    assert ((got.double() - want).abs() <= tol).all()
    for _ in range(5):
        assert torch.equal(got, kv.attention(s.cache, s.batch, q))


@pytest.mark.parametrize("scale", [0.0, 0.03, 5.0])
def test_sharp_and_flat_softmax(kv, scale):
    """Scores from nearly equal to one that outweighs all others, of both signs and large."""
    s = Setup([(1, 500), (3, 90)], 2, 128, 32, seed=3)
    filled = s.fill(kv, seed=31, scale=3.0)
    q = normal(s.tokens, 8, 128, seed=6) * 4
    got = kv.attention(s.cache, s.batch, q, scale=scale)
    want, tol = attention64(s, filled, q, scale or 128 ** -0.5, 0)
    assert ((got.double() - want).abs() <= tol).all()


def test_a_sequence_that_is_not_finite_stays_alone(kv):
    s = Setup([(1, 40), (1, 50), (1, 45)], 1, 128, 16, seed=4)
    filled = s.fill(kv, seed=41)
    q = normal(3, 8, 128, seed=6)
    clean = kv.attention(s.cache, s.batch, q)
    one = Setup.__new__(Setup)
    one.__dict__.update(s.__dict__)
    # the last token of sequence 1 becomes NaN in the second group of its values
    k, v = normal(3, 1, 128, seed=8), normal(3, 1, 128, seed=9)
    kv.append(s.cache, s.batch, k, v)
    before = kv.attention(s.cache, s.batch, q)
    v[1, 0, 100] = math.nan
    kv.append(s.cache, s.batch, k, v)
    got = kv.attention(s.cache, s.batch, q)
    assert torch.isnan(got[1, :, 64:]).all() and torch.equal(got[1, :, :64], before[1, :, :64])
    assert torch.equal(got[0], before[0]) and torch.equal(got[2], before[2])
    assert torch.isfinite(clean).all() and len(filled) == 3


@pytest.mark.parametrize("offset", [0, 1, 4])
def test_attention_takes_any_strides(kv, offset):
    s = Setup([(5, 70), (1, 30)], 2, 128, 16, seed=5)
    s.fill(kv, seed=51)
    q = normal(s.tokens, 8, 128, seed=6)
    want = kv.attention(s.cache, s.batch, q)
    room = torch.zeros(s.tokens, 8 * 128 + 8 + offset, device="cuda", dtype=torch.bfloat16)
    qs = room[:, offset:offset + 1024].unflatten(1, (8, 128))
    qs.copy_(q)
    o = torch.full((8, s.tokens, 136 + offset), 7.0, device="cuda", dtype=torch.bfloat16)
    out = o[:, :, offset:offset + 128].transpose(0, 1)
    kv.attention(s.cache, s.batch, qs, out=out)
    assert torch.equal(out, want)
    assert (o[:, :, :offset] == 7.0).all() and (o[:, :, offset + 128:] == 7.0).all()


@pytest.mark.parametrize("hq,hkv,dim", [(8, 2, 128), (6, 1, 64)])
def test_one_piece_or_many_give_the_same_rows(kv, hq, hkv, dim):
    """A prompt in one call, and its tokens one call at a time, each over the cache as it was then."""
    total = 77
    s = Setup([(total, total)], hkv, dim, 16, seed=6)
    s.fill(kv, seed=61)
    q = normal(total, hq, dim, seed=7)
    whole = kv.attention(s.cache, s.batch, q).double()
    for t in (0, 1, 15, 16, 40, 76):
        batch = symar.KVBatch(torch.tensor([t + 1], dtype=torch.int32, device="cuda"), s.table)
        one = kv.attention(s.cache, batch, q[t:t + 1]).double()
        # both are within the bound of the same value; twice a bf16 rounding of values below 4 and of the probabilities
        assert (whole[t] - one[0]).abs().max() <= 4 * 2.0 ** -8 * 4


def test_bad_page_numbers_and_positions_are_reported(kv):
    c = symar.KVContext.on_torch()
    s = Setup([(1, 40), (1, 20)], 1, 128, 16, seed=7)
    s.fill(kv, seed=71)
    q, k = normal(2, 8, 128, seed=1), normal(2, 1, 128, seed=2)
    good = c.attention(s.cache, s.batch, q)
    for bad_page in (-1, s.cache.pages.shape[0], 1 << 30):
        table = s.table.clone()
        table[1, 1] = bad_page
        batch = symar.KVBatch(s.lengths, table)
        for go in (lambda: c.append(s.cache, batch, k, k), lambda: c.read(s.cache, batch, 2), lambda: c.attention(s.cache, batch, q)):
            go()
            code, seq, position = c.status()
            assert code == symar.ERR_INVAL and seq == 1 and 16 <= position < 20
            c.reset()
            assert c.status()[0] == symar.OK
    # a sequence that is longer than its row of the table
    long = symar.KVBatch(torch.tensor([40, 49], dtype=torch.int32, device="cuda"), s.table)
    c.append(s.cache, long, k, k)
    assert c.status() == (symar.ERR_INVAL, 1, 48)
    c.reset()
    # a position beyond the table of rotations
    c.append(s.cache, s.batch, k, k, q=q, rotations=symar.rope_table(39, 128))
    assert c.status() == (symar.ERR_INVAL, 0, 39)
    c.reset()
    s.fill(kv, seed=71)
    assert torch.equal(c.attention(s.cache, s.batch, q), good) and c.status()[0] == symar.OK
    c.destroy()


def test_graph_replay_follows_the_lengths(kv):
    """A captured step: lengths, tokens and tables change between replays, the calls do not."""
    s = Setup([(1, 200), (1, 90)], 2, 128, 16, seed=8)
    s.fill(kv, seed=81)
    table = symar.rope_table(256, 128)
    q, k, v = normal(2, 16, 128, seed=1), normal(2, 2, 128, seed=2), normal(2, 2, 128, seed=3)
    qo, out = torch.empty_like(q), torch.empty_like(q)

    def step():
        kv.append(s.cache, s.batch, k, v, q=q, q_out=qo, rotations=table)
        kv.attention(s.cache, s.batch, qo, out=out)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
    for lengths in ([200, 90], [150, 1], [193, 0]):
        s.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        q.copy_(normal(2, 16, 128, seed=sum(lengths)))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out)
        if lengths[1] == 0:
            assert (out[1] == 0).all()


def test_a_long_pool_passes_32_bit_offsets(kv):
    """Pages beyond 4 GiB of the pool."""
    dim, page, heads = 128, 64, 8
    each = symar.load().symar_kv_page_bytes(heads, dim, page)
    pages = (5 << 30) // each
    cache = symar.PagedKV(torch.empty(pages, heads, each // heads, dtype=torch.uint8, device="cuda"), dim, page)
    cache.pages[-4:].fill_(255)
    lengths = torch.tensor([100], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 100], dtype=torch.int32, device="cuda")
    far = symar.KVBatch(lengths, torch.tensor([[pages - 1, pages - 3]], dtype=torch.int32, device="cuda"), start)
    near_cache = symar.PagedKV.zeros(4, heads, dim, page)
    near = symar.KVBatch(lengths, torch.tensor([[0, 2]], dtype=torch.int32, device="cuda"), start)
    k, v, q = (normal(100, h, dim, seed=i) for i, h in enumerate((heads, heads, 8)))
    got = []
    for c, b in ((cache, far), (near_cache, near)):
        kv.append(c, b, k, v)
        got.append((*kv.read(c, b, 100), kv.attention(c, b, q)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_no_tokens(kv):
    s = Setup([(0, 5), (0, 0)], 2, 128, 16, single=False)
    empty = torch.empty(0, 2, 128, device="cuda", dtype=torch.bfloat16)
    q = torch.empty(0, 8, 128, device="cuda", dtype=torch.bfloat16)
    assert kv.append(s.cache, s.batch, empty, empty, q=q).shape == (0, 8, 128)
    assert kv.read(s.cache, s.batch, 0)[0].shape == (0, 2, 128)
    assert kv.attention(s.cache, s.batch, q).shape == (0, 8, 128)


def test_python_refusals(kv):
    s = Setup([(1, 5)], 2, 128, 16)
    k, q = normal(1, 2, 128, seed=1), normal(1, 8, 128, seed=2)
    for go in (lambda: kv.append(s.cache, s.batch, k, k.float()), lambda: kv.append(s.cache, s.batch, k[:, :1], k),
               lambda: kv.append(s.cache, s.batch, k, k, q=q[..., :64]), lambda: kv.append(s.cache, s.batch, k.half(), k.half()),
               lambda: kv.append(s.cache, s.batch, k, k, rotations=torch.zeros(8, 64, device="cuda")),
               lambda: kv.attention(s.cache, s.batch, q.float()), lambda: kv.attention(s.cache, s.batch, q[:, :7]),
               lambda: kv.attention(s.cache, s.batch, normal(2, 8, 128, seed=1)),
               lambda: symar.PagedKV(s.cache.pages[:, :, :-1], 128, 16), lambda: symar.PagedKV(s.cache.pages, 96, 16),
               lambda: symar.KVBatch(s.lengths.long(), s.table), lambda: symar.KVBatch(s.lengths, s.table.repeat(2, 1)),
               lambda: symar.KVBatch(s.lengths, s.table, torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(symar.SymarError):
            go()
