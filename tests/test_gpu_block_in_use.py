"""The quantized block in use, on the GPU: rows to 8 bits, the integer projection, the paged cache and the
attention over it, each against its definition in plain numpy / torch (fp64, and fp32 steps where the definition
rounds)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_34866_amd import jab

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _problem(dtype, rows, d=64, hq=4, hkv=2, dh=64, sym=False, rope=0.0, batch=1):
    return jab.problem(batch, rows, d, hq, hkv, dh, 32, DT[dtype], scheme=jab.SYM if sym else jab.ASYM, rope_theta=rope)


# ------------------------------------------------------------------ rows
def _rows_plain(x):
    """codes and scales by fp32 steps, as numpy rounds them"""
    x = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        top = np.abs(x).max(1)
        s = (top / np.float32(127)).astype(np.float32)
        s[s == 0] = 1
        q = np.clip(np.rint(x / s[:, None]), -127, 127)
    bad = ~np.isfinite(x).all(1)
    s[bad], q[bad] = np.nan, 0
    return q.astype(np.int8), s


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,d", [(1, 32), (3, 96), (7, 512), (5, 544), (2, 4096), (3, 4128), (1, 16416)])
def test_quant_rows(dtype, rows, d):
    x = torch.randn((rows + 4, d), generator=_gen(rows * d), device="cuda") * 3
    x[0] = 0
    x[1, d - 1], x[2, 0], x[3, 5] = math.inf, math.nan, -math.inf
    x[4, ::3] = 0.5 * x[4].abs().max() / 127 * 5            # many quotients next to or on a tie
    x = x.to(DT[dtype])
    q, s = jab.quant_rows(_problem(dtype, 1, d=d), x)
    want_q, want_s = _rows_plain(x)
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


def test_quant_rows_of_subnormals():
    x = torch.full((2, 64), 1e-44, device="cuda")
    x[1, 3] = 3e-38
    q, s = jab.quant_rows(_problem("f32", 1), x)
    want_q, want_s = _rows_plain(x)
    np.testing.assert_array_equal(s.cpu().numpy(), want_s)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q)


# ------------------------------------------------------------------ projection
def _project_plain(xq, sx, wq, sw, dt):
    acc = (xq.double() @ wq.double().t().contiguous()).float()           # whole sums below 2^31, exact in fp64
    return (acc * (sx[:, None] * sw)).to(dt)


# tokens and shapes of each kernel: few tokens, small tiles (K a multiple of 32, 64, 128), 256-tiles
PROJ = [(1, 32, 4, 2, 16), (5, 96, 4, 2, 16), (16, 4096, 8, 2, 64), (17, 160, 4, 4, 64), (33, 64, 12, 12, 64),
        (64, 1056, 8, 2, 128), (65, 32, 4, 2, 16), (70, 96, 4, 1, 16), (200, 64, 4, 2, 64), (129, 768, 12, 12, 64),
        (700, 160, 32, 8, 128), (1024, 192, 32, 8, 128), (1000, 384, 32, 8, 128), (300, 1024, 4, 2, 64),
        (2000, 1024, 32, 8, 128), (2048, 1152, 32, 8, 128), (1801, 2048, 32, 8, 128)]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,d,hq,hkv,dh", PROJ)
def test_project_int_is_exact(dtype, M, d, hq, hkv, dh):
    p, g = _problem(dtype, M, d, hq, hkv, dh), _gen(M + d)
    xq = torch.randint(-128, 128, (1, M, d), generator=g, device="cuda").to(torch.int8)
    wq = torch.randint(-128, 128, (p.rows, d), generator=g, device="cuda").to(torch.int8)
    sx = torch.rand((1, M), generator=g, device="cuda") * 1e-3
    sw = torch.rand(p.rows, generator=g, device="cuda") * 1e-3
    out = torch.full((1, M, p.rows), 7.0, dtype=DT[dtype], device="cuda")
    assert jab.project_int(p, xq, sx, wq, sw, out=out) is out
    assert torch.equal(out[0], _project_plain(xq[0], sx[0], wq, sw, DT[dtype]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,d", [(9, 96), (16, 1024), (20, 64), (20, 1056), (32, 2048), (32, 544), (33, 160), (64, 96)])
def test_project_int_few_tokens_wide(dtype, M, d):
    """1023 tiles of 16 weight rows: four to a workgroup, the last one short; 513: two."""
    test_project_int_is_exact(dtype, M, d, 341, 341, 16)
    test_project_int_is_exact(dtype, M, d, 171, 171, 16)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,d", [(300, 768), (3, 1024), (2, 1056), (1, 2080)])
def test_quant_rows_of_middle_sizes(dtype, rows, d):
    test_quant_rows(dtype, rows, d)


@pytest.mark.parametrize("M", [3, 100])
def test_project_int_largest_sums(M):
    """All codes -128 at the largest d_model: sums of 2^14 * 131040 stay in 32 bits."""
    d = 131040
    p = _problem("f32", M, d, 4, 2, 16)
    xq = torch.full((1, M, d), -128, dtype=torch.int8, device="cuda")
    wq = torch.full((p.rows, d), -128, dtype=torch.int8, device="cuda")
    one = torch.ones((1, M), device="cuda")
    y = jab.project_int(p, xq, one, wq, torch.ones(p.rows, device="cuda"))
    assert bool((y == float(np.float32(16384 * d))).all())


def test_project_int_nan_scale_marks_its_row_only():
    p = _problem("bf16", 70)
    x = torch.randn((1, 70, 64), device="cuda", generator=_gen(1)).bfloat16()
    x[0, 3, 5] = math.nan
    xq, sx = jab.quant_rows(p, x)
    wq, sw = jab.quant_rows(p, torch.randn((p.rows, 64), device="cuda", generator=_gen(2)).bfloat16())
    bad = jab.project_int(p, xq, sx, wq, sw)[0].isnan()
    assert bool(bad[3].all()) and int(bad.sum()) == p.rows


# ------------------------------------------------------------------ cache
class Setup:
    """A paged batch: sequences with (past, new) tokens, pages in a random order, the cache's unwritten places
    full of codes 255, scales NaN."""

    def __init__(self, dtype, seqs, hq=4, hkv=2, dh=64, bits=8, sym=False, rope=0.0, page=64, seed=0, spare_rows=2,
                 extra_cols=1, max_new=None):
        self.seqs, self.bits, self.sym, self.dh, self.hq, self.hkv, self.page = seqs, bits, sym, dh, hq, hkv, page
        self.rope, self.dtype = rope, DT[dtype]
        self.M = sum(n for _, n in seqs) + spare_rows
        self.p = _problem(dtype, self.M, 64, hq, hkv, dh, sym, rope)
        need = [(a + n + page - 1) // page for a, n in seqs]
        rng = np.random.default_rng(seed)
        order = rng.permutation(sum(need) + 2)
        pages = np.full((len(seqs), max(need) + extra_cols), -1, np.int32)
        k = 0
        for i, n in enumerate(need):
            pages[i, :n] = order[k:k + n]
            k += n
        self.pages = torch.tensor(pages, device="cuda")
        self.past = torch.tensor([a for a, _ in seqs], dtype=torch.int32, device="cuda")
        self.start = torch.tensor(np.cumsum([0] + [n for _, n in seqs]), dtype=torch.int32, device="cuda")
        self.cache = jab.Cache.empty(self.p, bits, page, sum(need) + 2)
        for t in self.cache.tensors:
            if t is not None:
                t.fill_(255 if t.dtype == torch.uint8 else math.nan)
        self.rows = jab.CacheRows(self.pages, self.past, self.start, max_new or max(n for _, n in seqs))
        self.gen = _gen(seed + 100)

    def y(self, rows, scale=1.0):
        y = torch.randn((1, rows, self.p.rows), generator=self.gen, device="cuda")
        y[..., : self.hq * self.dh] *= scale
        return y.to(self.dtype)

    def history(self):
        """Writes every sequence's past through its own call; returns the rows written [seq][past][R]."""
        out = []
        for i, (a, _) in enumerate(self.seqs):
            if a == 0:
                out.append(torch.empty((0, self.p.rows), dtype=self.dtype, device="cuda"))
                continue
            y = self.y(a)
            one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")       # noqa: E731
            p = _problem({v: k for k, v in DT.items()}[self.dtype], a, 64, self.hq, self.hkv, self.dh, self.sym, self.rope)
            jab.cache_write(p, self.cache, jab.CacheRows(self.pages[i:i + 1].contiguous(), one([0]), one([0, a]), a), y)
            out.append(y[0])
        return out


def _turned(x, pos, theta):
    """The rotary embedding in fp64 on [rows][heads][dh], rounded to fp32."""
    half = x.shape[-1] // 2
    ang = pos.astype(np.float64)[:, None] * theta ** (-2.0 * np.arange(half) / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half].astype(np.float64), x[..., half:].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def _encode(x, bits, sym):
    """codes, scale, zero of fp32 rows by fp32 steps"""
    x = x.astype(np.float32)
    f = np.float32
    with np.errstate(all="ignore"):
        if sym:
            q = 2 ** (bits - 1) - 1
            s = np.abs(x).max(-1) / f(q)
            s[s == 0] = 1
            return (np.clip(np.rint(x / s[..., None]), -q, q) + q).astype(np.uint8), s, np.full(s.shape, q, np.uint8)
        n = 2 ** bits - 1
        lo, hi = np.minimum(x.min(-1), 0), np.maximum(x.max(-1), 0)
        s = (hi - lo) / f(n)
        s[s == 0] = 1
        z = np.clip(np.rint(-lo / s), 0, n)
        return np.clip(np.rint(x / s[..., None]) + z[..., None], 0, n).astype(np.uint8), s, z.astype(np.uint8)


def _places(su):
    """(row, sequence, position, page, place) of every row of a sequence"""
    pages = su.pages.cpu().numpy()
    row = 0
    for i, (a, n) in enumerate(su.seqs):
        for t in range(a, a + n):
            yield row, i, t, int(pages[i, t // su.page]), t % su.page
            row += 1


def _stored(su, page, at):
    """codes [2][hkv][dh], scales and zero-points [2][hkv] at a place of the cache"""
    k, v, ks, vs, kz, vz = [None if t is None else t[page].cpu().numpy() for t in su.cache.tensors]
    kc, vc = k[:, at], v[:, at // 32, :, at % 32]
    un = (lambda b: np.concatenate([b & 15, b >> 4], -1)) if su.bits == 4 else (lambda b: b)
    z = [np.full(su.hkv, 2 ** (su.bits - 1) - 1) if su.sym else t[:, at] for t in (kz, vz)]
    return np.stack([un(kc), un(vc)]), np.stack([ks[:, at], vs[:, at]]), np.stack(z)


CACHE = [  # dtype, head_dim, bits, symmetric, rope, page, (past, new) of the sequences
    ("bf16", 128, 8, False, 0.0, 64, [(0, 1)]),
    ("bf16", 128, 8, False, 10000.0, 32, [(31, 2), (5, 1), (100, 3), (63, 1)]),
    ("bf16", 64, 4, True, 0.0, 64, [(7, 70), (0, 33), (62, 5)]),
    ("f16", 64, 4, False, 10000.0, 128, [(0, 129), (127, 40), (3, 1)]),
    ("f16", 16, 8, True, 10000.0, 32, [(0, 37), (30, 36)]),
    ("f32", 16, 4, False, 0.0, 32, [(1, 1), (2, 31), (0, 64)]),
    ("f32", 128, 4, False, 10000.0, 256, [(250, 20)]),
    ("f32", 64, 8, True, 0.0, 64, [(33, 4), (32, 5), (1, 90)]),
    ("bf16", 16, 4, True, 0.0, 64, [(0, 5), (9, 1)]),
]


@pytest.mark.parametrize("dtype,dh,bits,sym,rope,page,seqs", CACHE)
def test_cache_write_and_read(dtype, dh, bits, sym, rope, page, seqs):
    su = Setup(dtype, seqs, dh=dh, bits=bits, sym=sym, rope=rope, page=page)
    y = su.y(su.M)
    jab.cache_write(su.p, su.cache, su.rows, y)
    k = torch.full((1, su.M, su.hkv * dh), 3.0, dtype=su.dtype, device="cuda")
    v = k.clone()
    jab.cache_read(su.p, su.cache, su.rows, k, v)
    yn = y[0].float().cpu().numpy()
    kv = np.stack([k[0].float().cpu().numpy(), v[0].float().cpu().numpy()]).reshape(2, su.M, su.hkv, dh)
    written = np.zeros(su.cache.tensors[2].shape[::2], bool)
    flips = total = 0
    for row, _, t, page_i, at in _places(su):
        x = yn[row, su.hq * dh:].reshape(2, su.hkv, dh).copy()
        if rope:
            x[0] = _turned(x[0][None], np.array([t]), rope)[0]
        codes, scale, zero = _stored(su, page_i, at)
        for m in range(2):
            q, s, z = _encode(x[m], bits, sym)
            if rope and m == 0:     # libraries' fp64 cosines may differ in the last place, the key by one fp32 step
                np.testing.assert_allclose(scale[m], s, rtol=2.0 ** -22)
                assert np.abs(codes[m].astype(int) - q).max() <= 1
                flips, total = flips + int((codes[m] != q).sum()), total + q.size
            else:
                np.testing.assert_array_equal(scale[m], s)
                np.testing.assert_array_equal(zero[m], z)
                np.testing.assert_array_equal(codes[m], q)
            val = (codes[m].astype(np.float32) - zero[m][:, None].astype(np.float32)) * scale[m][:, None]
            np.testing.assert_array_equal(kv[m, row], torch.from_numpy(val).to(su.dtype).float().numpy())
        written[page_i, at] = True
    assert flips <= 1e-4 * total + 1
    # nothing else was touched
    assert bool((k[0, su.M - 2:] == 3).all()) and bool((v[0, su.M - 2:] == 3).all())
    kc, vc, ks, vs, kz, vz = [None if t is None else t.cpu().numpy() for t in su.cache.tensors]
    free = ~written
    assert (kc.transpose(0, 2, 1, 3)[free] == 255).all()
    assert (vc.transpose(0, 2, 4, 1, 3).reshape(kc.shape[0], page, su.hkv, -1)[free] == 255).all()
    assert np.isnan(ks.transpose(0, 2, 1)[free]).all() and np.isnan(vs.transpose(0, 2, 1)[free]).all()
    if not sym:
        assert (kz.transpose(0, 2, 1)[free] == 255).all() and (vz.transpose(0, 2, 1)[free] == 255).all()


def test_cache_far_positions():
    """The rotary angle at position 2^30: fp64 throughout."""
    far = 1 << 30
    su = Setup("f32", [(0, 1)], rope=10000.0, page=256, spare_rows=0)
    cols = far // 256 + 1
    pages = torch.full((1, cols), -1, dtype=torch.int32, device="cuda")
    pages[0, -1] = 1
    rows = jab.CacheRows(pages, torch.tensor([far], dtype=torch.int32, device="cuda"), su.start, 1)
    y = su.y(1)
    jab.cache_write(su.p, su.cache, rows, y)
    x = y[0, 0, 4 * 64:6 * 64].cpu().numpy().reshape(1, 2, 64)
    want = _turned(x, np.array([far]), 10000.0)[0]
    codes, scale, zero = _stored(su, 1, 0)
    got = (codes[0].astype(np.float64) - zero[0][:, None]) * scale[0][:, None]
    # half a step of the grid; an angle of 2^30 rad in fp64 is good to 2^-22
    assert np.abs(got - want).max() <= (0.5 + 1e-3) * scale[0].max()


def test_cache_values_that_are_not_finite():
    su = Setup("f32", [(0, 6)], page=32)
    y = su.y(su.M)
    k0, v0 = 4 * 64, 6 * 64
    y[0, 1, k0 + 3], y[0, 2, v0 + 64] = math.nan, math.inf
    y[0, 3, k0], y[0, 3, k0 + 1] = 3e38, -3e38             # the range overflows
    y[0, 4, k0:k0 + 64] = 0
    jab.cache_write(su.p, su.cache, su.rows, y)
    k, v = jab.cache_read(su.p, su.cache, su.rows)
    kb, vb = k[0, :6].reshape(6, 2, 64).isnan().all(-1).cpu(), v[0, :6].reshape(6, 2, 64).isnan().all(-1).cpu()
    want_k, want_v = torch.zeros(6, 2, dtype=torch.bool), torch.zeros(6, 2, dtype=torch.bool)
    want_k[1, 0] = want_k[3, 0] = want_v[2, 1] = True
    assert torch.equal(kb, want_k) and torch.equal(vb, want_v)
    assert torch.equal(k[0, :6].reshape(6, 2, 64).isnan().any(-1).cpu(), want_k)
    assert bool((k[0, 4, :64] == 0).all())


def test_cache_bad_tables():
    """Pages outside the pool, tokens past the last column, rows past the batch: not stored, not seen, no access."""
    su = Setup("bf16", [(0, 40), (20, 40), (0, 8)], page=32, extra_cols=0)
    pages = su.pages.clone()
    pages[0, 1], pages[1, 0] = 1 << 30, -7
    start = torch.tensor([0, 40, 80, 10 ** 9], dtype=torch.int32, device="cuda")
    past = torch.tensor([0, 2 ** 31 - 1, -5], dtype=torch.int32, device="cuda")
    rows = jab.CacheRows(pages, past, start, 40)
    y = su.y(su.M)
    jab.cache_write(su.p, su.cache, rows, y)
    k = torch.full((1, su.M, su.hkv * su.dh), 3.0, dtype=su.dtype, device="cuda")
    v = k.clone()
    jab.cache_read(su.p, su.cache, rows, k, v)
    assert bool((k[0, 32:40] == 0).all()) and bool((v[0, 32:40] == 0).all())       # the bad page
    assert bool((k[0, 40:80] == 3).all())                                          # past the columns
    assert not bool((k[0, :32] == 0).all(1).any()) and not bool((k[0, 80:] == 3).all(1).any())
    a = jab.attn_cache(su.p, su.cache, rows, y)
    assert bool(a[0, :40].isfinite().all()) and bool(a[0, 80:].isfinite().all())
    # a descending start: no rows
    rows = jab.CacheRows(su.pages, su.past, torch.tensor([50, 40, 30, -4], dtype=torch.int32, device="cuda"), 40)
    before = [None if t is None else t.clone() for t in su.cache.tensors]
    jab.cache_write(su.p, su.cache, rows, y)
    for t, b in zip(su.cache.tensors, before):
        assert t is None or torch.equal(t.view(torch.uint8), b.view(torch.uint8))


# ------------------------------------------------------------------ attention
def _values(su, host, i, length):
    """keys and values [2][length][hkv][dh] of sequence i in fp64, from the cache's codes (host: its tensors)"""
    pages, out = su.pages.cpu().numpy(), []
    kc, vc, ks, vs, kz, vz = host
    for c, s, z, tr in ((kc, ks, kz, False), (vc, vs, vz, True)):
        rows = []
        for col in range((length + su.page - 1) // su.page):
            b = c[pages[i, col]]
            if tr:
                b = b.transpose(0, 1, 3, 2).reshape(su.hkv, su.page, -1)
            if su.bits == 4:
                b = np.concatenate([b & 15, b >> 4], -1)
            zz = 2 ** (su.bits - 1) - 1 if su.sym else z[pages[i, col]].astype(np.float64)[..., None]
            rows.append((b.astype(np.float64) - zz) * s[pages[i, col]].astype(np.float64)[..., None])
        out.append(np.concatenate(rows, 1)[:, :length].transpose(1, 0, 2))
    return np.stack(out)


def _largest_scale(su, host, i, length):
    """the largest value scale of sequence i per query head"""
    s = host[3][su.pages[i, : (length + su.page - 1) // su.page].cpu().numpy()].astype(np.float64)
    s = s.transpose(1, 0, 2).reshape(su.hkv, -1)[:, :length].max(1)
    return np.repeat(s, su.hq // su.hkv)


def _attend(su, y):
    """The definition in fp64 and, per output element, how far the kernel may be: with u the step of the fp16
    parts (2^-11 one part, 2^-22 two), a weight is off by u relative, a logit by (u + (dh + 8) 2^-24) S, S = sum |q k| /
    sqrt(dh), which moves a weight by twice that; fp32 sums over n keys by (n / 16 + 64) 2^-24; all times
    sum p |v|; and half a step of the output's type.

    What is small is held to absolute steps.  The smallest step of fp16 is 2^-24.  A query row is scaled so that its
    largest element lies in 2^3 .. 2^4: an element is off by at most 2^-25, which is 2^-28 of the row's largest.
    A weight p sv is scaled by 2^6 / 2^E with 2^E at most twice the largest sv: it is off by at most 2^-25 2^-6 2 max sv =
    2^-30 max sv, times a code difference of at most 255 and the n keys (l is at least 1: the reference's own
    key counts 1).  And fp32 has no step below 2^-149."""
    yn = y[0].double().cpu().numpy()
    u = 2.0 ** (-11 if su.dtype == torch.bfloat16 else -22)
    want, tol = np.zeros((su.M, su.hq * su.dh)), np.zeros((su.M, su.hq * su.dh))
    row = 0
    host = [None if t is None else t.cpu().numpy() for t in su.cache.tensors]
    for i, (a, n) in enumerate(su.seqs):
        if n == 0:
            continue
        q = yn[row:row + n, : su.hq * su.dh].reshape(n, su.hq, su.dh)
        if su.rope:
            q = _turned(q, np.arange(a, a + n), su.rope)
        k, v = _values(su, host, i, a + n)
        k, v = np.repeat(k, su.hq // su.hkv, 1), np.repeat(v, su.hq // su.hkv, 1)
        z = np.einsum("nhd,thd->hnt", q, k) / math.sqrt(su.dh)
        S = np.einsum("nhd,thd->hnt", np.abs(q), np.abs(k)) / math.sqrt(su.dh)
        late = np.arange(a + n)[None] > np.arange(a, a + n)[:, None]
        z[:, late] = -np.inf
        S[:, late] = 0
        w = np.exp(z - z.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        o = np.einsum("hnt,thd->nhd", w, v)
        delta = (u + (su.dh + 8) * 2.0 ** -24) * S.max(-1)                   # [h][n]
        delta += 2.0 ** -28 * np.abs(q).max(-1).T * np.abs(k).sum(-1).max(0)[:, None] / math.sqrt(su.dh)
        rel = u + 2 * delta + ((a + n) / 16 + 64) * 2.0 ** -24
        A = np.einsum("hnt,thd->nhd", w, np.abs(v))
        want[row:row + n] = o.reshape(n, -1)
        t = A * rel.T[..., None] + np.abs(o) * torch.finfo(su.dtype).eps / 2 + 2.0 ** -149
        t = t + ((a + n) * 255 * 2.0 ** -30 * _largest_scale(su, host, i, a + n))[None, :, None]
        if su.dtype == torch.float16:
            t = t + 2.0 ** -25                             # half a step of its subnormals
        tol[row:row + n] = t.reshape(n, -1)
        row += n
    return want, tol


def _check_attention(su, y, out=None):
    a = torch.full((1, su.M, su.hq * su.dh), 9.0, dtype=su.dtype, device="cuda") if out is None else out
    if out is None:
        jab.attn_cache(su.p, su.cache, su.rows, y, out=a)
    got = a[0].double().cpu().numpy()
    want, tol = _attend(su, y)
    n = sum(n for _, n in su.seqs)
    off = np.abs(got - want)[:n] - tol[:n]
    assert np.isfinite(got[:n]).all()
    assert off.max() <= 0, (float(off.max()), np.unravel_index(off.argmax(), off.shape))
    assert (got[n:] == 9).all()                            # rows of no sequence


ATTN = [  # dtype, hq, hkv, head_dim, bits, symmetric, rope, page, (past, new)
    ("bf16", 8, 2, 128, 8, False, 10000.0, 64, [(100, 1), (0, 1), (31, 1), (640, 1), (32, 1)]),
    ("bf16", 8, 2, 128, 4, False, 10000.0, 32, [(77, 1), (500, 1)]),
    ("bf16", 8, 2, 64, 8, True, 0.0, 64, [(200, 3), (0, 4), (63, 1)]),
    ("bf16", 4, 4, 16, 8, False, 10000.0, 32, [(50, 1), (3, 2)]),
    ("f16", 12, 12, 64, 8, False, 0.0, 64, [(200, 1), (1, 1)]),
    ("f16", 8, 4, 64, 4, True, 10000.0, 128, [(129, 5), (0, 17)]),
    ("f16", 8, 1, 128, 8, False, 0.0, 256, [(300, 2)]),
    ("f16", 4, 4, 16, 4, False, 0.0, 32, [(33, 7)]),
    ("f32", 4, 4, 16, 8, False, 0.0, 32, [(0, 32), (0, 31)]),
    ("f32", 8, 2, 64, 8, True, 10000.0, 64, [(40, 1), (90, 9)]),
    ("f32", 8, 2, 128, 4, False, 10000.0, 64, [(100, 33)]),
    ("bf16", 32, 1, 64, 8, False, 0.0, 64, [(65, 1), (10, 2)]),        # 32 and 64 rows
    ("bf16", 8, 2, 128, 8, False, 10000.0, 64, [(90, 70), (0, 1), (5, 130)]),      # rows by waves
    ("bf16", 4, 4, 64, 4, False, 0.0, 64, [(0, 200), (33, 65)]),
    ("f32", 4, 2, 16, 4, True, 10000.0, 32, [(0, 100)]),
    ("f16", 16, 2, 128, 8, True, 10000.0, 128, [(260, 50)]),
]


@pytest.mark.parametrize("dtype,hq,hkv,dh,bits,sym,rope,page,seqs", ATTN)
def test_attention_over_the_cache(dtype, hq, hkv, dh, bits, sym, rope, page, seqs):
    su = Setup(dtype, seqs, hq, hkv, dh, bits, sym, rope, page)
    su.history()
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


@pytest.mark.parametrize("dtype,bits,seqs", [("bf16", 8, [(5000, 1)]), ("bf16", 4, [(9000, 1), (4, 1)]),
                                            ("f32", 8, [(3000, 2), (2999, 1)]), ("f16", 4, [(4000, 20)])])
def test_attention_with_a_split_key_axis(dtype, bits, seqs):
    su = Setup(dtype, seqs, 8, 2, 128 if bits == 8 else 64, bits, rope=10000.0, page=64)
    assert jab.attn_cache_workspace(su.p, su.cache, su.rows).numel() > 0
    su.history()
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


@pytest.mark.parametrize("dtype,bits,dh,seqs", [
    # one sequence far longer than the others, some without new tokens, cuts inside and between heads
    ("bf16", 8, 128, [(3, 1), (20000, 1), (0, 0), (900, 2), (40, 1), (0, 0), (2500, 1), (7, 3)]),
    ("f32", 4, 16, [(0, 0), (12000, 1), (5, 1), (5, 0), (700, 1), (0, 0)]),
    ("f16", 8, 64, [(100, 6)] * 30 + [(4000, 8)] + [(0, 1)] * 40),
    # tiles of many rows cut between workgroups
    ("bf16", 8, 64, [(3000, 150), (0, 0), (10, 70), (0, 400), (1500, 1)]),
    ("f32", 8, 16, [(0, 700), (2000, 40)]),
])
def test_attention_of_uneven_sequences(dtype, bits, dh, seqs):
    su = Setup(dtype, seqs, 8, 2, dh, bits, rope=10000.0, page=64, spare_rows=1)
    su.history()
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


@pytest.mark.parametrize("dtype,bits,dh,seqs", [
    # prompts without or with a short past: few blocks, many tiles of rows
    ("bf16", 8, 128, [(0, 300), (0, 17), (100, 256)]), ("f16", 4, 64, [(0, 140), (0, 0), (0, 512)]),
    ("f32", 8, 16, [(0, 640)]), ("bf16", 4, 64, [(300, 40)]),
])
def test_attention_of_short_prompts(dtype, bits, dh, seqs):
    su = Setup(dtype, seqs, 8, 2, dh, bits, rope=10000.0, page=32, spare_rows=1)
    assert jab.attn_cache_workspace(su.p, su.cache, su.rows).numel() > 0                 # shares
    su.history()
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


@pytest.mark.parametrize("new", [1, 20])
def test_attention_of_many_sequences(new):
    """More sequences than a workgroup scans: one workgroup per (sequence, head)."""
    rng = np.random.default_rng(5)
    seqs = [(int(a), int(n)) for a, n in zip(rng.integers(0, 60, 600), rng.integers(0, new + 1, 600))]
    su = Setup("bf16", seqs, 8, 2, 16, page=32)
    y0 = su.y(sum(a for a, _ in seqs))                     # all the histories in one call
    p = _problem("bf16", y0.shape[1], 64, 8, 2, 16)
    start = torch.tensor(np.cumsum([0] + [a for a, _ in seqs]), dtype=torch.int32, device="cuda")
    jab.cache_write(p, su.cache, jab.CacheRows(su.pages, torch.zeros_like(su.past), start, 60), y0)
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


def test_attention_more_new_tokens_than_told():
    su = Setup("bf16", [(10, 70), (0, 40)], 8, 2, 64, max_new=1, spare_rows=0)
    su.history()
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


@pytest.mark.parametrize("scale,vscale", [(1e-30, 1e30), (1e4, 1e-30), (40.0, 1.0)])
def test_attention_of_unusual_magnitudes(scale, vscale):
    """Queries and values far from 1; peaked softmaxes."""
    su = Setup("f32", [(150, 2)], 8, 2, 64, page=32)
    y0 = su.y(150, 1.0)
    y0[..., (8 + 2) * 64:] *= vscale
    one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")               # noqa: E731
    jab.cache_write(_problem("f32", 150, 64, 8, 2, 64), su.cache,
                    jab.CacheRows(su.pages, one([0]), one([0, 150]), 150), y0)
    y = su.y(su.M, scale)
    y[..., (8 + 2) * 64:] *= vscale
    if scale == 1e4:                                       # logits of 1e4: keys of 1e-3
        y[..., 8 * 64:10 * 64] *= 1e-3
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


def test_attention_values_of_very_different_scales():
    """Each token's values a power of two apart: the weights' scale follows the largest."""
    su = Setup("f32", [(0, 60)], 4, 2, 64, page=32)
    y = su.y(su.M, 1.0)
    y[0, :60, 6 * 64:] *= (2.0 ** (torch.arange(60, device="cuda") - 40))[:, None]
    jab.cache_write(su.p, su.cache, su.rows, y)
    _check_attention(su, y)


def test_attention_rows_that_see_nothing():
    su = Setup("bf16", [(40, 2), (8, 1), (5, 40)], 8, 2, 64, page=32, spare_rows=1)
    su.history()
    y = su.y(su.M, 2.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    pages = su.pages.clone()
    pages[1] = -1                                          # nothing of sequence 1
    pages[2, 0] = 1 << 20                                  # not the first page of sequence 2
    a = torch.full((1, su.M, 8 * 64), 9.0, dtype=su.dtype, device="cuda")
    jab.attn_cache(su.p, su.cache, jab.CacheRows(pages, su.past, su.start, 40), y, out=a)
    assert bool((a[0, 2] == 0).all())
    assert bool((a[0, 3:3 + 27] == 0).all()) and bool(a[0, 30:43].isfinite().all())
    assert not bool((a[0, 30:43] == 0).all(1).any()) and bool((a[0, 43] == 9).all())


@pytest.mark.parametrize("past", [40, 5000])
def test_attention_single_tokens_without_their_first_pages(past):
    """A decoding step whose first pages are gone sees the rest, and 0 where all are gone."""
    su = Setup("bf16", [(past, 1), (past, 1)], 8, 2, 64, page=32, spare_rows=0)
    su.history()
    y = su.y(2, 2.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    gone = past // 32                                      # the new token's own page stays
    pages = su.pages.clone()
    pages[0, :gone] = -1
    pages[1] = -1
    a = jab.attn_cache(su.p, su.cache, jab.CacheRows(pages, su.past, su.start, 1), y)[0]
    assert bool((a[1] == 0).all())
    # the same tokens as a short sequence of their own (no rotary embedding: positions do not matter)
    n = past + 1 - 32 * gone
    one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")               # noqa: E731
    b = jab.attn_cache(_problem("bf16", 1, 64, 8, 2, 64), su.cache,
                       jab.CacheRows(su.pages[:1, gone:].contiguous(), one([n - 1]), one([0, 1]), 1), y[:, :1].contiguous())[0]
    # half a step of bf16 each, and the weights' 2^-11 of sum p |v|, at most the largest |v|
    v = jab.cache_read(_problem("bf16", n, 64, 8, 2, 64), su.cache,
                       jab.CacheRows(su.pages[:1, gone:].contiguous(), one([0]), one([0, n]), n))[1].abs().max().item()
    assert float((a[0] - b[0]).abs().max()) <= 2 * (2.0 ** -8 + 2.0 ** -11) * v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("first,second", [(40, 3), (3, 2)])                          # many rows, few rows
def test_attention_nan_stays_in_its_rows(dtype, first, second):
    su = Setup(dtype, [(0, first), (0, second)], 8, 2, 64, page=32, spare_rows=0)
    y = su.y(su.M, 2.0)
    y[0, 2, 3] = math.nan                                  # a query of head 0
    y[0, first + 1, 8 * 64 + 1] = math.inf                 # a key of head 0, sequence 1: seen by its rows from there on
    y[0, 1, 11 * 64 + 5] = math.nan                        # a value of head 1, sequence 0
    jab.cache_write(su.p, su.cache, su.rows, y)
    bad = jab.attn_cache(su.p, su.cache, su.rows, y)[0].reshape(su.M, 8, 64).isnan()
    want = torch.zeros(su.M, 8, dtype=torch.bool, device="cuda")
    want[2, 0] = True
    want[first + 1:, :4] = True
    want[1:first, 4:] = True
    assert torch.equal(bad.any(-1), want) and torch.equal(bad.all(-1), want)


def test_attention_steps_as_one_prompt():
    """A prompt written and attended in chunks gives what the whole prompt gives: every row is the same function
    of its query and the cache."""
    n = 75
    whole = Setup("f32", [(0, n)], 8, 2, 64, rope=10000.0, page=32, spare_rows=0)
    y = whole.y(n, 3.0)
    jab.cache_write(whole.p, whole.cache, whole.rows, y)
    a = jab.attn_cache(whole.p, whole.cache, whole.rows, y)
    one = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")               # noqa: E731
    cache = jab.Cache.empty(whole.p, 8, 32, whole.cache.struct.n_pages)
    at = 0
    for step in (1, 1, 30, 1, 33, 9):
        p, rows = _problem("f32", step, 64, 8, 2, 64, rope=10000.0), jab.CacheRows(whole.pages, one([at]), one([0, step]), step)
        part = y[:, at:at + step].contiguous()
        jab.cache_write(p, cache, rows, part)
        b = jab.attn_cache(p, cache, rows, part)
        # the two differ by the order of fp32 sums alone
        torch.testing.assert_close(b, a[:, at:at + step], rtol=2e-5, atol=2e-6)
        at += step
    written = (whole.pages[0, :-1] >= 0).sum()
    used = whole.pages[0, :written].long()
    assert torch.equal(cache.tensors[0][used][0], whole.cache.tensors[0][used][0])


def test_block_from_tokens_to_attention():
    """Tokens quantized, projected in integers, cached and attended, against the same chain in fp64 from the
    dequantized operands."""
    d, hq, hkv, dh = 256, 8, 2, 64
    su = Setup("bf16", [(0, 40), (0, 33), (0, 7)], hq, hkv, dh, rope=10000.0, spare_rows=0)
    p = _problem("bf16", su.M, d, hq, hkv, dh, rope=10000.0)
    x = torch.randn((1, su.M, d), generator=su.gen, device="cuda").bfloat16()
    w = (torch.randn((p.rows, d), generator=su.gen, device="cuda") * 0.1).bfloat16()
    wq, sw = jab.quant_rows(p, w)
    xq, sx = jab.quant_rows(p, x)
    y = jab.project_int(p, xq, sx, wq, sw)
    # whole sums first: scaled operands would leave 1e-17 where the sum is 0
    y64 = (xq[0].double() @ wq.double().t().contiguous()) * sx[0].double()[:, None] * sw.double()
    # half a step of bf16 and three fp32 roundings
    assert bool(((y[0].double() - y64).abs() <= y64.abs() * (2.0 ** -8 + 2.0 ** -22)).all())
    # and it is the float projection up to the grids: half a step of each operand
    full = x[0].double() @ w.double().t().contiguous()
    slack = 0.5 * (sx[0].double()[:, None] * w.double().abs().sum(1) + sw.double() * x[0].double().abs().sum(1)[:, None]
                   + 0.5 * d * sx[0].double()[:, None] * sw.double())
    assert bool(((y64 - full).abs() <= slack).all())
    jab.cache_write(p, su.cache, su.rows, y)
    su.p = p
    _check_attention(su, y)


# ------------------------------------------------------------------ streams and graphs
@pytest.mark.parametrize("bits,seqs", [(8, [(700, 1), (90, 2)]), (4, [(300, 70), (0, 33)])])
def test_pages_behind_4_gib(bits, seqs):
    """The same pages at the front of a small cache and behind 2^32 bytes of codes: bitwise the same results."""
    got = []
    for big in (False, True):
        su = Setup("bf16", seqs, 8, 2, 128, bits, rope=10000.0, page=256, spare_rows=0)
        if big:
            n = (1 << 32) // (256 * 2 * 128 * bits // 8)
            used = su.cache.tensors[0].shape[0]
            su.cache = jab.Cache.empty(su.p, bits, 256, n + used)
            su.pages += torch.where(su.pages >= 0, n, 0).to(torch.int32)
        su.history()
        y = su.y(su.M, 3.0)
        jab.cache_write(su.p, su.cache, su.rows, y)
        got.append(jab.cache_read(su.p, su.cache, su.rows) + (jab.attn_cache(su.p, su.cache, su.rows, y),))
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


def test_another_stream_and_repeats():
    su = Setup("bf16", [(700, 1), (33, 1)], 8, 2, 128, page=64, spare_rows=0)
    su.history()
    y = su.y(su.M, 3.0)
    jab.cache_write(su.p, su.cache, su.rows, y)
    a = jab.attn_cache(su.p, su.cache, su.rows, y)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        jab.cache_write(su.p, su.cache, su.rows, y)
        b = jab.attn_cache(su.p, su.cache, su.rows, y)
    st.synchronize()
    assert torch.equal(a, b)                               # bitwise: no order of sums depends on the run


def test_captured_step_follows_the_tables():
    """A captured decoding step, replayed with other rows and lengths, against the eager step each time."""
    steps, hq, hkv, dh, d = 5, 8, 2, 128, 256
    su = Setup("bf16", [(40, steps), (300, steps)], hq, hkv, dh, rope=10000.0, page=32, spare_rows=0, max_new=1)
    su.history()
    p = _problem("bf16", 2, d, hq, hkv, dh, rope=10000.0)
    wq, sw = jab.quant_rows(p, (torch.randn((p.rows, d), generator=su.gen, device="cuda") * 0.1).bfloat16())
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    past, x = su.past.clone(), torch.zeros((1, 2, d), dtype=torch.bfloat16, device="cuda")
    rows = jab.CacheRows(su.pages, past, start, 1)
    ws = jab.attn_cache_workspace(p, su.cache, rows)
    out = torch.empty((1, 2, hq * dh), dtype=torch.bfloat16, device="cuda")

    def step(cache, out):
        xq, sx = jab.quant_rows(p, x)
        y = jab.project_int(p, xq, sx, wq, sw)
        jab.cache_write(p, cache, rows, y)
        return jab.attn_cache(p, cache, rows, y, ws=ws, out=out)

    other = jab.Cache(p, 8, 32, *[t.clone() for t in su.cache.tensors])              # the eager steps' cache
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(su.cache, out)                                # position 40: written again by the first replay
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(su.cache, out)
    for k in range(steps):
        x.copy_(torch.randn((1, 2, d), generator=su.gen, device="cuda"))
        past.copy_(su.past + k)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = step(other, torch.empty_like(out))
        torch.cuda.synchronize()
        assert torch.equal(got, want), k
