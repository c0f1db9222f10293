"""The operators around the products of a serving step: norm into block formats, the quantized paged cache, attention over it.

Conversions are compared bit for bit with the CPU oracle, attention with softmax attention in 64 bits on the de-converted cache.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import wide
from paper_2510_14557_amd import mxp, synth

gpu = pytest.mark.gpu
FMTS = {"MXFP4": mxp.MXFP4, "MXFP4P": mxp.MXFP4P, "MXFP4PP": mxp.MXFP4PP, "MXFP6": mxp.MXFP6, "MXFP6P": mxp.MXFP6P, "MXFP8": mxp.MXFP8,
        "MXFP8P": mxp.MXFP8P}
PLAIN = (mxp.MXFP4, mxp.MXFP6, mxp.MXFP8)
FOUR = ["MXFP4", "MXFP4P", "MXFP4PP"]
U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}          # half a step, relative


def quantize(x, fmt):
    """Oracle bytes of fp32 rows or bf16 bits."""
    return oracle.quantize(x, fmt) if fmt <= mxp.MXFP4PP else wide.quantize(x, fmt)


def dequantize(q, fmt):
    return np.asarray(oracle.dequantize(q, fmt) if fmt <= mxp.MXFP4PP else wide.dequantize(q, fmt), dtype=np.float64)


def host(t):
    return t.float().cpu().numpy()


def same_bytes(got, want, fmt):
    e, s, i = (t.cpu().numpy() for t in got)
    assert (s == want[1]).all() and (e == want[0]).all()
    if fmt not in PLAIN:
        assert (i == want[2]).all()


# ---- norm -----------------------------------------------------------------------------------------------------------
SPECIAL = [0.0, -0.0, 1e-39, 2.0 ** -125, -(2.0 ** -124), 7.5, 7.9, -7.0, 5.0, 3.0e38, 0.25, 0.75, 2.5, -3.5, 448.0, 460.0]


def special_weight(K, bf16, seed=5):
    rng = np.random.default_rng(seed)
    w = (rng.standard_normal(K) * np.exp2(rng.integers(-3, 4, K))).astype(np.float32)
    for b in range(0, K - 31, 32):
        kind = b // 32 % 7
        if kind == 0:
            w[b:b + 32] = 0.0
            w[b + 3] = SPECIAL[b // 32 % len(SPECIAL)]
        elif kind == 1:
            w[b:b + 32] = rng.choice(SPECIAL[5:], 32)
        elif kind == 2:
            w[b + 7] = [np.inf, np.nan, -np.inf][b // 32 % 3]
        elif kind == 3:
            w[b:b + 32] *= np.float32(2.0 ** -122)
        elif kind == 4:
            w[b + 9] *= 2.0 ** 9
    return synth.bf16_bits_to_f32(synth.f32_to_bf16_bits(w)) if bf16 else w


@gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("K", [32, 512, 4096, 16384, 32768])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_norm_of_signs_is_the_weight_bit_for_bit(fmt, K, dt):
    """Rows of +-2^a have the root mean square 2^a exactly (K a power of two, sums below 2^24): y = +-weight, special values included."""
    f = FMTS[fmt]
    rng = np.random.default_rng(K)
    sign = rng.choice([-1.0, 1.0], (3, K)).astype(np.float32)
    x = torch.from_numpy(sign * np.array([[1.0], [4.0], [0.125]], np.float32)).to("cuda", dt)
    w = special_weight(K, dt == torch.bfloat16)
    q, h = mxp.rmsnorm_quantize(x, torch.from_numpy(w).to("cuda", dt), f, eps=0.0)
    assert h is x
    with np.errstate(invalid="ignore"):
        same_bytes(q, quantize(sign * w, f), f)


@gpu
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,K", [(1, 4096), (5, 32), (37, 1056), (3, 16384), (2, 16416), (2, 33056)])
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
def test_norm_against_64_bits(fmt, rows, K, dt, residual):
    """Quantized values lie between those of y (1 - d) and y (1 + d): a lane sums at most 33056 / 1024 / 8 < 5 groups of 8 squares in a
    row and ten partial sums follow, so the sum is within 64 * 2^-24, y within half of that and four roundings: d = 2^-18."""
    f = FMTS[fmt]
    x = torch.from_numpy(synth.activations(rows, K, 1, 3, dtype="f32")).to("cuda", dt)
    r = torch.from_numpy(synth.activations(rows, K, 1, 4, dtype="f32")).to("cuda", dt) if residual else None
    w = (1 + 0.1 * torch.randn(K, generator=torch.Generator().manual_seed(K))).to("cuda", dt)
    q, h = mxp.rmsnorm_quantize(x, w, f, residual=r, eps=1e-5)
    want_h = (x.float() + r.float()).to(dt) if residual else x
    assert torch.equal(h, want_h)
    a = h.double().cpu().numpy()
    y = a / np.sqrt((a * a).mean(-1, keepdims=True) + 1e-5) * w.double().cpu().numpy()
    ends = [dequantize(quantize((y * (1 + d)).astype(np.float32), f), f) for d in (-2.0 ** -18, 2.0 ** -18)]
    got = dequantize(tuple(t.cpu().numpy() for t in q), f)
    assert (got >= np.minimum(*ends)).all() and (got <= np.maximum(*ends)).all()


@gpu
def test_norm_in_place_strided_and_rows_of_nothing():
    gen = torch.Generator(device="cuda").manual_seed(1)
    for K in (2048, 20000):                                       # in registers, in two passes
        wide_x = torch.randn((9, K + 64), generator=gen, device="cuda").bfloat16()
        wide_r = torch.randn((9, K + 32), generator=gen, device="cuda").bfloat16()
        w = torch.randn(K, generator=gen, device="cuda").bfloat16()
        x, r = wide_x[:, 32:32 + K], wide_r[:, :K]
        want_q, want_h = mxp.rmsnorm_quantize(x.contiguous(), w, mxp.MXFP8P, residual=r.contiguous())
        keep = wide_x.clone(), wide_r.clone()
        for out in (r, x):                                        # h over the residual, then over x (from the values before)
            wide_x.copy_(keep[0]); wide_r.copy_(keep[1])
            q, h = mxp.rmsnorm_quantize(x, w, mxp.MXFP8P, residual=r, h=out)
            assert h is out and torch.equal(out, want_h) and all(torch.equal(a, b) for a, b in zip(q, want_q))
        assert torch.equal(wide_x[:, :32], keep[0][:, :32]) and torch.equal(wide_x[:, 32 + K:], keep[0][:, 32 + K:])
        assert torch.equal(wide_r[:, K:], keep[1][:, K:])
        copy = torch.empty_like(want_h)                           # h without a residual: a copy of x
        mxp.rmsnorm_quantize(keep[0][:, 32:32 + K], w, mxp.MXFP8P, h=copy)
        assert torch.equal(copy, keep[0][:, 32:32 + K])
    z = torch.zeros((4, 64), device="cuda")
    z[1, 3], z[2, 40] = float("nan"), float("inf")
    (e, s, i), _ = mxp.rmsnorm_quantize(z, torch.ones(64, device="cuda"), mxp.MXFP4P, eps=1e-6)
    assert s.tolist() == [[0, 0], [255, 255], [0, 255], [0, 0]]   # NaN spoils the row; Inf: others 0 / Inf, itself NaN
    (e, s, i), _ = mxp.rmsnorm_quantize(z[3:], torch.ones(64, device="cuda"), mxp.MXFP4P, eps=0.0)
    assert s.tolist() == [[255, 255]]                             # 0 / 0
    for shape in ((0, 64), (3, 0)):
        (e, s, i), _ = mxp.rmsnorm_quantize(torch.empty(shape, device="cuda"), torch.empty(shape[1], device="cuda"), mxp.MXFP8)
        assert e.shape[0] == shape[0] and e.numel() == 0


@gpu
@pytest.mark.parametrize("K", [64, 1056, 16416])
def test_norm_of_more_rows_than_a_grid_has(K):
    """Rows behind the 16384 workgroups of a launch, of one wavefront, of several and in two passes: as calls of 1000 rows have them."""
    n = 2 * 16384 + 333 if K < 16000 else 16384 + 333
    gen = torch.Generator(device="cuda").manual_seed(K)
    x, r = (torch.randn((n, K), generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(K, generator=gen, device="cuda")
    q, h = mxp.rmsnorm_quantize(x, w, mxp.MXFP8P, residual=r)
    for at in (0, 16000, 16384, n - 1000):
        rows = slice(at, at + 1000)
        part, hp = mxp.rmsnorm_quantize(x[rows], w, mxp.MXFP8P, residual=r[rows])
        assert torch.equal(h[rows], hp) and all(torch.equal(a[rows], b) for a, b in zip(q, part))


# ---- the cache ------------------------------------------------------------------------------------------------------
def records(e, s, i, n_pages, T, H, D, fmt):
    """Oracle bytes of rows [page][token][head] as the cache's records [page][head][bytes]."""
    parts = []
    for a, width in ((e, D // 2), (s, D // 32), (i, D // 32))[:2 if fmt == mxp.MXFP4 else 3]:
        parts.append(a.reshape(n_pages, T, H, width).transpose(0, 2, 1, 3).reshape(n_pages, H, T * width))
    return np.concatenate(parts, -1)


@gpu
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,D,n", [(16, 1, 64, 1), (16, 8, 128, 77), (64, 3, 128, 200), (256, 5, 64, 311), (32, 2, 256, 50), (128, 7, 256, 3)])
def test_cache_write_and_read_bit_for_bit(fmt, dt, T, H, D, n):
    f = FMTS[fmt]
    rng = np.random.default_rng(n)
    n_pages = n // T + 3
    slots = rng.permutation(n_pages * T)[:n].astype(np.int64)
    qkv = synth.activations(n, 3 * H * D, 2, n % 7, dtype="f32").reshape(n, 3 * H, D)
    qkv[:, :, :32] *= np.exp2(rng.integers(-130, 100, (n, 3 * H, 1))).astype(np.float32)
    qkv[0, :, 32:64] = 0
    qkv[-1, 1::2, 40], qkv[-1, ::2, 33] = np.inf, np.nan
    x = torch.from_numpy(qkv).to("cuda", dt)
    k, v = x[:, H:2 * H], x[:, 2 * H:]                            # slices of a joint projection
    bits = synth.f32_to_bf16_bits(qkv) if dt == torch.bfloat16 else qkv
    skipped = slots.copy()
    skipped[::5] = [-1, n_pages * T, -(2 ** 40), 2 ** 40][n % 4]
    cache = mxp.cache_empty(n_pages, T, H, D, f)
    cache.data.fill_(0xA5)
    mxp.cache_write(cache, k, v, torch.from_numpy(skipped).cuda())
    kept = skipped == slots
    want = np.full(tuple(cache.data.shape), 0xA5, np.uint8)
    values = []
    for part, rows in ((0, bits[:, H:2 * H]), (1, bits[:, 2 * H:])):
        e, s, i = oracle.quantize(np.ascontiguousarray(rows).reshape(n * H, D), f)
        values.append(oracle.dequantize((e, s, i), f).reshape(n, H, D))
        full = []
        for a in (e, s, i):
            b = np.full((n_pages * T, H, a.shape[1]), 0xA5, np.uint8)
            b[slots[kept]] = a.reshape(n, H, -1)[kept]
            full.append(b)
        want[:, :, part] = records(*full, n_pages, T, H, D, f)
    assert (cache.data.cpu().numpy() == want).all()
    for out_dt in (torch.bfloat16, torch.float32):
        room = torch.full((n, 2 * H + 1, D), 7.0, dtype=out_dt, device="cuda")
        got = mxp.cache_read(cache, torch.from_numpy(skipped).cuda(), out=(room[:, :H], room[:, H:2 * H]))
        for g, val in zip(got, values):
            np.testing.assert_array_equal(g.double().cpu().numpy(), np.where(kept[:, None, None], val, 0.0))
        assert (room[:, 2 * H] == 7).all()
    twice = torch.from_numpy(np.repeat(slots[kept][:1], 5)).cuda()   # a slot may be read more than once
    np.testing.assert_array_equal(mxp.cache_read(cache, twice, torch.float32)[1].double().cpu().numpy(), np.repeat(values[1][kept][:1], 5, 0))


@gpu
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,H,n", [(64, 7, 20011), (128, 5, 13999), (256, 8, 4099)])
def test_cache_of_many_rows(fmt, dt, D, H, n):
    """Enough rows for the launch with several groups per lane: the records are mxp_quantize's bytes, what is read mxp_dequantize's values."""
    f, T = FMTS[fmt], 64
    gen = torch.Generator(device="cuda").manual_seed(D)
    n_pages = n // T + 2
    slots = torch.randperm(n_pages * T, generator=gen, device="cuda")[:n]
    k, v = (torch.randn((n, H, D), generator=gen, device="cuda").mul_(torch.exp2(torch.randint(-9, 9, (n, 1, 1), generator=gen, device="cuda").float())).to(dt)
            for _ in range(2))
    given = slots.clone()
    given[::7] = -1
    cache = mxp.cache_empty(n_pages, T, H, D, f)
    cache.data.fill_(0xA5)
    mxp.cache_write(cache, k, v, given)
    kept = given >= 0
    for part, x, back in zip((0, 1), (k, v), mxp.cache_read(cache, given, dt)):
        q = mxp.quantize(x.view(n * H, D), f)
        at = 0
        for a, width in zip(q, (D // 2, D // 32, D // 32)[:2 if f == mxp.MXFP4 else 3]):
            want = torch.full((n_pages * T, H, width), 0xA5, dtype=torch.uint8, device="cuda")
            want[slots[kept]] = a.view(n, H, width)[kept]
            got = cache.data[:, :, part, at:at + T * width].reshape(n_pages, H, T, width).transpose(1, 2).reshape(n_pages * T, H, width)
            assert torch.equal(got, want)
            at += T * width
        assert torch.equal(back, torch.where(kept[:, None, None], mxp.dequantize(q, f, dt).view(n, H, D), 0.0))


@gpu
def test_cache_of_more_tiles_than_a_grid_has():
    """Tokens behind the 65535th tile of 8 (head_dim 256): the first and the last of them as the dense conversions have them."""
    n, D = 65535 * 8 + 21, 256
    x = torch.randn((2, n, 1, D), device="cuda", generator=torch.Generator("cuda").manual_seed(3)).bfloat16()
    c = mxp.cache_empty(-(-n // 256), 256, 1, D, mxp.MXFP4P)
    slots = torch.arange(n, device="cuda")
    mxp.cache_write(c, x[0], x[1], slots)
    got = mxp.cache_read(c, slots, torch.bfloat16)
    for g, want in zip(got, x):
        assert torch.equal(g.view(n, D), mxp.dequantize(mxp.quantize(want.view(n, D), mxp.MXFP4P), mxp.MXFP4P, torch.bfloat16))


@gpu
def test_cache_beyond_32_bit_offsets():
    """Pages above 4 GiB: written, read and attended to as the first ones are."""
    T, H, D, f = 256, 8, 128, mxp.MXFP4P
    n_pages = 18500
    size = mxp.cache_bytes(n_pages, T, H, D, f)
    assert size > 5 << 30
    cache = mxp.cache_empty(n_pages, T, H, D, f)
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((300, H, D), generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((1, 16, D), generator=gen, device="cuda").bfloat16()
    kv_len = torch.tensor([300], dtype=torch.int32, device="cuda")
    outs = []
    for pages in ((0, 1), (n_pages - 1, n_pages - 2)):
        table = torch.tensor([pages], dtype=torch.int32, device="cuda")
        t = torch.arange(300, device="cuda")
        slots = table[0, t // T].long() * T + t % T
        mxp.cache_write(cache, k, v, slots)
        outs.append(mxp.cache_read(cache, slots, torch.float32) + (mxp.attention(q, cache, table, kv_len, out_dtype=torch.float32),))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# ---- attention ------------------------------------------------------------------------------------------------------
class Batch:
    """Sequences in a cache of quantized random rows; every slot that no sequence has is poisoned with NaN blocks."""

    def __init__(self, fmt, T, H, G, D, kv, nq, seed=0, gaps=False, garbage=True):
        rng = np.random.default_rng(seed)
        self.f, self.T, self.H, self.G, self.D, self.kv, self.nq = FMTS[fmt], T, H, G, D, kv, nq
        per = [-(-n // T) for n in kv]
        self.n_pages = n_pages = sum(per) + 2
        names = rng.permutation(n_pages)
        self.table = np.full((len(kv), max(max(per), 1) + 1), -1, np.int32)
        at = 0
        for s, p in enumerate(per):
            self.table[s, :p] = names[at:at + p]
            at += p
        raw = rng.standard_normal((2, n_pages * T * H, D)).astype(np.float32)
        raw[0] *= np.where(rng.random((1, D)) < 0.05, 6.0, 1.0).astype(np.float32)
        self.q3 = [oracle.quantize(r, self.f) for r in raw]
        self.val = [oracle.dequantize(q, self.f).reshape(n_pages * T, H, D) for q in self.q3]
        self.slots = [self.table[s, np.arange(n) // T].astype(np.int64) * T + np.arange(n) % T for s, n in enumerate(kv)]
        if garbage:
            free = np.ones(n_pages * T, bool)
            for sl in self.slots:
                free[sl] = False
            for e, sc, ix in self.q3:
                sc.reshape(n_pages * T, H, -1)[free] = 255
        self.start = np.concatenate([[0], np.cumsum(nq)]).astype(np.int32)
        self.q = torch.from_numpy(rng.standard_normal((int(self.start[-1]), H * G, D)).astype(np.float32)).bfloat16().cuda()

    def poison(self, seq, t, blocks, part):
        """NaN blocks in a visible token's keys (0) or values (1)."""
        slot = self.slots[seq][t]
        self.q3[part][1].reshape(self.n_pages * self.T, self.H, -1)[slot, :, blocks] = 255
        for b in blocks:
            self.val[part][slot, :, 32 * b:32 * b + 32] = np.nan

    def cache(self):
        data = np.stack([records(*q, self.n_pages, self.T, self.H, self.D, self.f) for q in self.q3], 2)
        return mxp.KVCache(torch.from_numpy(np.ascontiguousarray(data)).cuda(), self.T, self.H, self.D, self.f)

    def call(self, cache=None, **kw):
        n = len(self.kv)
        kw.setdefault("lse", torch.full((self.q.shape[0], self.H * self.G), 77.0, device="cuda"))
        kw.setdefault("max_q", max(self.nq + [1]))
        kw.setdefault("max_kv", max(self.kv))
        out = mxp.attention(kw.pop("q", self.q), cache or self.cache(), torch.from_numpy(self.table).cuda(),
                            torch.tensor(self.kv, dtype=torch.int32, device="cuda"),
                            q_start=None if self.nq == [1] * n else torch.from_numpy(self.start).cuda(), **kw)
        return out, kw["lse"]

    def check(self, out, lse, causal=True, window=0, scale=None, hidden=lambda s: None):
        """Against 64 bits.  An output is off by at most
            2 e S + p S + a S + u |o|,    S = sum p |v| / sum p,
        e: a score's error, 2 (D + 8) 2^-24 of the largest visible scale * sum |q k| (the product's sums and the roundings behind it),
        once in p and once in the sum; p: the rounding of p to one bf16 term (2^-8, bf16 output) or three (2^-24); a: fp32 sums over the
        tokens and joins, (tokens + 64) 2^-24, exp2 and the division in the 64; u: the output's own rounding."""
        scale = self.D ** -0.5 if scale is None else scale
        got, got_lse, qh = out.double().cpu().numpy(), lse.double().cpu().numpy(), self.q.double().cpu().numpy()
        p_err, u = (2.0 ** -8, U[torch.bfloat16]) if out.dtype == torch.bfloat16 else (2.0 ** -24, U[torch.float32])
        for s, n in enumerate(self.kv):
            m, rows = self.nq[s], slice(int(self.start[s]), int(self.start[s + 1]))
            k, v = (x[self.slots[s]].transpose(1, 0, 2) for x in self.val)         # [H][n][D]
            q = qh[rows].reshape(m, self.H, self.G, self.D).transpose(1, 0, 2, 3).reshape(self.H, m * self.G, self.D)
            pos = (n - m + np.arange(m) if causal else np.full(m, n - 1)).repeat(self.G)[None, :, None]
            t = np.arange(n)
            seen = np.broadcast_to((t <= pos) & ((t > pos - window) if window else True), (self.H, m * self.G, n)).copy()
            if hidden(s) is not None:
                seen[:, :, hidden(s)] = False
            z = np.where(seen, scale * (q @ k.transpose(0, 2, 1)), -np.inf)
            size = np.where(seen, abs(scale) * (abs(q) @ abs(k).transpose(0, 2, 1)), 0.0).max(-1, initial=0.0)
            with np.errstate(invalid="ignore", divide="ignore"):
                top = z.max(-1, initial=-np.inf)
                p = np.where(seen, np.exp(z - np.where(np.isneginf(top), 0.0, top)[..., None]), 0.0)
                total = p.sum(-1)
                d = np.where(total == 0, 1.0, total)[..., None]
                if np.isnan(v).any():                                              # an invisible token's values do not count
                    bad = np.isnan(v)
                    o = p @ np.where(bad, 0.0, v) / d
                    o[(seen.astype(float) @ bad.astype(float)) > 0] = np.nan
                    S = p @ np.where(bad, 0.0, abs(v)) / d
                else:
                    o, S = p @ v / d, p @ abs(v) / d
                want_lse = np.where(total == 0, -np.inf, top + np.log(total))
            e = 2 * (self.D + 8) * 2.0 ** -24 * size
            a = (n + 64) * 2.0 ** -24
            tol = (2 * e[..., None] + p_err + a) * S + u * abs(o)
            shape = lambda x: x.reshape((self.H, m, self.G) + x.shape[2:]).swapaxes(0, 1).reshape((m, self.H * self.G) + x.shape[2:])
            o, tol, want_lse, lse_tol = (shape(x) for x in (o, tol, want_lse, e + a + abs(np.where(np.isfinite(want_lse), want_lse, 0)) * 2.0 ** -22))
            g, gl = got[rows], got_lse[rows]
            assert (np.isnan(g) == np.isnan(o)).all() and (np.isnan(gl) == np.isnan(want_lse)).all()
            ok = ~np.isnan(o)
            assert (abs(g - o)[ok] <= tol[ok]).all(), (s, (abs(g - o) / tol)[ok].max())
            fine = np.isfinite(want_lse)
            assert (gl[~fine & ~np.isnan(want_lse)] == -np.inf).all()
            off = abs(gl[fine] - want_lse[fine]) / lse_tol[fine]
            assert (off <= 1).all(), (s, off.max())


ODD = [1, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129, 255, 257, 600]


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("D,T,H,G", [(64, 16, 2, 1), (128, 16, 2, 4), (128, 64, 1, 8), (256, 32, 1, 16), (64, 256, 3, 7), (128, 32, 1, 20), (256, 128, 2, 17)])
def test_attention_one_query_each(out, fmt, D, T, H, G):
    b = Batch(fmt, T, H, G, D, ODD, [1] * len(ODD), seed=D + G)
    b.check(*b.call(out_dtype=out))


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("G", [3, 20])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_every_launch_of_few_rows(out, fmt, G, D):
    """Up to 16 and up to 32 rows of a head; whole sequences by a workgroup, with a compute unit to itself and not, and shares of them."""
    for kv in ([100, 300], [2200, 40], [50] * 130):
        b = Batch(fmt, 32, 2, G, D, kv, [1] * len(kv), seed=G)
        b.check(*b.call(out_dtype=out))


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("D,T,H,G", [(64, 32, 2, 3), (128, 16, 1, 4), (256, 16, 1, 2), (128, 128, 2, 1)])
@pytest.mark.parametrize("window", [0, 40])
def test_attention_ragged_queries(out, fmt, D, T, H, G, window):
    """A few queries (one workgroup's rows), many, none, and more queries than tokens: the first of them see nothing."""
    for kv, nq in (([5, 40, 0, 333, 64], [5, 3, 2, 8, 0]), ([300, 130, 7, 64, 1], [300, 41, 20, 64, 1]), ([70], [130])):
        b = Batch(fmt, T, H, G, D, kv, nq, seed=window + G)
        b.check(*b.call(out_dtype=out, window=window), window=window)


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_both_launches_of_many_rows(out, fmt, D):
    """Many rows behind long contexts, dealt out in shares; the same tokens without their contexts, whole tiles of rows."""
    b = Batch(fmt, 64, 2, 2, D, [2600, 1300], [70, 45], seed=31)
    assert mxp.attention_workspace_bytes(2, 115, 70, 2600, 4, 2, D) > 0
    b.check(*b.call(out_dtype=out))
    b = Batch(fmt, 64, 2, 2, D, [70, 45], [70, 45], seed=32)
    assert mxp.attention_workspace_bytes(2, 115, 70, 70, 4, 2, D) == 0
    b.check(*b.call(out_dtype=out))


@gpu
@pytest.mark.parametrize("nq", [[1, 1], [6, 40]])
def test_attention_not_causal_and_other_scales(nq):
    b = Batch("MXFP4P", 16, 2, 4, 128, [77, 200], nq, seed=3)
    b.check(*b.call(causal=False, scale=0.3, out_dtype=torch.float32), causal=False, scale=0.3)
    b.check(*b.call(scale=-0.2), scale=-0.2)
    b.check(*b.call(scale=0.0), scale=0.0)


@gpu
@pytest.mark.parametrize("G,n", [(1, 1), (4, 2), (4, 50)])
def test_attention_splits_long_sequences(G, n):
    """Long sequences next to short and empty ones: parts without a visible token among them."""
    kv = [5000, 3, 0, 777, 2049]
    b = Batch("MXFP4P", 64, 2, G, 128, kv, [n, n, 1, n, n], seed=n)
    rows = int(b.start[-1])
    assert mxp.attention_workspace_bytes(5, rows, n, 5000, 2 * G, 2, 128) > 0
    out, lse = b.call(out_dtype=torch.float32)
    b.check(out, lse)
    again = b.call(out_dtype=torch.float32)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])              # no order that changes
    b.check(*b.call(window=300), window=300)


@gpu
@pytest.mark.parametrize("n", [1, 4, 60])
def test_attention_bounds_are_hints(n):
    """Bounds below the true sizes change the launch, not the result; bounds far above them neither."""
    b = Batch("MXFP4", 16, 1, 4, 64, [700, 90], [n, n], seed=9)
    for max_q, max_kv in ((1, 1), (n, 100), (1, 700), (5000, 1 << 20), (0, 0)):
        b.check(*b.call(max_q=max_q, max_kv=max_kv, out_dtype=torch.float32))


@gpu
def test_attention_a_prompt_among_single_queries():
    """One long prompt, many sequences of one query, bounds for the longest, an empty sequence between."""
    kv, nq = [1500] + [1 + 37 * i for i in range(60)] + [0, 3000], [1500] + [1] * 61 + [5]
    b = Batch("MXFP4P", 64, 2, 4, 64, kv, nq, seed=21)
    for out in (torch.bfloat16, torch.float32):
        b.check(*b.call(out_dtype=out))
        b.check(*b.call(out_dtype=out, window=100), window=100)
    b.check(*b.call(causal=False), causal=False)


@gpu
def test_attention_many_sequences():
    """More sequences than the lanes that add up their lengths, each of its own length, some without queries."""
    rng = np.random.default_rng(2)
    kv = [int(x) for x in rng.integers(0, 90, 1500)]
    kv[700] = 4000
    b = Batch("MXFP4", 16, 1, 2, 64, kv, [1] * 1500, seed=22)
    b.check(*b.call())
    nq = [int(x) for x in rng.integers(0, 3, 1500)]
    b = Batch("MXFP4", 16, 1, 2, 64, kv, nq, seed=23)
    b.check(*b.call(max_kv=4000, out_dtype=torch.float32))


@gpu
@pytest.mark.parametrize("n", [1, 3, 70])
def test_attention_pages_that_are_not_there(n):
    """Entries outside the cache hide their tokens; the last page's tokens behind kv_len hold NaN blocks throughout."""
    b = Batch("MXFP4P", 16, 2, 2, 128, [200, 95, 33], [n] * 3, seed=4)
    gone = {0: [0, 3, 12], 1: [1], 2: [0, 1, 2]}
    for s, pages in gone.items():
        b.table[s, pages] = [-1, b.n_pages, 2 ** 31 - 1][s]
    hide = lambda s: [t for t in range(b.kv[s]) if t // 16 in gone[s]]
    for out in (torch.bfloat16, torch.float32):
        o, lse = b.call(out_dtype=out)
        b.check(o, lse, hidden=hide)
        if n <= 33:
            assert (o[2 * n:] == 0).all() and (lse[2 * n:] == -float("inf")).all()


@gpu
@pytest.mark.parametrize("G,n", [(2, 1), (2, 6), (4, 90)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_nan_blocks_count_where_they_are_seen(G, n, D):
    """NaN blocks of keys and values in the last tokens: the queries before them are not touched."""
    b = Batch("MXFP4P", 16, 2, G, D, [150, 95], [n, n], seed=6)
    b.poison(0, 150 - (n + 1) // 2, [1], 1)
    b.poison(0, 149, [0], 1)
    b.poison(1, 94, [D // 32 - 1], 0)
    o, lse = b.call(out_dtype=torch.float32)
    b.check(o, lse)
    if n > 1:
        assert not o[0].isnan().any() and not o[n].isnan().any()


@gpu
@pytest.mark.parametrize("kv,n", [(3000, 1), (20000, 1), (3000, 40), (5000, 40)])
def test_attention_nan_values_of_no_weight_count_too(kv, n):
    """A NaN block among tokens whose weights are all zero in fp32: no part of a split sequence may be passed over."""
    b = Batch("MXFP4P", 64, 1, 2, 64, [kv], [n], seed=12)
    b.q[..., 0] = 64.0                                        # its product with channel 0 decides
    e, s, i = (x.reshape(b.n_pages * 64, 1, -1) for x in b.q3[0])
    for tokens, x in ((slice(0, kv // 2), -64.0), (slice(kv // 2, kv), 64.0)):
        slots = b.slots[0][tokens]
        rows = np.zeros((len(slots), 64), np.float32)
        rows[:, 0] = x
        for to, q in zip((e, s, i), oracle.quantize(rows, b.f)):
            to[slots, 0] = q.reshape(len(slots), -1)
        b.val[0][slots, 0] = rows
    b.poison(0, 5, [1], 1)
    for out in (torch.bfloat16, torch.float32):
        o, lse = b.call(out_dtype=out)
        assert o[..., 32:].isnan().all() and not o[..., :32].isnan().any() and lse.isfinite().all()
        b.check(o, lse)


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("kv,nq,window", [([150, 33, 77], [1, 1, 1], 40), ([150, 64], [5, 5], 45), ([300, 130], [60, 20], 45), ([5000, 900], [2, 2], 3000),
                                          ([4100], [70], 2500)])
def test_attention_slots_in_front_of_a_window_may_hold_anything(out, fmt, D, kv, nq, window):
    """Slots that nobody sees, before a window and behind the last token, hold bytes that no conversion leaves: scale bytes 253 to 255,
    scales below their delta.  Few and many rows, whole tiles and shares."""
    b = Batch(fmt, 16, 2, 2, D, kv, nq, seed=16)
    if window > 1000:
        assert mxp.attention_workspace_bytes(len(kv), int(b.start[-1]), max(nq), max(kv), 4, 2, D, window=window) > 0
    unseen = np.ones(b.n_pages * 16, bool)
    for n, m, slots in zip(kv, nq, b.slots):
        unseen[slots[max(n - m - window + 1, 0):]] = False
    assert sum(unseen[slots].sum() for slots in b.slots) > 0
    rng = np.random.default_rng(17)
    for e, s, i in (tuple(x.reshape(b.n_pages * 16, 2, -1) for x in q) for q in b.q3):
        for x, values in ((e, range(256)), (s, (1, 2, 253, 254, 255)), (i, range(256))):
            x[unseen] = rng.choice(values, x[unseen].shape)
    b.check(*b.call(out_dtype=out, window=window), window=window)


@gpu
@pytest.mark.parametrize("fmt", FOUR)
@pytest.mark.parametrize("n", [1, 10, 40])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_attention_nan_and_zero_blocks_whatever_their_index_bytes(fmt, n, D):
    """A scale byte of 255 is NaN and one of 0 zeros, in keys and values, also with a position and a delta left in the index byte."""
    b = Batch(fmt, 16, 2, 2, D, [150, 95, 40], [n] * 3, seed=18)
    for seq, t, block, part, index in ((0, 149, 0, 0, 0xE9), (1, 94, D // 32 - 1, 1, 0xE9), (2, 39, 0, 0, 0x29), (2, 38, D // 32 - 1, 1, 0x29)):
        b.poison(seq, t, [block], part)
        b.q3[part][2].reshape(b.n_pages * 16, 2, -1)[b.slots[seq][t], :, block] = index
        if seq == 2:
            b.q3[part][1].reshape(b.n_pages * 16, 2, -1)[b.slots[2][t], :, block] = 0
            b.val[part][b.slots[2][t], :, 32 * block:32 * block + 32] = 0
    o, lse = b.call(out_dtype=torch.float32)
    assert o[n - 1].isnan().all() and lse[n - 1].isnan().all() and not o[2 * n:].isnan().any()
    b.check(o, lse)


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 12, 40])
@pytest.mark.parametrize("period,max_kv", [(128, 1100), (256, 1)])
def test_attention_large_values_behind_a_lagging_maximum(out, D, n, period, max_kv):
    """Values up to 2^117, scores that rise by 2^7 (base 2) without the weights being rescaled: sum p |v| with p <= 1 stays below
    1024 * 2^117, so nothing overflows on the way to a finite result."""
    b = Batch("MXFP4P", 64, 1, 2, D, [1024], [n], seed=19)
    assert (mxp.attention_workspace_bytes(1, n, n, max_kv, 2, 1, D) > 0) == (max_kv > 1)
    b.q.zero_()
    b.q[..., 0] = 4.84375                                     # * 4 * 0.25 * log2(e) = 6.99
    rows = np.zeros((2, 1024, D), np.float32)
    rows[0, np.arange(1024) // period % 2 == 1, 0] = 4.0
    rows[1] = 2.0 ** 116 * (1 + 0.99 * np.random.default_rng(20).random((1024, D)))
    for part in (0, 1):
        q = oracle.quantize(rows[part], b.f)
        for to, x in zip(b.q3[part], q):
            to.reshape(b.n_pages * 64, -1)[b.slots[0]] = x
        b.val[part][b.slots[0], 0] = oracle.dequantize(q, b.f)
    o, lse = b.call(out_dtype=out, scale=0.25, max_kv=max_kv)
    assert o.isfinite().all()
    b.check(o, lse, scale=0.25)


@gpu
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv", [200, 3000])
@pytest.mark.parametrize("n", [1, 12, 40])
def test_attention_scores_beyond_fp32_are_not_taken_for_nothing_seen(out, kv, n):
    """Products of scale and score above 2^128: NaN in O and lse; the rows of zero scores beside them are averages of the values."""
    b = Batch("MXFP4P", 16, 1, 2, 64, [kv], [n], seed=21)
    b.q[:, 0] = 0
    o, lse = b.call(out_dtype=out, scale=2e38)
    assert o[:, 1].isnan().all() and lse[:, 1].isnan().all()
    b.q[:, 1] = 0
    both, both_lse = b.call(out_dtype=out)
    both[:, 0], both_lse[:, 0] = o[:, 0], lse[:, 0]
    b.check(both, both_lse)


@gpu
@pytest.mark.parametrize("T,D,kv,n,max_kv,splits", [
    (16, 64, [9000], 1, 1, False), (16, 128, [9000], 1, 1, False),               # eight wavefronts: 8192 tokens per lookup
    (16, 64, [9000] + [20] * 260, 1, 1, False), (32, 256, [9000], 10, 1, False),  # four: 4096
    (16, 64, [20000], 1, 600, True), (16, 128, [20000], 3, 600, True),           # the same in shares
    (16, 64, [2500], 40, 1, False), (16, 128, [2500, 1100], 40, 1, False), (16, 256, [2500], 20, 1, False),   # many rows: 1024
    (16, 64, [9000], 40, 1100, True), (16, 128, [9000], 40, 1100, True)])
def test_attention_looks_pages_up_again(T, D, kv, n, max_kv, splits):
    """Runs of tokens longer than the page numbers that a wavefront holds at once; a bound on kv_len below the truth makes them so long."""
    H, G = 1, 3 if n == 10 else 2
    b = Batch("MXFP4P", T, H, G, D, kv, [n] * len(kv), seed=24)
    assert (mxp.attention_workspace_bytes(len(kv), n * len(kv), n, max_kv, H * G, H, D) > 0) == splits
    for out in (torch.bfloat16, torch.float32):
        b.check(*b.call(out_dtype=out, max_kv=max_kv))


@gpu
@pytest.mark.parametrize("D,kv,n,least", [(64, 140000, 1, 257), (128, 20000, 1, 65), (256, 20000, 2, 65)])
def test_attention_joins_of_many_parts(D, kv, n, least):
    """One sequence and one key-value head in more than 64 and more than 256 parts."""
    b = Batch("MXFP4P", 64, 1, 4, D, [kv], [n], seed=25)
    # a share leaves room for two parts of 16 rows: D values, maximum and sum; and its record
    assert mxp.attention_workspace_bytes(1, n, n, kv, 4, 1, D) >= least * (2 * 16 * (D + 2) * 4 + 16)
    for out in (torch.bfloat16, torch.float32):
        b.check(*b.call(out_dtype=out))


@gpu
@pytest.mark.parametrize("n", [1, 12, 40])
def test_attention_of_zero_scores_whatever_the_scale(n):
    """Any finite scale is taken, also one whose product with log2(e) is not: 0 times it is 0, and O the average of the values."""
    b = Batch("MXFP4P", 16, 1, 2, 64, [200], [n], seed=26)
    b.q.zero_()
    for scale in (3.4e38, -3.4e38, 1e-45):
        b.check(*b.call(out_dtype=torch.float32, scale=scale))


@gpu
def test_attention_strides_rows_of_no_sequence_and_device_side_lengths():
    """q a slice of a joint projection, out with gaps; rows before the first and behind the last sequence stay as they are."""
    b = Batch("MXFP4P", 32, 2, 3, 64, [50, 120], [4, 30], seed=8)
    joint = torch.full((40, 10, 64), float("nan"), device="cuda").bfloat16()
    joint[3:37, 2:8] = b.q
    for dt in (torch.bfloat16, torch.float32):
        room = torch.full((40, 8, 64), 5.0, dtype=dt, device="cuda")
        lse = torch.full((40, 6), 5.0, device="cuda")
        start = torch.from_numpy(b.start + 3).cuda()
        mxp.attention(joint[:, 2:8], b.cache(), torch.from_numpy(b.table).cuda(), torch.tensor(b.kv, dtype=torch.int32, device="cuda"),
                      q_start=start, max_q=30, max_kv=120, out=room[:, 1:7], lse=lse)
        b.check(room[3:37, 1:7], lse[3:37])
        assert (room[:3] == 5).all() and (room[37:] == 5).all() and (room[:, 0] == 5).all() and (room[:, 7] == 5).all()
        assert (lse[:3] == 5).all() and (lse[37:] == 5).all()
    none = mxp.attention(b.q[:0], b.cache(), torch.from_numpy(b.table).cuda()[:0], torch.empty(0, dtype=torch.int32, device="cuda"))
    assert none.shape == (0, 6, 64)


@gpu
def test_attention_large_scores_and_flushed_blocks():
    """Scores in the hundreds, one key far ahead of all others, blocks of zeros: the running maximum carries them."""
    b = Batch("MXFP4P", 16, 1, 4, 128, [400, 400], [1, 60], seed=11, garbage=False)
    b.q *= 30
    for part in (0, 1):
        sc = b.q3[part][1]
        sc[::7] = 0
        b.q3[part][0].reshape(len(sc), -1, 16)[::7] = 0
        b.q3[part][2][::7] = 0
        b.val[part] = oracle.dequantize(b.q3[part], b.f).reshape(b.val[part].shape)
    for out in (torch.bfloat16, torch.float32):
        b.check(*b.call(out_dtype=out))


# ---- together -------------------------------------------------------------------------------------------------------
def test_refusals_before_anything_is_launched():
    """Status codes of the entry points for what they do not take, on the CPU: nothing is enqueued."""
    import ctypes as C
    L = mxp.lib()
    buf = (C.c_uint8 * 4096)()
    addr = (C.addressof(buf) + 15) & ~15
    p, odd, N = C.c_void_p(addr), C.c_void_p(addr + 2), None
    B, F = mxp.BF16, mxp.F32
    norm = lambda x=p, r=p, dt=B, rows=4, K=64, lx=64, lr=64, w=p, wd=B, eps=1e-6, h=p, lh=64, f=mxp.MXFP8, e=p, s=p, i=p: \
        L.mxp_rmsnorm_quantize(x, r, dt, rows, K, lx, lr, w, wd, eps, h, lh, f, e, s, i, None)
    assert norm(f=7) == -5 and norm(f=-1) == -5 and norm(dt=2) == -4 and norm(wd=2) == -4
    assert norm(K=48) == -2 and norm(rows=-1) == -2 and norm(eps=-1.0) == -2 and norm(eps=float("nan")) == -2 and norm(eps=float("inf")) == -2
    assert norm(lx=32) == -2 and norm(lr=32) == -2 and norm(lh=32) == -2
    assert norm(x=N) == -1 and norm(w=N) == -1 and norm(e=N) == -1 and norm(s=N) == -1 and norm(f=mxp.MXFP8P, i=N) == -1
    assert norm(x=odd) == -3 and norm(r=odd) == -3 and norm(h=odd) == -3 and norm(w=odd) == -3 and norm(lx=68) == -3 and norm(e=odd) == -3
    assert norm(K=(1 << 21) + 32, lx=1 << 22, lr=1 << 22, lh=1 << 22) == -8 and norm(rows=0, x=N) == 0 and norm(K=0, x=N) == 0

    size = lambda n=4, T=16, H=2, D=128, f=1: L.mxp_cache_bytes(n, T, H, D, f)
    assert size() == 4 * 2 * 2 * 16 * 72 and size(f=0) == 4 * 2 * 2 * 16 * 68
    assert [size(n=0), size(T=8), size(T=48), size(T=512), size(H=0), size(D=96), size(D=0), size(f=5), size(f=9)] == [0] * 9
    for call in (lambda k=p, v=p, dt=B, n=3, lk=256, lv=256, sl=p, c=p, pages=4, T=16, H=2, D=128, f=1: L.mxp_cache_write(k, v, dt, n, lk, lv, sl, c, pages, T, H, D, f, None),
                 lambda k=p, v=p, dt=B, n=3, lk=256, lv=256, sl=p, c=p, pages=4, T=16, H=2, D=128, f=1: L.mxp_cache_read(c, pages, T, H, D, f, sl, n, k, v, dt, lk, lv, None)):
        assert call(f=3) == -8 and call(f=8) == -5 and call(T=17) == -8 and call(D=32) == -8 and call(pages=0) == -2 and call(H=0) == -2
        assert call(dt=3) == -4 and call(n=-1) == -2 and call(lk=255) == -2 and call(lv=128) == -2 and call(lk=260) == -3
        assert call(k=N) == -1 and call(v=N) == -1 and call(sl=N) == -1 and call(c=N) == -1 and call(n=0, k=N) == 0
        assert call(k=odd) == -3 and call(c=odd) == -3 and call(sl=odd) == -3

    def attn(Q=p, qd=B, lq=1024, rows=3, heads=8, qs=p, kl=p, tb=p, lt=4, n=2, mq=3, mk=64, scale=0.1, causal=1, win=0, c=p, pages=4, T=16, H=2, D=128, f=1,
             O=p, od=B, lo=1024, lse=p, ws=N, wb=0):
        return L.mxp_attention(Q, qd, lq, rows, heads, qs, kl, tb, lt, n, mq, mk, scale, causal, win, c, pages, T, H, D, f, O, od, lo, lse, ws, wb, None)
    assert attn(f=6) == -8 and attn(f=11) == -5 and attn(D=96) == -8 and attn(T=8) == -8 and attn(pages=0) == -2
    assert attn(qd=5) == -4 and attn(od=5) == -4 and attn(qd=F) == -8
    assert attn(heads=7) == -2 and attn(heads=0) == -2 and attn(rows=-1) == -2 and attn(mq=-1) == -2 and attn(mk=-1) == -2 and attn(win=-1) == -2
    assert attn(causal=0, win=5) == -2 and attn(scale=float("inf")) == -2 and attn(scale=float("nan")) == -2 and attn(lt=-1) == -2
    assert attn(qs=N) == -2                                       # one row per sequence, and three rows for two
    assert attn(lq=1000) == -2 and attn(lo=512) == -2 and attn(lq=1028) == -3 and attn(lo=1028) == -3
    assert [attn(Q=N), attn(kl=N), attn(tb=N), attn(c=N), attn(O=N)] == [-1] * 5
    assert [attn(Q=odd), attn(O=odd), attn(c=odd), attn(qs=odd), attn(kl=odd), attn(tb=odd), attn(lse=odd)] == [-3] * 7
    assert attn(rows=1 << 28) == -8 and attn(rows=1 << 24, n=1 << 24, qs=N, mq=1, heads=2) == -8 and attn(rows=0, Q=N) == 0 and attn(n=0, Q=N) == 0
    need = mxp.attention_workspace_bytes(2, 3, 3, 100000, 8, 2, 128)
    assert need > 0 and attn(mk=100000) == -6 and attn(mk=100000, ws=p, wb=need - 1) == -6
    assert mxp.attention_workspace_bytes(0, 3, 3, 100000, 8, 2, 128) == 0 == mxp.attention_workspace_bytes(2, 3, 3, 100000, 7, 2, 128)


def test_binding_refuses_what_does_not_fit():
    """Tensors elsewhere than on the current GPU, and with no GPU at all: an exception, never another route."""
    x = torch.zeros((4, 64))
    c = mxp.KVCache(torch.zeros((4, 2, 2, 16 * 36), dtype=torch.uint8), 16, 2, 64, mxp.MXFP4P)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)
    for call in (lambda: mxp.rmsnorm_quantize(x, x[0]), lambda: mxp.cache_write(c, x.view(2, 2, 64), x.view(2, 2, 64), torch.zeros(2, dtype=torch.int64)),
                 lambda: mxp.cache_read(c, torch.zeros(2, dtype=torch.int64)),
                 lambda: mxp.attention(torch.zeros((1, 2, 64)).bfloat16(), c, i32(1, 1), i32(1))):
        with pytest.raises(mxp.MxpError, match="current GPU"):
            call()
    with pytest.raises(mxp.MxpError, match="no cache"):
        mxp.cache_empty(4, 24, 2, 64)


@gpu
def test_binding_refuses_shapes_and_types():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    c = mxp.cache_empty(4, 16, 2, 64)
    i32 = lambda *s: z(*s, dt=torch.int32)
    sl = z(3, dt=torch.int64)
    k = z(3, 2, 64)
    bad = [lambda: mxp.rmsnorm_quantize(z(4, 64), z(32)), lambda: mxp.rmsnorm_quantize(z(4, 64), z(64), residual=z(4, 64, dt=torch.float32)),
           lambda: mxp.rmsnorm_quantize(z(4, 64), z(64), residual=z(3, 64)), lambda: mxp.rmsnorm_quantize(z(4, 48), z(48)),
           lambda: mxp.rmsnorm_quantize(z(64, 4).t(), z(64)), lambda: mxp.rmsnorm_quantize(z(4, 64), z(64), eps=-1.0),
           lambda: mxp.cache_write(c, k, k, sl.int()), lambda: mxp.cache_write(c, k, k.float(), sl), lambda: mxp.cache_write(c, k, k[:2], sl),
           lambda: mxp.cache_write(c, z(3, 64, 2).transpose(1, 2), k, sl), lambda: mxp.cache_write(c._replace(page_tokens=32), k, k, sl),
           lambda: mxp.cache_write(c._replace(data=c.data.flatten()), k, k, sl), lambda: mxp.cache_write(c._replace(fmt=mxp.MXFP4), k, k, sl),
           lambda: mxp.cache_read(c, sl[::2]), lambda: mxp.cache_read(c, sl, out=(k, k.float())),
           lambda: mxp.attention(z(1, 4, 128), c, i32(1, 1), i32(1)), lambda: mxp.attention(z(1, 4, 64), c, i32(2, 1), i32(1)),
           lambda: mxp.attention(z(1, 4, 64), c, z(1, 1, dt=torch.int64), i32(1)), lambda: mxp.attention(z(1, 4, 64), c, i32(1, 1), i32(1), q_start=i32(1)),
           lambda: mxp.attention(z(2, 4, 64), c, i32(1, 1), i32(1)), lambda: mxp.attention(z(1, 3, 64), c, i32(1, 1), i32(1)),
           lambda: mxp.attention(z(1, 4, 64, dt=torch.float32), c, i32(1, 1), i32(1)), lambda: mxp.attention(z(1, 4, 64), c, i32(1, 1), i32(1), lse=z(1, 4)),
           lambda: mxp.attention(z(1, 4, 64), c, i32(1, 1), i32(1), causal=False, window=3),
           lambda: mxp.attention(z(1, 4, 64), c, i32(1, 4000), i32(1), workspace=z(16, dt=torch.uint8))]
    for n, call in enumerate(bad):
        with pytest.raises((mxp.MxpError, TypeError)):
            call()
            pytest.fail("call %d was taken" % n)


@gpu
def test_native_calls_are_taken_and_equal_the_general_code(monkeypatch):
    """The binding's native part takes the ordinary calls of each operator, and gives what the general code gives."""
    b = Batch("MXFP4PP", 16, 2, 4, 128, [4000, 33, 100], [1, 1, 1], seed=13)
    r = Batch("MXFP4P", 32, 2, 2, 64, [50, 120], [4, 30], seed=14)
    cb, cr = b.cache(), r.cache()
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, res = (torch.randn((5, 96), generator=gen, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(96, generator=gen, device="cuda")
    k, v = (torch.randn((7, 4, 128), generator=gen, device="cuda")[:, :2] for _ in range(2))
    slots = torch.tensor([3, -1, 40, 7, 100, 9, 31], device="cuda")

    def calls():
        mxp.cache_write(cb, k, v, slots)
        q, h = mxp.rmsnorm_quantize(x, w, mxp.MXFP6P, residual=res)
        q2, x2 = mxp.rmsnorm_quantize(x, w, mxp.MXFP4PP, eps=0.5)
        return [*q, h, *q2, x2, cb.data.clone(), *mxp.cache_read(cb, slots), *mxp.cache_read(cb, slots, torch.float32), *b.call(cb), *b.call(cb, max_kv=None, max_q=None),
                *r.call(cr, out_dtype=torch.float32, window=9), *r.call(cr, causal=False, scale=1)]

    taken = []
    native = mxp._native()

    class Noting:
        def __getattr__(self, name):
            def call(*args):
                out = getattr(native, name)(*args)
                taken.append((name, out is not None))
                return out
            return call

    monkeypatch.setattr(mxp, "_fast", Noting())
    got = calls()
    if not isinstance(native, mxp._NoNative):
        assert len(taken) == 9 and all(ok for _, ok in taken), taken
    monkeypatch.setattr(mxp, "_fast", mxp._NoNative())
    for a, w_ in zip(got, calls()):
        assert a.dtype == w_.dtype and torch.equal(a.view(torch.uint8) if a.dtype == torch.uint8 else a, w_)


class Layer:
    """The attention half of a layer as a serving program runs it: norm, joint projection, cache, attention, next residual."""

    def __init__(self, n_seq=3, H=2, G=2, D=64, T=16, pages=6):
        gen = torch.Generator(device="cuda").manual_seed(0)
        self.H, self.G, self.D, self.T, self.n = H, G, D, T, n_seq
        K = 256
        self.w = (1 + 0.1 * torch.randn(K, generator=gen, device="cuda")).bfloat16()
        self.qw = mxp.quantize((torch.randn(((G + 2) * H * D, K), generator=gen, device="cuda") * 0.06).bfloat16(), mxp.MXFP4P)
        self.cache = mxp.cache_empty(n_seq * pages, T, H, D)
        self.table = torch.randperm(n_seq * pages, generator=gen, device="cuda").to(torch.int32).view(n_seq, pages)
        self.kv_len = torch.zeros(n_seq, dtype=torch.int32, device="cuda")
        self.x, self.r = (torch.randn((n_seq, K), generator=gen, device="cuda").bfloat16() for _ in range(2))
        need = mxp.attention_workspace_bytes(n_seq, n_seq, 1, pages * T, G * H, H, D)
        self.ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def step(self):
        q8, self.h = mxp.rmsnorm_quantize(self.x, self.w, mxp.MXFP8, residual=self.r)
        self.act = q8
        self.qkv = mxp.gemm(q8, mxp.MXFP8, self.qw, mxp.MXFP4P, torch.bfloat16).view(self.n, -1, self.D)
        t = self.kv_len.long()
        slots = self.table.gather(1, (t // self.T)[:, None])[:, 0].long() * self.T + t % self.T
        HG = self.H * self.G
        mxp.cache_write(self.cache, self.qkv[:, HG:HG + self.H], self.qkv[:, HG + self.H:], slots)
        self.kv_len += 1
        self.o = mxp.attention(self.qkv[:, :HG], self.cache, self.table, self.kv_len, max_kv=self.table.shape[1] * self.T, workspace=self.ws)


@gpu
def test_a_layer_step_by_step():
    """Every stage of a decode loop against 64 bits on what the stage before it left."""
    L = Layer()
    kept = [[], []]
    for step in range(20):
        L.x = L.x.roll(step, 1)
        L.step()
        act = mxp.dequantize(L.act, mxp.MXFP8).double().cpu()
        qw = mxp.dequantize(L.qw, mxp.MXFP4P).double().cpu()
        y = (act @ qw.T).view(L.n, -1, L.D)
        got = L.qkv.double().cpu()
        assert ((got - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -15 * (act.abs() @ qw.abs().T).view_as(y)).all()
        HG = L.H * L.G
        for part, rows in ((0, got[:, HG:HG + L.H]), (1, got[:, HG + L.H:])):
            b = np.ascontiguousarray(rows.float().numpy()).reshape(-1, L.D)
            kept[part].append(oracle.dequantize(oracle.quantize(b, oracle.MXFP4P), oracle.MXFP4P).reshape(L.n, L.H, L.D))
        k, v = (np.stack(x, 1).repeat(L.G, 2) for x in kept)                 # [n][t][heads][D]
        q = got[:, :HG].numpy()
        z = np.einsum("nhd,nthd->nht", q, k) * L.D ** -0.5
        p = np.exp(z - z.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        o, S = np.einsum("nht,nthd->nhd", p, v), np.einsum("nht,nthd->nhd", p, abs(v))
        size = np.einsum("nhd,nthd->nht", abs(q), abs(k)).max() * L.D ** -0.5
        tol = (4 * (L.D + 8) * 2.0 ** -24 * size + 2.0 ** -8 + 100 * 2.0 ** -24) * S + 2.0 ** -8 * abs(o)
        assert (abs(L.o.double().cpu().numpy() - o) <= tol).all()


@gpu
@pytest.mark.parametrize("own_stream", [False, True])
def test_a_layer_captured_and_replayed(own_stream):
    """The step in a HIP graph: every replay, with eager work and new inputs in between, against the eager step on a twin."""
    L, E = Layer(), Layer()
    L.step(); E.step()                                            # (first calls set launch attributes)
    L.kv_len.zero_(); E.kv_len.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.step()
    L.kv_len.zero_()
    side = torch.cuda.Stream()
    for step in range(6):
        new = torch.randn(L.x.shape, generator=torch.Generator().manual_seed(step)).bfloat16().cuda()
        L.x.copy_(new); E.x.copy_(new)
        graph.replay()
        if own_stream:                                            # the eager step on a stream of its own
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                E.step()
            torch.cuda.current_stream().wait_stream(side)
        else:
            E.step()
        torch.cuda.synchronize()
        assert torch.equal(L.o, E.o) and torch.equal(L.h, E.h) and torch.equal(L.kv_len, E.kv_len)
        torch.randn(1000, device="cuda").sum().item()


class LongLayer(Layer):
    """A layer with room for thousands of tokens, so that attention is dealt out in shares and joined, and a product behind it."""

    def __init__(self):
        super().__init__(pages=256)
        gen = torch.Generator(device="cuda").manual_seed(1)
        assert mxp.attention_workspace_bytes(self.n, self.n, 1, 256 * self.T, self.G * self.H, self.H, self.D) > 0
        self.qo = mxp.quantize((torch.randn((256, self.G * self.H * self.D), generator=gen, device="cuda") * 0.06).bfloat16(), mxp.MXFP4P)
        self.past = [torch.randn((256 * self.T, self.n * self.H, self.D), generator=gen, device="cuda").bfloat16() for _ in range(2)]

    def begin(self, lengths):
        """Contexts of these lengths, written by an eager prefill; the layer's step then goes on from there."""
        for s, n in enumerate(lengths):
            t = torch.arange(n, device="cuda")
            mxp.cache_write(self.cache, *(p[:n, s * self.H:(s + 1) * self.H] for p in self.past), self.table[s, t // self.T].long() * self.T + t % self.T)
        self.kv_len.copy_(torch.tensor(lengths, dtype=torch.int32))

    def step(self):
        super().step()
        self.y = mxp.gemm(mxp.quantize(self.o.view(self.n, -1), mxp.MXFP8), mxp.MXFP8, self.qo, mxp.MXFP4P, torch.bfloat16)

    def results(self):
        return self.h, self.qkv, self.o, self.y, self.kv_len

    def expected(self):
        """The attention in 64 bits on the cache's tokens, and how far an output may be off: Batch.check's bound for bf16."""
        outs = []
        for s, n in enumerate(self.kv_len.tolist()):
            t = torch.arange(n, device="cuda")
            k, v = (x.double().cpu().numpy().repeat(self.G, 1) for x in mxp.cache_read(self.cache, self.table[s, t // self.T].long() * self.T + t % self.T, torch.float32))
            q = self.qkv[s, :self.H * self.G].double().cpu().numpy()
            z = np.einsum("hd,thd->ht", q, k) * self.D ** -0.5
            p = np.exp(z - z.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            o, S = np.einsum("ht,thd->hd", p, v), np.einsum("ht,thd->hd", p, abs(v))
            size = np.einsum("hd,thd->ht", abs(q), abs(k)).max() * self.D ** -0.5
            outs.append((o, (4 * (self.D + 8) * 2.0 ** -24 * size + 2.0 ** -8 + (n + 64) * 2.0 ** -24) * S + 2.0 ** -8 * abs(o)))
        return (np.stack(x) for x in zip(*outs))


LENGTHS = ([0, 0, 0], [1, 3000, 0], [4000, 4090, 2222], [5, 6, 7], [0, 4095, 130])   # before a step; shares without work among them


@gpu
@pytest.mark.parametrize("own_stream", [False, True])
def test_a_layer_with_split_sequences_captured_and_replayed(own_stream):
    """The parts' workspace and the joins in a HIP graph: replays at lengths set from outside, each against the eager step and 64 bits."""
    L, E = LongLayer(), LongLayer()
    L.step(); E.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.step()
    side = torch.cuda.Stream()
    for turn, lengths in enumerate(LENGTHS * 2):
        new = torch.randn(L.x.shape, generator=torch.Generator().manual_seed(turn)).bfloat16().cuda()
        for layer in (L, E):
            layer.x.copy_(new)
            layer.begin(lengths)
        L.ws.fill_(255)                                       # nothing is kept in the workspace from call to call
        graph.replay()
        if own_stream:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                E.step()
            torch.cuda.current_stream().wait_stream(side)
        else:
            E.step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(L.results(), E.results()))
        o, tol = L.expected()
        assert (abs(L.o.double().cpu().numpy() - o) <= tol).all()


@gpu
def test_two_layers_on_two_streams():
    """Whole layers, attention dealt out in shares, on two streams at once: as one after the other."""
    layers = [LongLayer(), LongLayer()]
    for i, layer in enumerate(layers):
        layer.x.mul_(i + 1)
    want = []
    for lengths in LENGTHS:
        for layer in layers:
            layer.begin(lengths)
            layer.step()
            want.append([x.clone() for x in layer.results()])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    got = [[], []]
    for layer, stream, out in zip(layers, streams, got):
        stream.wait_stream(torch.cuda.current_stream())
    for lengths in LENGTHS:
        for layer, stream, out in zip(layers, streams, got):
            with torch.cuda.stream(stream):
                layer.begin(lengths)
                layer.step()
                out.append([x.clone() for x in layer.results()])
    torch.cuda.synchronize()
    for i in range(2):
        for a, b in zip(got[i], want[i::2]):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


@gpu
def test_two_streams_with_workspaces_of_their_own():
    """Split sequences on two streams at once: each call's parts lie in its own workspace."""
    b = [Batch("MXFP4P", 64, 2, 4, 128, [4000, 900], [1, 1], seed=s) for s in (1, 2)]
    caches = [x.cache() for x in b]
    want = [x.call(c) for x, c in zip(b, caches)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in b]
    for _ in range(5):
        got = []
        for x, c, s in zip(b, caches, streams):
            with torch.cuda.stream(s):
                got.append(x.call(c))
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for gs, ws in zip(got, want) for g, w in zip(gs, ws))
