"""Pages of an 8-bit cache (kf_page_*) against a plain model of them: who holds which page, every code and scale to the bit, a
token's attention against its definition in 64 bits; refusals (no GPU); calls in a row as a server makes them."""
import math

import numpy as np
import pytest
import torch

import paper_2403_09054_amd as kf
from paper_2403_09054_amd import binding

TYPES = {kf.BF16: torch.bfloat16, kf.F16: torch.float16}
U = 2.0 ** -24  # half a step of fp32
P = kf.PAGE_TOKENS


def expect(status, fn, *a, **k):
    with pytest.raises(kf.KeyformerError) as e:
        fn(*a, **k)
    assert e.value.status == status, e.value
    assert len(str(e.value)) > 20


# ---------------------------------------------------------------- refusals (nothing is launched)
def fake(**over):
    kw = dict(K=0x10000, V=0x20000, k_scale=0x30000, v_scale=0x40000, table=0x50000, len=0x60000, refs=0x70000, L=2, B=3, H=4, d=128, pages=100,
              max_pages=20, dtype=kf.BF16)
    kw.update(over)
    return kf.Pages(**kw)


WS = (0x100000, 1 << 40)
CALLS = {
    "reserve": lambda p, ws=WS, n=4: kf.kf_page_reserve(p, n, workspace=ws, stream=0),
    "write": lambda p, ws=WS, k=0x1000, v=0x2000, n=4, rows=0: kf.kf_page_write(p, k, v, n, rows, workspace=ws, stream=0),
    "step": lambda p, ws=WS, q=0x1000, k=0x2000, v=0x3000, out=0x4000, scale=0.1, m_hint=0: kf.kf_page_step(p, q, k, v, scale, out, m_hint, workspace=ws, stream=0),
    "fork": lambda p, ws=WS, parent=0x1000: kf.kf_page_fork(p, parent, workspace=ws, stream=0),
    "free": lambda p, ws=WS: kf.kf_page_free(p, 0x1000, workspace=ws, stream=0),
    "compact": lambda p, ws=WS, keep=0x1000, k=64: kf.kf_page_compact(p, keep, k, workspace=ws, stream=0),
}


@pytest.mark.parametrize("name", CALLS)
def test_page_refusals(name):
    call = CALLS[name]
    for bad in (dict(L=0), dict(B=0), dict(H=0), dict(d=0), dict(pages=0), dict(max_pages=0), dict(q_per_kv=-1), dict(dtype=9), dict(dtype=kf.BF16_Q4), dict(K=None),
                dict(V=None), dict(k_scale=None), dict(v_scale=None), dict(table=None), dict(len=None), dict(refs=None), dict(K=0x10008), dict(V=0x20004),
                dict(max_pages=1 << 25), dict(L=1 << 15, B=1 << 9, H=2)):
        expect(binding.KF_EINVAL, call, fake(**bad))
    for bad in (dict(d=96), dict(d=512), dict(dtype=kf.F32), dict(q_per_kv=3), dict(q_per_kv=16), dict(B=8193)):
        expect(binding.KF_EUNSUPPORTED, call, fake(**bad))
    for bad in (None, (0x100000, 64), (0x100004, 1 << 40)):
        expect(binding.KF_EWORKSPACE, call, fake(), ws=bad)


def test_page_refusals_of_one_call():
    for bad in (dict(n=0), dict(n=-1)):
        expect(binding.KF_EINVAL, CALLS["reserve"], fake(), **bad)
    for bad in (dict(k=None), dict(v=None), dict(k=0x1008), dict(n=0), dict(n=5, rows=4)):
        expect(binding.KF_EINVAL, CALLS["write"], fake(), **bad)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q=0x1004), dict(scale=math.nan), dict(scale=math.inf), dict(m_hint=-1), dict(m_hint=20 * P + 1)):
        expect(binding.KF_EINVAL, CALLS["step"], fake(), **bad)
    expect(binding.KF_EINVAL, CALLS["fork"], fake(), parent=None)
    for bad in (dict(keep=None), dict(k=0), dict(k=20 * P + 1)):
        expect(binding.KF_EINVAL, CALLS["compact"], fake(), **bad)
    expect(binding.KF_EUNSUPPORTED, CALLS["write"], fake(L=1 << 15, B=4, H=64), n=1 << 20)
    expect(binding.KF_EUNSUPPORTED, CALLS["compact"], fake(L=1 << 15, B=4, H=64, max_pages=1 << 20), k=1 << 20)
    assert kf.kf_page_workspace_bytes(fake(d=96)) == 0 < kf.kf_page_workspace_bytes(fake())
    expect(binding.KF_EUNSUPPORTED, kf.new_page_workspace, fake(d=96), device="cpu")


def test_launches_of_2_to_the_32_threads_are_refused():
    """Before any launch of the call: the step's own is smaller than the one that joins its splits, for each head of a unit."""
    units = dict(L=1 << 9, B=1 << 9, H=1 << 6)
    expect(binding.KF_EUNSUPPORTED, CALLS["write"], fake(**units), n=1)
    expect(binding.KF_EUNSUPPORTED, CALLS["compact"], fake(**units), k=64)
    expect(binding.KF_EUNSUPPORTED, CALLS["step"], fake(max_pages=1000, **units))
    expect(binding.KF_EUNSUPPORTED, CALLS["step"], fake(L=80, B=8192, H=8, q_per_kv=8, max_pages=65))
    expect(binding.KF_EUNSUPPORTED, CALLS["write"], fake(L=1, B=1, H=1), n=(1 << 31) - 1)


@pytest.mark.parametrize("L,B,H,G,d,max_pages", [(32, 1, 32, 1, 128, 64), (32, 4, 32, 1, 128, 64), (32, 8, 32, 1, 128, 64), (32, 8, 8, 4, 128, 64),
                                                 (32, 1, 8, 4, 128, 512), (80, 1, 1, 8, 256, 4000), (28, 16, 3, 2, 64, 7), (2000, 1, 2, 1, 64, 300)])
def test_a_workspace_serves_any_number_of_layers(L, B, H, G, d, max_pages):
    """Fewer units take more splits each: the records of a layer can be more than those of all."""
    of = dict(B=B, H=H, q_per_kv=G, d=d, max_pages=max_pages, pages=4096)
    whole = kf.kf_page_workspace_bytes(fake(L=L, **of))
    assert all(whole >= kf.kf_page_workspace_bytes(fake(L=l, **of)) > 0 for l in range(1, L))


# ---------------------------------------------------------------- codes, written apart from any 8-bit type of torch
MAGNITUDE = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])
VALUE = np.concatenate([MAGNITUDE, [math.nan], -MAGNITUDE, [math.nan]])


def exponent(a):
    m, e = math.frexp(a)
    return -117 if a == 0 else min(max(e - 9 if m <= 0.875 else e - 8, -117), 119)


def encode(x, e):
    """float64 array -> codes: the nearest, of two as near the even one; what is not finite 0x7F."""
    bad = ~np.isfinite(x)
    y = np.where(bad, 0.0, np.abs(x)) * 2.0 ** -e
    hi = np.clip(np.searchsorted(MAGNITUDE, y), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = MAGNITUDE[hi] - y, y - MAGNITUDE[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return np.where(bad, 127, c + 128 * np.signbit(np.where(bad, 0.0, x))).astype(np.uint8)


def largest(x):
    return float(np.max(np.abs(x[np.isfinite(x)]), initial=0.0))


def test_codes_of_the_model():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(VALUE)) and np.array_equal(t[~np.isnan(t)], VALUE[~np.isnan(t)])
    x = np.concatenate([np.random.default_rng(0).standard_normal(2000) * 100, VALUE[:126] + np.diff(VALUE[:127]) / 2, [0.0, -0.0, 448.0, -448.0, 2.0 ** -10, 3e-4]])
    assert np.array_equal(encode(x, 0), torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    for a, e in ((448.0, 0), (448.5, 1), (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -117), (1e-40, -117), (3.4e38, 120 - 1), (2.0 ** -9, -17)):
        assert exponent(a) == e


class Model:
    """The pages as lists and arrays on the host."""

    def __init__(self, L, B, H, d, pages, max_pages):
        self.of = (L, B, H, d, pages, max_pages)
        self.K, self.V = np.zeros((L, pages, H, P, d), np.uint8), np.zeros((L, pages, H, d, P), np.uint8)
        self.ks, self.vs = np.ones((L, pages, H), np.float32), np.ones((L, pages, H), np.float32)
        self.rows, self.len, self.refs, self.errors = [[] for _ in range(B)], [0] * B, [0] * pages, 0

    def take(self, k):
        free = [p for p, r in enumerate(self.refs) if r == 0][:k]
        if len(free) < k:
            return None
        for p in free:
            self.refs[p] = 1
        return free

    def drop(self, b):
        for p in self.rows[b]:
            self.refs[p] -= 1
        self.rows[b], self.len[b] = [], 0

    def reserve(self, n, counts=None):
        for b, add in enumerate(counts or [n] * len(self.len)):
            if not 1 <= add <= n:
                continue
            k = -(-(self.len[b] + add) // P)
            got = self.take(k - len(self.rows[b])) if k <= self.of[5] else None
            if got is None:
                self.errors += 1
                continue
            self.rows[b] += got
            self.len[b] += add

    def put(self, x, scale, page, rows, slots):
        """x[l, page, h, slot] <- rows [H, slots, d], for all layers' [L, H, slots, d]."""
        L, _, H, _, _, _ = self.of
        for l in range(L):
            for h in range(H):
                new, s0 = rows[l, h], slots[0]
                e = exponent(largest(new))
                if s0 > 0:
                    was = int(math.log2(scale[l, page, h]))
                    e = max(e, was)
                    if e > was:
                        x[l, page, h, :s0] = encode(VALUE[x[l, page, h, :s0]], e - was)
                x[l, page, h, s0:slots[1]] = encode(new, e)
                scale[l, page, h] = 2.0 ** e

    def write(self, k, v, counts):
        """k, v [L, B, H, rows, d] float64"""
        for b, add in enumerate(counts):
            first = self.len[b] - add
            for j in range(first // P, -(-self.len[b] // P)):
                a, e = max(first, j * P), min(self.len[b], j * P + P)
                for x, scale, rows in ((self.K, self.ks, k), (self.V.transpose(0, 1, 2, 4, 3), self.vs, v)):
                    self.put(x, scale, self.rows[b][j], rows[:, b, :, a - first:e - first], (a - j * P, e - j * P))

    def held(self, l, b, h):
        """Keys and values of a unit as they stand, [len, d] float64"""
        K = [VALUE[self.K[l, p, h]] * float(self.ks[l, p, h]) for p in self.rows[b]]
        V = [VALUE[self.V[l, p, h].T] * float(self.vs[l, p, h]) for p in self.rows[b]]
        return (np.concatenate(x)[:self.len[b]] if x else np.zeros((0, self.of[3])) for x in (K, V))

    def fork(self, parent):
        B = self.of[1]
        go = [b for b in range(B) if parent[b] != b]
        for b in list(go):
            if not 0 <= parent[b] < B or parent[parent[b]] != parent[b]:
                self.errors += 1
                go.remove(b)
        for b in go:
            self.drop(b)
        for b in go:
            full = self.len[parent[b]] // P
            self.rows[b] = self.rows[parent[b]][:full]
            for p in self.rows[b]:
                self.refs[p] += 1
        for b in go:
            n = self.len[parent[b]]
            if n % P:
                got = self.take(1)
                if got is None:
                    self.errors += 1
                    self.drop(b)
                    continue
                src = self.rows[parent[b]][n // P]
                for x in (self.K, self.V, self.ks, self.vs):
                    x[:, got[0]] = x[:, src]
                self.rows[b] = self.rows[b] + got
            self.len[b] = n

    def free(self, which):
        for b, w in enumerate(which):
            if w:
                self.drop(b)

    def compact(self, keep, k, which):
        """keep [L, B, H, k]"""
        L, B, H, d, _, _ = self.of
        got = {}
        for b in range(B):
            if which[b] and self.len[b] > k:
                got[b] = self.take(-(-k // P))
                if got[b] is None:
                    self.errors += 1
                    del got[b]
        for b, pages in got.items():
            for l in range(L):
                for h in range(H):
                    for x, scale, rows in zip((self.K, self.V.transpose(0, 1, 2, 4, 3)), (self.ks, self.vs), self.held(l, b, h)):
                        for j, p in enumerate(pages):
                            mine = keep[l, b, h, j * P:j * P + P]
                            there = (mine >= 0) & (mine < self.len[b])
                            self.errors += int((~there).sum()) if x is self.K else 0
                            new = np.where(there[:, None], rows[np.where(there, mine, 0)], 0.0)
                            e = exponent(largest(new))
                            x[l, p, h, :len(mine)] = encode(new, e)
                            scale[l, p, h] = 2.0 ** e
        for b, pages in got.items():
            self.drop(b)
            self.rows[b], self.len[b] = pages, k

    def same(self, c, ws, what):
        torch.cuda.synchronize()
        B, max_pages = self.of[1], self.of[5]
        assert c.len.tolist() == self.len, what
        assert c.table.tolist() == [r + [-1] * (max_pages - len(r)) for r in self.rows], what
        assert c.refs.tolist() == self.refs, what
        assert np.array_equal(c.k_scale.cpu().numpy(), self.ks) and np.array_equal(c.v_scale.cpu().numpy(), self.vs), what
        for name, got, want in (("K", c.K, self.K), ("V", c.V, self.V)):
            bad = np.argwhere(got.cpu().numpy() != want)
            if len(bad):
                pytest.fail("%s: %s differs at %d places, first %s: %s, not %s" % (what, name, len(bad), bad[:4].tolist(), got.cpu().numpy()[tuple(bad[0])], want[tuple(bad[0])]))
        assert int(ws[:4].view(torch.int32)) == self.errors, what


def both(L, B, H, d, pages, max_pages, dtype=kf.BF16, G=1):
    c = kf.Pages.allocate(L, B, H, d, pages, max_pages, dtype, q_per_kv=G)
    return c, kf.new_page_workspace(c), Model(L, B, H, d, pages, max_pages)


def rows_of(g, L, B, H, n, d, dtype, spread=3.0):
    """Rows whose sizes differ, so that scales grow on the way."""
    x = torch.randn((L, B, H, n, d), generator=g) * torch.exp2(spread * torch.randn((L, B, H, n, 1), generator=g))
    return x.to(TYPES[dtype])


def grow(c, ws, m, g, n, counts=None, spread=3.0):
    L, B, H, d, _, _ = m.of
    x = [rows_of(g, L, B, H, n, d, c.dtype, spread) for _ in range(2)]
    dev = None if counts is None else torch.tensor(counts, dtype=torch.int32).cuda()
    kf.kf_page_reserve(c, n, dev, workspace=ws)
    kf.kf_page_write(c, x[0].cuda(), x[1].cuda(), n, seq_n=dev, workspace=ws)
    m.reserve(n, counts)
    m.write(x[0].double().numpy(), x[1].double().numpy(), [a if 1 <= a <= n else 0 for a in counts or [n] * B])


# ---------------------------------------------------------------- rows in
@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(64, kf.BF16), (128, kf.F16), (256, kf.BF16)])
def test_rows_are_held_to_the_bit(d, dtype):
    L, B, H = 2, 4, 3
    c, ws, m = both(L, B, H, d, 60, 8, dtype)
    g = torch.Generator().manual_seed(d)
    c.K.fill_(0x7F), c.V.fill_(0x7F)  # pages hold anything before
    m.K[:], m.V[:] = 0x7F, 0x7F
    for n, counts in ((1, None), (62, None), (1, [1, 0, 1, 5]), (2, None), (64, [64, 1, 63, 3]), (100, [7, 100, 0, 65]), (130, [0, -3, 129, 130])):
        grow(c, ws, m, g, n, counts)
        m.same(c, ws, (n, counts))


@pytest.mark.gpu
def test_rows_of_any_values_and_a_stage_with_room_behind():
    """Zeros, the smallest and largest numbers, infinities, NaN; rows of a cache with more rows than the prompt has."""
    for dtype in (kf.BF16, kf.F16):
        L, B, H, d, n, cap = 1, 2, 2, 64, 70, 90
        c, ws, m = both(L, B, H, d, 10, 3, dtype)
        dt, g = TYPES[dtype], torch.Generator().manual_seed(4)
        k = torch.randn((L, B, H, cap, d), generator=g).to(dt)
        v = torch.randn((L, B, H, cap, d), generator=g).to(dt)
        big, tiny = torch.finfo(dt).max, torch.finfo(dt).smallest_normal / 8
        k[0, 0, 0, :64] = 0.0
        k[0, 0, 1, 3], k[0, 0, 1, 9, 7] = big, -big
        k[0, 1, 0, 5, 2], k[0, 1, 0, 6, 1], k[0, 1, 0, 8, 63] = math.inf, -math.inf, math.nan
        k[0, 1, 1] = tiny
        v[0, 0, 0, 2, 2], v[0, 0, 0, 66, 5] = math.nan, math.inf
        v[0, 0, 1, :, ::2] *= 2.0 ** -12
        v[0, 1, 0, :64] = -0.0
        v[0, 1, 1, 64] = math.nan
        v[0, 1, 1, 65:] = math.inf
        k[..., n:, :] = math.nan  # behind the rows
        kf.kf_page_reserve(c, n, workspace=ws)
        kf.kf_page_write(c, k.cuda(), v.cuda(), n, cap, workspace=ws)
        m.reserve(n)
        m.write(k.double().numpy(), v.double().numpy(), [n] * B)
        m.same(c, ws, dtype)


# ---------------------------------------------------------------- who holds which page
@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(4))
def test_calls_in_any_order_leave_the_pages_of_the_model(seed):
    rng, g = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
    L, B, H, d = 2, 9, 2, 64
    c, ws, m = both(L, B, H, d, int(rng.integers(25, 45)), 7)  # too few for everybody
    for i in range(24):
        what = rng.choice(["grow", "grow", "fork", "free", "compact"])
        if what == "grow":
            n = int(rng.choice([1, 3, 64, 65, 150]))
            before = list(m.len)
            counts = [int(x) for x in rng.integers(0, n + 1, B)]
            x = [rows_of(g, L, B, H, n, d, c.dtype) for _ in range(2)]
            dev = torch.tensor(counts, dtype=torch.int32).cuda()
            kf.kf_page_reserve(c, n, dev, workspace=ws)
            m.reserve(n, counts)
            m.same(c, ws, (i, what, counts))
            got = [a - b for a, b in zip(m.len, before)]  # who found room
            kf.kf_page_write(c, x[0].cuda(), x[1].cuda(), n, seq_n=torch.tensor(got, dtype=torch.int32).cuda(), workspace=ws)
            m.write(x[0].double().numpy(), x[1].double().numpy(), got)
        elif what == "fork":
            parent = list(range(B))
            for b in rng.choice(B, 4, replace=False):
                parent[b] = int(rng.integers(-1, B + 1))
            kf.kf_page_fork(c, torch.tensor(parent, dtype=torch.int32).cuda(), workspace=ws)
            m.fork(parent)
        elif what == "free":
            which = [int(x) for x in rng.random(B) < 0.25]
            kf.kf_page_free(c, torch.tensor(which, dtype=torch.int32).cuda(), workspace=ws)
            m.free(which)
        else:
            k = int(rng.choice([1, 40, 64, 100, 128]))
            which = [int(x) for x in rng.random(B) < 0.5]
            keep = np.full((L, B, H, k), -1, np.int32)
            for b in range(B):
                if m.len[b] > k:
                    for l in range(L):
                        for h in range(H):
                            keep[l, b, h] = np.sort(rng.choice(m.len[b], k, replace=False))
            kf.kf_page_compact(c, torch.from_numpy(keep).cuda(), k, torch.tensor(which, dtype=torch.int32).cuda(), workspace=ws)
            m.compact(keep, k, which)
        m.same(c, ws, (i, what))
    kf.kf_page_free(c, None, workspace=ws)
    m.free([1] * B)
    m.same(c, ws, "all")
    assert m.refs == [0] * m.of[4]


@pytest.mark.gpu
def test_kept_tokens_in_any_order_twice_and_none_such():
    L, B, H, d = 1, 2, 2, 128
    c, ws, m = both(L, B, H, d, 20, 5, kf.F16)
    g = torch.Generator().manual_seed(1)
    grow(c, ws, m, g, 200)
    # what is no number stays none, and does not ask for a scale
    page = m.rows[0][1]
    c.K[0, page, 1, 3, 7], c.V[0, page, 0, 11, 5], c.V[0, page, 0, 12, 5] = 0xFF, 0x7F, 0xFF
    m.K[0, page, 1, 3, 7], m.V[0, page, 0, 11, 5], m.V[0, page, 0, 12, 5] = 0xFF, 0x7F, 0xFF
    k = 70
    keep = np.random.default_rng(0).integers(0, 200, (L, B, H, k)).astype(np.int32)
    keep[0, 0, 1, 0], keep[0, 0, 0, 1], keep[0, 0, 0, 2] = 67, 69, 69
    keep[0, 1, 0, 3], keep[0, 1, 1, 69] = -1, 200
    kf.kf_page_compact(c, torch.from_numpy(keep).cuda(), k, workspace=ws)
    m.compact(keep, k, [1, 1])
    m.same(c, ws, "kept")
    kf.kf_page_compact(c, torch.from_numpy(keep).cuda(), k, workspace=ws)  # no more tokens than that: as they are
    m.same(c, ws, "again")


@pytest.mark.gpu
def test_tables_that_are_none_and_rows_without_room():
    L, B, H, d = 1, 4, 2, 64
    c, ws, m = both(L, B, H, d, 12, 3)
    g = torch.Generator().manual_seed(2)
    grow(c, ws, m, g, 70)
    c.table[1, 0] = 99          # no such page
    c.len[2] = 3 * P + 1        # more than a row of the table has room for
    kf.kf_page_fork(c, torch.tensor([0, 1, 2, 1], dtype=torch.int32).cuda(), workspace=ws)
    assert c.len.tolist() == [70, 70, 3 * P + 1, 0] and int(ws[:4].view(torch.int32)) == 1 and c.table[3].tolist() == [-1] * 3
    kf.kf_page_fork(c, torch.tensor([2, 1, 2, 3], dtype=torch.int32).cuda(), workspace=ws)
    assert c.len.tolist() == [70, 70, 3 * P + 1, 0] and int(ws[:4].view(torch.int32)) == 2
    kf.kf_page_reserve(c, 1, workspace=ws)
    assert c.len.tolist() == [71, 71, 3 * P + 1, 1] and int(ws[:4].view(torch.int32)) == 3
    keep = torch.zeros((L, B, H, 5), dtype=torch.int32, device="cuda")
    kf.kf_page_compact(c, keep, 5, torch.tensor([0, 1, 1, 0], dtype=torch.int32).cuda(), workspace=ws)
    assert c.len.tolist() == [71, 71, 3 * P + 1, 1] and int(ws[:4].view(torch.int32)) == 5
    x = torch.randn((L, B, H, 80, d)).bfloat16().cuda()
    K = c.K.clone()
    kf.kf_page_write(c, x, x, 80, workspace=ws)  # no row has so many tokens: each unit left out and counted
    assert torch.equal(K, c.K) and int(ws[:4].view(torch.int32)) == 5 + B * H
    for n in (0, 65):  # a page number that is none, of a page that is written
        kf.kf_page_write(c, x, x, 66, 80, seq_n=torch.tensor([0, n, 0, 0], dtype=torch.int32).cuda(), workspace=ws)
    assert int(ws[:4].view(torch.int32)) == 5 + B * H + H
    kf.kf_page_free(c, None, workspace=ws)
    assert c.len.tolist() == [0] * B and bool((c.table == -1).all()) and int(ws[:4].view(torch.int32)) == 6 + B * H + H


# ---------------------------------------------------------------- a token's step
@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(kf.BF16, 128), (kf.F16, 64)])
def test_a_page_that_several_hold_is_not_written(dtype, d):
    """A reservation that found no page, and rows written all the same: the last full page is the other sequence's too."""
    L, B, H = 2, 3, 2
    c, ws, m = both(L, B, H, d, 3, 3, dtype)
    g = torch.Generator().manual_seed(8)
    grow(c, ws, m, g, P, [P, 0, P])
    for x in (c, m):
        kf.kf_page_fork(x, torch.tensor([0, 0, 2], dtype=torch.int32).cuda(), workspace=ws) if x is c else x.fork([0, 0, 2])
    grow(c, ws, m, g, 40, [0, 0, 40])  # no page is free now
    kf.kf_page_reserve(c, 1, torch.tensor([1, 1, 0], dtype=torch.int32).cuda(), workspace=ws)
    m.reserve(1, [1, 1, 0])
    m.same(c, ws, "nothing reserved")
    q, k, v = (rows_of(g, L, B, H, 1, d, dtype).cuda() for _ in range(3))
    on = torch.tensor([1, 1, 0], dtype=torch.int32).cuda()
    out = torch.zeros((L, B, H, d), device="cuda")
    kf.kf_page_step(c, q, k, v, 0.1, out, seq_n=on, workspace=ws)
    m.errors += L * 2 * H
    m.same(c, ws, "step")
    kf.kf_page_write(c, k, v, 1, seq_n=on, workspace=ws)
    m.errors += L * 2 * H
    m.same(c, ws, "write")


@pytest.mark.gpu
def test_a_page_number_that_is_none_beside_a_scale_that_is_no_number():
    """The tokens of a page that there is not are left out; what page 0 holds does not come in their place."""
    c, ws, m = both(1, 1, 1, 64, 4, 3)
    g = torch.Generator().manual_seed(9)
    fill(c, ws, m, g, [150])
    c.table[0] = torch.tensor([1, 77, 2])
    for x in (c.K, c.V):
        x[:, 1:3] = x[:, [0, 2]].clone()
        x[:, 0] = 0x7F
    for x in (c.k_scale, c.v_scale):
        x[:, 1:3] = x[:, [0, 2]].clone()
        x[:, 0] = math.nan
    q, k, v = (torch.randn((1, 1, 1, 64), generator=g).bfloat16() for _ in range(3))
    out = torch.zeros((1, 1, 1, 64), device="cuda")
    kf.kf_page_step(c, q.cuda(), k.cuda(), v.cuda(), 0.125, out, workspace=ws)
    K, V = m.held(0, 0, 0)
    at = [j for j in range(149) if j // P != 1]
    want, tol = step_oracle(K[at], V[at], *(x[0, 0, 0].double().numpy() for x in (q, k, v)), 0.125, 0.0)
    assert (np.abs(out[0, 0, 0].double().cpu().numpy() - want) <= tol).all()


def step_oracle(K, V, q, kn, vn, scale, slope):
    """One head: held rows [m, d], the token's own -> its output and how far it may be off: d U of a logit's magnitudes and 6 U of its own size, 2^-21 of
    the exponential, 2^-20 for the two halves of 11 bits that a probability is held in (2^-34 of the largest where they become subnormal), the sums."""
    K, V = np.concatenate([K, kn[None]]), np.concatenate([V, vn[None]])
    gap = np.arange(len(K) - 1, -1, -1.0)
    x = K @ q * scale - slope * gap
    w = np.exp(x - x.max())
    p = w / w.sum()
    e = (np.abs(K) @ np.abs(q) * abs(scale) * len(q) * U + 6 * U * (np.abs(x) + slope * gap)).max()
    out, size = p @ V, p @ np.abs(V)
    return out, size * (2 * e + 2.0 ** -21 + 2.0 ** -20 + (len(K) + 80) * U) + 2.0 ** -34 * np.abs(V).sum(0) + 2 * U * np.abs(out) + 1e-38


STEPS = [  # L, B, H, G, d, dtype, alibi, lengths before, m_hint
    (1, 1, 1, 1, 64, kf.BF16, False, [0], 0),
    (1, 3, 2, 4, 128, kf.BF16, False, [1, 63, 64], 65),
    (2, 2, 2, 8, 256, kf.F16, True, [65, 127], 0),
    (1, 4, 3, 2, 64, kf.F16, True, [0, 200, 128, 191], 201),
    (1, 2, 1, 1, 128, kf.F16, False, [1500, 31], 1501),
    (2, 1, 4, 8, 128, kf.BF16, True, [700], 0),
    (1, 2, 2, 1, 256, kf.BF16, False, [640, 300], 100),   # a hint below the length shapes the launch, no more
    (1, 40, 32, 1, 64, kf.BF16, False, [70 + i for i in range(40)], 128),
]


def fill(c, ws, m, g, lens, spread=0.0):
    if max(lens):
        grow(c, ws, m, g, max(lens), lens, spread)


def take_step(c, ws, m, g, slopes=None, m_hint=0, seq=None, scale=None):
    """A step on both sides, compared."""
    L, B, H, d, _, _ = m.of
    G, dt = c.q_per_kv, TYPES[c.dtype]
    scale = d ** -0.5 if scale is None else scale
    q, k, v = (torch.randn((L, B, h, d), generator=g).to(dt) for h in (H * G, H, H))
    on = [1] * B if seq is None else [int(x == 1) for x in seq]
    dev = None if seq is None else torch.tensor(seq, dtype=torch.int32).cuda()
    kf.kf_page_reserve(c, 1, dev, workspace=ws)
    out = torch.full((L, B, H * G, d), 7.0, device="cuda")
    kf.kf_page_step(c, q.cuda(), k.cuda(), v.cuda(), scale, out, m_hint, None if slopes is None else slopes.cuda(), dev, workspace=ws)
    got = out.double().cpu().numpy()
    q, k, v = (x.double().numpy() for x in (q, k, v))
    for b in range(B):
        for l in range(L):
            for h in range(H):
                K, V = m.held(l, b, h)
                for i in range(h * G, h * G + G):
                    if not on[b]:
                        assert not got[l, b, i].any()
                        continue
                    want, tol = step_oracle(K, V, q[l, b, i], k[l, b, h], v[l, b, h], scale, 0.0 if slopes is None else float(slopes[i]))
                    err = np.abs(got[l, b, i] - want)
                    assert (err <= tol).all(), (l, b, i, m.len[b], float((err - tol).max()), float(err.max()))
    m.reserve(1, on)
    m.write(k[:, :, :, None], v[:, :, :, None], on)


@pytest.mark.gpu
@pytest.mark.parametrize("case", STEPS, ids=lambda c: "x".join(map(str, c[:5])))
def test_steps_match_the_definition(case):
    L, B, H, G, d, dtype, alibi, lens, m_hint = case
    pages = sum(-(-(n + 5) // P) for n in lens) + 1
    c, ws, m = both(L, B, H, d, pages, -(-(max(lens) + 5) // P), dtype, G)
    c.K.fill_(0x7F), c.V.fill_(0x7F)  # what no token holds is no number
    m.K[:], m.V[:] = 0x7F, 0x7F
    g = torch.Generator().manual_seed(len(lens) + d)
    fill(c, ws, m, g, lens)
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / (H * G)) for h in range(H * G)]) if alibi else None
    for _ in range(2 if B > 10 else 4):
        take_step(c, ws, m, g, slopes, m_hint)
        m.same(c, ws, case)


@pytest.mark.gpu
def test_steps_of_some_sequences_and_scales_that_grow():
    L, B, H, d = 1, 4, 2, 128
    c, ws, m = both(L, B, H, d, 30, 6, kf.BF16, 2)
    g = torch.Generator().manual_seed(3)
    fill(c, ws, m, g, [62, 5, 130, 191], 2.0)
    for seq in ([1, 1, 1, 1], [1, 0, 1, 2], [0, 1, -1, 1], [1, 1, 0, 0]):
        take_step(c, ws, m, g, seq=seq)
        m.same(c, ws, seq)
    # a token far larger than its page's, then one far smaller
    for size in (300.0, 2.0 ** -20, 1e30):
        k = torch.randn((L, B, H, d), generator=g).bfloat16() * size
        out = torch.zeros((L, B, 2 * H, d), device="cuda")
        kf.kf_page_reserve(c, 1, workspace=ws)
        kf.kf_page_step(c, torch.zeros((L, B, 2 * H, d), dtype=torch.bfloat16, device="cuda"), k.cuda(), k.cuda(), 0.1, out, workspace=ws)
        m.reserve(1)
        m.write(k.double().numpy()[:, :, :, None], k.double().numpy()[:, :, :, None], [1] * B)
        m.same(c, ws, size)


@pytest.mark.gpu
def test_steps_without_a_token_and_pages_that_are_none():
    L, B, H, d = 1, 3, 2, 64
    c, ws, m = both(L, B, H, d, 10, 3)
    g = torch.Generator().manual_seed(5)
    fill(c, ws, m, g, [130, 0, 100])
    q, k, v = (torch.randn((L, B, H, d), generator=g).bfloat16() for _ in range(3))
    c.len[2] = 3 * P + 1
    c.table[0, 1] = -5
    out = torch.full((L, B, H, d), 7.0, device="cuda")
    kf.kf_page_step(c, q.cuda(), k.cuda(), v.cuda(), 0.125, out, workspace=ws)
    torch.cuda.synchronize()
    assert not bool(out[0, 1:].any())
    assert int(ws[:4].view(torch.int32)) == 2 * H + H  # units without a token or with too many, and a page of each head
    for h in range(H):  # the second page's tokens are left out
        K, V = m.held(0, 0, h)
        at = [j for j in range(129) if j // P != 1]
        want, tol = step_oracle(K[at], V[at], *(x[0, 0, h].double().numpy() for x in (q, k, v)), 0.125, 0.0)
        assert (np.abs(out[0, 0, h].double().cpu().numpy() - want) <= tol).all()


@pytest.mark.gpu
def test_infinite_logits_and_numbers_that_are_none():
    L, B, H, d = 1, 2, 1, 64
    c, ws, m = both(L, B, H, d, 6, 2)
    g = torch.Generator().manual_seed(6)
    fill(c, ws, m, g, [100, 100])
    q, k, v = (torch.ones((L, B, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    k[0, 0, 0, 0] = -math.inf   # the token itself takes no part
    c.V[0, c.table[1, 0].item(), 0, 5, 7] = 0x7F
    kf.kf_page_reserve(c, 1, workspace=ws)
    out = torch.zeros((L, B, H, d), device="cuda")
    kf.kf_page_step(c, q, k, v, 0.125, out, workspace=ws)
    K, V = m.held(0, 0, 0)
    w = np.exp(K.sum(1) * 0.125 - (K.sum(1) * 0.125).max())
    want = w @ V / w.sum()
    assert np.abs(out[0, 0, 0].double().cpu().numpy() - want).max() < 1e-4
    assert torch.isnan(out[0, 1, 0]).nonzero().flatten().tolist() == [5]


@pytest.mark.gpu
def test_layers_one_after_the_other_are_all_at_once():
    L, B, H, d, G = 3, 2, 2, 128, 2
    runs = []
    for apart in (False, True):
        c = kf.Pages.allocate(L, B, H, d, 20, 5, kf.BF16, q_per_kv=G)
        ws, g = kf.new_page_workspace(c), torch.Generator().manual_seed(8)
        lens = torch.tensor([90, 150], dtype=torch.int32).cuda()
        k, v = (torch.randn((L, B, H, 150, d), generator=g).bfloat16().cuda() for _ in range(2))
        outs = []
        parts = [(c.layer(l), slice(l, l + 1)) for l in range(L)] if apart else [(c, slice(0, L))]
        kf.kf_page_reserve(c, 150, lens, workspace=ws)
        for p, at in parts:
            kf.kf_page_write(p, k[at], v[at], 150, seq_n=lens, workspace=ws)
        for _ in range(3):
            q, kn, vn = (torch.randn((L, B, h, d), generator=g).bfloat16().cuda() for h in (H * G, H, H))
            out = torch.zeros((L, B, H * G, d), device="cuda")
            kf.kf_page_reserve(c, workspace=ws)
            for p, at in parts:
                kf.kf_page_step(p, q[at], kn[at], vn[at], d ** -0.5, out[at], 256, workspace=ws)
            outs.append(out)
        runs.append((outs, [x.clone() for x in (c.K, c.V, c.k_scale, c.v_scale, c.table, c.len, c.refs)]))
    assert all(torch.equal(x, y) for x, y in zip(runs[0][0], runs[1][0])) and all(torch.equal(x, y) for x, y in zip(runs[0][1], runs[1][1]))


@pytest.mark.gpu
def test_a_layer_of_many_units_in_the_workspace_of_all_and_of_one():
    """All layers are 1024 units of a split each, a layer 64 units of several: either in the other's workspace, where that serves it."""
    L, B, H, d, n = 16, 1, 64, 128, 1000
    c = kf.Pages.allocate(L, B, H, d, 16, 64, kf.BF16)
    whole, one, g = kf.new_page_workspace(c), kf.new_page_workspace(c.layer(0)), torch.Generator().manual_seed(21)
    k, v = (torch.randn((L, B, H, n, d), generator=g).bfloat16().cuda() for _ in range(2))
    kf.kf_page_reserve(c, n, workspace=one)
    kf.kf_page_write(c, k, v, n, workspace=one)
    table = c.table[0, :16].cpu()
    for i, ws in enumerate((whole, one)):
        q, kn, vn = (torch.randn((L, B, H, d), generator=g).bfloat16() for _ in range(3))
        heads = [(0, 0), (7, 33), (15, 63)]
        held = [[(codes[l, table, h].view(torch.float8_e4m3fn).double() * by[l, table, h, None, None].double()).cpu() for codes, by in ((c.K, c.k_scale), (c.V, c.v_scale))]
                for l, h in heads]
        out = torch.zeros((L, B, H, d), device="cuda")
        kf.kf_page_reserve(c, workspace=ws)
        for l in range(L):
            at = slice(l, l + 1)
            kf.kf_page_step(c.layer(l), q[at].cuda(), kn[at].cuda(), vn[at].cuda(), d ** -0.5, out[at], workspace=ws)
        for (l, h), (K, V) in zip(heads, held):
            K, V = K.reshape(-1, d)[:n + i].numpy(), V.transpose(1, 2).reshape(-1, d)[:n + i].numpy()
            want, tol = step_oracle(K, V, *(x[l, 0, h].double().numpy() for x in (q, kn, vn)), d ** -0.5, 0.0)
            assert (np.abs(out[l, 0, h].double().cpu().numpy() - want) <= tol).all(), (i, l, h)
    assert int(whole[:4].view(torch.int32)) == 0 == int(one[:4].view(torch.int32))


@pytest.mark.gpu
def test_a_token_captured_and_replayed_is_a_token_each_time():
    """Room and step in one graph, replayed across page borders, with eager work between, against the same calls one by one."""
    L, B, H, d = 2, 3, 2, 64
    c, ws, m = both(L, B, H, d, 12, 4)
    g = torch.Generator().manual_seed(11)
    fill(c, ws, m, g, [60, 62, 127])
    e = kf.Pages(**{**c.__dict__, **{x: getattr(c, x).clone() for x in ("K", "V", "k_scale", "v_scale", "table", "len", "refs")}})
    we = ws.clone()
    q, k, v = (torch.zeros((L, B, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    out, want = torch.zeros((L, B, H, d), device="cuda"), torch.zeros((L, B, H, d), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kf.kf_page_reserve(c, workspace=ws)
        kf.kf_page_step(c, q, k, v, 0.125, out, workspace=ws)
    for i in range(6):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g).bfloat16())
        graph.replay()
        kf.kf_page_reserve(e, workspace=we)
        kf.kf_page_step(e, q, k, v, 0.125, want, workspace=we)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        for x in ("K", "V", "k_scale", "v_scale", "table", "len", "refs"):
            assert torch.equal(getattr(c, x), getattr(e, x)), (i, x)


@pytest.mark.gpu
def test_a_page_beyond_32_bits():
    """A pool of more than 2^32 bytes of keys: its last pages hold what the first would."""
    L, B, H, d = 1, 1, 32, 256
    pages = (1 << 32) // (H * P * d) + 3
    c, ws, m = both(L, B, H, d, pages, 2)[0], None, None
    ws = kf.new_page_workspace(c)
    c.refs.fill_(1)
    c.refs[-2:] = 0
    small, wsm = kf.Pages.allocate(L, B, H, d, 2, 2), None
    wsm = kf.new_page_workspace(small)
    g = torch.Generator().manual_seed(12)
    k, v = (torch.randn((L, B, H, 70, d), generator=g).bfloat16().cuda() for _ in range(2))
    q, kn, vn = (torch.randn((L, B, H, d), generator=g).bfloat16().cuda() for _ in range(3))
    outs = []
    for x, w in ((c, ws), (small, wsm)):
        out = torch.zeros((L, B, H, d), device="cuda")
        kf.kf_page_reserve(x, 70, workspace=w)
        kf.kf_page_write(x, k, v, 70, workspace=w)
        kf.kf_page_reserve(x, workspace=w)
        kf.kf_page_step(x, q, kn, vn, d ** -0.5, out, workspace=w)
        outs.append(out)
    assert c.table.tolist() == [[pages - 2, pages - 1]]
    assert torch.equal(outs[0], outs[1]) and torch.equal(c.K[:, -2:], small.K) and torch.equal(c.V[:, -2:], small.V)


@pytest.mark.gpu
def test_a_search_over_pages_from_prompt_to_tokens():
    """kf_norm_rotate -> kf_prompt_attend and kf_page_write -> (kf_beam_select -> kf_page_fork -> kf_page_reserve -> kf_page_step)... and a compaction by
    what kf_prefill_score and kf_select_evict kept."""
    R, W, H, G, d, n = 2, 3, 2, 2, 64, 90
    B, V = R * W, 50
    c, ws, m = both(1, B, H, d, 40, 4, kf.BF16, G)
    g = torch.Generator().manual_seed(21)
    x = torch.randn((R, n, (G + 2) * H, d), generator=g).bfloat16().cuda()
    stage = kf.Cache.allocate(1, R, H, d, n, kf.BF16, q_per_kv=G)
    Q = torch.zeros((R, H * G, n, d), dtype=torch.bfloat16, device="cuda")
    q, k, v = x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]
    freq = (0.5 ** torch.arange(32).float()).cuda()
    kf.kf_norm_rotate(kf.Rows(B=R, n=n, H=H, d=d, dtype=kf.BF16, q_per_kv=G, q_stride=q.stride()[:2], k_stride=k.stride()[:2], v_stride=v.stride()[:2],
                              rotate=kf.ROTATE_HALVES, rot_dim=d, inv_freq=freq), q, k, v, Q, stage.K[0], stage.V[0])
    p = kf.Prompt(B=R, n=n, m=n, H=H, q_per_kv=G, d=d, dtype=kf.BF16, scale=0.125)
    out = torch.zeros((R, n, H * G, d), dtype=torch.bfloat16, device="cuda")
    kf.kf_prompt_attend(p, Q, stage.K[0], stage.V[0], out, workspace=kf.new_prompt_workspace(p))
    # the prompts go into the first beam of each request
    first = [n if b % W == 0 else 0 for b in range(B)]
    k0, v0 = (torch.zeros((1, B, H, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k0[:, ::W], v0[:, ::W] = stage.K, stage.V
    counts = torch.tensor(first, dtype=torch.int32).cuda()
    kf.kf_page_reserve(c, n, counts, workspace=ws)
    kf.kf_page_write(c, k0, v0, n, seq_n=counts, workspace=ws)
    m.reserve(n, first)
    m.write(k0.double().cpu().numpy(), v0.double().cpu().numpy(), first)
    kf.kf_page_fork(c, torch.tensor([b // W * W for b in range(B)], dtype=torch.int32).cuda(), workspace=ws)
    m.fork([b // W * W for b in range(B)])
    m.same(c, ws, "prompts")
    beams = kf.Beams(R, W, V)
    bw, score = kf.new_beam_workspace(beams), torch.zeros(B, device="cuda")
    parent, token = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    for _ in range(5):
        kf.kf_beam_select(beams, torch.randn((B, V), generator=g).cuda() * 3, score, parent, token, score, workspace=bw)
        kf.kf_page_fork(c, parent, workspace=ws)
        m.fork(parent.tolist())
        take_step(c, ws, m, g, m_hint=n + 5)
        m.same(c, ws, "token")
    # what the scores of the prompt keep
    wq = kf.new_workspace(stage, n)
    kf.kf_prefill_score(stage, Q, n, 1.0, 0.125, kf.NOISE_GUMBEL, torch.arange(R, dtype=torch.int64, device="cuda"), workspace=wq)
    kept = torch.zeros((1, R, H, 40), dtype=torch.int32, device="cuda")
    kf.kf_select_evict(stage, 40, 10, kept, workspace=wq)
    keep = torch.cat([kept.repeat_interleave(W, 1), torch.arange(n, n + 5, dtype=torch.int32, device="cuda").expand(1, B, H, 5)], -1).contiguous()
    kf.kf_page_compact(c, keep, 45, workspace=ws)
    m.compact(keep.cpu().numpy(), 45, [1] * B)
    m.same(c, ws, "kept")
    take_step(c, ws, m, g)
    m.same(c, ws, "after")


@pytest.mark.gpu
def test_thousands_of_sequences():
    """More rows of the table than a workgroup has threads, and fewer pages than they ask for."""
    L, B, H, d = 1, 2500, 1, 64
    c, ws, m = both(L, B, H, d, 2300, 2)
    g = torch.Generator().manual_seed(11)
    counts = [int(x) for x in torch.randint(0, 90, (B,), generator=g)]
    kf.kf_page_reserve(c, 80, torch.tensor(counts, dtype=torch.int32).cuda(), workspace=ws)
    m.reserve(80, counts)
    m.same(c, ws, "reserved")
    assert m.errors > 0 and 0 < min(x for x in m.len if x) < 80  # some found no page, of those behind them some did
    x = rows_of(g, L, B, H, 80, d, kf.BF16)
    held = [n if 1 <= n <= 80 and m.len[b] == n else 0 for b, n in enumerate(counts)]
    kf.kf_page_write(c, x.cuda(), x.cuda(), 80, seq_n=torch.tensor(held, dtype=torch.int32).cuda(), workspace=ws)
    m.write(x.double().numpy(), x.double().numpy(), held)
    which = [int(b % 3 == 0) for b in range(B)]
    kf.kf_page_free(c, torch.tensor(which, dtype=torch.int32).cuda(), workspace=ws)
    m.free(which)
    parent = [b if b % 3 else b + 1 if b + 1 < B else b for b in range(B)]
    kf.kf_page_fork(c, torch.tensor(parent, dtype=torch.int32).cuda(), workspace=ws)
    m.fork(parent)
    m.same(c, ws, "forked")
    keep = torch.randint(0, 5, (L, B, H, 5), generator=g, dtype=torch.int32)
    kf.kf_page_compact(c, keep.cuda(), 5, workspace=ws)
    m.compact(keep.numpy(), 5, [1] * B)
    m.same(c, ws, "compacted")


@pytest.mark.gpu
def test_two_caches_on_two_streams():
    """Calls at once, each cache with a workspace of its own: as one after the other."""
    g = torch.Generator().manual_seed(12)
    sets = []
    for lens in ([900, 1300, 20], [1200, 64, 700]):
        c, ws, m = both(1, 3, 4, 128, 64, 32, kf.BF16, 2)
        fill(c, ws, m, g, lens)
        q, k, v = (torch.randn((1, 3, h, 128), generator=g).bfloat16().cuda() for h in (8, 4, 4))
        sets.append((c, ws, q, k, v, [torch.zeros((1, 3, 8, 128), device="cuda") for _ in range(2)]))
    torch.cuda.synchronize()
    for c, ws, q, k, v, out in sets:
        kf.kf_page_step(c, q, k, v, 0.1, out[0], workspace=ws)  # (the last token's place each time: nothing is reserved)
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (c, ws, q, k, v, out) in zip(streams, sets):
            with torch.cuda.stream(s):
                kf.kf_page_step(c, q, k, v, 0.1, out[1], workspace=ws)
    torch.cuda.synchronize()
    for c, ws, q, k, v, out in sets:
        assert bool(out[0].any()) and torch.equal(out[0], out[1]) and int(ws[:4].view(torch.int32)) == 0
