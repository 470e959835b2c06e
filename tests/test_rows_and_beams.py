"""Rows of a projection (kf_norm_rotate) and the selection of a beam search (kf_beam_select) against plain
definitions in 64 bits, their refusals (no GPU), and their replay from a HIP graph."""
import math

import numpy as np
import pytest
import torch

import paper_2403_09054_amd as kf
from paper_2403_09054_amd import binding

TYPES = {kf.F32: torch.float32, kf.BF16: torch.bfloat16, kf.F16: torch.float16}
U = 2.0 ** -24  # half a step of fp32


def expect(status, fn, *a, **k):
    with pytest.raises(kf.KeyformerError) as e:
        fn(*a, **k)
    assert e.value.status == status, e.value
    assert len(str(e.value)) > 20


# ---------------------------------------------------------------- refusals (nothing is launched)
def test_rows_refusals():
    def call(q=0x1000, k=0x2000, v=0x3000, Q=0x4000, K=0x5000, V=0x6000, **over):
        r = dict(B=2, n=5, H=4, d=128, dtype=kf.BF16, rotate=kf.ROTATE_HALVES, rot_dim=64, inv_freq=0x7000)
        r.update(over)
        kf.kf_norm_rotate(kf.Rows(**r), q, k, v, Q, K, V, stream=0)

    for bad in (dict(B=0), dict(n=0), dict(H=0), dict(d=0), dict(q_per_kv=-1), dict(dtype=5), dict(kv_rows=4), dict(q=None), dict(K=None),
                dict(q=None, k=None, v=None, Q=None, K=None, V=None), dict(q=0x1008), dict(V=0x6004), dict(q_weight=0x7008),
                dict(q_stride=(-8, 512)), dict(k_stride=(2560, 516)), dict(rotate=3), dict(rot_dim=63), dict(rot_dim=130), dict(rot_dim=0),
                dict(inv_freq=None), dict(pos0=-1), dict(q_weight=0x7000, eps=-1.0), dict(k_weight=0x7000, eps=float("nan"))):
        expect(binding.KF_EINVAL, call, **bad)
    expect(binding.KF_EUNSUPPORTED, call, d=96)
    expect(binding.KF_EUNSUPPORTED, call, dtype=kf.F32, d=256)
    assert binding.lib().kf_norm_rotate(None, 1, 1, 1, 1, 1, 1, None) == binding.KF_EINVAL


def test_beam_refusals():
    ws = (0x100000, 1 << 40)

    def call(logits=0x1000, score=0x2000, parent=0x3000, token=0x4000, new_score=0x5000, done=None, new_done=None, workspace=ws, **over):
        b = dict(R=2, W=4, V=1000, dtype=kf.BF16)
        b.update(over)
        kf.kf_beam_select(kf.Beams(**b), logits, score, parent, token, new_score, done=done, new_done=new_done, workspace=workspace, stream=0)

    for bad in (dict(R=0), dict(W=0), dict(V=0), dict(dtype=9), dict(logits=None), dict(score=None), dict(parent=None), dict(token=None),
                dict(new_score=None), dict(logits=0x1001), dict(row_stride=999), dict(row_stride=-1), dict(done=0x6000), dict(new_done=0x6000, eos=1000)):
        expect(binding.KF_EINVAL, call, **bad)
    for bad in (dict(W=33), dict(V=500001)):
        expect(binding.KF_EUNSUPPORTED, call, **bad)
    for bad in (None, (0x100000, 64), (0x100004, 1 << 40)):
        expect(binding.KF_EWORKSPACE, call, workspace=bad)
    assert kf.kf_beam_workspace_bytes(kf.Beams(2, 33, 1000)) == 0 < kf.kf_beam_workspace_bytes(kf.Beams(2, 32, 1000))
    expect(binding.KF_EUNSUPPORTED, kf.new_beam_workspace, kf.Beams(2, 33, 1000), device="cpu")


# ---------------------------------------------------------------- rows
def rows_oracle(x, w, eps, pos, freq, style, rot):
    """[B, n, heads, d] -> [B, heads, n, d], and what bounds an error in 32 bits: |a| + |b| of each rotated pair, else |x|."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    size = x.abs()
    if style != kf.ROTATE_NONE:
        t = pos.double()[:, :, None, None] * freq.double()
        a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if style == kf.ROTATE_PAIRS else (x[..., :rot // 2], x[..., rot // 2:rot])
        u, v, m = a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos(), a.abs() + b.abs()
        size = size.clone()
        x = x.clone()
        for y, (p, q) in ((x, (u, v)), (size, (m, m))):
            if style == kf.ROTATE_PAIRS:
                y[..., 0:rot:2], y[..., 1:rot:2] = p, q
            else:
                y[..., :rot // 2], y[..., rot // 2:rot] = p, q
    return x.transpose(1, 2), size.transpose(1, 2)


def assert_rows(got, want, size, dt, what):
    # the sum of squares: 13 roundings at most, halved by the root; root, division, two products: 11 U of the normed element.
    # Cosine and sine: the turn rounded to 32 bits (3.2 U), the function (2 U), product and sum (2 U).  Then the final rounding.
    tol = 20 * U * size + torch.finfo(dt).eps / 2 * want.abs() + 2.0 ** -25 * (dt == torch.float16)  # (half a step of the smallest halves)
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol).all()), (what, float((err - tol).max()))


ROWS = [  # B, n, H, G, d, dtype, style, rot, norm, extra cache rows, far, padded
    (1, 1, 1, 1, 64, kf.F32, kf.ROTATE_PAIRS, 64, False, 0, 0, False),
    (1, 1, 16, 1, 256, kf.BF16, kf.ROTATE_PAIRS, 64, False, 0, 3000, False),
    (3, 1, 2, 8, 128, kf.BF16, kf.ROTATE_HALVES, 128, True, 5, 1000000, False),
    (2, 2, 3, 2, 64, kf.F16, kf.ROTATE_HALVES, 2, True, 1, 9, False),
    (2, 3, 2, 1, 128, kf.F32, kf.ROTATE_HALVES, 36, True, 0, 200, True),
    (2, 4, 2, 4, 128, kf.F16, kf.ROTATE_PAIRS, 22, False, 3, 70, False),
    (1, 7, 5, 1, 256, kf.F16, kf.ROTATE_HALVES, 254, True, 0, 100, False),
    (5, 37, 2, 2, 128, kf.BF16, kf.ROTATE_HALVES, 64, True, 11, 50, True),
    (2, 513, 4, 1, 64, kf.BF16, kf.ROTATE_NONE, 0, True, 0, 0, True),
    (1, 300, 3, 3, 256, kf.BF16, kf.ROTATE_HALVES, 256, False, 0, 2 ** 31 - 400, False),
    (1, 9, 70, 1, 128, kf.F32, kf.ROTATE_NONE, 0, False, 0, 0, False),
]


def rows_case(rng, B, n, H, G, d, dtype, style, rot, norm, extra, far, padded, fused):
    dt = TYPES[dtype]
    HQ = H * G
    if fused:  # one projection, queries, keys and values side by side, and a gap behind
        x = torch.from_numpy(rng.standard_normal((B, n, HQ + 2 * H + 1, d))).to(dt)
        q, k, v = x[:, :, :HQ], x[:, :, HQ:HQ + H], x[:, :, HQ + H:HQ + 2 * H]
    else:
        q, k, v = (torch.from_numpy(rng.standard_normal((B, n, h, d))).to(dt) for h in (HQ, H, H))
    w = [(torch.from_numpy(1.0 + 0.3 * rng.standard_normal(d)).to(dt)) if norm else None for _ in range(2)]
    freq = torch.from_numpy((10000.0 ** (-2.0 * np.arange(max(rot // 2, 1)) / max(rot, 1))).astype(np.float32))
    start = torch.from_numpy(rng.integers(0, far + 1, B).astype(np.int32))
    lens = torch.from_numpy(rng.integers(1, n + 1, B).astype(np.int32)) if padded else None
    return dt, q, k, v, w, freq, start, lens


@pytest.mark.gpu
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("case", ROWS, ids=lambda c: "x".join(map(str, c)))
def test_rows_match_the_definition(case, fused):
    B, n, H, G, d, dtype, style, rot, norm, extra, far, padded = case
    rng = np.random.default_rng(sum(case[:5]))
    dt, q, k, v, w, freq, start, lens = rows_case(rng, *case, fused)
    base = [t.cuda() for t in ((q._base,) if fused else (q, k, v))]
    if fused:
        HQ = H * G
        dq, dk, dv = base[0][:, :, :HQ], base[0][:, :, HQ:HQ + H], base[0][:, :, HQ + H:HQ + 2 * H]
        st = dict(q_stride=dq.stride()[:2], k_stride=dk.stride()[:2], v_stride=dv.stride()[:2])
    else:
        (dq, dk, dv), st = base, {}
    Q = torch.full((B, H * G, n, d), 7.0, dtype=dt, device="cuda")
    K, V = (torch.full((B, H, n + extra, d), 7.0, dtype=dt, device="cuda") for _ in range(2))
    dw = [None if x is None else x.cuda() for x in w]
    rows = kf.Rows(B=B, n=n, H=H, d=d, dtype=dtype, q_per_kv=G, kv_rows=n + extra, q_weight=dw[0], k_weight=dw[1], eps=1e-5, rotate=style,
                   rot_dim=rot, inv_freq=freq.cuda(), seq_pos=start.cuda(), seq_n=None if lens is None else lens.cuda(), **st)
    kf.kf_norm_rotate(rows, dq, dk, dv, Q, K, V)
    torch.cuda.synchronize()
    pos = start[:, None].long() + torch.arange(n)
    ok = (torch.arange(n)[None, :] < (lens[:, None] if lens is not None else n))[:, None, :, None]
    seven = torch.tensor(7.0, dtype=torch.float64)
    for name, got, x, wt in (("Q", Q, q, w[0]), ("K", K[:, :, :n], k, w[1])):
        want, size = rows_oracle(x, wt, 1e-5, pos, freq, style, rot)
        assert_rows(got, torch.where(ok, want, seven), torch.where(ok, size, 0.0), dt, name)
    assert torch.equal(V[:, :, :n].cpu(), torch.where(ok, v.transpose(1, 2), torch.tensor(7.0, dtype=dt)))
    assert bool((K[:, :, n:] == 7.0).all()) and bool((V[:, :, n:] == 7.0).all())  # rows behind stay as they were


@pytest.mark.gpu
def test_rows_left_out_kinds_one_position_and_bad_lengths():
    g = torch.Generator().manual_seed(5)
    B, n, H, d = 3, 6, 2, 128
    q, k, v = (torch.randn((B, n, H, d), generator=g).bfloat16().cuda() for _ in range(3))
    freq = (0.5 ** torch.arange(32).float()).cuda()
    of = dict(B=B, n=n, H=H, d=d, dtype=kf.BF16, rotate=kf.ROTATE_HALVES, rot_dim=64, inv_freq=freq, pos0=41)
    full = [torch.zeros((B, H, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    kf.kf_norm_rotate(kf.Rows(**of), q, k, v, *full)
    want, size = rows_oracle(q.cpu(), None, 0.0, torch.arange(41, 41 + n).expand(B, n), freq.cpu(), kf.ROTATE_HALVES, 64)
    assert_rows(full[0], want, size, torch.bfloat16, "Q")
    for only in range(3):  # each kind alone gives what all together give
        ins, outs = [None] * 3, [None] * 3
        ins[only], outs[only] = (q, k, v)[only], torch.zeros_like(full[only])
        kf.kf_norm_rotate(kf.Rows(**of), *ins, *outs)
        assert torch.equal(outs[only], full[only])
    # a length that is none leaves its sequence out
    for bad in (-1, 0, n + 1):
        Q = torch.full_like(full[0], 3.0)
        kf.kf_norm_rotate(kf.Rows(seq_n=torch.tensor([n, bad, 2], dtype=torch.int32).cuda(), **of), q, None, None, Q, None, None)
        assert torch.equal(Q[0], full[0][0]) and bool((Q[1] == 3.0).all()) and torch.equal(Q[2, :, :2], full[0][2, :, :2]) and bool((Q[2, :, 2:] == 3.0).all())


@pytest.mark.gpu
def test_rows_carry_nan_and_infinity_of_their_own_row_only():
    x = torch.randn((1, 4, 2, 64), generator=torch.Generator().manual_seed(1)).half().cuda()
    x[0, 1, 0, 3] = float("nan")
    x[0, 2, 1, 60] = float("inf")
    Q = torch.zeros((1, 2, 4, 64), dtype=torch.float16, device="cuda")
    w = torch.ones(64, dtype=torch.float16, device="cuda")
    kf.kf_norm_rotate(kf.Rows(B=1, n=4, H=2, d=64, dtype=kf.F16, q_weight=w, rotate=kf.ROTATE_PAIRS, rot_dim=32, inv_freq=torch.ones(16).cuda()),
                      x, None, None, Q, None, None)
    bad = torch.isnan(Q).any(-1)[0].cpu()
    assert bad.tolist() == [[False, True, False, False], [False, False, True, False]]
    assert bool(torch.isnan(Q[0, 0, 1]).all())


# ---------------------------------------------------------------- beams
def beam_oracle(x, score, done, eos, R, W):
    """The definition in float64: (parent, token, new_score, new_done, rank), and each request's candidates in order,
    (-total, beam, -logit, word), W of each beam."""
    x = x.double().numpy()
    V = x.shape[1]
    parent, token, rank, nd = (np.zeros(R * W, np.int64) for _ in range(4))
    new, every = np.zeros(R * W), []
    for r in range(R):
        found = []
        for i in range(W):
            row, sc = r * W + i, float(score[r * W + i])
            if done is not None and done[row]:
                t = -math.inf if math.isnan(sc) else sc
                found.append((-t, i, 0.0, eos))
                continue
            with np.errstate(all="ignore"):
                top = np.nanmax(x[row]) if not np.isnan(x[row]).all() else -math.inf
                ref = 0.0 if top == -math.inf else top
                lse = ref + np.log(np.exp(x[row] - ref).sum())
                tot = sc + (x[row] - lse)
            tot = np.where(np.isnan(tot), -math.inf, tot)
            lg = np.where(np.isnan(x[row]), -math.inf, x[row]) + 0.0
            order = np.lexsort((np.arange(V), -lg))[:W]
            found += [(-tot[v], i, -lg[v], int(v)) for v in order]
        every.append(sorted(found))
        found = every[-1][:W]
        taken, rows = set(), []
        for c in found:
            rows.append(c[1] if c[1] not in taken else None)
            taken.add(c[1])
        left = [i for i in range(W) if i not in taken]
        for j, c in enumerate(found):
            at = r * W + (rows[j] if rows[j] is not None else left.pop(0))
            parent[at], token[at], rank[at], new[at] = r * W + c[1], c[3], j, -c[0]
            nd[at] = int((done is not None and done[r * W + c[1]] != 0) or c[3] == eos)
    return parent, token, new, nd, rank, every, [0] * (R * W) if done is None else [int(v != 0) for v in done], eos


def run_beams(x, score, done, eos, R, W, dtype, pad=0, shift=0, in_place=False):
    V = x.shape[1]
    dt = TYPES[dtype]
    store = torch.full((R * W * (V + pad) + shift,), float("nan"), dtype=dt)  # what lies between the rows is not looked at
    store[shift:].view(R * W, V + pad)[:, :V] = x
    store = store.cuda()
    logits = store[shift:]
    sc = torch.from_numpy(np.asarray(score, np.float32)).cuda()
    dn = None if done is None else torch.from_numpy(np.asarray(done, np.int32)).cuda()
    b = kf.Beams(R=R, W=W, V=V, dtype=dtype, row_stride=V + pad if pad else 0, eos=eos)
    parent, token, rank = (torch.full((R * W,), -9, dtype=torch.int32, device="cuda") for _ in range(3))
    new = sc if in_place else torch.zeros_like(sc)
    nd = None if eos < 0 else (dn if in_place and dn is not None else torch.full((R * W,), -9, dtype=torch.int32, device="cuda"))
    kf.kf_beam_select(b, logits, sc, parent, token, new, done=dn, new_done=nd, rank=rank, workspace=kf.new_beam_workspace(b))
    torch.cuda.synchronize()
    return parent.cpu().numpy(), token.cpu().numpy(), new.cpu().numpy(), None if nd is None else nd.cpu().numpy(), rank.cpu().numpy()


def assert_beams(got, want, what="", x=None, score=None):
    """Equal to the definition.  Totals of different beams that differ by less than what 32-bit exponentials resolve may change
    places: an exponential is off by 2.4 U, a sum of up to 8 of them by 7 U more, the rest is in 64 bits, so a total is
    off by at most 10 U, and 20 U tell two apart.  (Rows of the same logits in another order have equal totals by the
    definition, and sums that differ in their last bits.)  Within a beam, and between beams of the same logits and score, the order is
    exact."""
    parent, token, new, nd, rank = got
    R, W = len(want[5]), len(parent) // len(want[5])
    for r in range(R):
        z = slice(r * W, r * W + W)
        assert sorted(rank[z]) == list(range(W)), what
        rows = r * W + np.argsort(rank[z])  # the request's rows, best first
        picks = [(int(parent[i]) - r * W, int(token[i])) for i in rows]
        total = {(c[1], c[3]): -c[0] for c in want[5][r]}
        assert len(set(picks)) == W and all(p in total for p in picks), (what, picks)
        for j, p in enumerate(picks):
            best = -want[5][r][j][0]
            assert total[p] == best or abs(total[p] - best) <= 20 * U, (what, j, p, total[p], best)
            w = total[p]
            assert np.float32(new[rows[j]]) == np.float32(w) or abs(new[rows[j]] - w) <= U * abs(w) + 10 * U, (what, j, new[rows[j]], w)
        for i in range(W):  # a beam's continuations are its best ones, in order
            mine = [c[3] for c in sorted((c for c in want[5][r] if c[1] == i), key=lambda c: (c[2], c[3]))]
            assert [t for b, t in picks if b == i] == mine[:sum(b == i for b, _ in picks)], (what, i)
        if x is not None:
            for i in range(W):
                for j in range(i + 1, W):
                    a, b = r * W + i, r * W + j
                    if score[a] == score[b] and torch.equal(x[a], x[b]):  # the lower of two equal beams is served first
                        for t in {t for q, t in picks if q == j}:
                            assert (i, t) in picks and picks.index((i, t)) < picks.index((j, t)), (what, i, j, t)
        taken, left = set(), sorted(set(range(W)) - {b for b, _ in picks})
        for j, (b, _) in enumerate(picks):  # numbering
            assert rows[j] == r * W + (left.pop(0) if b in taken else b), (what, j)
            taken.add(b)
        if nd is not None:
            assert all(nd[i] == int(want[6][int(parent[i])] or token[i] == want[7]) for i in rows), what
    assert np.array_equal(parent[parent], parent), "a parent continues itself"


BEAMS = [  # R, W, V, dtype, elements between rows, elements before the first
    (1, 1, 1, kf.F32, 0, 0), (2, 4, 1, kf.BF16, 0, 1), (3, 5, 7, kf.F16, 2, 3), (1, 32, 50, kf.BF16, 0, 0), (2, 32, 5003, kf.F32, 1, 2),
    (4, 4, 50257, kf.BF16, 0, 5), (1, 1, 50257, kf.F16, 0, 1), (300, 2, 129, kf.F32, 0, 1), (1, 16, 131072, kf.F32, 0, 0),
    (1, 32, 131073, kf.BF16, 7, 0), (2, 2, 499999, kf.F16, 0, 0), (1, 3, 499999, kf.F32, 0, 3), (17, 8, 2048, kf.F16, 0, 0), (64, 4, 8192, kf.BF16, 0, 0),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", BEAMS, ids=lambda c: "x".join(map(str, c)))
def test_beams_match_the_definition(case):
    R, W, V, dtype, pad, shift = case
    rng = np.random.default_rng(R + 10 * W + V)
    x = torch.from_numpy(3.0 * rng.standard_normal((R * W, V))).to(TYPES[dtype])
    score = -10 * rng.random(R * W)
    score = score.astype(np.float32)
    assert_beams(run_beams(x, score, None, -1, R, W, dtype, pad, shift), beam_oracle(x, score, None, -1, R, W))
    done = (rng.random(R * W) < 0.4).astype(np.int32) * 5
    eos = int(rng.integers(0, V))
    for in_place in (False, True):
        assert_beams(run_beams(x, score, done, eos, R, W, dtype, pad, shift, in_place), beam_oracle(x, score, done, eos, R, W), "ended")


def _special(kind, rng, rows, V):
    x = rng.standard_normal((rows, V)).astype(np.float32)
    if kind == "constant":
        x[:] = 1.5
    elif kind == "few values":  # ties everywhere, zeros of both signs among them
        x = rng.integers(-1, 2, (rows, V)).astype(np.float32)
        x[x == 0] *= np.where(rng.random((x == 0).sum()) < 0.5, -1.0, 1.0)
    elif kind == "rising":
        x = np.broadcast_to(np.arange(V, dtype=np.float32) / 64, (rows, V)).copy()
    elif kind == "falling":
        x = np.broadcast_to(-np.arange(V, dtype=np.float32) / 64, (rows, V)).copy()
    elif kind == "one left":  # a grammar leaves one word in some rows, none in others
        x[:] = -np.inf
        x[::2, V // 3] = 0.25
    elif kind == "lowest":
        x[:, 5:] = float(torch.finfo(torch.bfloat16).min)
    elif kind == "nan":
        x[1, V // 2] = np.nan
        x[2, :] = np.nan
    elif kind == "infinite":
        x[0, V // 2] = np.inf
    elif kind == "nothing":
        x[:] = -np.inf
    elif kind == "wide":  # sums of exponentials that only a reference keeps in range
        x = x * 300.0
    return torch.from_numpy(x)


@pytest.mark.gpu
@pytest.mark.parametrize("V", [3, 40, 6000])
@pytest.mark.parametrize("kind", ["constant", "few values", "rising", "falling", "one left", "lowest", "nan", "infinite", "nothing", "wide"])
def test_beams_ties_masks_and_infinities(kind, V):
    R, W = 2, 6
    rng = np.random.default_rng(3)
    for dtype in (kf.F32, kf.BF16, kf.F16):
        x = _special(kind, rng, R * W, V).to(TYPES[dtype])
        if dtype == kf.F16 and kind == "lowest":
            x = x.clamp(min=-65504.0)
        score = np.array([-1.0, -2.0, -2.0, -1.0, -30.0, -0.5] * R, np.float32)
        want = beam_oracle(x, score, None, -1, R, W)
        assert_beams(run_beams(x, score, None, -1, R, W, dtype), want, kind, x, score)
        # the first step: one beam lives; and scores that are no numbers
        first = np.array([0.0] + [-np.inf] * 4 + [np.nan] + [-np.inf] * 6, np.float32)
        assert_beams(run_beams(x, first, None, -1, R, W, dtype), beam_oracle(x, first, None, -1, R, W), kind + ", first step")
        done = np.array([0, 1, 0, 1, 0, 0] * R, np.int32)
        assert_beams(run_beams(x, score, done, 1, R, W, dtype), beam_oracle(x, score, done, 1, R, W), kind + ", ended")
        everyone = np.ones(R * W, np.int32)
        assert_beams(run_beams(x, score, everyone, 2, R, W, dtype), beam_oracle(x, score, everyone, 2, R, W), kind + ", all ended")


@pytest.mark.gpu
def test_rows_and_beams_replay_from_a_graph():
    torch.manual_seed(7)
    R, W, V, H, d = 3, 4, 9001, 4, 128
    B = R * W
    b = kf.Beams(R=R, W=W, V=V, dtype=kf.BF16, eos=3)
    ws = kf.new_beam_workspace(b)
    logits = torch.empty((B, V), dtype=torch.bfloat16, device="cuda")
    x = torch.empty((B, 1, 3 * H, d), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(B, dtype=torch.int32, device="cuda")
    freq = (0.9 ** torch.arange(d // 2).float()).cuda()
    st = x.stride()[:2]
    rows = kf.Rows(B=B, n=1, H=H, d=d, dtype=kf.BF16, q_stride=st, k_stride=st, v_stride=st, rotate=kf.ROTATE_HALVES, rot_dim=d, inv_freq=freq, seq_pos=pos)
    parts = (x[:, :, :H], x[:, :, H:2 * H], x[:, :, 2 * H:])

    def state():
        return dict(score=torch.zeros(B, device="cuda"), done=torch.zeros(B, dtype=torch.int32, device="cuda"),
                    ints=torch.zeros((3, B), dtype=torch.int32, device="cuda"), out=torch.zeros((3, B, H, 1, d), dtype=torch.bfloat16, device="cuda"))

    def step(s):
        kf.kf_norm_rotate(rows, *parts, s["out"][0], s["out"][1], s["out"][2])
        kf.kf_beam_select(b, logits, s["score"], s["ints"][0], s["ints"][1], s["score"], done=s["done"], new_done=s["done"], rank=s["ints"][2], workspace=ws)

    def fill(i):
        g = torch.Generator(device="cuda").manual_seed(100 + i)
        logits.copy_(4 * torch.randn(logits.shape, generator=g, device="cuda"))
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        pos.fill_(50 + i)

    eager, played = state(), state()
    fill(0)
    step(state())  # loads the kernels
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(played)
    for s in (eager, played):
        s["score"].zero_(), s["done"].zero_()
    for i in range(5):
        fill(i)
        graph.replay()
        step(eager)
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(eager[name], played[name]), (i, name)


@pytest.mark.gpu
def test_rows_and_beams_on_a_stream_of_their_own():
    torch.manual_seed(8)
    x = torch.randn((2, 40, 6, 64)).half().cuda()
    freq = torch.rand(32).cuda()
    logits = torch.randn((8, 3000)).cuda()
    b = kf.Beams(R=2, W=4, V=3000)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            Q = torch.zeros((2, 6, 40, 64), dtype=torch.float16, device="cuda")
            out = [torch.zeros(8, dtype=torch.int32, device="cuda") for _ in range(2)]
            new, score = torch.zeros(8, device="cuda"), torch.arange(8, device="cuda").float()
            ws = kf.new_beam_workspace(b)
            kf.kf_norm_rotate(kf.Rows(B=2, n=40, H=6, d=64, dtype=kf.F16, rotate=kf.ROTATE_PAIRS, rot_dim=64, inv_freq=freq), x, None, None, Q, None, None,
                              stream=stream)
            kf.kf_beam_select(b, logits, score, out[0], out[1], new, workspace=ws, stream=stream)
        stream.synchronize()
        got.append([Q, *out, new])
    assert all(torch.equal(p, q) for p, q in zip(*got))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [9, 70])
def test_rows_of_any_length_that_is_none_are_left_out(n):
    """Also lengths from which a later tile's first token cannot be taken away in 32 bits."""
    g = torch.Generator().manual_seed(6)
    low = -2 ** 31
    lens = torch.tensor([n, low, low + 7, low + n, -n, 2 ** 31 - 1, 1], dtype=torch.int32).cuda()
    B, H, d, room = len(lens), 2, 64, 16  # (rows behind a sequence's, as a padded batch has them)
    x = [torch.randn((B, n + room, H, d), generator=g).half().cuda() for _ in range(3)]
    Q = torch.full((B, H, n, d), 3.0, dtype=torch.float16, device="cuda")
    K, V = (torch.full((B, H, n + room, d), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    st = x[0].stride()[:2]
    kf.kf_norm_rotate(kf.Rows(B=B, n=n, H=H, d=d, dtype=kf.F16, kv_rows=n + room, q_stride=st, k_stride=st, v_stride=st, seq_n=lens), *x, Q, K, V)
    torch.cuda.synchronize()
    for got, src in zip((Q, K, V), x):
        want = torch.full_like(got, 3.0)
        for b, m in ((0, n), (B - 1, 1)):
            want[b, :, :m] = src[b, :m].transpose(0, 1)
        assert torch.equal(got, want)
