"""Attention over prompts (kf_prompt_attend) against its definition in 64 bits, its refusals (no GPU), what masked places may
hold, its replay from a HIP graph, and its place between kf_norm_rotate and kf_prefill_score."""
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
def test_prompt_refusals():
    def call(Q=0x1000, K=0x2000, V=0x3000, out=0x4000, workspace=(0x100000, 1 << 40), **over):
        p = dict(B=2, n=5, m=9, H=4, d=128, dtype=kf.BF16, scale=0.1)
        p.update(over)
        kf.kf_prompt_attend(kf.Prompt(**p), Q, K, V, out, workspace=workspace, stream=0)

    for bad in (dict(B=0), dict(n=0), dict(m=0), dict(H=0), dict(d=0), dict(q_per_kv=-1), dict(dtype=5), dict(dtype=kf.BF16_Q4), dict(Q=None), dict(K=None),
                dict(V=None), dict(out=None), dict(Q=0x1008), dict(V=0x3004), dict(out=0x4002), dict(scale=math.inf), dict(scale=math.nan),
                dict(q_stride=(-8, 512, 128)), dict(k_stride=(2560, 516, 128)), dict(out_stride=(8, 8, 4)), dict(q_start=0x5000, seq_n=0x6000),
                dict(k_start=0x5000, seq_m=0x6000), dict(n=1 << 30, q_per_kv=2), dict(H=1 << 24, q_per_kv=2)):
        expect(binding.KF_EINVAL, call, **bad)
    for bad in (dict(d=96), dict(dtype=kf.F32, d=256), dict(B=1 << 20, H=1 << 14), dict(k_stride=(0, 128, (1 << 26) + 8))):
        expect(binding.KF_EUNSUPPORTED, call, **bad)
    for bad in (None, (0x100000, 64), (0x100004, 1 << 40)):
        expect(binding.KF_EWORKSPACE, call, workspace=bad)
    assert binding.lib().kf_prompt_attend(None, 1, 1, 1, 1, 1, 1, None) == binding.KF_EINVAL
    assert kf.kf_prompt_workspace_bytes(kf.Prompt(1, 5, 5, 2, 96, kf.BF16, 1.0)) == 0
    expect(binding.KF_EUNSUPPORTED, kf.new_prompt_workspace, kf.Prompt(1, 5, 5, 2, 96, kf.BF16, 1.0), device="cpu")
    # few rows of many keys are shared out, and need room for it; many rows need none
    assert kf.kf_prompt_workspace_bytes(kf.Prompt(1, 1, 8000, 2, 128, kf.BF16, 1.0)) > kf.kf_prompt_workspace_bytes(kf.Prompt(64, 4096, 4096, 32, 128, kf.BF16, 1.0)) > 0


SHAPES = r"""
#include "kf_internal.h"
#include <cstdio>
int main() {  // shapes that the plan did not size its tiles and records for: refused, and nothing is launched
    const int type[][2] = {{KF_F32, 64}, {KF_F32, 128}, {KF_BF16, 64}, {KF_BF16, 128}, {KF_BF16, 256}, {KF_F16, 64}, {KF_F16, 256}};
    int calls = 0;
    for (auto& t : type)
        for (int n : {1, 100, 3000})
            for (int units : {1, 40, 700})
                for (int shape = 0; shape < 5; ++shape) {
                    kf::AttendArgs a = {};
                    a.B = units, a.H = 1, a.G = 1, a.n = n, a.m = 3000;
                    kf::plan_attend(&a, t[1], t[0]);
                    if (shape == a.shape) continue;
                    a.shape = shape;
                    if (kf::launch_attend(a, t[1], t[0], nullptr) != hipErrorInvalidValue) return printf("%d x %d, %d rows of %d: shape %d\n", t[0], t[1], n, units, shape), 1;
                    ++calls;
                }
    return calls > 200 ? 0 : 1;
}
"""


def test_a_shape_that_was_not_planned_is_refused(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(kf.lib_path())
    source, program = tmp_path / "shapes.hip", tmp_path / "shapes"
    source.write_text(SHAPES)
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "-std=c++17", "-I", os.path.join(root, "csrc"), str(source), "-o", str(program),
                    "-L", root, "-lkeyformer", f"-Wl,-rpath,{root}"], check=True, timeout=100)
    r = subprocess.run([str(program)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr


def test_launches_of_2_to_the_32_threads_are_refused():
    of = dict(n=1, m=1, d=128, dtype=kf.BF16, scale=1.0)
    assert kf.kf_prompt_workspace_bytes(kf.Prompt(B=4095, H=4097, **of)) > 0 == kf.kf_prompt_workspace_bytes(kf.Prompt(B=4096, H=4096, **of))
    for big in (dict(B=4096, H=4096), dict(B=1 << 12, H=1 << 9, n=1024), dict(B=(1 << 31) - 1, H=(1 << 24) - 1, n=1 << 30)):
        expect(binding.KF_EUNSUPPORTED, kf.kf_prompt_attend, kf.Prompt(**{**of, **big}), 0x1000, 0x2000, 0x3000, 0x4000, workspace=(0x100000, 1 << 40), stream=0)


# ---------------------------------------------------------------- the definition
def attend_oracle(q, k, v, scale, slope, dt):
    """One head: [nq, d], [nk, d] -> its rows, and how far a row may be off.

    A logit sums d products in 32 bits (d U of their magnitudes), a scale, the bias and the reference round (6 U of theirs); a term's
    relative error is that, twice (its own and the sum's), 2^-22 of the exponential, and its rounding to the element type for the
    product (none in fp32; 2^-25 of the largest term where halves become subnormal).  The sums of nk terms: nk U.  The row is rounded once."""
    q, k, v = q.double(), k.double(), v.double()
    nq, nk = q.shape[0], k.shape[0]
    gap = (torch.arange(nq)[:, None] + nk - nq - torch.arange(nk)).double()
    x = q @ k.T * scale - slope * gap
    see = gap >= 0
    x = torch.where(see, x, -math.inf)
    top = x.amax(1, keepdim=True) if nk else torch.zeros(nq, 1)
    w = torch.where(see, torch.exp(x - torch.where(top == -math.inf, 0.0, top)), 0.0)
    total = w.sum(1, keepdim=True)
    p = torch.where(total > 0, w / total, 0.0) if nk else w
    out, size = p @ v, p @ v.abs()
    e = torch.where(see, (q.abs() @ k.abs().T) * abs(scale) * q.shape[1] * U + 6 * U * (x.nan_to_num(0, 0, 0).abs() + slope * gap.abs()), 0.0)
    worst = e.amax(1, keepdim=True) if nk else torch.zeros(nq, 1)
    half = torch.finfo(dt).eps / 2
    rel = 2 * worst + 2.0 ** -21 + (0.0 if dt == torch.float32 else half) + (nk + 64) * U
    tol = size * rel + half * out.abs() + (2.0 ** -25 * v.abs().sum(0) + 2.0 ** -25 if dt == torch.float16 else 0.0)
    return out, tol + 1e-38


def oracle(Q, K, V, scale, slopes, G, dt):
    """[HQ, nq, d], [H, nk, d] -> [HQ, nq, d] and tolerances."""
    rows = [attend_oracle(Q[h], K[h // G], V[h // G], scale, 0.0 if slopes is None else float(slopes[h]), dt) for h in range(Q.shape[0])]
    return torch.stack([r[0] for r in rows]), torch.stack([r[1] for r in rows])


def near(got, want, tol, what):
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol).all()), (what, float((err - tol).max()), float(err.max()))


def slopes_of(HQ):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / HQ) for h in range(HQ)], dtype=torch.float32)


CASES = [  # B, n, m, H, G, d, dtype, alibi, layout
    (1, 1, 1, 1, 1, 64, kf.F32, False, "plain"),
    (1, 1, 1, 2, 2, 128, kf.BF16, True, "plain"),
    (2, 1, 700, 2, 4, 128, kf.BF16, False, "plain"),      # one row of many keys: shared out
    (1, 1, 3001, 1, 1, 256, kf.F16, True, "plain"),
    (2, 33, 33, 3, 1, 64, kf.F16, False, "cache"),
    (1, 127, 127, 2, 1, 128, kf.BF16, False, "plain"),
    (1, 128, 128, 2, 1, 128, kf.F16, True, "packed"),
    (2, 129, 129, 2, 2, 64, kf.BF16, True, "cache"),
    (1, 65, 191, 2, 3, 128, kf.BF16, False, "packed"),    # three query heads a cached head
    (3, 200, 200, 2, 1, 256, kf.BF16, True, "padded"),
    (4, 257, 400, 2, 4, 128, kf.F16, False, "padded"),
    (5, 300, 300, 2, 8, 64, kf.BF16, False, "packed"),
    (3, 100, 60, 2, 1, 128, kf.BF16, False, "padded"),    # more queries than keys: rows that see nothing
    (2, 70, 33, 1, 5, 64, kf.F32, True, "plain"),
    (2, 150, 150, 2, 2, 128, kf.F32, False, "packed"),
    (1, 40, 1000, 1, 2, 64, kf.F32, True, "cache"),
    (1, 513, 513, 1, 1, 256, kf.F16, False, "plain"),
    (1, 1100, 1100, 2, 1, 128, kf.BF16, True, "plain"),
    (1, 1025, 1025, 1, 2, 64, kf.BF16, False, "plain"),
    (70, 3, 5, 3, 2, 64, kf.BF16, False, "padded"),       # many short ones
]


def make(case, scale=None):
    """Inputs on the GPU, the description, and for each sequence the views of its rows."""
    B, n, m, H, G, d, dtype, alibi, layout = case
    dt, HQ, g = TYPES[dtype], H * G, torch.Generator().manual_seed(sum(case[:6]))
    rng = np.random.default_rng(sum(case[:6]) + 1)

    def normal(*shape):
        return torch.randn(shape, generator=g).to(dt).cuda()

    nq, nk = [n] * B, [m] * B
    if layout in ("padded", "packed"):
        nq = [n] + [int(x) for x in rng.integers(1, n + 1, B - 1)]
        nk = [m] + [max(0, x + int(rng.integers(m - n - 2, m - n + 1))) if m > n or layout == "padded" else x for x in nq[1:]]
        nk = [min(x, m) for x in nk]
    slopes = slopes_of(HQ) if alibi else None
    of = dict(B=B, n=n, m=m, H=H, q_per_kv=G, d=d, dtype=dtype, scale=scale if scale is not None else d ** -0.5, slopes=None if slopes is None else slopes.cuda())
    if layout == "packed":
        tq, tk = sum(nq), sum(nk)
        if tq == tk:  # one fused projection, and a gap behind
            x = normal(tq, HQ + 2 * H + 1, d)
            Q, K, V = x[:, :HQ], x[:, HQ:HQ + H], x[:, HQ + H:HQ + 2 * H]
        else:
            Q, K, V = normal(tq, HQ, d), normal(tk, H, d), normal(tk, H, d)
        out = torch.full((tq + 2, HQ, d), 7.0, dtype=dt, device="cuda")
        qs, ks = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (nq, nk))
        p = kf.Prompt(q_start=torch.from_numpy(qs).cuda(), k_start=torch.from_numpy(ks).cuda(), q_stride=(0, d, Q.stride(0)), k_stride=(0, d, K.stride(0)),
                      v_stride=(0, d, V.stride(0)), out_stride=(0, d, HQ * d), **of)
        views = [(Q[qs[b]:qs[b + 1]].transpose(0, 1), K[ks[b]:ks[b + 1]].transpose(0, 1), V[ks[b]:ks[b + 1]].transpose(0, 1), out[qs[b]:qs[b + 1]].transpose(0, 1)) for b in range(B)]
    else:
        cap = m + 13 if layout == "cache" else m
        Q, K, V = normal(B, HQ, n, d), normal(B, H, cap, d), normal(B, H, cap, d)
        if layout == "cache":  # rows behind the prompt belong to nobody
            K[:, :, m:], V[:, :, m:] = math.nan, math.inf
            of["k_stride"] = of["v_stride"] = K.stride()[:3]
            out = torch.full((B, HQ, n, d), 7.0, dtype=dt, device="cuda")
            of["out_stride"] = out.stride()[:3]
        else:
            out = torch.full((B, n, HQ, d), 7.0, dtype=dt, device="cuda")
        if layout == "padded":
            of["seq_n"], of["seq_m"] = (torch.tensor(x, dtype=torch.int32).cuda() for x in (nq, nk))
            for b in range(B):
                Q[b, :, nq[b]:], K[b, :, nk[b]:], V[b, :, nk[b]:] = math.nan, math.inf, math.nan
        p = kf.Prompt(**of)
        heads = out if layout == "cache" else out.transpose(1, 2)
        views = [(Q[b, :, :nq[b]], K[b, :, :nk[b]], V[b, :, :nk[b]], heads[b, :, :nq[b]]) for b in range(B)]
    return p, (Q, K, V, out), views, slopes, dt


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c)))
def test_attention_matches_the_definition(case):
    p, (Q, K, V, out), views, slopes, dt = make(case)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    torch.cuda.synchronize()
    for b, (q, k, v, o) in enumerate(views):
        want, tol = oracle(q.cpu(), k.cpu(), v.cpu(), p.scale, slopes, p.q_per_kv, dt)
        near(o, want, tol, (case, b))
        o.fill_(7.0)
    assert bool((out == 7.0).all())  # nothing else was written


MANY = [  # workgroups of 128 rows; heads that are a multiple of the XCDs and heads that are none
    (64, 130, 130, 16, 1, 128, kf.BF16, False, "padded"),
    (64, 130, 130, 16, 1, 128, kf.F16, True, "plain"),
    (64, 129, 140, 16, 1, 64, kf.BF16, True, "padded"),
    (64, 130, 130, 16, 1, 64, kf.F16, False, "packed"),
    (64, 130, 130, 16, 1, 64, kf.F32, True, "cache"),
    (32, 130, 130, 16, 1, 256, kf.BF16, True, "packed"),
    (32, 140, 200, 16, 1, 256, kf.F16, False, "padded"),
    (32, 70, 97, 8, 4, 128, kf.F32, False, "padded"),     # three blocks of 128 rows of four heads each, cut through a position
    (39, 70, 70, 9, 5, 64, kf.BF16, False, "packed"),
    (8, 2100, 2100, 8, 1, 128, kf.BF16, True, "plain"),   # far keys are looked for
    (5, 2100, 2111, 7, 2, 64, kf.F16, True, "padded"),    # blocks of a head dealt out over XCDs
    (5, 4100, 4100, 7, 1, 128, kf.BF16, False, "packed"),
]


def takes_128_rows(p):
    """The rule by which a call does."""
    return p.B * p.H * -(-p.n * p.q_per_kv // 128) >= (512 if p.d * (4 if p.dtype == kf.F32 else 2) > 256 else 1024)


@pytest.mark.gpu
@pytest.mark.parametrize("case", MANY, ids=lambda c: "x".join(map(str, c)))
def test_workgroups_of_128_rows_match_the_definition(case):
    p, (Q, K, V, out), views, slopes, dt = make(case)
    assert takes_128_rows(p)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    torch.cuda.synchronize()
    assert not bool((torch.cat([o.reshape(-1) for *_, o in views]).reshape(-1, p.d) == 7.0).all(1).any())  # every row was written
    for b, (q, k, v, o) in enumerate(views):
        G = p.q_per_kv
        for h in range(p.H) if p.n < 1000 else ((b + 3) % p.H,) if b < 3 or b == p.B - 1 else ():
            at = slice(h * G, h * G + G)
            want, tol = oracle(q[at].cpu(), k[h:h + 1].cpu(), v[h:h + 1].cpu(), p.scale, None if slopes is None else slopes[at], G, dt)
            near(o[at], want, tol, (case, b, h))
        o.fill_(7.0)
    assert bool((out == 7.0).all())  # nothing else was


@pytest.mark.gpu
@pytest.mark.parametrize("B,dtype,d", [(64, kf.BF16, 128), (64, kf.F16, 64), (32, kf.BF16, 256), (32, kf.F32, 128)])
def test_what_rows_of_a_workgroup_of_128_do_not_see_does_not_reach_them(B, dtype, d):
    n, m = 150, 190
    p, (Q, K, V, out), views, _, dt = make((B, n, m, 16, 1, d, dtype, False, "plain"))
    assert takes_128_rows(p)
    ws = kf.new_prompt_workspace(p)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=ws)
    clean = out.clone()
    for j in (0, m - n, m - n + 1, 90, 127, 128, m - 2, m - 1):
        first = max(0, j - (m - n))
        for tensor, value in ((V, math.nan), (V, math.inf), (K, math.nan)):
            keep = tensor[7, 5, j].clone()
            tensor[7, 5, j, 9] = value
            out.fill_(7.0)
            kf.kf_prompt_attend(p, Q, K, V, out, workspace=ws)
            tensor[7, 5, j] = keep
            got, was = out[7, :, 5].clone(), clean[7, :, 5]
            out[7, :, 5] = was
            assert torch.equal(out, clean)
            # a row that does not see it: sums as they were, but for the terms' order (their 2 * (m + 64) U of at most |v| = 6)
            near(got[:first], was[:first].double().cpu(), torch.finfo(dt).eps * was[:first].double().cpu().abs() + 12 * (m + 64) * U, (j, value))
            seen = got[first:].float()
            if tensor is K:
                assert bool(torch.isnan(seen).all())
            else:
                assert not bool(torch.isfinite(seen[:, 9]).any()) and bool(torch.isfinite(torch.cat([seen[:, :9], seen[:, 10:]], 1)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.0, -0.125, 40.0])
def test_scales_of_any_sign_and_size(scale):
    p, (Q, K, V, out), views, slopes, dt = make((2, 90, 90, 2, 1, 64, kf.BF16, True, "plain"), scale)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    for b, (q, k, v, o) in enumerate(views):
        want, tol = oracle(q.cpu(), k.cpu(), v.cpu(), scale, slopes, 1, dt)
        near(o, want, tol, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [(kf.BF16, 128), (kf.F16, 64), (kf.F16, 256), (kf.F32, 64)])
@pytest.mark.parametrize("n,m", [(200, 200), (3, 900)])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, d, n, m):
    """NaN and infinity in a value or key: the rows before it are what they were; the rows that see it are no numbers."""
    p, (Q, K, V, out), views, _, dt = make((1, n, m, 2, 1, d, dtype, False, "plain"))
    ws = kf.new_prompt_workspace(p)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=ws)
    clean = out.clone()
    for j in (0, m - n, m - n + 1, m - n // 2, m - 2, m - 1):
        first = max(0, j - (m - n))
        for tensor, value in ((V, math.nan), (V, math.inf), (K, math.nan)):
            keep = tensor[0, 1, j].clone()
            tensor[0, 1, j, 5] = value
            out.fill_(7.0)
            kf.kf_prompt_attend(p, Q, K, V, out, workspace=ws)
            assert torch.equal(out[0, :, 0], clean[0, :, 0])  # the other head
            near(out[0, :first, 1], clean[0, :first, 1].double().cpu(), 4 * torch.finfo(dt).eps * clean[0, :first, 1].double().cpu().abs() + 1e-3 * (dt != torch.float32) + 1e-5, (j, value))
            seen = out[0, first:, 1].float()
            if tensor is K:
                assert bool(torch.isnan(seen).all())
            else:
                assert not bool(torch.isfinite(seen[:, 5]).any())
                others = torch.cat([seen[:, :5], seen[:, 6:]], 1)
                assert bool(torch.isfinite(others).all())
            tensor[0, 1, j] = keep


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,H,G,n,m,packed", [(kf.BF16, 128, 2, 1, 2300, 2300, False), (kf.F16, 64, 1, 4, 700, 2100, False), (kf.F32, 64, 1, 2, 1100, 1100, True),
                                                    (kf.BF16, 256, 1, 1, 2048, 2200, True)])
def test_far_keys_are_left_out_only_where_they_cannot_matter(dtype, d, H, G, n, m, packed):
    """Slopes from steep to none and rising ones, a far key that is long, far keys and values that are no numbers: as the definition has it."""
    dt, HQ, g = TYPES[dtype], H * G, torch.Generator().manual_seed(n)
    Q, K, V = (torch.randn((h, r, d), generator=g).to(dt) for h, r in ((HQ, n), (H, m), (H, m)))
    scale = d ** -0.5
    slopes = torch.tensor([0.9, 0.02, 0.3, 0.0][:HQ])
    start = torch.tensor([0, n], dtype=torch.int32), torch.tensor([0, m], dtype=torch.int32)

    def run(slopes):
        out = torch.zeros((1, n, HQ, d), dtype=dt, device="cuda")
        of = dict(B=1, n=n, m=m, H=H, q_per_kv=G, d=d, dtype=dtype, scale=scale, slopes=slopes.cuda())
        if packed:
            p = kf.Prompt(q_start=start[0].cuda(), k_start=start[1].cuda(), **of)
            args = [x.transpose(0, 1).contiguous().cuda() for x in (Q, K, V)]
        else:
            p, args = kf.Prompt(**of), [x[None].cuda() for x in (Q, K, V)]
        assert binding.lib().kf_prompt_workspace_bytes(p.c_struct()) > 256  # it is long enough to look for far keys
        kf.kf_prompt_attend(p, *args, out, workspace=kf.new_prompt_workspace(p))
        return out[0].transpose(0, 1)

    def check(slopes, what):
        want, tol = oracle(Q, K, V, scale, slopes, G, dt)
        near(run(slopes), want, tol, what)

    check(slopes, "slopes")
    check(torch.full((HQ,), -0.004), "rising")
    far = m // 50
    keep = K[:, far].clone()
    K[:, far] = Q[::G, n - 1] * 40.0  # a key that the last row asks for, far away
    check(torch.full((HQ,), 0.1), "a long far key")
    K[:, far] = keep
    steep = torch.full((HQ,), 0.9)
    clean = run(steep).double().cpu()
    first = max(0, far - (m - n))
    for tensor, value in ((V, math.inf), (V, math.nan), (K, math.nan)):
        keep = tensor[0, far].clone()
        tensor[0, far, 3] = value
        got = run(steep).double().cpu()
        assert bool(torch.isfinite(got[:G, :first]).all()) and torch.equal(got[G:], clean[G:])
        bad = got[:G, first:, 3] if tensor is V else got[:G, first:]
        assert not bool(torch.isfinite(bad).any())
        tensor[0, far] = keep


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d,n,m,big", [(kf.F32, 64, 2304, 2304, 1e20), (kf.BF16, 128, 2304, 2304, 2.0 ** 34), (kf.BF16, 64, 2100, 2500, 1e30), (kf.F16, 64, 2304, 2304, 6e4)])
def test_far_values_that_are_large_and_elements_that_only_far_keys_have(dtype, d, n, m, big):
    """What a far key weighs times what it holds: finite values some powers of ten above their neighbours', and neighbours of zeros."""
    dt, g = TYPES[dtype], torch.Generator().manual_seed(m)
    Q, K, V = (torch.randn((1, r, d), generator=g).to(dt) for r in (n, m, m))
    V[0, 64:, 1] = 0.0
    V[0, 1500:1600] = 0.0                       # rows whose own key holds nothing
    alone = V.clone()
    for at in (5, 700):
        V[0, at] = (V[0, at].float() * 0.2 * big).to(dt)
    p = kf.Prompt(1, n, m, 1, d, dtype, 0.02, slopes=torch.tensor([0.02]).cuda())
    ws = kf.new_prompt_workspace(p)
    for v in (V, alone):
        out = torch.zeros((1, n, 1, d), dtype=dt, device="cuda")
        kf.kf_prompt_attend(p, Q[None].cuda(), K[None].cuda(), v[None].cuda(), out, workspace=ws)
        want, tol = oracle(Q, K, v, 0.02, torch.tensor([0.02]), 1, dt)
        near(out[0].transpose(0, 1), want, tol, "far values")


@pytest.mark.gpu
def test_far_keys_that_a_rising_bias_prefers():
    """The far end of a far tile has more of a negative slope than its near end: every row's first key outweighs its own."""
    n, d, slope, g = 2304, 128, -10.0, torch.Generator().manual_seed(3)
    row = torch.arange(n)
    Q = torch.nn.functional.one_hot(row % d, d).bfloat16()[None]
    K = torch.where(row >= n - d, -slope * row - 800.0, 0.0)[:, None].bfloat16() * Q
    V = torch.randn((1, n, d), generator=g).bfloat16()
    out = torch.zeros((1, n, 1, d), dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(1, n, n, 1, d, kf.BF16, 1.0, slopes=torch.tensor([slope]).cuda())
    kf.kf_prompt_attend(p, Q[None].cuda(), K[None].cuda(), V[None].cuda(), out, workspace=kf.new_prompt_workspace(p))
    want, tol = oracle(Q, K, V, 1.0, torch.tensor([slope]), 1, torch.bfloat16)
    near(out[0].transpose(0, 1), want, tol, "rising")


@pytest.mark.gpu
def test_many_light_keys_beside_a_heavy_one():
    """65535 keys of weight 2^-25.5 beside one of weight 1 have 1/700 of a row, in half precision too."""
    H, n, m, d, dt = 64, 256, 65536, 64, torch.float16
    K, V = torch.zeros((1, 1, m, d), dtype=dt), torch.ones((1, 1, m, d), dtype=dt)
    K[0, 0, 7, 0], V[0, 0, 7] = 17.6875, 0.0
    Q = torch.zeros((1, H, n, d), dtype=dt)
    Q[..., 0] = 1.0
    out = torch.zeros((1, n, H, d), dtype=dt, device="cuda")
    p = kf.Prompt(1, n, m, H, d, kf.F16, 1.0, k_stride=(0, 0, d), v_stride=(0, 0, d))
    kf.kf_prompt_attend(p, Q.cuda(), K.cuda(), V.cuda(), out, workspace=kf.new_prompt_workspace(p))
    light = (m - n + torch.arange(n)).double() * math.exp(-17.6875)
    want = (light / (1 + light))[:, None, None].expand(n, H, d)
    # a term's 2^-21 and 2^-12, the sums' (m + 64) U, and the row's rounding: 2^-12 (halves as small as 2^-10 are normal)
    near(out[0], want, want * (2.0 ** -21 + 2.0 ** -11 + (m + 64) * U), "light")


@pytest.mark.gpu
def test_keys_at_minus_infinity_and_sequences_that_are_none():
    d, n = 64, 40
    Q = torch.ones((1, 1, n, d), dtype=torch.bfloat16, device="cuda")
    K, V = torch.zeros_like(Q), torch.randn((1, 1, n, d), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    K[0, 0, :7, 0] = -math.inf   # the first rows see nothing else
    K[0, 0, 20, 3] = -math.inf
    out = torch.zeros((1, n, 1, d), dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(1, n, n, 1, d, kf.BF16, 1.0)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    assert bool((out[0, :7] == 0).all())
    use = torch.tensor([j >= 7 and j != 20 for j in range(n)])
    for i in (7, 19, 20, 39):
        mean = V[0, 0, :i + 1][use[:i + 1].cuda()].double().mean(0)
        assert bool(((out[0, i, 0].double() - mean).abs() <= 2.0 ** -7 * (mean.abs() + V[0, 0].double().abs().amax(0))).all())
    # lengths that are none leave their sequences out
    B = 5
    Q, K, V = (torch.randn((B, 2, 9, d), generator=torch.Generator().manual_seed(x)).half().cuda() for x in range(3))
    out = torch.full((B, 9, 2, d), 7.0, dtype=torch.float16, device="cuda")
    lens = [torch.tensor(x, dtype=torch.int32).cuda() for x in ([9, 0, 10, 4, -1], [9, 9, 9, 0, 9])]
    p = kf.Prompt(B, 9, 9, 2, d, kf.F16, 0.1, seq_n=lens[0], seq_m=lens[1])
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    want, tol = oracle(Q[0].cpu(), K[0].cpu(), V[0].cpu(), 0.1, None, 1, torch.float16)
    near(out[0].transpose(0, 1), want, tol, "whole")
    assert bool((out[1:3] == 7.0).all()) and bool((out[3, :4] == 0.0).all()) and bool((out[3, 4:] == 7.0).all()) and bool((out[4] == 7.0).all())
    starts = torch.tensor([0, 9, 9, 5, 14, 18], dtype=torch.int32).cuda()  # one empty, one that runs backwards
    q, k, v = (x.transpose(1, 2).reshape(-1, 2, d) for x in (Q, K, V))
    out = torch.full((45, 2, d), 7.0, dtype=torch.float16, device="cuda")
    p = kf.Prompt(B, 9, 9, 2, d, kf.F16, 0.1, q_start=starts, k_start=starts)
    kf.kf_prompt_attend(p, q, k, v, out, workspace=kf.new_prompt_workspace(p))
    for a, e in ((0, 9), (5, 14), (14, 18)):
        if a != 0:
            want, tol = oracle(q[a:e].transpose(0, 1).cpu(), k[a:e].transpose(0, 1).cpu(), v[a:e].transpose(0, 1).cpu(), 0.1, None, 1, torch.float16)
            near(out[a:e].transpose(0, 1)[:, -4:], want[:, -4:], tol[:, -4:], (a, e))
    assert bool((out[18:] == 7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("n,m", [(40, 40), (40, 600), (3, 3000), (2, 130)])
def test_rows_at_minus_infinity_are_zero_whatever_their_values_hold(n, m):
    """Rows that see keys, all of them at minus infinity: walked whole, by waves that share them, and in parts."""
    d = 64
    Q = torch.ones((1, 1, n, d), dtype=torch.bfloat16, device="cuda")
    K, V = torch.zeros((1, 1, m, d), dtype=torch.bfloat16, device="cuda"), torch.ones((1, 1, m, d), dtype=torch.bfloat16, device="cuda")
    K[..., 0] = -math.inf
    K[0, 0, -1, 0] = 0.0                         # the last row sees one that is not
    V[0, 0, ::3, 5], V[0, 0, 1::3, 6] = math.inf, math.nan
    V[0, 0, -1] = 3.0
    out = torch.full((1, n, 1, d), 7.0, dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(1, n, m, 1, d, kf.BF16, 1.0)
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    assert bool((out[0, :-1] == 0).all())
    assert bool((out[0, -1, 0, :5] == 3.0).all()) and bool((out[0, -1, 0, 7:] == 3.0).all())


@pytest.mark.gpu
def test_far_rows_pass_32_bits():
    """Keys whose byte offsets lie beyond 2^32: a head's rows far apart."""
    d, m, step = 128, 40, 1 << 26  # elements between tokens
    flat = torch.zeros(step * (m - 1) + d, dtype=torch.bfloat16, device="cuda")
    K = torch.as_strided(flat, (1, 1, m, d), (0, 0, step, 1))
    g = torch.Generator().manual_seed(1)
    K.copy_(torch.randn((1, 1, m, d), generator=g).bfloat16())
    Q, V = (torch.randn((1, 1, m, d), generator=g).bfloat16().cuda() for _ in range(2))
    out = torch.zeros((1, m, 1, d), dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(1, m, m, 1, d, kf.BF16, 0.1, k_stride=(0, 8, step))
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    want, tol = oracle(Q[0].cpu(), K[0].cpu(), V[0].cpu(), 0.1, None, 1, torch.bfloat16)
    near(out[0].transpose(0, 1), want, tol, "far")


@pytest.mark.gpu
def test_far_rows_pass_32_bits_inside_a_tile():
    """Tiles of 128 keys whose tokens lie 2^27 bytes apart, shared by workgroups of eight waves."""
    H, n, m, d, step = 40, 128, 130, 64, 1 << 26
    flat = torch.empty(step * (m - 1) + 2 * H * d, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.as_strided(flat, (1, H, m, d), (0, d, step, 1), i * H * d) for i in range(2))
    g = torch.Generator().manual_seed(2)
    for x in (K, V):
        x.copy_(torch.randn((1, H, m, d), generator=g).bfloat16())
    Q = torch.randn((1, H, n, d), generator=g).bfloat16().cuda()
    out = torch.zeros((1, n, H, d), dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(1, n, m, H, d, kf.BF16, 0.1, k_stride=(0, d, step), v_stride=(0, d, step))
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    want, tol = oracle(Q[0].cpu(), K[0].cpu(), V[0].cpu(), 0.1, None, 1, torch.bfloat16)
    near(out[0].transpose(0, 1), want, tol, "far")


@pytest.mark.gpu
def test_far_rows_pass_32_bits_inside_a_tile_of_eight_waves():
    """More than 512 keys, 2^27 bytes apart, and 65 to 256 workgroups: eight waves bring 64 rows of a tile of 128 at once."""
    H, n, m, d, step = 80, 9, 520, 64, 1 << 26
    flat = torch.empty(step * (m - 1) + 2 * H * d, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.as_strided(flat, (1, H, m, d), (0, d, step, 1), i * H * d) for i in range(2))
    g = torch.Generator().manual_seed(2)
    for x in (K, V):
        x.copy_(torch.randn((1, H, m, d), generator=g).bfloat16())
    Q = torch.randn((1, H, n, d), generator=g).bfloat16().cuda()
    out = torch.zeros((1, n, H, d), dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(1, n, m, H, d, kf.BF16, 0.1, k_stride=(0, d, step), v_stride=(0, d, step))
    kf.kf_prompt_attend(p, Q, K, V, out, workspace=kf.new_prompt_workspace(p))
    want, tol = oracle(Q[0].cpu(), K[0].cpu(), V[0].cpu(), 0.1, None, 1, torch.bfloat16)
    near(out[0].transpose(0, 1), want, tol, "far")


@pytest.mark.gpu
def test_replayed_graph_and_another_stream():
    for case in ((2, 130, 130, 2, 2, 128, kf.BF16, False, "plain"), (1, 2, 2000, 2, 1, 128, kf.BF16, False, "plain")):
        p, (Q, K, V, out), views, _, dt = make(case)
        ws = kf.new_prompt_workspace(p)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            kf.kf_prompt_attend(p, Q, K, V, out, workspace=ws)
        torch.cuda.current_stream().wait_stream(s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kf.kf_prompt_attend(p, Q, K, V, out, workspace=ws)
        for i in range(4):
            Q.copy_(torch.randn(Q.shape, generator=torch.Generator().manual_seed(i)).to(dt))
            eager = torch.zeros_like(out)
            kf.kf_prompt_attend(p, Q, K, V, eager, workspace=ws)
            out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager)


@pytest.mark.gpu
def test_a_prompts_layer_from_projection_to_reduced_cache():
    """kf_norm_rotate -> kf_prompt_attend and kf_prefill_score on the same rows -> kf_select_evict_into, padded prompts."""
    B, n, H, G, d = 3, 150, 2, 2, 128
    g = torch.Generator().manual_seed(9)
    x = torch.randn((B, n, (G + 2) * H, d), generator=g).bfloat16().cuda()
    lens = [150, 64, 97]
    seq = torch.tensor(lens, dtype=torch.int32).cuda()
    freq = (10000.0 ** (-torch.arange(32).float() / 32)).cuda()
    q, k, v = x[:, :, :G * H], x[:, :, G * H:(G + 1) * H], x[:, :, (G + 1) * H:]
    stage = kf.Cache.allocate(1, B, H, d, n, kf.BF16, q_per_kv=G)
    Q = torch.zeros((B, H * G, n, d), dtype=torch.bfloat16, device="cuda")
    st = dict(q_stride=q.stride()[:2], k_stride=k.stride()[:2], v_stride=v.stride()[:2])
    kf.kf_norm_rotate(kf.Rows(B=B, n=n, H=H, d=d, dtype=kf.BF16, q_per_kv=G, rotate=kf.ROTATE_HALVES, rot_dim=64, inv_freq=freq, seq_n=seq, **st), q, k, v, Q,
                      stage.K[0], stage.V[0])
    out = torch.zeros((B, n, H * G, d), dtype=torch.bfloat16, device="cuda")
    p = kf.Prompt(B=B, n=n, m=n, H=H, q_per_kv=G, d=d, dtype=kf.BF16, scale=d ** -0.5, seq_n=seq, seq_m=seq)
    kf.kf_prompt_attend(p, Q, stage.K[0], stage.V[0], out, workspace=kf.new_prompt_workspace(p))
    ws = kf.new_workspace(stage, n)
    seeds = torch.arange(B, dtype=torch.int64, device="cuda")
    kf.kf_prefill_score(stage, Q, n, 1.0, d ** -0.5, kf.NOISE_GUMBEL, seeds, workspace=ws, seq_n=seq)
    cache = kf.Cache.allocate(1, B, H, d, 65, kf.BF16, q_per_kv=G)
    kf.kf_select_evict_into(stage, cache, 0, 64, 16, workspace=ws)
    assert cache.len.flatten().tolist() == [64] * (B * H)
    for b in range(B):
        want, tol = oracle(Q[b, :, :lens[b]].cpu(), stage.K[0, b, :, :lens[b]].cpu(), stage.V[0, b, :, :lens[b]].cpu(), d ** -0.5, None, G, torch.bfloat16)
        near(out[b, :lens[b]].transpose(0, 1), want, tol, b)
        assert bool((out[b, lens[b]:] == 0).all())


@pytest.mark.gpu
def test_calls_at_once_and_twice_are_the_same_to_the_bit():
    """Two prompts on two streams with a workspace each, over and over: shared-out keys, far keys and whole walks."""
    g, calls = torch.Generator().manual_seed(4), []
    for B, n, m, H, G, slopes in ((2, 30, 3000, 4, 2, None), (1, 2100, 2100, 2, 1, slopes_of(2).cuda()), (3, 500, 500, 8, 1, None)):
        Q, K, V = (torch.randn((B, h, r, 128), generator=g).bfloat16().cuda() for h, r in ((H * G, n), (H, m), (H, m)))
        p = kf.Prompt(B, n, m, H, 128, kf.BF16, 0.09, q_per_kv=G, slopes=slopes)
        out = [torch.zeros((B, n, H * G, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        calls.append((p, (Q, K, V), out, kf.new_prompt_workspace(p)))
        kf.kf_prompt_attend(p, Q, K, V, out[0], workspace=calls[-1][3])
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (p, x, out, ws) in zip(streams, calls):
            with torch.cuda.stream(s):
                kf.kf_prompt_attend(p, *x, out[1], workspace=ws)
    torch.cuda.synchronize()
    for p, x, out, ws in calls:
        assert bool(out[0].any()) and torch.equal(out[0], out[1])
