"""Operators around a reduced cache, as cases that can be timed and compared with their plain form.

Three groups of calls, each through the package's public functions:

  beam    one selection of a beam search (kf_beam_select): log-probabilities of every beam's next token, the best
          continuations of each request, numbered so that kf_beam_fork can take them
  rotate  a projection's rows on their way to the caches (kf_norm_rotate): per-head norm of queries and keys,
          position rotation, and the turn from token-major to head-major rows
  step    one generation step (kf_decode_select_step) over a cache whose keys and values are held in 4 bits
  evict   the eviction after the prompt into such a cache (kf_select_evict_into): 16-bit rows -> 4-bit rows

A 4-bit row of d elements is d/2 bytes of codes (element c in byte c/2, even elements in the low half; sign, then the
magnitudes 0 1/2 1 3/2 2 3 4 6) and 16 scale bytes: byte g, less 127, is the exponent of two that the elements
[g*d/16, (g+1)*d/16) are multiplied by -- the smallest with which none of them is above 7.  Which bytes a row gets is
therefore fixed to the bit, and the caches are returned as the bytes they are.

Sizes are those of kf_workloads.CONFIGS (a layer, or a few layers, of them) or generic.
"""
import math

import numpy as np
import torch

own = False

RING = 8  # distinct generated tokens that the steps take in turn
TAU = (1.0, 2.0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _beam(name, R, W, V, dtype, ended=False, masked=0.0):
    return {"name": name, "call": "beam", "R": R, "W": W, "V": V, "dtype": dtype, "ended": ended, "masked": masked}


def _rotate(name, B, n, H, G, d, dtype, style, rot, norm, kv_rows, far=0, padded=False):
    return {"name": name, "call": "rotate", "B": B, "n": n, "H": H, "G": G, "d": d, "dtype": dtype, "style": style, "rot": rot,
            "norm": norm, "kv_rows": kv_rows, "far": far, "padded": padded}


def _step(name, L, B, H, d, k, w, n, T, dtype="bf16", layout="slot", G=1, alibi=False, outliers=0.0):
    return {"name": name, "call": "step", "L": L, "B": B, "H": H, "d": d, "k": k, "w": w, "n": n, "T": T, "dtype": dtype,
            "layout": layout, "G": G, "alibi": alibi, "outliers": outliers}


def _evict(name, L, B, H, d, n, k, w, dtype="bf16"):
    return {"name": name, "call": "evict", "L": L, "B": B, "H": H, "d": d, "n": n, "k": k, "w": w, "dtype": dtype}


def listed():
    return [
        # one request of 4 beams over a vocabulary of odd size: the rows are not aligned
        _beam("beam_request", 1, 4, 50257, "bf16"),
        # a serving batch, logits as a 32-bit head leaves them
        _beam("beam_batch", 64, 4, 50304, "f32"),
        # many beams, a large vocabulary of which a grammar rules out most, some hypotheses at their end
        _beam("beam_wide", 16, 16, 128000, "f16", ended=True, masked=0.7),
        # one generated token of a model that rotates neighbouring pairs of a quarter of each head: the smallest call
        _rotate("rotate_token", 1, 1, 16, 1, 256, "bf16", "pairs", 64, False, 1, far=2500),
        # one generated token of each sequence of a large batch, far into their texts, with normed heads
        _rotate("rotate_batch_token", 64, 1, 32, 1, 128, "bf16", "halves", 128, True, 1, far=100000),
        # the prompts of one layer, padded, straight into the cache that prompt scoring reads: the most bytes
        _rotate("rotate_prompts", 8, 4096, 32, 1, 128, "bf16", "halves", 128, True, 4096, padded=True),
        # grouped queries in half precision, odd lengths, half of each head rotated
        _rotate("rotate_grouped", 3, 1501, 8, 4, 64, "f16", "halves", 32, True, 1600, far=70),
        # serving one sequence: a layer of wide heads, one call
        _step("q4_token", 1, 1, 16, 256, 1024, 205, 2048, 512, outliers=0.01),
        # one layer of a large batch
        _step("q4_layer_step", 1, 64, 32, 128, 1024, 205, 2048, 1024),
        # eight layers with position bias in one call: the largest step
        _step("q4_layers_step", 8, 8, 32, 128, 2048, 410, 4096, 1024, alibi=True),
        # grouped queries in half precision, rows kept in order, a budget that is no multiple of anything
        _step("q4_grouped_ordered", 2, 8, 8, 128, 1501, 300, 3002, 512, dtype="f16", layout="ordered", G=4),
        # the eviction after the prompts of one layer
        _evict("q4_evict_layer", 1, 16, 32, 128, 2048, 1024, 205),
    ]


def draw(rng):
    """One more case: sizes over the whole range, their logarithms even."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("beam", "rotate", "step", "step", "evict"))
    if kind == "beam":
        V, W = log(200, 150000), log(1, 16)
        case = _beam("", max(1, min(log(1, 128), int(3e7 / (W * V)))), W, V, rng.choice(("f32", "bf16", "f16")), rng.random() < 0.5,
                     rng.choice((0.0, 0.0, 0.9)))
    elif kind == "rotate":
        d, H, G = rng.choice((64, 128, 256)), rng.choice((2, 8, 12, 16, 32)), rng.choice((1, 1, 2, 4, 8))
        n = rng.choice((1, log(2, 6000)))
        B = max(1, min(log(1, 64), int(1.2e8 / (n * H * (G + 2) * d))))
        rot = rng.choice((d, d // 2, d // 4, 2 * log(1, d // 2)))
        case = _rotate("", B, n, H, G, d, rng.choice(("bf16", "bf16", "f16", "f32")) if d < 256 else rng.choice(("bf16", "f16")),
                       rng.choice(("pairs", "halves")), rot, rng.random() < 0.5, n + rng.choice((0, 1, log(1, 1000))), log(1, 100000),
                       rng.random() < 0.3)
    else:
        d, H, B = rng.choice((64, 128, 128, 256)), rng.choice((2, 8, 12, 16, 32)), log(1, 64)
        dtype = rng.choice(("bf16", "bf16", "f16"))
        if kind == "step":
            k, G = log(64, 9830), rng.choice((1, 1, 1, 2, 4, 8))
            B = max(1, min(B, int(5e8 / (H * k * d))))
            L = max(1, min(log(1, 16), int(5e8 / (B * H * k * d))))
            case = _step("", L, B, H, d, k, int(k * rng.uniform(0.05, 0.4)), 2 * k, 1024, dtype, rng.choice(("slot", "slot", "ordered")), G,
                         rng.random() < 0.3, rng.choice((0.0, 0.005, 0.01)))
        else:
            n = log(100, 20000)
            k = max(2, int(n * rng.uniform(0.2, 0.6)))
            B = max(1, min(B, int(2e8 / (H * n * d))))
            case = _evict("", max(1, min(log(1, 4), int(2e8 / (B * H * n * d)))), B, H, d, n, k, int(k * rng.uniform(0.05, 0.4)), dtype)
    del case["name"]
    return case


# ---------------------------------------------------------------- inputs
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + stream * 7919 + 20240309) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(shape, dt, g):
    return torch.randn(shape, generator=g, device="cuda").to(dt)


def _scale_rows(K, frac, g):
    """A share of the key rows four times as long: the tokens that attract attention."""
    return K if frac <= 0 else K * torch.where(torch.rand(K.shape[:-1], generator=g, device="cuda") < frac, 4.0, 1.0).to(K.dtype).unsqueeze(-1)


def _pack(x):
    """[..., d] in any floating type -> [..., d/2 + 16] bytes."""
    d = x.shape[-1]
    v = x.float().unflatten(-1, (16, d // 16))
    m, e = torch.frexp(v.abs().amax(-1))                      # m in [1/2, 1): largest = m * 2^e
    e = torch.where(m == 0, torch.full_like(e, -126), torch.where(m <= 0.875, e - 3, e - 2).clamp(-126, 125))
    y = torch.ldexp(v.abs(), -e.unsqueeze(-1))
    code = (y > 0.25).byte() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0) + 8 * torch.signbit(v).byte()
    code = code.flatten(-2).unflatten(-1, (d // 2, 2))
    return torch.cat([code[..., 0] + 16 * code[..., 1], (e + 127).byte()], -1)


def _values(d):
    """The two elements that each of the 256 code bytes stands for."""
    mag = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    both = torch.cat([mag, -mag])
    b = torch.arange(256, device="cuda")
    return torch.stack([both[b & 15], both[b >> 4]], -1)


def _unpack(rows, d):
    """[..., d/2 + 16] bytes -> [..., d] float32."""
    c = _values(d)[rows[..., :d // 2].int()].flatten(-2).unflatten(-1, (16, d // 16))
    return torch.ldexp(c, rows[..., d // 2:].int().sub_(127).unsqueeze(-1)).flatten(-2)


def _slopes(case):
    HQ = case["H"] * case["G"]
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / HQ) for h in range(HQ)], dtype=torch.float32, device="cuda") if case["alibi"] else None


def _scale(case):
    return float(np.float32(1.0) / np.sqrt(np.float32(case["d"])))


def _prepare_beam(case, seed):
    R, W, V = case["R"], case["W"], case["V"]
    g = _gen(seed, 1)
    # a few likely words, a long tail; the beams of a request rank much the same words
    base = torch.randn((R, 1, V), generator=g, device="cuda") * 2.5
    x = base + torch.randn((R, W, V), generator=g, device="cuda")
    if case["masked"] > 0:
        x.masked_fill_(torch.rand((R, 1, V), generator=g, device="cuda") < case["masked"], -math.inf)
    s = {"case": case, "logits": x.view(R * W, V).to(TYPES[case["dtype"]]),
         "score": torch.sort(-20.0 - 4.0 * torch.rand((R, W), generator=g, device="cuda"), descending=True).values.view(-1)}
    s["done"] = (torch.rand(R * W, generator=g, device="cuda") < 0.2).int() if case["ended"] else None
    for name, t in (("parent", torch.int32), ("token", torch.int32), ("rank", torch.int32), ("new_score", torch.float32), ("new_done", torch.int32)):
        s[name] = torch.zeros(R * W, dtype=t, device="cuda")
    return s


def _prepare_rotate(case, seed):
    B, n, H, G, d, rows = (case[x] for x in ("B", "n", "H", "G", "d", "kv_rows"))
    dt, g = TYPES[case["dtype"]], _gen(seed, 2)
    # one fused projection: queries, keys, values of a token side by side
    qkv = _normal((B, n, (G + 2) * H, d), dt, g)
    q, k, v = qkv[:, :, :G * H], qkv[:, :, G * H:G * H + H], qkv[:, :, G * H + H:]
    i = torch.arange(case["rot"] // 2, device="cuda", dtype=torch.float64)
    s = {"case": case, "q": q, "k": k, "v": v, "freq": (10000.0 ** (-2.0 * i / case["rot"])).float(),
         "pos": torch.randint(0, case["far"] + 1, (B,), generator=g, device="cuda", dtype=torch.int32),
         "rows": torch.randint(max(1, n // 4), n + 1, (B,), generator=g, device="cuda", dtype=torch.int32) if case["padded"] else None,
         "qw": None, "kw": None}
    if case["norm"]:
        s["qw"], s["kw"] = ((1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2))
    s["Q"] = torch.zeros((B, H * G, n, d), dtype=dt, device="cuda")
    s["K"], s["V"] = (torch.zeros((B, H, rows, d), dtype=dt, device="cuda") for _ in range(2))
    return s


def _prepare_step(case, seed):
    L, B, H, d, k, w, G = (case[x] for x in ("L", "B", "H", "d", "k", "w", "G"))
    dt, g = TYPES[case["dtype"]], _gen(seed, 3)
    U, cap, t = L * B * H, k + 1, case["T"] // 2  # a run begins in the middle of the generation
    s = {"case": case, "t": t}
    s["K"] = _pack(_scale_rows(_normal((L, B, H, cap, d), dt, g), case["outliers"], g))
    s["V"] = _pack(_normal((L, B, H, cap, d), dt, g))
    # the w newest positions, and k-w of the others; scores: what the key tokens gathered since the prompt, and, in the
    # window, what a token of that age has gathered so far
    q0 = case["n"] + t - 2  # position of the newest cached token
    keys = torch.rand((U, q0 + 1 - w), generator=g, device="cuda").topk(k - w, dim=1).indices.sort(dim=1).values
    pos = torch.zeros((U, cap), dtype=torch.int32, device="cuda")
    pos[:, :k - w] = keys.int()
    pos[:, k - w:k] = torch.arange(q0 + 1 - w, q0 + 1, device="cuda", dtype=torch.int32)
    noise = torch.randn((U, k), generator=g, device="cuda")
    score = torch.zeros((U, cap), dtype=torch.float32, device="cuda")
    score[:, :k - w] = 0.3 + torch.exp(0.7 * noise[:, :k - w])
    age = torch.arange(w, 0, -1, device="cuda", dtype=torch.float32) / (k + 1)
    score[:, k - w:k] = age * torch.exp(0.4 * noise[:, k - w:])
    if case["layout"] == "slot":  # the entries in any order, as a generation in this layout leaves them
        perm = torch.rand((U, k), generator=g, device="cuda").argsort(dim=1)
        pos[:, :k], score[:, :k] = pos[:, :k].gather(1, perm), score[:, :k].gather(1, perm)
    s["pos"], s["score"] = pos.view(L, B, H, cap), score.view(L, B, H, cap)
    s["len"] = torch.full((L, B, H), k, dtype=torch.int32, device="cuda")
    s["q"] = _normal((RING, L, B, H * G, d), dt, g)
    s["kn"] = _scale_rows(_normal((RING, L, B, H, d), dt, g), case["outliers"], g)
    s["vn"] = _normal((RING, L, B, H, d), dt, g)
    s["out"] = torch.zeros((L, B, H * G, d), dtype=torch.float32, device="cuda")
    s["seeds"] = torch.arange(B, dtype=torch.int64, device="cuda") ^ (20240309 + int(seed))
    s["slopes"] = _slopes(case)
    return s


def _prepare_evict(case, seed):
    L, B, H, d, n, k = (case[x] for x in ("L", "B", "H", "d", "n", "k"))
    dt, g = TYPES[case["dtype"]], _gen(seed, 4)
    U = L * B * H
    s = {"case": case, "K": _normal((L, B, H, n, d), dt, g), "V": _normal((L, B, H, n, d), dt, g)}
    # column sums of a causal softmax: a token that i rows see gathers about log(n/i), widely spread
    mean = torch.log(n / (torch.arange(n, device="cuda", dtype=torch.float32) + 1.0)) + 1.0 / n
    s["score"] = (mean * torch.exp(0.8 * torch.randn((U, n), generator=g, device="cuda"))).view(L, B, H, n)
    s["pos"] = torch.arange(n, device="cuda", dtype=torch.int32).expand(L, B, H, n).contiguous()
    s["len"] = torch.full((L, B, H), n, dtype=torch.int32, device="cuda")
    s["K4"], s["V4"] = (torch.zeros((L, B, H, k + 1, d // 2 + 16), dtype=torch.uint8, device="cuda") for _ in range(2))
    s["score4"], s["pos4"] = (torch.zeros((L, B, H, k + 1), dtype=t, device="cuda") for t in (torch.float32, torch.int32))
    s["len4"] = torch.zeros((L, B, H), dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    return {"beam": _prepare_beam, "rotate": _prepare_rotate, "step": _prepare_step, "evict": _prepare_evict}[case["call"]](case, seed)


# ---------------------------------------------------------------- the framework's calls
def _own_beam(kf, s):
    case = s["case"]
    if "cfg" not in s:
        s["cfg"] = kf.Beams(R=case["R"], W=case["W"], V=case["V"], dtype=_code(kf, case), eos=2 if case["ended"] else -1)
        s["ws"] = kf.new_beam_workspace(s["cfg"])
    kf.kf_beam_select(s["cfg"], s["logits"], s["score"], s["parent"], s["token"], s["new_score"], done=s["done"],
                      new_done=s["new_done"] if case["ended"] else None, rank=s["rank"], workspace=s["ws"])
    return {x: s[x] for x in ("parent", "token", "rank", "new_score", "new_done")}


def _own_rotate(kf, s):
    case = s["case"]
    if "cfg" not in s:
        q, k, v = s["q"], s["k"], s["v"]
        s["cfg"] = kf.Rows(B=case["B"], n=case["n"], H=case["H"], d=case["d"], dtype=_code(kf, case), q_per_kv=case["G"], kv_rows=case["kv_rows"],
                           q_stride=q.stride()[:2], k_stride=k.stride()[:2], v_stride=v.stride()[:2], q_weight=s["qw"], k_weight=s["kw"],
                           eps=1e-6, rotate=kf.ROTATE_PAIRS if case["style"] == "pairs" else kf.ROTATE_HALVES, rot_dim=case["rot"],
                           inv_freq=s["freq"], seq_pos=s["pos"], seq_n=s["rows"])
    kf.kf_norm_rotate(s["cfg"], s["q"], s["k"], s["v"], s["Q"], s["K"], s["V"])
    return {x: s[x] for x in ("Q", "K", "V")}


def _code(kf, case, cached=False):
    return {"f32": kf.F32, "bf16": kf.BF16_Q4 if cached else kf.BF16, "f16": kf.F16_Q4 if cached else kf.F16}[case["dtype"]]


def _own_step(kf, s):
    case = s["case"]
    if "cache" not in s:
        s["cache"] = kf.Cache(K=s["K"], V=s["V"], score=s["score"], pos=s["pos"], len=s["len"], L=case["L"], B=case["B"], H=case["H"], d=case["d"],
                              cap=case["k"] + 1, dtype=_code(kf, case, True), q_per_kv=case["G"])
        s["ws"] = kf.new_workspace(s["cache"])
    t, r = s["t"], s["t"] % RING
    s["t"] += 1
    kf.kf_decode_select_step(s["cache"], s["q"][r], s["kn"][r], s["vn"][r], case["n"] + t - 1, case["k"] + 1,
                             kf.kf_tau(min(t, case["T"]), case["T"], *TAU), _scale(case), kf.NOISE_GUMBEL, s["seeds"], s["slopes"], s["out"],
                             k=case["k"], w=case["w"], layout=kf.LAYOUT_SLOT if case["layout"] == "slot" else kf.LAYOUT_ORDERED, workspace=s["ws"])
    return _live(s, case["k"])


def _own_evict(kf, s):
    case = s["case"]
    if "src" not in s:
        of = dict(L=case["L"], B=case["B"], H=case["H"], d=case["d"])
        s["src"] = kf.Cache(K=s["K"], V=s["V"], score=s["score"], pos=s["pos"], len=s["len"], cap=case["n"], dtype=_code(kf, case), **of)
        s["dst"] = kf.Cache(K=s["K4"], V=s["V4"], score=s["score4"], pos=s["pos4"], len=s["len4"], cap=case["k"] + 1, dtype=_code(kf, case, True), **of)
        s["ws"] = kf.new_workspace(s["src"])
    kf.kf_select_evict_into(s["src"], s["dst"], 0, case["k"], case["w"], None, s["ws"])
    return _kept(s)


def _live(s, k):
    return {"out": s["out"], "K": s["K"][..., :k, :], "V": s["V"][..., :k, :], "score": s["score"][..., :k], "pos": s["pos"][..., :k], "len": s["len"]}


def _kept(s):
    k = s["case"]["k"]
    return {"K": s["K4"][..., :k, :], "V": s["V4"][..., :k, :], "score": s["score4"][..., :k], "pos": s["pos4"][..., :k], "len": s["len4"]}


# ---------------------------------------------------------------- the plain forms
def _plain_beam(s):
    case = s["case"]
    R, W, V = case["R"], case["W"], case["V"]
    x = s["logits"].view(R, W, V)
    # a row's best W words, by logit and then by the lower number: one whole number orders them
    bits = x.float().view(torch.int32).long()
    key = torch.where(bits < 0, ~bits & 0xFFFFFFFF, bits | 0x80000000)
    best = ((key << 31) | (0x7FFFFFFF - torch.arange(V, device="cuda"))).topk(min(W, V), dim=-1).values
    token = 0x7FFFFFFF - (best & 0x7FFFFFFF)
    xd = x.double()
    lse = torch.logsumexp(xd, -1, keepdim=True)
    total = s["score"].view(R, W, 1).double() + (xd.gather(-1, token) - lse)
    total = torch.where(torch.isnan(total), -math.inf, total)
    if s["done"] is not None:  # a hypothesis at its end goes on as it is, by one continuation
        ended, first = s["done"].view(R, W, 1) != 0, torch.arange(token.shape[-1], device="cuda") == 0
        token = torch.where(ended, 2, token)
        total = torch.where(ended, s["score"].view(R, W, 1).double(), total)
        order = torch.where(ended & ~first, 1, 0).flatten(1)  # no continuations: behind everything
    else:
        order = torch.zeros_like(total, dtype=torch.int64).flatten(1)
    at = torch.sort(total.flatten(1), dim=1, descending=True, stable=True).indices
    at = at.gather(1, torch.sort(order.gather(1, at), dim=1, stable=True).indices)[:, :W]
    p, tok, tot = at // token.shape[-1], token.flatten(1).gather(1, at), total.flatten(1).gather(1, at)
    # the best continuation of a beam keeps its row, the others take the rows that died, lowest first
    j = torch.arange(W, device="cuda")
    same = p[:, :, None] == p[:, None, :]
    first = ~(same & (j[None, :] < j[:, None])).any(-1)
    used = (p[:, :, None] == j).any(1)
    free = torch.sort(used.int(), dim=1, stable=True).indices
    row = torch.where(first, p, free.gather(1, (torch.cumsum(~first, 1) - 1).clamp(min=0)))
    base = torch.arange(R, device="cuda")[:, None] * W
    at = (base + row).flatten()
    s["parent"][at], s["token"][at] = (base + p).flatten().int(), tok.flatten().int()
    s["rank"][at], s["new_score"][at] = j.expand(R, W).flatten().int(), tot.flatten().float()
    if s["done"] is not None:
        s["new_done"][at] = ((s["done"].view(R, W).gather(1, p) != 0) | (tok == 2)).flatten().int()
    return {x: s[x] for x in ("parent", "token", "rank", "new_score", "new_done")}


def _normed(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()


def _turned(x, cos, sin, rot, style):
    a, b = (x[..., :rot:2], x[..., 1:rot:2]) if style == "pairs" else (x[..., :rot // 2], x[..., rot // 2:rot])
    both = (a * cos - b * sin, a * sin + b * cos)
    return torch.cat([torch.stack(both, -1).flatten(-2) if style == "pairs" else torch.cat(both, -1), x[..., rot:]], -1)


def _plain_rotate(s):
    case = s["case"]
    B, n, rot = case["B"], case["n"], case["rot"]
    at = s["pos"].double()[:, None] + torch.arange(n, device="cuda")
    angle = (at[:, :, None] * s["freq"].double())[:, :, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _turned(_normed(s["q"], s["qw"]), cos, sin, rot, case["style"]).to(s["Q"].dtype).transpose(1, 2)
    k = _turned(_normed(s["k"], s["kw"]), cos, sin, rot, case["style"]).to(s["K"].dtype).transpose(1, 2)
    v = s["v"].transpose(1, 2)
    if s["rows"] is not None:  # what lies behind a sequence stays as it is
        ok = (torch.arange(n, device="cuda") < s["rows"][:, None])[:, None, :, None]
        q, k, v = (torch.where(ok, x, y) for x, y in ((q, s["Q"]), (k, s["K"][:, :, :n]), (v, s["V"][:, :, :n])))
    s["Q"].copy_(q)
    s["K"][:, :, :n] = k
    s["V"][:, :, :n] = v
    return {x: s[x] for x in ("Q", "K", "V")}


def _mix32(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _mix64(z):
    z = z ^ ((z >> 32) & 0xFFFFFFFF)
    z = z * 0x6A09E667F3BCC909
    z = z ^ ((z >> 29) & 0x7FFFFFFFF)
    z = z * (0xBB67AE8584CAA73B - (1 << 64))
    return z ^ ((z >> 32) & 0xFFFFFFFF)


def _noise(seeds, L, HQ, q_pos, pos):
    """Gumbel adjustment of every (layer, sequence, query head) for keys at `pos` [L, B, HQ, m] (see kf_noise_bits)."""
    lh = (torch.arange(L, device="cuda")[:, None, None] << 32) | torch.arange(HQ, device="cuda")
    u = _mix64(_mix64(seeds + (0x9E3779B97F4A7C15 - (1 << 64)))[None, :, None] + lh)
    lo, hi = u & 0xFFFFFFFF, (u >> 32) & 0xFFFFFFFF
    row = _mix32((_mix32(lo ^ ((q_pos * 0x9E3779B9) & 0xFFFFFFFF)) + hi) & 0xFFFFFFFF)
    bits = _mix32(row[..., None] ^ ((pos * 0x243F6A89) & 0xFFFFFFFF))
    return -torch.log(-torch.log((2 * (bits >> 9) + 1).double() * 2.0 ** -24))


def _tau32(t, T):
    return float(np.float32(TAU[0]) + np.float32(min(t, T)) * (np.float32(TAU[1] - TAU[0]) / np.float32(T)))


def _plain_step(s):
    case = s["case"]
    L, B, H, d, k, w, G = (case[x] for x in ("L", "B", "H", "d", "k", "w", "G"))
    U, t, r = L * B * H, s["t"], s["t"] % RING
    s["t"] += 1
    q_pos, tau = case["n"] + t - 1, _tau32(t, case["T"])
    q, kn, vn = s["q"][r].view(U, G, d).float(), s["kn"][r].view(U, 1, d), s["vn"][r].view(U, 1, d)
    K, V, pos, score = s["K"].view(U, k + 1, -1), s["V"].view(U, k + 1, -1), s["pos"].view(U, k + 1), s["score"].view(U, k + 1)
    # the new token is appended; its own key and value enter this step as they were given
    K[:, k:], V[:, k:], pos[:, k], score[:, k] = _pack(kn), _pack(vn), q_pos, 0.0
    x = torch.cat([_unpack(K[:, :k], d) @ q.transpose(1, 2).contiguous(), kn.float() @ q.transpose(1, 2).contiguous()], 1) * _scale(case)  # [U, m, G]
    if s["slopes"] is not None:
        x -= s["slopes"].view(1, H, G).expand(L * B, H, G).reshape(U, 1, G) * (q_pos - pos)[:, :, None]
    p = torch.softmax(x, 1).transpose(1, 2).contiguous()
    s["out"].copy_((p[:, :, :k].contiguous() @ _unpack(V[:, :k], d) + p[:, :, k:] * vn.float()).view(L, B, H * G, d))
    zeta = _noise(s["seeds"], L, H * G, q_pos, pos.view(L, B, H, 1, k + 1).expand(L, B, H, G, k + 1).reshape(L, B, H * G, k + 1).long())
    y = (x.transpose(1, 2) + zeta.view(U, G, k + 1)) / tau
    score += torch.softmax(y, -1).sum(1).float()
    # one token leaves: the smallest score outside the window of the w newest, the later one of equals
    f = torch.where(pos <= q_pos - w, score, math.inf)
    e = torch.where(f == f.amin(1, keepdim=True), pos, -1).argmax(1, keepdim=True)
    if case["layout"] == "slot":  # the new token takes its place
        u = torch.arange(U, device="cuda")[:, None]
        K[u, e], V[u, e], pos[u, e], score[u, e] = K[:, k:], V[:, k:], pos[:, k:], score[:, k:]
    else:
        gap = torch.arange(k, device="cuda") >= e
        pos[:, :k], score[:, :k] = torch.where(gap, pos[:, 1:], pos[:, :k]), torch.where(gap, score[:, 1:], score[:, :k])
        gap = gap[:, :, None]
        K[:, :k], V[:, :k] = torch.where(gap, K[:, 1:], K[:, :k]), torch.where(gap, V[:, 1:], V[:, :k])
    return _live(s, k)


def _plain_evict(s):
    case = s["case"]
    n, k, w = case["n"], case["k"], case["w"]
    # the k-w best of the tokens before the window, the earlier one of equals, then the window; in order
    bits = s["score"][..., :n - w].view(torch.int32).long()
    key = torch.where(bits < 0, ~bits & 0xFFFFFFFF, bits | 0x80000000)
    best = ((key << 31) | (0x7FFFFFFF - torch.arange(n - w, device="cuda"))).topk(k - w, dim=-1).values
    keep = torch.sort(0x7FFFFFFF - (best & 0x7FFFFFFF), dim=-1).values
    keep = torch.cat([keep, torch.arange(n - w, n, device="cuda").expand(*keep.shape[:-1], w)], -1)
    rows = keep[..., None].expand(*keep.shape, case["d"])
    s["K4"][..., :k, :], s["V4"][..., :k, :] = _pack(s["K"].gather(-2, rows)), _pack(s["V"].gather(-2, rows))
    s["score4"][..., :k], s["pos4"][..., :k] = s["score"].gather(-1, keep), s["pos"].gather(-1, keep)
    s["len4"].copy_(s["len"].clamp(max=k))
    return _kept(s)


def run(s):
    call = s["case"]["call"]
    if own:
        import paper_2403_09054_amd as kf
        return {"beam": _own_beam, "rotate": _own_rotate, "step": _own_step, "evict": _own_evict}[call](kf, s)
    return {"beam": _plain_beam, "rotate": _plain_rotate, "step": _plain_step, "evict": _plain_evict}[call](s)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    eb = 4 if case["dtype"] == "f32" else 2
    if case["call"] == "beam":  # the logits, once
        return {"bytes": case["R"] * case["W"] * (float(case["V"]) * eb + 24), "flops": 4.0 * case["R"] * case["W"] * case["V"]}
    d, H = case["d"], case["H"]
    if case["call"] == "rotate":  # every row in and out
        rows = float(case["B"]) * case["n"] * (0.625 if case["padded"] and case["n"] > 1 else 1.0)
        return {"bytes": rows * H * (case["G"] + 2) * 2.0 * d * eb, "flops": rows * H * (case["G"] + 1) * 7.0 * d}
    U, k, row = case["L"] * case["B"] * H, case["k"], d // 2 + 16
    if case["call"] == "step":
        G = case["G"]
        # K and V rows, scores and positions in; scores out; q, k_new, v_new in, the attention output out
        b = k * (2.0 * row + 12) + (G + 2) * d * 2.0 + 4.0 * G * d
        # the window's rows move down by one slot (the slot layout stores one row)
        b += (case["w"] if case["layout"] == "ordered" else 1) * (2.0 * row + 8)
        return {"bytes": U * b, "flops": U * G * (k + 1) * 4.0 * d}
    return {"bytes": U * (case["n"] * 4.0 + k * (2.0 * d * 2 + 2.0 * row + 12)), "flops": 0.0}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_beam(case, seed):
    """New scores only: the rest are choices among given values."""
    s = _prepare_beam(case, seed)
    R, W, V = case["R"], case["W"], case["V"]
    new = torch.zeros(R * W, dtype=torch.float64)
    for r in range(R):
        x = s["logits"][r * W:(r + 1) * W].double()
        top = x.amax(1, keepdim=True)
        logp = x - (top + torch.log(torch.exp(x - top).sum(1, keepdim=True)))
        found = []  # (-total, row, -logit, word)
        for i in range(W):
            sc = float(s["score"][r * W + i])
            if s["done"] is not None and int(s["done"][r * W + i]):
                found.append((-sc, i, 0.0, 2))
                continue
            few = torch.nonzero(logp[i] >= torch.topk(logp[i], min(W, V)).values[-1]).flatten()
            lp, xs = logp[i][few].cpu().numpy(), x[i][few].cpu().numpy()
            mine = [(-(sc + float(a)), i, -float(b), int(v)) for a, b, v in zip(lp, xs, few.cpu().numpy())]
            found += sorted(mine)[:W]
        found = sorted(found)[:W]
        rows = {}
        for j, c in enumerate(found):
            if c[1] not in rows.values():
                rows[j] = c[1]
        left = [i for i in range(W) if i not in rows.values()]
        for j, c in enumerate(found):
            new[r * W + (rows[j] if j in rows else left.pop(0))] = -c[0]
    return {"parent": None, "token": None, "rank": None, "new_score": new, "new_done": None}


def _exact_rotate(case, seed):
    s = _prepare_rotate(case, seed)
    B, n, d, rot = case["B"], case["n"], case["d"], case["rot"]
    got = {}
    for name, x, w in (("Q", s["q"], s["qw"]), ("K", s["k"], s["kw"])):
        full = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
        for b in range(B):
            m = n if s["rows"] is None else int(s["rows"][b])
            y = x[b, :m].double()
            if w is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + 1e-6) * w.double()
            angle = torch.outer(int(s["pos"][b]) + torch.arange(m, device="cuda", dtype=torch.float64), s["freq"].double())
            turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]
            if case["style"] == "pairs":
                z = torch.view_as_real(torch.view_as_complex(y[..., :rot].unflatten(-1, (rot // 2, 2)).contiguous()) * turn).flatten(-2)
            else:
                z = torch.complex(y[..., :rot // 2].contiguous(), y[..., rot // 2:rot].contiguous()) * turn
                z = torch.cat([z.real, z.imag], -1)
            full[b, :, :m] = torch.cat([z, y[..., rot:]], -1).transpose(0, 1)
        got[name] = full
    return {**got, "V": None}


def _exact_step(case, seed):
    s = _prepare_step(case, seed)
    L, B, H, d, k, w, G = (case[x] for x in ("L", "B", "H", "d", "k", "w", "G"))
    U, t, r = L * B * H, s["t"], s["t"] % RING
    q_pos, tau = case["n"] + t - 1, _tau32(t, case["T"])
    q, kn, vn = (s[x][r].view(U, -1, d).double() for x in ("q", "kn", "vn"))
    pos, f = s["pos"].view(U, k + 1).long(), s["score"].view(U, k + 1).double()
    pos[:, k], f[:, k] = q_pos, 0.0
    zeta = _noise(s["seeds"], L, H * G, q_pos, pos.view(L, B, H, 1, k + 1).expand(L, B, H, G, k + 1).reshape(L, B, H * G, k + 1)).view(U, G, k + 1)
    out, score = torch.empty((U, G, d), dtype=torch.float64, device="cuda"), torch.empty((U, k), dtype=torch.float64, device="cuda")
    some = max(1, int(1e8 // ((k + 1) * d)))

    def rows(packed, new):
        c = packed[:, :k, :d // 2].int()
        c = torch.stack([c & 15, c >> 4], -1).flatten(-2)
        h = (c >> 1) & 3  # exponent of a code; its last bit is the mantissa
        mag = torch.where(h == 0, (c & 1) * 0.5, (2.0 + (c & 1)) * torch.exp2(h.double() - 2.0))
        two = torch.exp2(packed[:, :k, d // 2:].double() - 127.0).repeat_interleave(d // 16, -1)
        return torch.cat([torch.where(c >= 8, -mag, mag) * two, new], 1)

    for a in range(0, U, some):
        z = slice(a, min(U, a + some))
        x = (q[z] @ rows(s["K"].view(U, k + 1, -1)[z], kn[z]).transpose(1, 2).contiguous()) * _scale(case)
        if s["slopes"] is not None:
            heads = torch.arange(a, z.stop, device="cuda") % H
            x = x - s["slopes"].double().view(H, G)[heads][:, :, None] * (q_pos - pos[z])[:, None, :]
        out[z] = torch.softmax(x, -1) @ rows(s["V"].view(U, k + 1, -1)[z], vn[z])
        fn = f[z] + torch.softmax((x + zeta[z]) / tau, -1).sum(1)
        e = torch.where(pos[z] <= q_pos - w, fn, math.inf).argmin(1, keepdim=True)
        if case["layout"] == "slot":
            score[z] = fn.scatter(1, e, fn[:, k:])[:, :k]
        else:
            j = torch.arange(k, device="cuda")[None, :]
            score[z] = fn.gather(1, j + (j >= e))
    return {"out": out.view(L, B, H * G, d), "K": None, "V": None, "score": score.view(L, B, H, k), "pos": None, "len": None}


def exact(case, seed):
    if case["call"] == "evict":
        return None  # a choice among the given scores, moves, and bytes that are fixed
    return {"beam": _exact_beam, "rotate": _exact_rotate, "step": _exact_step}[case["call"]](case, seed)
