"""The prompt's attention and a paged cache of 8 bits, as cases that can be timed and compared with their plain form.

Groups of calls, each through the package's public functions:

  prompt   attention over prompts (kf_prompt_attend): causal, grouped heads, padded or packed sequences, or the last rows of
           longer ones
  step     one generated token of every sequence (kf_page_step): attention over 8-bit pages, and the token's own row
  admit    sequences that ended give their pages back, new prompts take pages and are written (kf_page_free,
           kf_page_reserve, kf_page_write), in one part or in two
  fork     the beams of a search take over their parents' pages (kf_page_fork)
  compact  a request goes on with a part of a prompt that others keep in full (kf_page_fork, kf_page_compact)

A page holds 64 tokens of every layer and head: key codes [64][d], value codes [d][64], of 8 bits (E4M3: sign, four exponent
bits, three of mantissa), and for each tensor and head one power of two that they are multiplied by -- the smallest, from
2^-117 to 2^119, with which no finite element of the page's rows is above 448.  A row that needs a larger one than its page
has makes the page's older codes be rounded again.  Which codes a page gets is therefore fixed to the bit; they are returned as
8-bit floating numbers, beside their scales.

Sizes are those of kf_workloads.CONFIGS (a layer, or a few layers, of them) or generic.
"""
import math

import numpy as np
import torch

own = False

PAGE = 64
RING = 8  # distinct generated tokens that the steps take in turn
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _prompt(name, B, n, m, H, G, d, dtype="bf16", alibi=False, ragged="none", outliers=0.0):
    return {"name": name, "call": "prompt", "B": B, "n": n, "m": m, "H": H, "G": G, "d": d, "dtype": dtype, "alibi": alibi,
            "ragged": ragged, "outliers": outliers}


def _step(name, L, B, H, G, d, length, dtype="bf16", alibi=False, ragged=False, outliers=0.0):
    return {"name": name, "call": "step", "L": L, "B": B, "H": H, "G": G, "d": d, "length": length, "dtype": dtype, "alibi": alibi,
            "ragged": ragged, "outliers": outliers}


def _admit(name, L, B, new, H, d, n, dtype="bf16", ragged=False, parts=1):
    return {"name": name, "call": "admit", "L": L, "B": B, "new": new, "H": H, "d": d, "n": n, "dtype": dtype, "ragged": ragged, "parts": parts}


def _fork(name, L, R, W, H, d, length):
    return {"name": name, "call": "fork", "L": L, "R": R, "W": W, "H": H, "d": d, "length": length}


def _compact(name, L, B, H, d, n, k):
    return {"name": name, "call": "compact", "L": L, "B": B, "H": H, "d": d, "n": n, "k": k}


def listed():
    return [
        # one prompt of a model with wide heads, one layer
        _prompt("prompt_wide_heads", 1, 2048, 2048, 16, 1, 256, outliers=0.01),
        # the prompts of a batch of 8 with position bias, one layer: the largest
        _prompt("prompt_layer", 8, 4096, 4096, 32, 1, 128, alibi=True),
        # a serving engine's prompts of very different lengths, packed one behind the other, grouped heads in half precision
        _prompt("prompt_packed", 24, 3000, 3000, 8, 4, 128, dtype="f16", ragged="packed"),
        # the last part of long prompts that are taken in parts
        _prompt("prompt_part", 4, 512, 8192, 8, 8, 128, outliers=0.005),
        # serving one sequence with grouped heads: the smallest call
        _step("page_token", 1, 1, 8, 4, 128, 1501),
        # one layer of a large batch, sequences of all ages
        _step("page_layer_step", 1, 64, 32, 1, 128, 2048, ragged=True),
        # one layer of one long sequence: few, long units
        _step("page_long_step", 1, 1, 32, 1, 128, 32768, outliers=0.005),
        # eight layers of a batch of 8 with position bias in one call: the largest step
        _step("page_layers_step", 8, 8, 32, 1, 128, 4096, alibi=True),
        # a long prompt comes in: one layer
        _admit("admit_long", 1, 1, 1, 32, 128, 32768),
        # half of a batch ends and new prompts take their places, in two parts each, grouped heads in half precision
        _admit("admit_batch", 4, 32, 16, 8, 128, 2000, dtype="f16", ragged=True, parts=2),
        # 16 requests of 4 beams go on after a choice
        _fork("fork_beams", 16, 16, 4, 8, 128, 1801),
        # half of the prompts' tokens leave, four layers of eight requests
        _compact("compact_prompts", 4, 8, 32, 128, 2048, 1024),
    ]


def draw(rng):
    """One more case: sizes over the whole range, their logarithms even."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("prompt", "prompt", "prompt", "step", "step", "step", "admit", "fork", "compact"))
    d, H = rng.choice((64, 128, 128, 256)), rng.choice((2, 8, 12, 16, 32))
    dtype, alibi, outliers = rng.choice(("bf16", "bf16", "f16")), rng.random() < 0.3, rng.choice((0.0, 0.005, 0.01))
    if kind == "prompt":
        if d < 256 and rng.random() < 0.15:
            dtype = "f32"
        n, G = log(1, 6000), rng.choice((1, 1, 2, 4, 8))
        m = n if rng.random() < 0.7 else n + log(1, 8000)
        G = max(1, min(G, int(1.5e9 / (H * n * m))))
        B = max(1, min(log(1, 64), int(5.4e11 / (H * G * n * m * max(d, 128))), int(2e8 / (H * G * (n + m) * d))))
        # fp32 products cost more: as much less of them
        B = max(1, B // 8) if dtype == "f32" else B
        case = _prompt("", B, n, m, H, G, d, dtype, alibi, rng.choice(("none", "padded", "packed")), outliers)
    elif kind == "step":
        length, G = log(1, 40000), rng.choice((1, 1, 1, 2, 4, 8))
        B = max(1, min(log(1, 128), int(2.6e8 / (H * length * d))))
        L = max(1, min(log(1, 16), int(2.6e8 / (B * H * length * d))))
        case = _step("", L, B, H, G, d, length, dtype, alibi, rng.random() < 0.5, outliers)
    elif kind == "admit":
        n = log(1, 32768)
        B = max(1, min(log(1, 64), int(1.3e8 / (H * n * d))))
        L = max(1, min(log(1, 8), int(1.3e8 / (B * H * n * d))))
        case = _admit("", L, B, rng.randint(1, B), H, d, n, dtype, rng.random() < 0.5, rng.choice((1, 2)) if n > 1 else 1)
    elif kind == "fork":
        W, length = log(2, 16), log(1, 8000)
        page = PAGE * H * d * (_pages_of(length) + W)  # of a request and layer
        R = max(1, min(log(1, 32), int(5.6e8 / page)))
        case = _fork("", max(1, min(log(1, 32), int(5.6e8 / (R * page)))), R, W, H, d, length)
    else:
        n = log(2, 16000)
        B = max(1, min(log(1, 32), int(2.6e8 / (H * n * d))))
        case = _compact("", max(1, min(log(1, 8), int(2.6e8 / (B * H * n * d)))), B, H, d, n, max(1, int(n * rng.uniform(0.1, 0.7))))
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


def _slopes(case):
    HQ = case["H"] * case["G"]
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / HQ) for h in range(HQ)], dtype=torch.float32, device="cuda") if case["alibi"] else None


def _scale(case):
    return float(np.float32(1.0) / np.sqrt(np.float32(case["d"])))


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _lengths(count, most, spread, seed=None):
    """Lengths that a program knows of its sequences: spread evenly over so many powers of two up to `most`, in an order of the seed's."""
    v = [max(1, int(round(most * 2.0 ** (-spread * i / count)))) for i in range(count)]
    if seed is not None:
        np.random.RandomState((int(seed) * 7 + count * 13 + most) & 0x7FFFFFFF).shuffle(v)
    return v


def _prepare_prompt(case, seed):
    B, n, m, H, G, d = (case[x] for x in ("B", "n", "m", "H", "G", "d"))
    dt, g = TYPES[case["dtype"]], _gen(seed, 1)
    s = {"case": case, "slopes": _slopes(case)}
    # a prompt of n rows of which none came before, or n rows behind others of the same sequence
    s["nq"] = [n] * B if case["ragged"] == "none" else _lengths(B, n, math.log2(n) if case["ragged"] == "packed" else 2.0, seed)
    s["nk"] = [x + m - n for x in s["nq"]]
    if case["ragged"] == "packed":
        # a fused projection's rows, token by token, and the keys and values of all tokens likewise
        tq, tk = sum(s["nq"]), sum(s["nk"])
        q = _normal((tq, (G + 2) * H if tq == tk else G * H, d), dt, g)
        kv = q[:, G * H:] if tq == tk else _normal((tk, 2 * H, d), dt, g)
        s["Q"], s["K"], s["V"] = q[:, :G * H], kv[:, :H], kv[:, H:]
        s["K"].copy_(_scale_rows(s["K"], case["outliers"], g))
        s["q_start"], s["k_start"] = (np.concatenate([[0], np.cumsum(x)]).tolist() for x in (s["nq"], s["nk"]))
        s["q_at"], s["k_at"] = _ints(s["q_start"]), _ints(s["k_start"])
        s["out"] = torch.zeros((tq, G * H, d), dtype=dt, device="cuda")
    else:
        # head by head, as the rows of a projection are left for prompt scoring and the caches
        s["Q"] = _normal((B, G * H, n, d), dt, g)
        s["K"], s["V"] = _scale_rows(_normal((B, H, m, d), dt, g), case["outliers"], g), _normal((B, H, m, d), dt, g)
        s["seq_n"], s["seq_m"] = (_ints(s["nq"]), _ints(s["nk"])) if case["ragged"] == "padded" else (None, None)
        s["out"] = torch.zeros((B, n, G * H, d), dtype=dt, device="cuda")  # token by token, as the next projection reads it
    return s


def _pool(case, L, B, H, d, pages, max_pages):
    """Empty pages: what a server holds for all its sequences."""
    return {"case": case, "L": L, "B": B, "H": H, "d": d, "pages": pages, "max_pages": max_pages,
            "K": torch.zeros((L, pages, H, PAGE, d), dtype=torch.uint8, device="cuda"),
            "V": torch.zeros((L, pages, H, d, PAGE), dtype=torch.uint8, device="cuda"),
            "k_scale": torch.ones((L, pages, H), device="cuda"), "v_scale": torch.ones((L, pages, H), device="cuda"),
            "table": torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda"),
            "len": torch.zeros(B, dtype=torch.int32, device="cuda"), "refs": torch.zeros(pages, dtype=torch.int32, device="cuda")}


def _pages_of(n):
    return (n + PAGE - 1) // PAGE


def _fill(s, lens, g, outliers, owners=None):
    """Sequences of these lengths in pages all over the pool.  owners[b]: the row whose full pages row b shares."""
    B, pages = s["B"], s["pages"]
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(int(torch.randint(1 << 30, (1,), generator=g, device="cuda")))).tolist()
    table, refs, at = np.full((B, s["max_pages"]), -1, np.int32), np.zeros(pages, np.int32), 0
    for b in range(B):
        full = lens[b] // PAGE if owners is not None and owners[b] != b else 0
        for j in range(_pages_of(lens[b])):
            if j < full:
                table[b, j] = table[owners[b], j]
            else:
                table[b, j] = order[at]
                at += 1
            refs[table[b, j]] += 1
    s["table"], s["refs"], s["len"] = torch.from_numpy(table).cuda(), torch.from_numpy(refs).cuda(), _ints(lens)
    for l in range(s["L"]):  # a layer at a time: the values before their rounding are four times as large
        x = _scale_rows(torch.randn((pages, s["H"], PAGE, s["d"]), generator=g, device="cuda"), outliers, g)
        e = _exponent(x.abs().amax((-2, -1)))
        s["K"][l], s["k_scale"][l] = _codes(x, e[..., None, None]), torch.exp2(e.float())
        x = torch.randn((pages, s["H"], s["d"], PAGE), generator=g, device="cuda")
        e = _exponent(x.abs().amax((-2, -1)))
        s["V"][l], s["v_scale"][l] = _codes(x, e[..., None, None]), torch.exp2(e.float())


def _prepare_step(case, seed):
    L, B, H, G, d, n = (case[x] for x in ("L", "B", "H", "G", "d", "length"))
    dt, g = TYPES[case["dtype"]], _gen(seed, 2)
    lens = _lengths(B, n, 2.0, seed) if case["ragged"] else [n] * B
    s = _pool(case, L, B, H, d, sum(map(_pages_of, lens)) + 3, _pages_of(n) + 1)
    _fill(s, lens, g, case["outliers"])
    s |= {"lens": lens, "slopes": _slopes(case), "t": 0, "out": torch.zeros((L, B, H * G, d), device="cuda"),
          "q": _normal((RING, L, B, H * G, d), dt, g), "v": _normal((RING, L, B, H, d), dt, g),
          "k": _scale_rows(_normal((RING, L, B, H, d), dt, g), case["outliers"], g)}
    return s


def _prepare_admit(case, seed):
    L, B, H, d, n, new = (case[x] for x in ("L", "B", "H", "d", "n", "new"))
    dt, g = TYPES[case["dtype"]], _gen(seed, 3)
    lens = _lengths(B, n, 2.0, seed) if case["ragged"] else [n] * B
    # the rows that ended and the prompts that take their places, spread over the batch
    r = np.random.RandomState((int(seed) * 11 + B) & 0x7FFFFFFF)
    which = sorted(r.choice(B, new, replace=False).tolist())
    fresh = _lengths(new, n, 2.0, seed + 1) if case["ragged"] else [n] * new
    s = _pool(case, L, B, H, d, sum(map(_pages_of, lens)) + sum(map(_pages_of, fresh)) + 5, _pages_of(n) + 2)
    _fill(s, lens, g, 0.0)
    first = [0] * B
    for b, x in zip(which, fresh):
        first[b] = x
    s["parts"] = [first]
    if case["parts"] == 2:  # a first part, and what is left
        cut = [int(x * 0.4) for x in first]
        s["parts"] = [cut, [x - c for x, c in zip(first, cut)]]
    s["which"] = _ints([int(b in which) for b in range(B)])
    s["counts"], s["k"], s["v"], at = [_ints(p) for p in s["parts"]], [], [], [0] * B
    for p in s["parts"]:
        s["k"].append(_normal((L, B, H, max(p + [1]), d), dt, g))
        s["v"].append(_normal((L, B, H, max(p + [1]), d), dt, g))
    # which pages of which sequences a part touches, as a program that knows its prompts' lengths counts them
    s["touch"] = []
    for p in s["parts"]:
        pairs = [(b, j, at[b], p[b]) for b in range(B) if p[b] for j in range(at[b] // PAGE, _pages_of(at[b] + p[b]))]
        s["touch"].append(torch.tensor(pairs, dtype=torch.int64, device="cuda").reshape(-1, 4).unbind(1))
        at = [a + x for a, x in zip(at, p)]
    return s


def _prepare_fork(case, seed):
    L, R, W, H, d, n = (case[x] for x in ("L", "R", "W", "H", "d", "length"))
    g, B = _gen(seed, 4), R * W
    r = np.random.RandomState((int(seed) * 17 + B) & 0x7FFFFFFF)
    lens = [x for x in _lengths(R, n, 1.0, seed) for _ in range(W)]
    # about a third of a request's hypotheses die; their rows go to continuations of the others
    parent = []
    for q in range(R):
        alive = sorted(r.choice(W, max(1, W - r.binomial(W, 0.35)), replace=False).tolist())
        parent += [q * W + (i if i in alive else alive[r.randint(len(alive))]) for i in range(W)]
    s = _pool(case, L, B, H, d, sum(_pages_of(x) + W for x in lens[::W]) + 3, _pages_of(n) + 1)
    _fill(s, lens, g, 0.0, [b // W * W for b in range(B)])
    s |= {"lens": lens, "parent": _ints(parent), "parent_host": parent}
    return s


def _prepare_compact(case, seed):
    L, B, H, d, n, k = (case[x] for x in ("L", "B", "H", "d", "n", "k"))
    g = _gen(seed, 5)
    s = _pool(case, L, 2 * B, H, d, B * (_pages_of(n) + 1 + _pages_of(k)) + 2, _pages_of(n) + 1)
    _fill(s, [n] * B + [0] * B, g, 0.005)  # the first half of the rows keep their prompts; the others are requests
    s["parent"] = _ints(list(range(B)) * 2)
    # the last fifth, and the tokens that gathered the most before it
    w = max(0, min(k // 5, k - 1))
    keys = torch.rand((L * B * H, n - w), generator=g, device="cuda").topk(k - w, dim=1).indices.sort(dim=1).values
    keep = torch.cat([keys, torch.arange(n - w, n, device="cuda").expand(L * B * H, w)], 1).int().view(L, B, H, k)
    s["keep"] = torch.cat([torch.full_like(keep, -1), keep], 1)
    s["which"] = _ints([0] * B + [1] * B)
    return s


def prepare(case, seed):
    return {"prompt": _prepare_prompt, "step": _prepare_step, "admit": _prepare_admit, "fork": _prepare_fork, "compact": _prepare_compact}[case["call"]](case, seed)


# ---------------------------------------------------------------- the framework's calls
def _code(kf, case):
    return {"f32": kf.F32, "bf16": kf.BF16, "f16": kf.F16}[case.get("dtype", "bf16")]


def _own_prompt(kf, s):
    case = s["case"]
    if "cfg" not in s:
        of = dict(B=case["B"], n=case["n"], m=case["m"], H=case["H"], q_per_kv=case["G"], d=case["d"], dtype=_code(kf, case), scale=_scale(case),
                  slopes=s["slopes"])
        if case["ragged"] == "packed":
            rows = {x: (0, case["d"], t.stride(0)) for x, t in (("q_stride", s["Q"]), ("k_stride", s["K"]), ("v_stride", s["V"]), ("out_stride", s["out"]))}
            s["cfg"] = kf.Prompt(q_start=s["q_at"], k_start=s["k_at"], **rows, **of)
        else:
            o = s["out"].stride()
            s["cfg"] = kf.Prompt(seq_n=s["seq_n"], seq_m=s["seq_m"], q_stride=s["Q"].stride()[:3], k_stride=s["K"].stride()[:3],
                                 v_stride=s["V"].stride()[:3], out_stride=(o[0], o[2], o[1]), **of)
        s["ws"] = kf.new_prompt_workspace(s["cfg"])
    kf.kf_prompt_attend(s["cfg"], s["Q"], s["K"], s["V"], s["out"], workspace=s["ws"])
    return s["out"]


def _own_pages(kf, s):
    if "cache" not in s:
        s["cache"] = kf.Pages(K=s["K"], V=s["V"], k_scale=s["k_scale"], v_scale=s["v_scale"], table=s["table"], len=s["len"], refs=s["refs"],
                              L=s["L"], B=s["B"], H=s["H"], d=s["d"], pages=s["pages"], max_pages=s["max_pages"], dtype=_code(kf, s["case"]),
                              q_per_kv=s["case"].get("G", 1))
        s["ws"] = kf.new_page_workspace(s["cache"])
    return s["cache"], s["ws"]


def _own_step(kf, s):
    cache, ws = _own_pages(kf, s)
    r = s["t"] % RING
    s["t"] += 1
    kf.kf_page_step(cache, s["q"][r], s["k"][r], s["v"][r], _scale(s["case"]), s["out"], m_hint=s["case"]["length"], slopes=s["slopes"], workspace=ws)
    return {"out": s["out"], **_held(s)}


def _own_admit(kf, s):
    cache, ws = _own_pages(kf, s)
    kf.kf_page_free(cache, s["which"], workspace=ws)
    for p in range(len(s["parts"])):
        rows = s["k"][p].shape[3]
        kf.kf_page_reserve(cache, rows, s["counts"][p], workspace=ws)
        kf.kf_page_write(cache, s["k"][p], s["v"][p], rows, seq_n=s["counts"][p], workspace=ws)
    return _whole(s)


def _own_fork(kf, s):
    cache, ws = _own_pages(kf, s)
    kf.kf_page_fork(cache, s["parent"], workspace=ws)
    return _whole(s)


def _own_compact(kf, s):
    cache, ws = _own_pages(kf, s)
    kf.kf_page_fork(cache, s["parent"], workspace=ws)
    kf.kf_page_compact(cache, s["keep"], s["case"]["k"], which=s["which"], workspace=ws)
    return _whole(s)


def _held(s):
    return {"K": s["K"].view(torch.float8_e4m3fn), "V": s["V"].view(torch.float8_e4m3fn), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _whole(s):
    return {**_held(s), "table": s["table"], "len": s["len"], "refs": s["refs"]}


# ---------------------------------------------------------------- the plain forms
def _exponent(a):
    """Exponent of the scale of a page whose largest finite magnitude is `a`."""
    m, e = torch.frexp(a)
    return torch.where(a == 0, -117, torch.where(m <= 0.875, e - 9, e - 8).clamp(-117, 119)).int()


def _codes(x, e):
    """Elements -> codes, with the exponents `e` of their scales."""
    y = torch.ldexp(x, -e)
    return torch.where(torch.isfinite(y), y, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _attend(q, k, v, first, scale, slopes):
    """[B, HQ, nq, d] queries, [B, H, nk, d] keys and values in 32 bits; query i stands at key first + i."""
    B, HQ, nq, d = q.shape
    H, nk = k.shape[1], k.shape[2]
    x = (q.reshape(B * H, -1, d) @ k.reshape(B * H, nk, d).transpose(1, 2).contiguous()).view(B, HQ, nq, nk)
    x *= scale
    i, j = torch.arange(nq, device="cuda")[:, None] + first, torch.arange(nk, device="cuda")
    if slopes is not None:
        x -= slopes[:, None, None] * (i - j)
    x.masked_fill_(j > i, -math.inf)
    x = torch.softmax(x, -1)
    return (x.view(B * H, -1, nk) @ v.reshape(B * H, nk, d)).view(B, HQ, nq, d)


def _plain_prompt(s):
    case, sc = s["case"], _scale(s["case"])
    if case["ragged"] == "none":
        s["out"].copy_(_attend(s["Q"].float(), s["K"].float(), s["V"].float(), case["m"] - case["n"], sc, s["slopes"]).transpose(1, 2))
        return s["out"]
    for b, (nq, nk) in enumerate(zip(s["nq"], s["nk"])):  # each sequence has lengths of its own
        if case["ragged"] == "packed":
            rq, rk = slice(s["q_start"][b], s["q_start"][b] + nq), slice(s["k_start"][b], s["k_start"][b] + nk)
            q, k, v, out = s["Q"][rq].transpose(0, 1), s["K"][rk].transpose(0, 1), s["V"][rk].transpose(0, 1), s["out"][rq]
        else:
            q, k, v, out = s["Q"][b, :, :nq], s["K"][b, :, :nk], s["V"][b, :, :nk], s["out"][b, :nq]
        out.copy_(_attend(q.float()[None], k.float()[None], v.float()[None], nk - nq, sc, s["slopes"])[0].transpose(0, 1))
    return s["out"]


def _plain_rows(s, tensor, scale, x, at, where, older):
    """Rows into pages.  x [L, N, H, 64, d]: a page's new rows, those of `where` [N, 64]; `older` [N, 64]: rows it held before."""
    codes, sc = s[tensor][:, at], s[scale][:, at]
    if tensor == "V":
        x, where, older = x.transpose(-1, -2), where[:, None, None, :], older[:, None, None, :]
    else:
        where, older = where[:, None, :, None], older[:, None, :, None]
    size = torch.where(where & torch.isfinite(x), x.abs(), 0.0).amax((-2, -1))
    had = older.flatten(1).any(1)[None, :, None]
    old = torch.frexp(sc)[1].int() - 1
    e = _exponent(size)
    e = torch.where(had, torch.maximum(e, old), e)
    again = _codes(torch.ldexp(_values(codes), old[..., None, None]), e[..., None, None])
    s[tensor][:, at] = torch.where(where, _codes(x, e[..., None, None]), torch.where(older, again, codes))
    s[scale][:, at] = torch.exp2(e.float())


def _plain_step(s):
    case = s["case"]
    L, B, H, G, d = (case[x] for x in ("L", "B", "H", "G", "d"))
    r, n = s["t"] % RING, s["max_pages"] * PAGE
    s["t"] += 1
    q, kn, vn = s["q"][r].float().view(L, B, H, G, d), s["k"][r].float().view(L, B, H, 1, d), s["v"][r].float().view(L, B, H, 1, d)
    at = s["table"].long().clamp(min=0)
    K = (_values(s["K"])[:, at] * s["k_scale"][:, at][..., None, None]).permute(0, 1, 3, 2, 4, 5).reshape(L, B, H, n, d)
    V = (_values(s["V"])[:, at] * s["v_scale"][:, at][..., None, None]).permute(0, 1, 3, 2, 5, 4).reshape(L, B, H, n, d)
    j, last = torch.arange(n, device="cuda"), s["len"].long() - 1
    V.masked_fill_((j >= last[:, None])[None, :, None, :, None], 0.0)
    x = torch.cat([q.reshape(-1, G, d) @ K.view(-1, n, d).transpose(1, 2).contiguous(), q.reshape(-1, G, d) @ kn.reshape(-1, d, 1)], -1) * _scale(case)
    x = x.view(L, B, H, G, n + 1)
    if s["slopes"] is not None:
        x[..., :n] -= s["slopes"].view(H, G, 1) * (last[:, None] - j)[None, :, None, None, :]
    x[..., :n].masked_fill_((j >= last[:, None])[None, :, None, None, :], -math.inf)
    p = torch.softmax(x, -1)
    s["out"].copy_(((p[..., :n].reshape(-1, G, n) @ V.view(-1, n, d)).view(L, B, H, G, d) + p[..., n:] * vn).view(L, B, H * G, d))
    # the token's own row
    b = torch.arange(B, device="cuda")
    page, slot = s["table"][b, last // PAGE].long(), last % PAGE
    lane = torch.arange(PAGE, device="cuda")
    for tensor, scale, row in (("K", "k_scale", kn), ("V", "v_scale", vn)):
        _plain_rows(s, tensor, scale, row.expand(L, B, H, PAGE, d), page, lane == slot[:, None], lane < slot[:, None])
    return {"out": s["out"], **_held(s)}


def _plain_free(s, which):
    drop = (which != 0)[:, None] & (s["table"] >= 0)
    s["refs"].index_add_(0, s["table"].clamp(min=0).flatten().long(), -drop.flatten().int())
    s["table"].copy_(torch.where((which != 0)[:, None], -1, s["table"]))
    s["len"].copy_(torch.where(which != 0, 0, s["len"]))


def _plain_take(s, have, want):
    """Sequence b's pages have[b]..want[b]-1 are the free ones with the lowest numbers, in the order of the sequences."""
    j = torch.arange(s["max_pages"], device="cuda")
    new = (j >= have[:, None]) & (j < want[:, None])
    free = torch.sort((s["refs"] != 0).int(), stable=True).indices
    nth = (torch.cumsum(new.flatten(), 0) - 1).view(new.shape).clamp(0, s["pages"] - 1)
    s["table"].copy_(torch.where(new, free[nth].int(), s["table"]))
    s["refs"].index_add_(0, s["table"].clamp(min=0).flatten().long(), new.flatten().int())


def _plain_admit(s):
    _plain_free(s, s["which"])
    for p, (b, j, start, count) in enumerate(s["touch"]):
        after = s["len"] + s["counts"][p]
        _plain_take(s, _pages_of(s["len"]), _pages_of(after))
        s["len"].copy_(after)
        pos = j[:, None] * PAGE + torch.arange(PAGE, device="cuda")
        new, older = (pos >= start[:, None]) & (pos < (start + count)[:, None]), pos < start[:, None]
        at, row = s["table"][b, j].long(), (pos - start[:, None]).clamp(0, s["k"][p].shape[3] - 1)
        for tensor, scale, x in (("K", "k_scale", s["k"][p]), ("V", "v_scale", s["v"][p])):
            # [L, N, H, 64, d] of [L, B, H, rows, d]
            rows = x.permute(1, 3, 0, 2, 4)[b[:, None], row].permute(2, 0, 3, 1, 4).float()
            _plain_rows(s, tensor, scale, rows, at, new, older)
    return _whole(s)


def _plain_fork(s):
    B = s["B"]
    parent, b = s["parent"].long(), torch.arange(B, device="cuda")
    moved = parent != b
    held = s["table"].clone()
    _plain_free(s, moved.int())
    n = torch.where(moved, s["len"][parent], s["len"])
    full = n // PAGE
    j = torch.arange(s["max_pages"], device="cuda")
    share = moved[:, None] & (j < full[:, None])
    s["table"].copy_(torch.where(share, held[parent], s["table"]))
    s["refs"].index_add_(0, s["table"].clamp(min=0).flatten().long(), share.flatten().int())
    _plain_take(s, torch.where(moved, full, 0), torch.where(moved, _pages_of(n), 0))
    s["len"].copy_(n)
    # the last page, where it is not full, is copied; where there is none to copy, a page is copied onto itself
    last = (full * (n % PAGE != 0)).clamp(max=s["max_pages"] - 1)
    some = moved & (n % PAGE != 0)
    at, own_at = held[parent, last].long(), s["table"][b, last].long()
    keeps = held[torch.argmin(moved.int()), 0].long()  # a page that stays as it is: of a row that goes on by itself
    at, own_at = torch.where(some, at, keeps), torch.where(some, own_at, keeps)
    for x in ("K", "V", "k_scale", "v_scale"):
        s[x][:, own_at] = s[x][:, at]
    return _whole(s)


def _plain_compact(s):
    _plain_fork(s)
    L, H, d, k = s["L"], s["H"], s["d"], s["case"]["k"]
    B, P = s["case"]["B"], _pages_of(k)
    rows = torch.arange(B, 2 * B, device="cuda")
    if s["case"]["n"] <= k:
        return _whole(s)
    keep = s["keep"][:, B:].long()  # [L, B, H, k]
    at = s["table"][rows].long()    # the pages before
    pad = torch.nn.functional.pad(keep, (0, P * PAGE - k))
    live = (torch.arange(P * PAGE, device="cuda") < k).view(P, PAGE)
    held = at.view(1, B, 1, -1).expand(L, B, H, -1).gather(3, pad // PAGE)  # the page of each kept token
    l, h = torch.arange(L, device="cuda").view(L, 1, 1, 1), torch.arange(H, device="cuda").view(1, 1, H, 1)
    new = {}
    for tensor, scale in (("K", "k_scale"), ("V", "v_scale")):
        c = s[tensor][l, held, h, pad % PAGE] if tensor == "K" else s[tensor][l, held, h, :, pad % PAGE]
        x = torch.ldexp(_values(c), torch.frexp(s[scale][l, held, h])[1].int().unsqueeze(-1) - 1).view(L, B, H, P, PAGE, d)
        e = _exponent(torch.where(live[:, :, None] & torch.isfinite(x), x.abs(), 0.0).amax((-2, -1)))
        new[tensor], new[scale] = _codes(x, e[..., None, None]).transpose(2, 3), torch.exp2(e.float()).transpose(2, 3)
    # new pages, then the old ones go
    before = s["table"].clone()
    s["table"][rows] = -1
    zero = torch.zeros(2 * B, dtype=torch.int64, device="cuda")
    _plain_take(s, zero, torch.where(torch.arange(2 * B, device="cuda") >= B, P, 0))
    drop = (before >= 0) & (torch.arange(2 * B, device="cuda") >= B)[:, None]
    s["refs"].index_add_(0, before.clamp(min=0).flatten().long(), -drop.flatten().int())
    s["len"][rows] = k
    to = s["table"][rows][:, :P].long()
    # what lies behind the last kept token stays as it was
    s["K"][:, to] = torch.where(live[:, None, :, None], new["K"], s["K"][:, to])
    s["V"][:, to] = torch.where(live[:, None, None, :], new["V"].transpose(-1, -2), s["V"][:, to])
    s["k_scale"][:, to], s["v_scale"][:, to] = new["k_scale"], new["v_scale"]
    return _whole(s)


def run(s):
    call = s["case"]["call"]
    if own:
        import paper_2403_09054_amd as kf
        return {"prompt": _own_prompt, "step": _own_step, "admit": _own_admit, "fork": _own_fork, "compact": _own_compact}[call](kf, s)
    return {"prompt": _plain_prompt, "step": _plain_step, "admit": _plain_admit, "fork": _plain_fork, "compact": _plain_compact}[call](s)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    d, H = case["d"], case["H"]
    if case["call"] == "prompt":
        eb, G = 4 if case["dtype"] == "f32" else 2, case["G"]
        nq = [case["n"]] * case["B"] if case["ragged"] == "none" else _lengths(case["B"], case["n"], math.log2(case["n"]) if case["ragged"] == "packed" else 2.0)
        more = case["m"] - case["n"]
        pairs = sum(x * (x + 1) / 2 + x * more for x in nq)
        return {"bytes": sum((2.0 * G * x + 2.0 * (x + more)) * H * d * eb for x in nq), "flops": 4.0 * pairs * H * G * d}
    if case["call"] == "step":
        L, B, G = case["L"], case["B"], case["G"]
        tokens = sum(_lengths(B, case["length"], 2.0) if case["ragged"] else [case["length"]] * B)
        return {"bytes": L * H * (2.0 * tokens * d + B * (2.0 * (G + 2) * d + 4.0 * G * d + 2.0 * d)), "flops": 4.0 * L * H * G * d * tokens}
    if case["call"] == "admit":
        tokens = sum(_lengths(case["new"], case["n"], 2.0) if case["ragged"] else [case["n"]] * case["new"])
        return {"bytes": 6.0 * case["L"] * H * d * tokens, "flops": 0.0}
    if case["call"] == "fork":  # a page in and out of about a third of the rows
        rows = max(1.0, 0.35 * case["R"] * (case["W"] - 1))
        return {"bytes": rows * case["L"] * H * 2.0 * 2.0 * PAGE * d, "flops": 0.0}
    # the kept rows in and out, and the fork's copies of the last pages
    last = 2.0 * 2.0 * PAGE * d if case["n"] % PAGE else 0.0
    return {"bytes": case["B"] * case["L"] * H * (4.0 * d * case["k"] + last), "flops": 0.0}


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_attend(q, k, v, first, scale, slope):
    """One head of one sequence: [nq, d], [nk, d] -> [nq, d]."""
    i = torch.arange(q.shape[0], device="cuda", dtype=torch.float64)[:, None] + first
    gap = i - torch.arange(k.shape[0], device="cuda", dtype=torch.float64)
    x = torch.mm(q.double(), k.double().t()) * scale - slope * gap
    x = torch.where(gap < 0, -math.inf, x)
    w = torch.exp(x - x.amax(1, keepdim=True))
    return torch.mm(w, v.double()) / w.sum(1, keepdim=True)


def _exact_prompt(case, seed):
    s = _prepare_prompt(case, seed)
    B, H, G, d = (case[x] for x in ("B", "H", "G", "d"))
    if sum(a * b for a, b in zip(s["nq"], s["nk"])) * H * G * d > 8e11:
        return None
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        nq, nk = s["nq"][b], s["nk"][b]
        for h in range(H * G):
            if case["ragged"] == "packed":
                a, c = s["q_start"][b], s["k_start"][b]
                q, k, v, o = s["Q"][a:a + nq, h], s["K"][c:c + nk, h // G], s["V"][c:c + nk, h // G], out[a:a + nq, h]
            else:
                q, k, v, o = s["Q"][b, h, :nq], s["K"][b, h // G, :nk], s["V"][b, h // G, :nk], out[b, :nq, h]
            slope = 0.0 if s["slopes"] is None else float(s["slopes"][h])
            for x in range(0, nq, 2048):
                y = min(nq, x + 2048)
                see = nk - nq + y  # keys that the rows before y see
                o[x:y] = _exact_attend(q[x:y], k[:see], v[:see], nk - nq + x, _scale(case), slope)
    return out


def _exact_step(case, seed):
    s = _prepare_step(case, seed)
    L, B, H, G, d = (case[x] for x in ("L", "B", "H", "G", "d"))
    out = torch.zeros((L, B, H * G, d), dtype=torch.float64, device="cuda")
    c = torch.arange(256, device="cuda")
    e, m = (c >> 3) & 15, (c & 7).double()
    stands = torch.where(e == 0, m * 2.0 ** -9, (8.0 + m) * torch.exp2(e.double() - 10.0)) * torch.where(c >= 128, -1.0, 1.0)
    for l in range(L):
        for b in range(B):
            n = s["lens"][b]
            at = s["table"][b, :_pages_of(n)].long()
            K = (stands[s["K"][l, at].long()] * s["k_scale"][l, at].double()[..., None, None]).permute(1, 0, 2, 3).reshape(H, -1, d)[:, :n - 1]
            V = (stands[s["V"][l, at].long()] * s["v_scale"][l, at].double()[..., None, None]).permute(1, 0, 3, 2).reshape(H, -1, d)[:, :n - 1]
            K, V = (torch.cat([x, y[0, l, b].double()[:, None]], 1) for x, y in ((K, s["k"]), (V, s["v"])))
            x = (s["q"][0, l, b].double().view(H, G, 1, d) * _scale(case) * K[:, None]).sum(-1) if n < 64 else \
                torch.bmm(s["q"][0, l, b].double().view(H, G, d) * _scale(case), K.transpose(1, 2).contiguous())
            if s["slopes"] is not None:
                x = x - s["slopes"].double().view(H, G, 1) * (n - 1 - torch.arange(n, device="cuda", dtype=torch.float64))
            w = torch.exp(x - x.amax(-1, keepdim=True))
            out[l, b] = (torch.bmm(w, V) / w.sum(-1, keepdim=True)).view(H * G, d)
    return {"out": out, "K": None, "V": None, "k_scale": None, "v_scale": None}


def exact(case, seed):
    if case["call"] == "prompt":
        return _exact_prompt(case, seed)
    if case["call"] == "step":
        return _exact_step(case, seed)
    return None  # page numbers, moves, and codes that are fixed to the bit
