"""The operators around the retained rows of a streaming video dialogue, and what they are timed on.

  rotary    positions with three axes (time, height, width) turned into the rotation of Q and K, before the rows are attended to
            and kept
  cache     retained rows held in 8 bits: quantised as they are written, and read back
  decode    one step of several ragged streams over such caches, the new row quantised and kept
  prefill   a frame, or a question, over such a cache: the carrier's row, or all rows, quantised and kept

What a row of 8 bits is: for every token and KV head, of K and of V, x is held as the whole number q = rint(x / s) (ties to
even), -127..127, beside s = max(ceil8(max|x| / 127), 2^-126), where ceil8 goes up to the next number of 8 significant bits
(a bfloat16).  It stands for q * s.
"""
import ctypes
import random

import torch

own = False

DEV = "cuda:0"
NEAREST = 2.0 ** -126


def listed():
    return [
        # one decoding step's positions: a token for each of 16 streams, layer by layer: latency
        dict(name="rotary_step", kind="rotary", dtype="bf16", hq=28, hkv=4, dim=128, layers=28, tokens=16, pairing="halves", inverse=False),
        # a frame of 13 x 13 tokens and its carrier, in four layers
        dict(name="rotary_frame", kind="rotary", dtype="bf16", hq=28, hkv=4, dim=128, layers=4, tokens=170, pairing="halves", inverse=False),
        # a long run in one call, turned back (what the gradients of a rotation are, and rows that are to be turned anew)
        dict(name="rotary_long", kind="rotary", dtype="bf16", hq=28, hkv=4, dim=128, layers=1, tokens=16384, pairing="halves", inverse=True),
        # the tiny fp32 configuration's heads, over 64 frames of 49 + 1 tokens
        dict(name="rotary_fp32", kind="rotary", dtype="f32", hq=4, hkv=1, dim=64, layers=1, tokens=3200, pairing="adjacent", inverse=False),
        # a frame's carrier rows of 28 layers at once, and what is kept of them
        dict(name="cache_carrier", kind="cache", hkv=4, caches=28, rows=4424, tokens=1),
        # a question's rows of 28 layers
        dict(name="cache_question", kind="cache", hkv=4, caches=28, rows=4552, tokens=37),
        # uncompressed caches of the visual rows of 64 frames, turned into 8 bits layer after layer, four of them here
        dict(name="cache_dense", kind="cache", hkv=4, caches=4, rows=0, tokens=11016),
        # one user's answer after a short video
        dict(name="decode_one", kind="decode", hq=28, hkv=4, layers=28, streams=1, lo=700, hi=700, lens_seed=0),
        # 16 ragged streams of 512..8192 carriers and 128 text rows
        dict(name="decode_16", kind="decode", hq=28, hkv=4, layers=28, streams=16, lo=640, hi=8320, lens_seed=3),
        # a question of 37 tokens after a short video
        dict(name="prefill_question", kind="prefill", hq=28, hkv=4, layers=28, rows=711, tokens=37, kept="all"),
        # hours into a video: one frame through the attention of all 28 layers
        dict(name="prefill_frame", kind="prefill", hq=28, hkv=4, layers=28, rows=4424, tokens=170, kept="carrier"),
        # the same frame over an uncompressed cache
        dict(name="prefill_dense", kind="prefill", hq=28, hkv=4, layers=4, rows=11016, tokens=170, kept="carrier"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "cache", "cache", "decode", "decode", "decode", "prefill", "prefill"])
    hq, hkv = rng.choice([(28, 4), (28, 4), (28, 4), (16, 2), (24, 8), (12, 6), (5, 5), (8, 1)])
    if kind == "rotary":
        f32 = rng.random() < 0.3
        c = dict(kind=kind, dtype="f32" if f32 else "bf16", hq=hq, hkv=hkv, dim=rng.choice([64, 128]) if f32 else 128,
                 layers=rng.choice([1, 4, 28]), tokens=_log_int(rng, 1, 16384), pairing=rng.choice(["halves", "halves", "adjacent"]),
                 inverse=rng.random() < 0.3)
    elif kind == "cache":
        c = dict(kind=kind, hkv=hkv, caches=_log_int(rng, 1, 112), rows=rng.choice([0, _log_int(rng, 1, 8192)]), tokens=_log_int(rng, 1, 11016))
    elif kind == "decode":
        lo = _log_int(rng, 1, 4096)
        c = dict(kind=kind, hq=hq, hkv=hkv, layers=rng.choice([4, 28]), streams=_log_int(rng, 1, 96), lo=lo, hi=lo + rng.randint(0, 8320 - lo),
                 lens_seed=rng.randrange(1000))
    else:
        c = dict(kind=kind, hq=hq, hkv=hkv, layers=rng.choice([1, 4, 28]), rows=_log_int(rng, 1, 11016),
                 tokens=rng.choice([_log_int(rng, 1, 256), rng.randint(100, 192)]), kept=rng.choice(["carrier", "all"]))
    # no more than the largest listed one
    while _cost(c) > 7.0e9 or work(c)["bytes"] > 2.4e9:
        key = max((k for k in ("layers", "caches", "streams", "tokens") if c.get(k, 1) > 1), key=lambda k: c[k])
        c[key] //= 2
    return c


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def _lens(c):
    r = random.Random(c["lens_seed"])
    return [r.randint(c["lo"], c["hi"]) for _ in range(c["streams"])]


def _sections(dim):
    return (dim // 8, dim * 3 // 16, dim * 3 // 16)


THETA = 1e6


def work(case):
    c, kind = case, case["kind"]
    if kind == "rotary":
        values = c["layers"] * c["tokens"] * (c["hq"] + c["hkv"]) * c["dim"]
        return {"bytes": 2 * values * (4 if c["dtype"] == "f32" else 2) + c["layers"] * 12 * c["tokens"], "flops": 3 * values}
    hkv = c["hkv"]
    row8 = 2 * hkv * (128 + 2)  # K and V of a row: a byte a value and 2 for each head's scale
    row16 = 2 * hkv * 256
    if kind == "cache":
        n = c["caches"] * c["tokens"]
        return {"bytes": n * 2 * (row16 + row8), "flops": n * 8 * hkv * 128}
    hq = c["hq"]
    if kind == "decode":
        rows = sum(_lens(c))
        return {"bytes": c["layers"] * (rows * row8 + c["streams"] * (2 * row16 + 2 * row8 + 2 * hq * 256)),
                "flops": c["layers"] * 4 * hq * 128 * (rows + c["streams"])}
    T, L = c["tokens"], c["rows"]
    kept = T if c["kept"] == "all" else 1
    return {"bytes": c["layers"] * (L * row8 + T * (2 * hq * 256 + row16) + kept * (2 * row8 + row16)),
            "flops": c["layers"] * 4 * hq * 128 * (T * L + T * (T + 1) // 2)}


# ------------------------------------------------------------------------------------------------ inputs
class _Draw:
    """Normal draws on the GPU, from the seed alone."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed)

    def __call__(self, *dims, sigma=0.5, dtype=torch.bfloat16):
        return torch.randn(dims, generator=self.g, device=DEV, dtype=dtype).mul_(sigma)


def _rows(rn, n, rows, hkv):
    """K or V rows: some channels and some tokens are several times the others, as projections' outputs are."""
    x = rn(n, rows, hkv, 128)
    loud = 1 + 7 * (torch.rand((n, 1, hkv, 128), generator=rn.g, device=DEV) < 0.03)
    size = 0.5 + 1.5 * torch.rand((n, rows, hkv, 1), generator=rn.g, device=DEV)
    return x.mul_(loud.to(x.dtype)).mul_(size.to(x.dtype))


def _positions(rng, tokens):
    """Time, height and width of the tokens of consecutive frames of 13 x 13 tokens and their carrier (at the middle), somewhere
    into a stream."""
    at = rng.randrange(0, 200000)
    t = torch.arange(tokens, dtype=torch.int64)
    frame, i = t // 170, t % 170
    i = torch.where(i == 169, torch.full_like(i, 84), i)
    return torch.stack([at + frame, at + i // 13, at + i % 13]).to(torch.int32).to(DEV)


def _inputs(case, seed):
    """The tensors of a case, the retained rows as they were before they were quantised."""
    c, rn, kind = case, _Draw(seed), case["kind"]
    if kind == "rotary":
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        return dict(q=rn(c["layers"], c["tokens"], c["hq"], c["dim"], dtype=dt), k=rn(c["layers"], c["tokens"], c["hkv"], c["dim"], dtype=dt),
                    pos=_positions(random.Random(seed), c["tokens"]))
    if kind == "cache":
        return dict(k=_rows(rn, c["caches"], c["tokens"], c["hkv"]), v=_rows(rn, c["caches"], c["tokens"], c["hkv"]))
    if kind == "decode":
        n, most = c["layers"] * c["streams"], max(_lens(c))
        return dict(k=_rows(rn, n, most, c["hkv"]), v=_rows(rn, n, most, c["hkv"]), q=rn(c["layers"], c["streams"], c["hq"], 128, sigma=1.0),
                    kn=_rows(rn, n, 1, c["hkv"]), vn=_rows(rn, n, 1, c["hkv"]))
    n, T = c["layers"], c["tokens"]
    return dict(k=_rows(rn, n, c["rows"], c["hkv"]), v=_rows(rn, n, c["rows"], c["hkv"]), q=rn(n, T, c["hq"], 128, sigma=1.0),
                kn=_rows(rn, n, T, c["hkv"]), vn=_rows(rn, n, T, c["hkv"]))


def prepare(case, seed):
    s = dict(case=case, **_inputs(case, seed))
    return _prepare_own(s) if own else _prepare_plain(s)


def _caches(c):
    """How many caches a case has, the rows that are retained in each, the rows that a pass keeps, and the rows there is room for."""
    if c["kind"] == "cache":
        return c["caches"], c["rows"], c["tokens"], c["rows"] + c["tokens"] + 5
    if c["kind"] == "decode":
        return c["layers"] * c["streams"], max(_lens(c)), 1, max(_lens(c)) + 64
    return c["layers"], c["rows"], c["tokens"] if c["kept"] == "all" else 1, c["rows"] + c["tokens"]


def _prepare_plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rotary":
        return s
    n, rows, _, cap = _caches(c)
    s["cache"] = [_held(n, cap, c["hkv"]) for _ in "kv"]
    if kind != "cache":
        for held, r in zip(s["cache"], (s.pop("k"), s.pop("v"))):
            held["q"][:, :rows], held["s"][:, :rows] = _quantise(r)
    if kind == "decode":
        s["new"] = torch.tensor(_lens(c), device=DEV).repeat(c["layers"])
        s["mask"] = torch.arange(rows + 1, device=DEV)[None, :] <= s["new"][:, None]
    return s


def _prepare_own(s):
    import paper_2503_09387_amd as vs
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rotary":
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["shape"] = vs.Shape.make(c["hq"], c["hkv"], c["dim"], c["dtype"])
        s["plan"] = vs.RotaryPlan(c["dim"], _sections(c["dim"]), THETA, vs.ROTARY_HALVES if c["pairing"] == "halves" else vs.ROTARY_ADJACENT)
        s["calls"] = [(s["q"][i], s["k"][i], s["q_out"][i], s["k_out"][i]) for i in range(c["layers"])]
        return s
    n, rows, kept, s["cap"] = _caches(c)
    s["shape"] = vs.Shape.make(c.get("hq", c["hkv"]), c["hkv"], 128, "bf16")
    s["slab"] = torch.zeros((n, vs.cache8_bytes(s["shape"], s["cap"])), dtype=torch.uint8, device=DEV)
    lens, firsts = (ctypes.c_int32 * n)(), [rows] * n
    if kind == "cache":
        s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
        s["lens"] = lens
    else:
        vs.cache8_append(s["shape"], s["slab"], s["cap"], lens, s.pop("k"), s.pop("v"))
        s["out"] = torch.empty_like(s["q"])
        s["kept"] = [torch.empty((n, kept, c["hkv"], 128), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    if kind == "decode":
        S = c["streams"]
        firsts, s["first"] = _lens(c) * c["layers"], _lens(c)
        s["calls"] = [(s["slab"][i:i + S], (ctypes.c_int32 * S)(), s["q"][i // S], s["kn"][i:i + S, 0], s["vn"][i:i + S, 0], s["out"][i // S])
                      for i in range(0, n, S)]
        s["ws"] = vs.make_cache8_workspace(s["shape"], 0, s["cap"], S, DEV)
    elif kind == "prefill":
        s["calls"] = [(vs.Cache8(s["slab"][i], s["cap"]), s["q"][i], s["kn"][i], s["vn"][i], s["out"][i]) for i in range(n)]
        s["first_kept"] = c["tokens"] - kept
        s["ws"] = vs.make_cache8_workspace(s["shape"], c["tokens"], rows, 0, DEV)
    s["firsts"], s["after"] = (ctypes.c_int32 * n)(*firsts), (ctypes.c_int32 * n)(*[m + kept for m in firsts])
    return s


# ------------------------------------------------------------------------------------------------ a pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2503_09387_amd as vs
    c, kind, stream = s["case"], s["case"]["kind"], vs.current_stream_handle()
    if kind == "rotary":
        for q, k, q_out, k_out in s["calls"]:
            vs.rotary(s["shape"], s["plan"], s["pos"], q, k, q_out, k_out, inverse=c["inverse"], stream=stream)
        return [s["q_out"], s["k_out"]]
    if kind == "cache":
        s["lens"][:] = s["firsts"]  # (a pass starts where the one before it did)
        vs.cache8_append(s["shape"], s["slab"], s["cap"], s["lens"], s["k"], s["v"], stream=stream)
        vs.cache8_read(s["shape"], s["slab"], s["cap"], s["lens"], s["firsts"], s["k_out"], s["v_out"], stream=stream)
        return [s["k_out"], s["v_out"]]
    if kind == "decode":
        for slab, lens, q, kn, vn, out in s["calls"]:
            lens[:] = s["first"]
            vs.cache8_decode_attn(s["shape"], slab, s["cap"], lens, q, kn, vn, out, s["ws"], stream=stream)
    else:
        for cache, q, k, v, out in s["calls"]:
            cache.len = c["rows"]
            vs.cache8_prefill_attn(s["shape"], cache, q, k, v, out, s["ws"], first_kept=s["first_kept"], stream=stream)
    # the rows that the pass has kept, as what they stand for
    vs.cache8_read(s["shape"], s["slab"], s["cap"], s["after"], s["firsts"], *s["kept"], stream=stream)
    return [s["out"], *s["kept"]]


def _held(n, cap, hkv):
    return dict(q=torch.zeros((n, cap, hkv, 128), dtype=torch.int8, device=DEV), s=torch.zeros((n, cap, hkv, 1), dtype=torch.bfloat16, device=DEV))


def _quantise(x):
    """Rows [..][128] -> whole numbers and their scales."""
    x = x.float()
    most = x.abs().amax(-1, keepdim=True) / 127
    up = ((most.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32).clamp_min(NEAREST)
    return torch.round(x / up).to(torch.int8), up.to(torch.bfloat16)


def _value(held, sl):
    return held["q"][sl].float() * held["s"][sl].float()


def _attend(q, k, v, seen):
    """q [n][T][Hq][128] over k, v [n][L][Hkv][128], all in 32 bits; seen: what token t of cache i sees, broadcast to [n][T][L]."""
    n, T, hq, d = q.shape
    hkv = k.shape[2]
    g = hq // hkv
    qs = q.float().reshape(n, T, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, T * g, d)
    score = torch.matmul(qs, k.permute(0, 2, 3, 1).contiguous()).mul_(d ** -0.5).reshape(n, hkv, T, g, -1)
    score.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    p = torch.exp(score - score.amax(-1, keepdim=True))
    p = (p / p.sum(-1, keepdim=True)).reshape(n, hkv, T * g, -1)
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous()).reshape(n, hkv, T, g, d)
    return o.permute(0, 2, 1, 3, 4).reshape(n, T, hq, d).to(q.dtype)


def _rotate(x, cos, sin, halves):
    x, p = x.float(), cos.shape[-1]
    a, b = (x[..., :p], x[..., p:2 * p]) if halves else (x[..., 0:2 * p:2], x[..., 1:2 * p:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([a, b], -1) if halves else torch.stack([a, b], -1).flatten(-2)


def _run_plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rotary":
        n = c["dim"] // 2
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(_sections(c["dim"]), device=DEV), output_size=n)
        # (angles in 64 bits: far positions)
        angle = s["pos"].double()[axis].T * THETA ** (-torch.arange(n, device=DEV, dtype=torch.float64) / n)
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
        sin = -sin if c["inverse"] else sin
        return [_rotate(s[t], cos, sin, c["pairing"] == "halves").to(s[t].dtype) for t in "qk"]
    (ck, cv), rows = s["cache"], c.get("rows", 0)
    if kind == "cache":
        kept = slice(None), slice(rows, rows + c["tokens"])
        (ck["q"][kept], ck["s"][kept]), (cv["q"][kept], cv["s"][kept]) = _quantise(s["k"]), _quantise(s["v"])
        return [_value(h, kept).to(torch.bfloat16) for h in (ck, cv)]
    if kind == "decode":
        at = torch.arange(len(s["new"]), device=DEV), s["new"]
        for held, new in ((ck, s["kn"]), (cv, s["vn"])):
            q, sc = _quantise(new[:, 0])
            held["q"][at], held["s"][at] = q, sc
        seen = slice(None), slice(0, s["mask"].shape[1])
        q = s["q"].reshape(-1, 1, c["hq"], 128)
        # (what lies behind a stream's last row is zero)
        out = _attend(q, _value(ck, seen), _value(cv, seen), s["mask"][:, None, :]).reshape(s["q"].shape)
        return [out, *(_value(h, at)[:, None].to(torch.bfloat16) for h in (ck, cv))]
    T = c["tokens"]
    old = slice(None), slice(0, rows)
    seen = torch.arange(rows + T, device=DEV)[None, None, :] <= rows + torch.arange(T, device=DEV)[None, :, None]
    out = _attend(s["q"], torch.cat([_value(ck, old), s["kn"].float()], 1), torch.cat([_value(cv, old), s["vn"].float()], 1), seen)
    m = T if c["kept"] == "all" else 1
    kept = slice(None), slice(rows, rows + m)
    (ck["q"][kept], ck["s"][kept]), (cv["q"][kept], cv["s"][kept]) = _quantise(s["kn"][:, T - m:]), _quantise(s["vn"][:, T - m:])
    return [out, *(_value(h, kept).to(torch.bfloat16) for h in (ck, cv))]


# ------------------------------------------------------------------------------------------------ in 64 bits, from the definitions
def _stands_for(x):
    x = x.double()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True) / 127)
    s = torch.ldexp(torch.ceil(m * 256), e - 8).clamp_min(NEAREST)
    return torch.round(x / s) * s


def exact(case, seed):
    c, kind, x = case, case["kind"], _inputs(case, seed)
    if kind == "rotary":
        n = c["dim"] // 2
        freq = torch.exp(-torch.log(torch.tensor(THETA, dtype=torch.float64)) * torch.arange(n, dtype=torch.float64) / n).to(DEV)
        a, b, _ = _sections(c["dim"])
        pos = x["pos"].double()
        angle = torch.cat([pos[0][:, None] * freq[:a], pos[1][:, None] * freq[a:a + b], pos[2][:, None] * freq[a + b:]], 1)
        turn = torch.polar(torch.ones_like(angle), -angle if c["inverse"] else angle)[:, None, :]
        outs = []
        for t in (x["q"], x["k"]):
            t = t.double()
            z = torch.complex(t[..., :n], t[..., n:]) if c["pairing"] == "halves" else torch.view_as_complex(t.unflatten(-1, (n, 2)).contiguous())
            z = z * turn
            outs.append(torch.cat([z.real, z.imag], -1) if c["pairing"] == "halves" else torch.view_as_real(z).flatten(-2))
        return outs
    if kind == "cache":
        return [_stands_for(x["k"]), _stands_for(x["v"])]
    if _cost(c) > 7.5e9:
        return None
    g = c["hq"] // c["hkv"]
    out = torch.empty(x["q"].shape, dtype=torch.float64, device=DEV)
    scale = 128 ** -0.5
    if kind == "decode":
        lens = _lens(c)
        for l in range(c["layers"]):
            for i, m in enumerate(lens):
                j = l * c["streams"] + i
                k, v = (torch.cat([_stands_for(x[a][j, :m]), _stands_for(x[b][j])]) for a, b in (("k", "kn"), ("v", "vn")))
                for h in range(c["hkv"]):
                    w = torch.softmax(x["q"][l, i, h * g:(h + 1) * g].double() @ k[:, h].T * scale, 1)
                    out[l, i, h * g:(h + 1) * g] = w @ v[:, h]
        return [out, _stands_for(x["kn"]), _stands_for(x["vn"])]
    T, L = c["tokens"], c["rows"]
    hidden = torch.ones((T, L + T), dtype=torch.bool, device=DEV).triu(L + 1)
    for l in range(c["layers"]):
        k, v = (torch.cat([_stands_for(x[a][l]), x[b][l].double()]) for a, b in (("k", "kn"), ("v", "vn")))
        for h in range(c["hq"]):
            z = (x["q"][l, :, h].double() @ k[:, h // g].T * scale).masked_fill(hidden, -torch.inf)
            out[l, :, h] = torch.softmax(z, 1) @ v[:, h // g]
    m = T if c["kept"] == "all" else 1
    return [out, _stands_for(x["kn"][:, T - m:]), _stands_for(x["vn"][:, T - m:])]
