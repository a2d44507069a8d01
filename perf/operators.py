"""Operators of a key-value cache held in 4 bits: written as keys and values arrive, read back, attended over.

What the cache is: every group of `group` channels of a token's head vector keeps a scale s and a minimum m in fp16 and one
4-bit code c a channel; it stands for the value fp16(s c + m).  With x' the group's values within +-65504,

  m = fp16(min x'),  s = (max x' - m) / 15 rounded to fp16 toward zero (at least 0),
  c = (x' - m) / s rounded to the nearest whole number, halves to even, held to 0 .. 15 (0 where s is 0);

a group with a NaN or an infinity stands for NaN.  Codes are bytes [seqs, kv_heads, rows, d / 2], channel 2j in the low half of
byte j; scales and minima are fp16 [seqs, kv_heads, d / group, rows, 2].

Kinds of case, each a pass as a serving program makes it:

  write   the keys and values of new tokens into the cache, and the values that the cache now stands for
  read    keys and values of a cache as dense vectors
  step    one decoding step of one layer: the new tokens written, then attention of one query per head
  attend  softmax attention of one query, of several (each sees the tokens up to its own), over a cache

Inputs: N(0,1) values and queries, N(0,1) keys with eight channels per head ten times larger.
"""
import math

import torch

own = False

LIMIT = 65504.0   # the largest fp16


def _case(kind, **over):
    c = dict(kind=kind, dtype="f16", seqs=1, kv_heads=8, q_heads=32, d=128, group=64, rows=4096, new=1, queries=1, ragged=False)
    c.update(over)
    return c


def listed():
    cases = {
        # the prompt of the benchmark's layer, 32 key-value heads: written once, and what the cache then stands for
        "write_prompt": _case("write", kv_heads=32, q_heads=32, new=4096),
        # a padded batch of prompts behind shared beginnings of other lengths, odd sizes, one scale a head vector
        "write_ragged_bf16": _case("write", dtype="bf16", seqs=6, group=128, rows=4300, new=2111, ragged=True),
        # the smallest configuration's type, heads of 64 channels
        "write_f32": _case("write", dtype="f32", seqs=2, kv_heads=4, q_heads=4, d=64, group=32, rows=1024, new=1000),
        # the dense keys and values of the benchmark's layer rebuilt
        "read_layer": _case("read", kv_heads=32, q_heads=32),
        # long caches of several sequences for a program that works on fp32
        "read_long_f32": _case("read", dtype="f32", seqs=4, d=64, group=32, rows=32768, ragged=True),
        # serving one sequence with a short context: the smallest call, latency counts
        "step_short": _case("step", rows=517),
        # serving a batch of sequences of different lengths
        "step_batch_bf16": _case("step", dtype="bf16", seqs=64, group=128, rows=2048, ragged=True),
        # long contexts, one query head per key-value head, the finest groups
        "attend_long": _case("attend", seqs=4, kv_heads=32, group=32, rows=32768),
        # the largest caches: eight sequences of different lengths, four query heads per key-value head
        "attend_gqa_ragged_bf16": _case("attend", dtype="bf16", seqs=8, rows=131072, ragged=True),
        # several drafted tokens of every sequence looked at together
        "attend_drafts": _case("attend", seqs=16, rows=8192, queries=5, ragged=True),
        # a chunk of a long prompt over the cache of the chunks before it and its own
        "attend_prompt": _case("attend", rows=10240, queries=2048),
        # fp32 queries, heads of 64 channels, two query heads per key-value head
        "attend_f32": _case("attend", dtype="f32", seqs=2, q_heads=16, d=64, group=32),
    }
    return [dict(c, name=name) for name, c in cases.items()]


# The most that a drawn case may ask for: the vectors of the largest listed caches of each kind, and the products of the prompt chunk.
_MOST_VECTORS = {"write": 32 * 4096, "read": 4 * 8 * 32768, "step": 8 * 8 * 131072 // 8, "attend": 8 * 8 * 131072}
_MOST_FLOPS = 4.0 * 128 * 32 * 2048 * 9216


def _spread(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    kind = rng.choice(["write", "write", "read", "step", "step", "attend", "attend", "attend", "attend"])
    kv_heads, share = rng.choice([(32, 1), (32, 1), (8, 4), (8, 4), (4, 8), (16, 2), (1, 1), (2, 7)])
    d = rng.choice([128, 128, 128, 64])
    c = _case(kind, dtype=rng.choice(["f16", "f16", "bf16", "bf16", "f32"]), kv_heads=kv_heads, q_heads=kv_heads * share, d=d,
              group=rng.choice([g for g in (32, 64, 128) if g <= d]), ragged=rng.random() < 0.4)
    blocks = _MOST_VECTORS[kind] // kv_heads
    c["seqs"] = min(_spread(rng, 1, 64), blocks // 64)
    c["rows"] = _spread(rng, 64, min(131072, blocks // c["seqs"]))
    if kind == "write":
        c["new"] = _spread(rng, 1, c["rows"])
    if kind == "attend" and rng.random() < 0.5:
        c["queries"] = _spread(rng, 2, min(2048, c["rows"]))
        most = 32 if c["dtype"] == "f32" else 1   # fp32 queries: a few, not whole prompts
        c["queries"] = max(1, min(c["queries"], int(_MOST_FLOPS / most / (4.0 * d * c["q_heads"] * c["seqs"] * c["rows"]))))
    return c


# ---------------------------------------------------------------------------------------------------------------------
_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _lengths(case):
    """Tokens of every sequence: all rows, or a batch whose shortest sequence has about half."""
    B, T = case["seqs"], case["rows"]
    return [T - (b * T) // (2 * B) if case["ragged"] else T for b in range(B)]


def _write_rows(case):
    """First row and number of the new tokens of every sequence: they end where the sequence does."""
    lens, n = _lengths(case), case["new"]
    counts = [max(1, n - (b * n) // (2 * case["seqs"])) if case["ragged"] else n for b in range(case["seqs"])]
    counts = [min(k, length) for k, length in zip(counts, lens)]
    return [length - k for k, length in zip(counts, lens)], counts


def _vectors(case, gen, heads, tokens, keys=False):
    """[heads, tokens, d]"""
    x = torch.randn(heads, tokens, case["d"], device="cuda", generator=gen)
    if keys:
        gain = torch.ones(heads, 1, case["d"], device="cuda")
        gain.scatter_(2, torch.rand(heads, 1, case["d"], device="cuda", generator=gen).argsort(dim=2)[..., :8], 10.0)
        x *= gain
    return x.to(_TYPES[case["dtype"]])


def _quantised(x, group):
    """Codes and (s, m) of vectors x [..., rows, d]: uint8 [..., rows, d], fp16 [..., d / group, rows, 2].  In 64 bits: a code next
    to a half and a scale next to a step of fp16 are not to depend on the rounding of a difference."""
    g = x.double().unflatten(-1, (-1, group))
    bad = ~torch.isfinite(g).all(dim=-1, keepdim=True)
    g = torch.where(bad, 0.0, g).clamp(-LIMIT, LIMIT)
    m = g.amin(dim=-1, keepdim=True).half()
    span = (g.amax(dim=-1, keepdim=True) - m.double()).clamp(min=0)
    s = (span / 15).half()
    s = torch.where(15 * s.double() > span, (s.view(torch.int16) - 1).view(torch.float16), s)   # toward zero
    c = torch.where(s > 0, (g - m.double()) / s.double(), 0.0).round().clamp(0, 15).to(torch.uint8)
    params = torch.where(bad, float("nan"), torch.cat([s, m], dim=-1))
    return c.flatten(-2), params.movedim(-2, -3).contiguous()


def _packed(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _unpacked(codes, params):
    """Values, in fp32, of rows [..., rows, d / 2] with params [..., d / group, rows, 2]"""
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).float()
    s, m = params.movedim(-3, -2).float().split(1, dim=-1)
    return (c.unflatten(-1, (s.shape[-2], -1)) * s + m).half().float().flatten(-2)


def prepare(case, seed):
    c, dt = case, _TYPES[case["dtype"]]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    B, Hkv, d, T, NG = c["seqs"], c["kv_heads"], c["d"], c["rows"], c["d"] // c["group"]
    st = dict(case=c)
    for name in ("k", "v"):
        codes = torch.zeros(B, Hkv, T, d // 2, dtype=torch.uint8, device="cuda")
        params = torch.zeros(B, Hkv, NG, T, 2, dtype=torch.float16, device="cuda")
        for b in range(B if c["kind"] != "write" else 0):   # a sequence at a time: the 64-bit parts stay small
            x, params[b] = _quantised(_vectors(c, gen, Hkv, T, name == "k"), c["group"])
            codes[b] = _packed(x)
        st["codes_" + name], st["params_" + name] = codes, params
        if c["kind"] in ("write", "step"):   # tokens as a projection leaves them: [seqs, tokens, heads, d], seen head by head
            x = torch.stack([_vectors(c, gen, Hkv, c["new"], name == "k") for _ in range(B)])
            st["new_" + name] = x.transpose(1, 2).contiguous().transpose(1, 2)
    st["q"] = torch.randn(B, c["queries"], c["q_heads"], d, device="cuda", generator=gen).to(dt).transpose(1, 2)
    pos, counts = _write_rows(c)
    st["pos"] = torch.tensor(pos, dtype=torch.int32, device="cuda")
    st["counts"] = torch.tensor(counts, dtype=torch.int32, device="cuda")
    st["lens"] = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    return st


# ---------------------------------------------------------------------------------------------------------------------
def _write(st):
    """The new tokens' codes and parameters into the cache; the values they stand for, zeros where a sequence has no token"""
    c, t = st["case"], torch.arange(st["case"]["new"], device="cuda")
    fresh = t < st["counts"][:, None]
    b, t = fresh.nonzero(as_tuple=True)
    rows, out = st["pos"].long()[b] + t, []
    for name in ("k", "v"):
        x, params = _quantised(st["new_" + name], c["group"])
        codes = _packed(x)
        st["codes_" + name][b, :, rows] = codes[b, :, t]
        st["params_" + name][b, :, :, rows] = params[b, :, :, t]
        out.append(torch.where(fresh[:, None, :, None], _unpacked(codes, params), 0.0).to(_TYPES[c["dtype"]]))
    return tuple(out)


def _read(st):
    held = torch.arange(st["case"]["rows"], device="cuda") < st["lens"][:, None]
    return tuple(torch.where(held[:, None, :, None], _unpacked(st["codes_" + n], st["params_" + n]), 0.0).to(_TYPES[st["case"]["dtype"]])
                 for n in ("k", "v"))


def _attend(st):
    c = st["case"]
    B, Hkv, n, T, d = c["seqs"], c["kv_heads"], c["queries"], c["rows"], c["d"]
    q = st["q"].float().reshape(B, Hkv, -1, d)   # a key-value head's queries: head by head, token by token
    k, v = (_unpacked(st["codes_" + x], st["params_" + x]) for x in ("k", "v"))
    score = (q @ k.transpose(2, 3).contiguous()) / math.sqrt(d)
    limit = st["lens"][:, None] - n + torch.arange(n, device="cuda")   # the token that each query stands at
    seen = (torch.arange(T, device="cuda") <= limit[..., None])[:, None, None]
    score = score.view(B, Hkv, -1, n, T).masked_fill(~seen, -math.inf).view(B, Hkv, -1, T)
    top = score.amax(dim=-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    out = p @ v / p.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    return out.view(B, c["q_heads"], n, d).to(st["q"].dtype)


def _run_own(st):
    import paper_2412_11741_amd as csr
    c, K, V = st["case"], (st["codes_k"], st["params_k"]), (st["codes_v"], st["params_v"])
    if c["kind"] == "read":
        dt = _TYPES[c["dtype"]]
        return csr.csr_q4_read(*K, counts=st["lens"], out_dtype=dt), csr.csr_q4_read(*V, counts=st["lens"], out_dtype=dt)
    if c["kind"] == "write":
        return csr.csr_q4_write(st["new_k"], *K, st["new_v"], *V, pos=st["pos"], counts=st["counts"], values=True)
    if c["kind"] == "attend":
        return csr.csr_q4_attn(st["q"], *K, *V, seq_lens=st["lens"])
    new = csr.csr_q4_write(st["new_k"], *K, st["new_v"], *V, pos=st["pos"], values=True)
    return (csr.csr_q4_attn(st["q"], *K, *V, seq_lens=st["lens"]),) + new


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "read":
        return _read(state)
    if kind == "write":
        return _write(state)
    if kind == "attend":
        return _attend(state)
    new = _write(state)
    return (_attend(state),) + new


# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    e, lens = {"f16": 2, "bf16": 2, "f32": 4}[c["dtype"]], _lengths(c)
    vector = c["d"] // 2 + 4 * (c["d"] // c["group"])   # bytes of a head vector in the cache
    pairs, n = 2.0 * c["kv_heads"], c["queries"]         # a key and a value per head
    byts = flops = 0.0
    if c["kind"] in ("write", "step"):
        new = pairs * sum(_write_rows(c)[1])
        byts += new * (2 * c["d"] * e + vector)
        flops += new * c["d"] * 6.0
        if c["kind"] == "write":   # zeros behind the shorter sequences
            byts += (pairs * c["seqs"] * c["new"] - new) * c["d"] * e
    if c["kind"] == "read":
        byts += pairs * (sum(lens) * vector + c["seqs"] * c["rows"] * c["d"] * e)
        flops += pairs * sum(lens) * c["d"] * 2.0
    if c["kind"] in ("step", "attend"):
        byts += pairs * sum(lens) * vector + 2.0 * c["seqs"] * c["q_heads"] * n * c["d"] * e
        seen = sum(max(0, length - n + i + 1) for length in lens for i in range(n))
        flops += 4.0 * c["d"] * c["q_heads"] * seen
    return {"bytes": byts, "flops": flops}


def exact(case, seed):
    """run()'s outputs from the definitions in 64 bits, sequence by sequence"""
    st = prepare(case, seed)
    c, d, group = case, case["d"], case["group"]
    lens, (pos, counts) = _lengths(c), _write_rows(c)

    def values(s, m, code):   # fp16(s c + m): both terms are fp16's, their sum is exact in 64 bits
        return (s.double() * code + m.double()).half().double()

    def written(x):   # [heads, tokens, d]
        x = x.double().reshape(x.shape[0], x.shape[1], d // group, group).clamp(-65504, 65504)
        m = x.min(dim=3).values.half().double()
        span = x.max(dim=3).values - m
        s = (span.clamp(min=0) / 15).half().double()
        below = torch.nextafter(s.half(), torch.full_like(s, -1).half()).double()
        s = torch.where(s * 15 > span.clamp(min=0), below, s)
        u = (x - m[..., None]) / torch.where(s > 0, s, torch.inf)[..., None]
        low = torch.floor(u)
        odd, rest = torch.remainder(low, 2), u - low
        code = (low + ((rest > 0.5) | ((rest == 0.5) & (odd == 1)))).clamp(0, 15)
        return values(s[..., None], m[..., None], code).reshape(x.shape[0], x.shape[1], d)

    def held(name, b, rows):   # [heads, rows, d] of sequence b
        codes, params = st["codes_" + name][b, :, :rows], st["params_" + name][b, :, :, :rows]
        code = torch.empty(codes.shape[0], rows, d, dtype=torch.float64, device=codes.device)
        code[..., 0::2], code[..., 1::2] = codes % 16, codes // 16
        s, m = (params[..., k].permute(0, 2, 1).repeat_interleave(group, dim=2) for k in (0, 1))
        return values(s, m, code)

    new, dense = {}, {"k": [], "v": []}
    for name in ("k", "v") if c["kind"] in ("write", "step") else ():
        new[name] = torch.zeros(c["seqs"], c["kv_heads"], c["new"], d, dtype=torch.float64, device="cuda")
        for b in range(c["seqs"]):
            new[name][b, :, :counts[b]] = written(st["new_" + name][b, :, :counts[b]])
    if c["kind"] == "write":
        return new["k"], new["v"]
    if c["kind"] == "read":
        for name in ("k", "v"):
            for b in range(c["seqs"]):
                x = torch.zeros(c["kv_heads"], c["rows"], d, dtype=torch.float64, device="cuda")
                x[:, :lens[b]] = held(name, b, lens[b])
                dense[name].append(x)
        return torch.stack(dense["k"]), torch.stack(dense["v"])
    n, share = c["queries"], c["q_heads"] // c["kv_heads"]
    out = torch.zeros(c["seqs"], c["q_heads"], n, d, dtype=torch.float64, device="cuda")
    for b in range(c["seqs"]):
        k, v = held("k", b, lens[b]), held("v", b, lens[b])
        if c["kind"] == "step":
            k[:, pos[b]], v[:, pos[b]] = new["k"][b, :, 0], new["v"][b, :, 0]
        at = torch.arange(lens[b], device="cuda")
        stands = lens[b] - n + torch.arange(n, device="cuda")
        for h in range(c["q_heads"]):
            score = (st["q"][b, h].double() @ k[h // share].T) * d ** -0.5
            score[at[None, :] > stands[:, None]] = -torch.inf
            some = stands >= 0
            out[b, h, some] = torch.softmax(score[some], dim=-1) @ v[h // share]
    return (out, new["k"], new["v"]) if c["kind"] == "step" else out
