"""The 4-bit cache on the GPU against its definition in 64 bits (tests/q4_reference.py).

Codes, parameters and values have to be the reference's, bit for bit.  Attention: what its roundings can amount to, counted
(see _bound)."""
import numpy as np
import pytest
import torch

import paper_2412_11741_amd as csr
from paper_2412_11741_amd import binding
from tests import q4_reference as ref
from tests.q4_plan import plan

pytestmark = pytest.mark.gpu

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF_STEP = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
NAN = float("nan")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(seed, *shape, dtype=F16, gain=None):
    x = torch.randn(*shape, device="cuda", generator=_gen(seed))
    return (x if gain is None else x * gain).to(dtype)


def _token_major(x):
    """The same [B, H, n, d] over memory [B, n, H, d]"""
    return x.transpose(1, 2).contiguous().transpose(1, 2)


def _np(t):
    return t.cpu().to(torch.float64).numpy() if t.dtype in (BF16, F16, F32) else t.cpu().numpy()


def _same(a, b):
    """Equal bit patterns of two fp16 arrays, NaNs of any kind alike"""
    return (np.asarray(a, np.float16).view(np.uint16) == np.asarray(b, np.float16).view(np.uint16)) | (np.isnan(a) & np.isnan(b))


def _hold(codes, params, want_codes, want_params, rows):
    """The cache's rows, [B][Hkv] each, are the wanted ones and the others still hold 0x77 / 7.0"""
    codes, params = codes.cpu().numpy(), params.cpu().numpy()
    for b, (first, count) in enumerate(rows):
        at = slice(first, first + count)
        assert (codes[b, :, at] == want_codes[b][:, :count]).all(), b
        assert _same(params[b, :, :, at], want_params[b][:, :, :count]).all(), b
        codes[b, :, at], params[b, :, :, at] = 0x77, 7.0
    assert (codes == 0x77).all() and (params == 7.0).all()


def _blank(B, Hkv, T, d, group):
    codes, params = csr.csr_q4_alloc(B, Hkv, T, d, group)
    return codes.fill_(0x77), params.fill_(7.0)


# ---- write and read -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("d,group", [(128, 32), (128, 64), (128, 128), (64, 32), (64, 64)])
@pytest.mark.parametrize("B,Hkv,n,T", [(1, 1, 1, 1), (2, 3, 37, 50), (3, 5, 1, 9), (1, 2, 517, 600), (2, 8, 1500, 1501)])
def test_written_rows_are_the_definitions(dtype, d, group, B, Hkv, n, T):
    gain = 10.0 ** torch.randint(-4, 4, (B, Hkv, n, 1), device="cuda", generator=_gen(n)).float()
    K, V = _randn(1, B, Hkv, n, d, dtype=dtype, gain=gain), _token_major(_randn(2, B, Hkv, n, d, dtype=dtype))
    K[0, 0, 0, :group] = 0.37                                    # a group without spread
    first = T - n
    cK, pK = _blank(B, Hkv, T, d, group)
    cV, pV = _blank(B, Hkv, T, d, 32)
    vals = csr.csr_q4_write(K, cK, pK, V, cV, pV, pos0=first, values=True)
    for X, c, p, g, got in ((K, cK, pK, group, vals[0]), (V, cV, pV, 32, vals[1])):
        codes, params = ref.quantise(_np(X), g)
        _hold(c, p, codes, params, [(first, n)] * B)
        want = torch.from_numpy(ref.values(codes, params)).to(dtype)
        assert got.dtype == dtype and torch.equal(got.cpu(), want)
        for out in (F16, BF16, F32):
            back = csr.csr_q4_read(c, p, pos0=first, out_dtype=out)
            assert back.shape == (B, Hkv, n, d) and torch.equal(back.cpu(), torch.from_numpy(ref.values(codes, params)).to(out))
    cK2, pK2 = _blank(B, Hkv, T, d, group)                       # one tensor, no values: the same cache
    assert csr.csr_q4_write(K, cK2, pK2, pos0=first) is None
    assert torch.equal(cK, cK2) and torch.equal(pK, pK2)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_codes_next_to_a_half(dtype):
    # every value at or next to the middle of two codes: steps of powers of two and others, minima far from and near zero
    d, group, n = 128, 32, 400
    r = np.random.default_rng(3)
    x = np.empty((1, 1, n, d))
    for t in range(n):
        for g in range(d // group):
            s = 2.0 ** r.integers(-12, 4) * r.integers(1024, 2048) / 1024
            m = r.choice([0.0, -7.5 * s, 100.0, -100.0, -3.0])
            u = np.concatenate([[0, 15], r.integers(0, 15, group - 2) + 0.5 + r.choice([0, 0, 1e-7, -1e-7, 1e-4, -1e-4], group - 2)])
            x[0, 0, t, g * group:(g + 1) * group] = np.float64(np.float16(m)) + s * u
    X = torch.from_numpy(x).cuda().to(dtype)
    c, p = _blank(1, 1, n, d, group)
    csr.csr_q4_write(X, c, p)
    codes, params = ref.quantise(_np(X), group)
    _hold(c, p, codes, params, [(0, n)])


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_values_at_the_ends_of_the_types(dtype):
    d, n = 64, 9
    x = torch.randn(1, 1, n, d, generator=torch.Generator().manual_seed(5))
    x[0, 0, 0, 3], x[0, 0, 1, 40], x[0, 0, 2, 63] = NAN, float("inf"), -float("inf")
    x[0, 0, 3, :2] = torch.tensor([65504.0, -65504.0])
    x[0, 0, 4] *= 6e4
    x[0, 0, 5] *= 2.0 ** -23
    x[0, 0, 6] = -0.0
    x[0, 0, 7] = 65504.0 if dtype != BF16 else 65280.0
    if dtype == F16:
        x = x.clamp(-65504, 65504).where(torch.isfinite(x), x)
    X = x.cuda().to(dtype)
    c, p = _blank(1, 1, n, d, 32)
    got = csr.csr_q4_write(X, c, p, values=True)
    codes, params = ref.quantise(_np(X), 32)
    _hold(c, p, codes, params, [(0, n)])
    want = ref.values(codes, params)
    assert _same(csr.csr_q4_read(c, p).cpu().numpy(), want).all()
    assert np.isnan(want[0, 0, :3]).any(axis=-1).all() and np.isfinite(want[0, 0, 3:]).all()
    assert torch.equal(torch.isnan(got).cpu(), torch.from_numpy(np.isnan(want)))


def test_ragged_batches_and_rows_outside_the_cache():
    B, Hkv, n, T, d, group = 5, 2, 9, 16, 128, 64
    K, V = _randn(7, B, Hkv, n, d), _randn(8, B, Hkv, n, d)
    pos = torch.tensor([0, 5, 12, -3, 40], dtype=torch.int32, device="cuda")
    counts = torch.tensor([9, 0, 9, 7, 3], dtype=torch.int32, device="cuda")
    K[1:2] = NAN                                                 # a sequence without tokens: what the padding holds is not looked at
    K[3, :, 7:] = NAN
    held = [(0, 9), (0, 0), (12, 4), (0, 4), (0, 0)]             # rows -3 .. -1 and 16 .. are nowhere
    source = [0, 0, 0, 3, 0]
    cK, pK = _blank(B, Hkv, T, d, group)
    cV, pV = _blank(B, Hkv, T, d, 128)
    vals = csr.csr_q4_write(K, cK, pK, V, cV, pV, pos=pos, counts=counts, values=True)
    for X, c, p, g, got in ((K, cK, pK, group, vals[0]), (V, cV, pV, 128, vals[1])):
        codes, params = ref.quantise(_np(X), g)
        _hold(c, p, [codes[b][:, s:] for b, s in enumerate(source)], [params[b][:, :, s:] for b, s in enumerate(source)], held)
        want = np.zeros((B, Hkv, n, d), np.float16)
        for b, (first, count) in enumerate(held):
            want[b, :, source[b]:source[b] + count] = ref.values(codes, params)[b, :, source[b]:source[b] + count]
        assert _same(got.cpu().numpy(), want).all()
        assert _same(csr.csr_q4_read(c, p, n=n, pos=pos, counts=counts).cpu().numpy(), want).all()
    shifted = torch.full_like(pos, 2)                            # pos0 and pos add up
    a, b_ = csr.csr_q4_read(cK, pK, n=3, pos0=1, pos=shifted), csr.csr_q4_read(cK, pK, n=3, pos0=3)
    assert torch.equal(a, b_)
    assert (csr.csr_q4_read(cK, pK, n=4, pos0=-4) == 0).all() and csr.csr_q4_read(cK, pK, pos0=16).shape[2] == 0


def test_outputs_and_inputs_of_other_orders():
    B, Hkv, n, d = 2, 3, 21, 64
    base = _randn(9, B, n, 3, Hkv, d)                            # a joint projection: [B, n, (q, k, v), H, d]
    K, V = base[:, :, 1].transpose(1, 2), base[:, :, 2].transpose(1, 2)
    c = [t for _ in range(4) for t in csr.csr_q4_alloc(B, Hkv, n, d, 32)]
    outK, outV = (_token_major(torch.empty(B, Hkv, n, d, dtype=F16, device="cuda")) for _ in range(2))
    got = csr.csr_q4_write(K, c[0], c[1], V, c[2], c[3], outK=outK, outV=outV)
    assert got[0] is outK and got[1] is outV
    want = csr.csr_q4_write(K.contiguous(), c[4], c[5], V.contiguous(), c[6], c[7], values=True)
    assert torch.equal(outK, want[0]) and torch.equal(outV, want[1])
    assert all(torch.equal(a, b) for a, b in zip(c[:4], c[4:]))
    one = base[:, :, 1, :1].transpose(1, 2).expand(B, Hkv, n, d)  # one head's keys for all: stride 0
    csr.csr_q4_write(one, c[0], c[1])
    csr.csr_q4_write(one.contiguous(), c[4], c[5])
    assert torch.equal(c[0], c[4]) and torch.equal(c[1], c[5])
    out = torch.full((B, n, Hkv, d), NAN, dtype=F32, device="cuda")
    assert csr.csr_q4_read(c[0], c[1], out=out.transpose(1, 2)).dtype == F32
    assert torch.equal(out.transpose(1, 2), csr.csr_q4_read(c[0], c[1], out_dtype=F32))


def test_a_batch_slice_of_a_cache_with_an_odd_number_of_rows():
    codes, params = csr.csr_q4_alloc(3, 1, 7, 64, 64)            # params of sequence 1 start at 28 bytes
    X = _randn(10, 2, 1, 7, 64)
    csr.csr_q4_write(X, codes[1:], params[1:])
    assert (codes[0] == 0).all() and torch.equal(csr.csr_q4_read(codes, params)[1:], csr.csr_q4_read(codes[1:], params[1:]))
    q = _randn(11, 2, 2, 64)
    a = csr.csr_q4_attn(q, codes[1:], params[1:], codes[1:], params[1:])
    b = csr.csr_q4_attn(q, codes[1:].clone(), params[1:].clone(), codes[1:].clone(), params[1:].clone())
    assert torch.equal(a, b)


# ---- attention ----------------------------------------------------------------------------------------------------------
def _bound(out, spread, size, T, d, q_dtype, out_dtype, one_p):
    """How far the kernel may be off.  Scores: products are exact (fp16 keys and queries; an fp32 query as two fp16 is 2^-22
    off), their d terms are summed in fp32 in any order, one more product, sum and exponential's argument each round; with the
    largest sum of |q k| these make an error e of a score, a factor 1 + 2 e of a probability over the sum of them.
    Probabilities as two fp16 are 2^-22 off, as one 2^-11; the exponential and the sums over a wave's T / 32 steps and the
    joining of parts, in fp32, 2^-24 each, the sum of probabilities alike."""
    e = size * ((d + 4) * 2.0 ** -24 + (2.0 ** -21 if q_dtype == F32 else 0.0)) + 16 * 2.0 ** -24
    p = (2.0 ** -11 if one_p else 2.0 ** -21) + (2 * (T / 32 * 8 + 64) + 8) * 2.0 ** -24
    return HALF_STEP[out_dtype] * np.abs(out) + spread * ((2 * e + p) * 1.01)[..., None] + 1e-30 + (2.0 ** -25 if out_dtype == F16 else 0.0)


def _filled(seed, B, Hkv, T, d, gk, gv):
    gain = torch.ones(Hkv, 1, d, device="cuda")
    gain[..., ::17] = 10.0                                       # outlier channels
    K, V = _randn(seed, B, Hkv, T, d, gain=gain), _randn(seed + 1, B, Hkv, T, d)
    cache = csr.csr_q4_alloc(B, Hkv, T, d, gk) + csr.csr_q4_alloc(B, Hkv, T, d, gv)
    csr.csr_q4_write(K, cache[0], cache[1])
    csr.csr_q4_write(V, cache[2], cache[3])
    return cache


def _check(q, cache, got, seq_lens=None, q_lens=None, causal=True, scale=0.0):
    k, v = (ref.values(cache[i].cpu().numpy(), cache[i + 1].cpu().numpy()) for i in (0, 2))
    q4, g4 = (t if t.dim() == 4 else t.unsqueeze(2) for t in (q, got))
    B, Hq, Tq, d = q4.shape
    T = k.shape[2]
    lens = [T] * B if seq_lens is None else [max(0, min(int(n), T)) for n in seq_lens]
    qn = [Tq] * B if q_lens is None else [max(0, min(int(n), Tq)) for n in q_lens]
    want, spread, size = ref.attention(_np(q4), k, v, lens, qn, scale or d ** -0.5, causal)
    one_p = q.dtype == BF16 or (Tq * (Hq // k.shape[1]) > 16 and q.dtype != F32)
    off = np.abs(_np(g4) - want) / _bound(want, spread, size, T, d, q.dtype, got.dtype, one_p)
    assert np.isfinite(off).all() and off.max() <= 1, off.max()
    return off.max()


SHAPES = [
    # B, Hq, Hkv, T, Tq, d, gk, gv
    (1, 1, 1, 1, 1, 128, 128, 128),
    (1, 1, 1, 31, 1, 64, 64, 32),
    (2, 4, 2, 33, 1, 128, 32, 64),
    (3, 8, 1, 129, 1, 64, 32, 64),
    (2, 14, 2, 517, 1, 128, 64, 32),
    (1, 40, 2, 300, 1, 128, 64, 64),        # 20 query heads per KV head: two tiles of rows
    (1, 6, 2, 2500, 1, 128, 32, 128),
    (2, 4, 2, 40, 3, 64, 64, 64),
    (2, 8, 2, 333, 7, 128, 64, 128),        # 28 rows
    (1, 4, 4, 100, 64, 64, 32, 32),
    (1, 8, 2, 700, 33, 128, 128, 32),       # 132 rows
    (2, 6, 2, 1111, 150, 64, 64, 32),
    (1, 2, 1, 260, 260, 128, 32, 64),       # a whole prompt
]


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention_is_the_definitions(dtype, shape):
    B, Hq, Hkv, T, Tq, d, gk, gv = shape
    cache = _filled(20, B, Hkv, T, d, gk, gv)
    q = _token_major(_randn(22, B, Hq, Tq, d, dtype=dtype))
    if Tq == 1:
        q = q[:, :, 0]
    _check(q, cache, csr.csr_q4_attn(q, *cache))
    lens = [T - (b * T) // 3 - b for b in range(B)]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for out_dtype in (dtype, F32 if dtype == F16 else F16):
        got = csr.csr_q4_attn(q, *cache, seq_lens=seq, out_dtype=out_dtype)
        assert got.dtype == out_dtype and got.shape == q.shape
        _check(q, cache, got, lens)
    if Tq > 1:
        qn = [max(0, Tq - 2 * b - 1) for b in range(B)]
        ql = torch.tensor(qn, dtype=torch.int32, device="cuda")
        _check(q, cache, csr.csr_q4_attn(q, *cache, seq_lens=seq, q_lens=ql), lens, qn)
        _check(q, cache, csr.csr_q4_attn(q, *cache, seq_lens=seq, q_lens=ql, causal=False, scale=0.3), lens, qn, False, 0.3)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("G,Tq", [(4, 1), (4, 40)])
def test_lengths_of_nothing_and_beyond(dtype, G, Tq):
    B, Hkv, T, d = 6, 2, 70, 128
    cache = _filled(30, B, Hkv, T, d, 32, 64)
    q = _randn(32, B, Hkv * G, Tq, d, dtype=dtype)
    lens, qn = [0, 1, -5, 1000, 33, 64], [Tq, Tq, Tq, Tq + 9, 0, -1]
    seq, ql = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, qn))
    for causal in (True, False):
        got = csr.csr_q4_attn(q, *cache, seq_lens=seq, q_lens=ql, causal=causal)
        _check(q, cache, got, lens, qn, causal)
        assert (got[0] == 0).all() and (got[2] == 0).all() and (got[4:] == 0).all()
    if Tq > 1:                                                   # queries ahead of the first token see nothing
        got = csr.csr_q4_attn(q, *cache, seq_lens=seq)
        assert (got[1, :, :-1] == 0).all() and (got[1, :, -1] != 0).any()
    empty = csr.csr_q4_alloc(B, Hkv, 0, d, 32) + csr.csr_q4_alloc(B, Hkv, 0, d, 64)
    assert (csr.csr_q4_attn(q, *empty) == 0).all()
    assert csr.csr_q4_attn(q[:, :, :0], *cache).shape == (B, Hkv * G, 0, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,Tq", [(2, 1), (2, 8), (4, 6), (4, 12), (4, 20), (1, 150)])
def test_what_lies_behind_the_last_token_stays_there(d, G, Tq):
    # parameters and codes of rows that nobody sees: NaN, infinities, products beyond fp16
    B, Hkv, T = 3, 2, 200
    lens = [157, 64, 1]
    cache = _filled(40, B, Hkv, T, d, 32, 32)
    q, seq = _randn(42, B, Hkv * G, Tq, d), torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = csr.csr_q4_attn(q, *cache, seq_lens=seq)
    for s, m in ((NAN, NAN), (float("inf"), 0.0), (0.0, -float("inf")), (60000.0, 1000.0), (NAN, 0.0)):
        for b, n in enumerate(lens):
            for k in (0, 2):
                cache[k][b, :, n:] = 0xff
                cache[k + 1][b, :, :, n:, 0], cache[k + 1][b, :, :, n:, 1] = s, m
        assert torch.equal(csr.csr_q4_attn(q, *cache, seq_lens=seq), want), (s, m)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("G,Tq,at", [(2, 1, 70), (2, 1, 199), (2, 9, 195), (4, 12, 190), (4, 30, 180), (1, 150, 60), (1, 150, 199)])
def test_a_token_that_is_no_number_reaches_those_who_see_it(dtype, G, Tq, at):
    B, Hkv, T, d = 1, 2, 200, 128
    q = _randn(52, B, Hkv * G, Tq, d, dtype=dtype)
    sees = torch.arange(T - Tq, T, device="cuda") >= at
    for side in (0, 2):
        cache = _filled(50, B, Hkv, T, d, 32, 32)
        want = csr.csr_q4_attn(q, *cache)
        row = torch.randn(B, Hkv, 1, d, device="cuda")
        row[0, 1, 0, 40] = NAN                                   # KV head 1, second group of channels
        csr.csr_q4_write(row, cache[side], cache[side + 1], pos0=at)
        got = csr.csr_q4_attn(q, *cache)
        hit = torch.zeros_like(got, dtype=torch.bool)
        hit[:, G:, sees, 0 if side == 0 else 32:d if side == 0 else 64] = True
        assert torch.equal(torch.isnan(got), hit)
        assert torch.equal(got[:, :, ~sees], want[:, :, ~sees])  # to the bit: nothing else changed for them


@pytest.mark.parametrize("G,Tq", [(4, 1), (4, 5), (4, 12), (4, 30)])
def test_scores_far_apart_and_large(G, Tq):
    # one token far above the others, at either end and in the middle; scores of thousands
    B, Hkv, T, d = 1, 1, 700, 128
    K, V = _randn(60, B, Hkv, T, d), _randn(61, B, Hkv, T, d)
    q = _randn(62, B, Hkv * G, Tq, d)
    for at in (0, 350, 669):
        k2 = K.clone()
        k2[0, 0, at] = q[0, 0, 0] * 3
        cache = csr.csr_q4_alloc(B, Hkv, T, d, 32) + csr.csr_q4_alloc(B, Hkv, T, d, 32)
        csr.csr_q4_write(k2, cache[0], cache[1], V, cache[2], cache[3])
        for scale in (0.0, 5.0, 1e-4):
            _check(q, cache, csr.csr_q4_attn(q, *cache, scale=scale), scale=scale)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_queries_beyond_the_range_of_fp16(dtype):
    cache = _filled(70, 1, 2, 90, 128, 64, 64)
    for size in (1e-38, 1e-20, 1e-6, 3e5, 1e15):
        q = _randn(72, 1, 4, 128, dtype=F32, gain=size).to(dtype)
        _check(q, cache, csr.csr_q4_attn(q, *cache, scale=0.1 / max(size, 1e-30), out_dtype=F32), scale=float(np.float32(0.1 / max(size, 1e-30))))
    q = torch.zeros(1, 4, 128, dtype=dtype, device="cuda")
    _check(q, cache, csr.csr_q4_attn(q, *cache, out_dtype=F32))


def test_long_contexts_of_even_scores_keep_every_token():
    # one token far above 60000 others that together weigh as much: probabilities of 2^-17 of the largest
    T, d = 60001, 64
    K, V = torch.zeros(1, 1, T, d, device="cuda"), _randn(80, 1, 1, T, d, dtype=F32) + 1.0
    q = torch.zeros(1, 1, d, device="cuda")
    q[..., 0] = 8.0
    K[0, 0, 1234, 0] = 11.0                                      # 88 / 8 = 11 above the rest: e^11 = 59874
    cache = csr.csr_q4_alloc(1, 1, T, d, 32) + csr.csr_q4_alloc(1, 1, T, d, 32)
    csr.csr_q4_write(K, cache[0], cache[1], V, cache[2], cache[3])
    for dtype in (F16, F32):
        _check(q.to(dtype), cache, csr.csr_q4_attn(q.to(dtype), *cache))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("B,Hq,Hkv,T,Tq", [(1, 2, 1, 700, 3), (1, 8, 2, 700, 6), (2, 8, 2, 700, 12), (1, 2, 2, 700, 150), (128, 2, 2, 300, 150)])
def test_other_rows_change_no_bit(B, Hq, Hkv, T, Tq, dtype):
    # one query of every sequence grows until its scores leave all others behind
    cache = _filled(86, B, Hkv, T, 128, 64, 64)
    q = _randn(88, B, Hq, Tq, 128, dtype=dtype)
    want = csr.csr_q4_attn(q, *cache)
    for size in (4.0, 64.0):
        loud = q.clone()
        loud[:, 0, 1] *= size
        got = csr.csr_q4_attn(loud, *cache)
        got[:, 0, 1] = want[:, 0, 1]
        assert torch.equal(got, want)


def test_the_same_call_gives_the_same_bits():
    cache = _filled(90, 2, 4, 5000, 128, 64, 64)
    q = _randn(92, 2, 8, 5, 128)
    first = csr.csr_q4_attn(q, *cache)
    assert all(torch.equal(csr.csr_q4_attn(q, *cache), first) for _ in range(5))


def test_other_layouts_of_queries_and_outputs():
    B, Hq, Hkv, Tq, T, d = 2, 8, 2, 5, 90, 64
    cache = _filled(95, B, Hkv, T, d, 32, 64)
    joint = _randn(97, B, Tq, 3, Hq, d)
    q = joint[:, :, 0].transpose(1, 2)
    want = csr.csr_q4_attn(q.contiguous(), *cache)
    out = torch.full((B, Tq, Hq, d), NAN, dtype=F16, device="cuda")
    assert csr.csr_q4_attn(q, *cache, out=out.transpose(1, 2)).data_ptr() == out.data_ptr()
    assert torch.equal(out.transpose(1, 2), want) and torch.equal(csr.csr_q4_attn(q, *cache), want)
    _check(q, cache, want)
    _check(q[:, :, 4], cache, csr.csr_q4_attn(q[:, :, 4], *cache))   # the last token alone: 4 rows, whose probabilities are rounded otherwise


# Calls of few workgroups go to the kernel of 16 rows each, whatever their rows are: those of 32, 64 and 256 need many pairs.
MANY = [
    # 16s of rows a workgroup, Hq, Hkv, T (twice that with heads of 64), Tq
    (1, 8, 2, 290, 90),                     # eight waves, several workgroups along the rows
    (2, 16, 4, 200, 7),
    (4, 16, 4, 400, 16),
    (4, 12, 4, 420, 19),                    # 57 rows
    (16, 2, 2, 200, 150),
    (16, 6, 2, 300, 99),                    # 297 rows: two workgroups, the second of 41
]


MANY_TYPES = [(shape, dtype) for shape in MANY for dtype in (F16, BF16, F32) if dtype != F32 or shape[0] <= 2]   # fp32 has the two smallest


def _many(tiles, Hq, Hkv, T, Tq, d, dtype):
    B = 2 if tiles == 1 else 128
    (got, blocks, _, alone), _ = plan(B, Hq, Hkv, T, Tq, d, {F32: 0, F16: 1, BF16: 2}[dtype])
    assert got == tiles and (tiles > 1 or (alone and blocks > 1))
    return B


@pytest.mark.parametrize("shape,dtype", MANY_TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_each_kernel_is_the_definitions(dtype, d, shape):
    tiles, Hq, Hkv, T, Tq = shape
    T *= 128 // d
    B = _many(tiles, Hq, Hkv, T, Tq, d, dtype)
    cache = _filled(210, B, Hkv, T, d, 32, 64)
    q = _token_major(_randn(212, B, Hq, Tq, d, dtype=dtype))
    r = np.random.default_rng(213)
    lens, qn = r.integers(0, T + 1, B), r.integers(0, Tq + 1, B)
    lens[0], qn[0], lens[1], qn[1] = T, Tq, T - 1, Tq - 1
    seq, ql = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, qn))
    at = sorted({0, 1, B // 2, B - 1})
    for causal in (True, False):
        got = csr.csr_q4_attn(q, *cache, seq_lens=seq, q_lens=ql, causal=causal)
        _check(q[at], tuple(c[at] for c in cache), got[at], lens[at], qn[at], causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", MANY)
def test_each_kernel_keeps_to_the_sequences_tokens(d, shape):
    tiles, Hq, Hkv, T, Tq = shape
    T *= 128 // d
    B = _many(tiles, Hq, Hkv, T, Tq, d, F16)
    cache = _filled(220, B, Hkv, T, d, 32, 32)
    q, seq = _randn(222, B, Hq, Tq, d), torch.arange(B, dtype=torch.int32, device="cuda") % (T - 1) + 1
    want = csr.csr_q4_attn(q, *cache, seq_lens=seq)
    assert torch.isfinite(want).all()
    behind = torch.arange(T, device="cuda") >= seq[:, None]
    for s, m in ((NAN, NAN), (float("inf"), 0.0), (60000.0, 1000.0)):
        for k in (0, 2):
            cache[k].masked_fill_(behind[:, None, :, None], 0xff)
            cache[k + 1][..., 0].masked_fill_(behind[:, None, None], s)
            cache[k + 1][..., 1].masked_fill_(behind[:, None, None], m)
        assert torch.equal(csr.csr_q4_attn(q, *cache, seq_lens=seq), want), (s, m)


@pytest.mark.parametrize("shape,dtype", MANY_TYPES)
def test_each_kernel_shows_a_token_that_is_no_number(dtype, shape):
    tiles, Hq, Hkv, T, Tq = shape
    d, G, B = 128, Hq // Hkv, _many(*shape, 128, dtype)
    q = _randn(232, B, Hq, Tq, d, dtype=dtype)
    for at in (T - Tq + Tq // 2, 5):
        sees = torch.arange(T - Tq, T, device="cuda") >= at
        for side in (0, 2):
            cache = _filled(230, B, Hkv, T, d, 32, 32)
            want = csr.csr_q4_attn(q, *cache)
            row = torch.randn(B, Hkv, 1, d, device="cuda")
            row[:, 1, 0, 40] = NAN                               # KV head 1, second group of channels
            csr.csr_q4_write(row, cache[side], cache[side + 1], pos0=at)
            got = csr.csr_q4_attn(q, *cache)
            hit = torch.zeros_like(got, dtype=torch.bool)
            hit[:, G:2 * G, sees, 0 if side == 0 else 32:d if side == 0 else 64] = True
            assert torch.equal(torch.isnan(got), hit)
            assert torch.equal(got[:, :, ~sees], want[:, :, ~sees])


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    r = np.random.default_rng(1000 + seed)
    d = int(r.choice([64, 128]))
    gk, gv = (int(r.choice([g for g in (32, 64, 128) if g <= d])) for _ in range(2))
    Hkv, G, B = int(r.integers(1, 4)), int(r.choice([1, 2, 3, 4, 7, 8])), int(r.integers(1, 4))
    T, Tq = int(np.exp(r.uniform(0, np.log(3000)))), int(np.exp(r.uniform(0, np.log(90)))) if seed % 2 else 1
    dtype = [F16, BF16, F32][seed % 3]
    cache = _filled(300 + seed, B, Hkv, T, d, gk, gv)
    q = _randn(400 + seed, B, Hkv * G, Tq, d, dtype=dtype)
    lens, qn = r.integers(0, T + 1, B).tolist(), r.integers(0, Tq + 1, B).tolist()
    lens[0], qn[0] = T, Tq
    seq, ql = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, qn))
    causal = bool(r.integers(0, 4))
    _check(q, cache, csr.csr_q4_attn(q, *cache, seq_lens=seq, q_lens=ql, causal=causal), lens, qn, causal)


# ---- together -----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_a_prompt_and_decoding_steps(dtype):
    # prompt of odd lengths written and attended to in two chunks, then tokens one by one; read back at the end
    B, Hq, Hkv, T, d, prompt, steps = 3, 8, 2, 160, 128, 97, 6
    lens = [97, 50, 3]
    K, V, Q = (_randn(100 + i, B, h, prompt + steps, d, dtype=dtype) for i, h in enumerate((Hkv, Hkv, Hq)))
    cache = _blank(B, Hkv, T, d, 64) + _blank(B, Hkv, T, d, 32)
    cK, pK, cV, pV = cache
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    done = [0] * B
    for first, chunk in ((0, 60), (60, 37)):
        n = [max(0, min(length - first, chunk)) for length in lens]
        at = slice(first, first + chunk)
        csr.csr_q4_write(K[:, :, at], cK, pK, V[:, :, at], cV, pV, pos0=first, counts=dev(n))
        done = [a + b for a, b in zip(done, n)]
        got = csr.csr_q4_attn(Q[:, :, at], *cache, seq_lens=dev(done), q_lens=dev(n))
        _check(Q[:, :, at], cache, got, done, n)
    assert done == lens
    for s in range(steps):
        at = slice(prompt + s, prompt + s + 1)
        csr.csr_q4_write(K[:, :, at], cK, pK, V[:, :, at], cV, pV, pos=dev(done))
        done = [a + 1 for a in done]
        got = csr.csr_q4_attn(Q[:, :, prompt + s], *cache, seq_lens=dev(done))
        _check(Q[:, :, prompt + s], cache, got, done)
    for X, c, p, g in ((K, cK, pK, 64), (V, cV, pV, 32)):
        back = csr.csr_q4_read(c, p, counts=dev(done))
        for b in range(B):
            rows = torch.cat([X[b, :, :lens[b]], X[b, :, prompt:]], dim=1)
            want = ref.values(*ref.quantise(_np(rows), g))
            assert _same(back[b, :, :done[b]].cpu().numpy(), want).all() and (back[b, :, done[b]:] == 0).all()
            assert (c[b, :, done[b]:] == 0x77).all() and (p[b, :, :, done[b]:] == 7.0).all()


def test_two_captured_steps_share_a_workspace():
    # graphs of a decoding step, replayed with eager work between; both use one workspace, one after the other
    B, Hq, Hkv, T, d = 2, 8, 2, 3000, 128
    cache = _filled(110, B, Hkv, T, d, 64, 64)
    st = [dict(K=_randn(120 + i, B, Hkv, 1, d), V=_randn(130 + i, B, Hkv, 1, d), q=_randn(140 + i, B, Hq, d),
               pos=torch.zeros(B, dtype=torch.int32, device="cuda"), lens=torch.ones(B, dtype=torch.int32, device="cuda"),
               out=torch.empty(B, Hq, d, dtype=F16, device="cuda")) for i in range(2)]
    desc = csr.q4_attn_desc(st[0]["q"].unsqueeze(2), cache[0], cache[1], cache[3], st[0]["out"].unsqueeze(2))
    ws = torch.empty(csr.csr_q4_attn_workspace_bytes(desc), dtype=torch.uint8, device="cuda")

    def step(x, out, ws=ws):
        csr.csr_q4_write(x["K"], cache[0], cache[1], x["V"], cache[2], cache[3], pos=x["pos"])
        csr.csr_q4_attn(x["q"], *cache, seq_lens=x["lens"], out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in st:
            step(x, x["out"])
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for x in st:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(x, x["out"])
        graphs.append(g)
    for k in range(4):
        for x, g in zip(st, graphs):
            x["pos"].copy_(torch.tensor([500 * k + 3, 700 * k], dtype=torch.int32))
            x["lens"].copy_(x["pos"] + 1)
            x["q"].copy_(_randn(150 + k, B, Hq, d))
            g.replay()
            eager = torch.empty_like(x["out"])
            torch.cuda.synchronize()
            step(x, eager, None)
            assert torch.equal(eager, x["out"]), k


def test_two_streams_at_once():
    cache = _filled(160, 2, 2, 6000, 128, 32, 32)
    qs = [_randn(162 + i, 2, 8, 128) for i in range(2)]
    want = [csr.csr_q4_attn(q, *cache) for q in qs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in qs], [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(csr.csr_q4_attn(qs[i], *cache))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])


def test_blocks_beyond_32_bits_of_bytes():
    # the last of the (sequence, head) blocks lies 4.2 GB into the codes
    B, Hkv, T, d = 1, 65, 1 << 20, 128
    codes = torch.empty(B, Hkv, T, d // 2, dtype=torch.uint8, device="cuda")
    params = torch.empty(B, Hkv, 1, T, 2, dtype=F16, device="cuda")
    n, first = 300, T - 300
    X = _randn(170, B, Hkv, n, d)
    assert torch.equal(csr.csr_q4_write(X, codes, params, pos0=first, values=True), csr.csr_q4_read(codes, params, pos0=first))
    c, p = csr.csr_q4_alloc(B, Hkv, n, d, 128)
    csr.csr_q4_write(X, c, p)
    assert torch.equal(codes[:, :, first:], c) and torch.equal(params[:, :, :, first:], p)
    params[:, :, :, :first] = 0.0                                # keys and values of zeros: every token before weighs e^0
    codes[:, :, :first] = 0
    q = _randn(171, B, Hkv, d)
    got = csr.csr_q4_attn(q, codes, params, codes, params, out_dtype=F32)
    v = csr.csr_q4_read(c, p, out_dtype=F32).double()[0]
    s = (v @ q[0].double().unsqueeze(-1)).squeeze(-1) * d ** -0.5
    want = (s.exp().unsqueeze(1) @ v).squeeze(1) / (s.exp().sum(-1, keepdim=True) + first)
    assert ((got[0].double() - want).norm(dim=-1) <= 1e-4 * want.norm(dim=-1) + 1e-9).all()


def test_both_ways_of_marshalling_agree(monkeypatch):
    B, Hq, Hkv, T, d = 2, 4, 2, 50, 64
    K, V, q = _randn(180, B, Hkv, 9, d), _randn(181, B, Hkv, 9, d), _randn(182, B, Hq, 3, d)
    pos = torch.tensor([3, 30], dtype=torch.int32, device="cuda")

    def all_calls():
        cache = csr.csr_q4_alloc(B, Hkv, T, d, 32) + csr.csr_q4_alloc(B, Hkv, T, d, 64)
        vals = csr.csr_q4_write(K, cache[0], cache[1], V, cache[2], cache[3], pos0=1, pos=pos, values=True)
        one = csr.csr_q4_write(K, cache[0], cache[1], pos0=20, values=True)
        return (*cache, *vals, one, csr.csr_q4_read(cache[0], cache[1], pos0=5, counts=pos), csr.csr_q4_attn(q, *cache, q_lens=pos),
                csr.csr_q4_attn(q[:, :, 0], *cache, seq_lens=pos + 9, causal=False, out_dtype=F32))
    fast = all_calls()
    monkeypatch.setattr(binding, "_native", binding._CtypesOnly)
    assert all(torch.equal(a, b) for a, b in zip(fast, all_calls()))


def test_refusals_name_the_mistake():
    B, Hq, Hkv, T, d = 2, 4, 2, 20, 64
    cK, pK = csr.csr_q4_alloc(B, Hkv, T, d, 32)
    K, q = _randn(190, B, Hkv, 5, d), _randn(191, B, Hq, d)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    write, read, attn = csr.csr_q4_write, csr.csr_q4_read, csr.csr_q4_attn
    cases = [
        (lambda: write(K[0], cK, pK), "K must be"), (lambda: write(K.double(), cK, pK), "dtype"), (lambda: write(K[:1], cK, pK), "K must have shape"),
        (lambda: write(K, cK, pK[:, :, :, :5]), "contiguous"), (lambda: write(K, cK, pK[:, :, :1].contiguous()[..., :1]), "paramsK"),
        (lambda: write(K, cK.int(), pK), "uint8"), (lambda: write(K, cK, pK.float()), "float16"),
        (lambda: write(K, cK, pK, K.float(), cK, pK), "V must have"), (lambda: write(K, cK, pK, None, cK), "without V"),
        (lambda: write(K, cK, pK, K, cK, pK, outK=K), "both or neither"), (lambda: write(K.transpose(2, 3), cK, pK), "K must have shape"),
        (lambda: write(K, cK, pK, pos=i32(3)), "pos must be"), (lambda: write(K, cK, pK, counts=i32(2).long()), "counts must be"),
        (lambda: write(K, cK, pK, outK=K.float()), "outK"), (lambda: write(K, cK, pK, pos0=1 << 41), "pos0"),
        (lambda: read(cK, pK, n=3, out=K), "out must have shape"), (lambda: read(cK, pK, out_dtype=torch.int8), "out_dtype"),
        (lambda: read(cK[:, :, 1:], pK), "contiguous"), (lambda: attn(q, cK, pK, cK[:, :1].contiguous(), pK[:, :1].contiguous()), "disagree"),
        (lambda: attn(q[:1], cK, pK, cK, pK), "q must have shape"), (lambda: attn(q[0], cK, pK, cK, pK), "q must be"),
        (lambda: attn(q[:, :3], cK, pK, cK, pK), "multiple of Hkv"), (lambda: attn(q, cK, pK, cK, pK, out=q[:1]), "out must have"),
        (lambda: attn(q, cK, pK, cK, pK, seq_lens=i32(3)), "seq_lens"), (lambda: attn(q, cK, pK, cK, pK, q_lens=i32(1)), "q_lens"),
        (lambda: attn(q, cK, pK, cK, pK, scale=-1.0), "scale"), (lambda: attn(q, cK, pK, cK, pK, out_dtype=torch.float64), "out_dtype"),
        (lambda: attn(torch.empty(B * Hq * d + 1, dtype=F16, device="cuda")[1:].view(B, Hq, d), cK, pK, cK, pK), "16-byte aligned"),
        (lambda: attn(q.cpu(), cK, pK, cK, pK), "GPU tensor"),
    ]
    for k, (call, words) in enumerate(cases):
        with pytest.raises((ValueError, csr.CsrError), match=words):
            call()
            pytest.fail(f"case {k} ({words}) was accepted")
    bad = csr.csr_q4_alloc(1, 1, 4, 64, 64)
    with pytest.raises(csr.CsrError, match="group"):             # four groups of 16
        csr.csr_q4_read(bad[0], torch.zeros(1, 1, 4, 4, 2, dtype=F16, device="cuda"))


def test_more_blocks_than_one_launch_takes():
    # 600000 (sequence, head) blocks: rows in two launches; the first, the last and those around the cut
    B, Hkv, n, d = 12, 50000, 64, 64
    X = torch.randn(1, 50, n, d, device="cuda", generator=_gen(200)).to(F16).repeat(B, Hkv // 50, 1, 1)
    X[3:] += 1.0
    codes, params = csr.csr_q4_alloc(B, Hkv, n, d, 64)
    vals = csr.csr_q4_write(X, codes, params, values=True)
    assert torch.equal(vals, csr.csr_q4_read(codes, params))
    for b, h in ((0, 0), (0, 49999), (10, 24287), (10, 24288), (10, 24289), (11, 49999)):   # 524288 blocks a launch
        want = ref.quantise(_np(X[b, h]), 64)
        assert (codes[b, h].cpu().numpy() == want[0]).all() and _same(params[b, h].cpu().numpy(), want[1]).all()
    assert torch.equal(vals[:3, :50], vals[:3, 50:100]) and torch.equal(vals[4:, :50], vals[4:, 49950:])
