"""The calls on a tied model's table against their float64 oracle, element by element.

Tolerances count roundings of half a step, u = eps / 2 (fp32 2^-24, bf16 2^-8):
  lookup    one product in fp32 and one rounding to the type: (2^-24 + u) |ref|; bit for bit with scale 1
  gradient  n terms: n sums and the scale in fp32, relative to the sum of magnitudes, and the rounding to the type of dW (with
            accumulate the sum with the old value is one rounding more): (n + 2) 2^-24 sum|terms| + u |ref|
  8 bits    equal
  logp      The 8-bit matrix unit adds products eight by eight, k = 8 g .. 8 g + 7: each is cut off below 2^-13 of 2^E, E the largest sum of two
            factors' exponents among the eight, so 2^E <= (largest |h|) (largest |w|) of the group.  The term with that E has 8 bits and
            loses nothing, the other seven less than 2^-13 2^E each: at most 7 2^-13 `cut` a logit.  What is left is fp32: products
            of 8-bit values are exact, d sums, each off by at most a whole step (cut off, not rounded) of a partial sum <= size,
            in the logit and in the sampled one, which is summed apart; the log-sum-exp adds roundings of the scaled exponent (a
            few 2^-24 of the largest |logit|), of 128 fp32 additions and of the exponentials (2^-16 in all), and results
            are rounded to fp32: 7 2^-13 cut + 2 d 2^-23 size + 2^-16 + 2^-21 (1 + top + |ref|)
"""
import numpy as np
import pytest
import torch

from oracle import table_oracle as orc

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def rb():
    from paper_2510_03515_amd import binding
    binding.load()
    assert torch.cuda.is_available()
    return binding


def _f64(t):
    return t.detach().double().cpu().numpy()


def _mask(kind, N, T, gen):
    if kind == "none":
        return None
    if kind == "empty":
        return torch.zeros((N, T), dtype=torch.uint8)
    length = torch.randint(0, T + 1, (N, 1), generator=gen)         # generations without a token among them
    mask = torch.arange(T)[None, :] < length
    if kind == "holes":
        mask &= torch.rand((N, T), generator=gen) < 0.6
    mask = mask.to(torch.uint8)
    if kind == "ragged" and N > 1:
        mask[0] = 0
        mask[-1] = 1
    return mask * (1 if kind == "ragged" else 7)                      # any value but 0 is valid


def _ids(kind, N, T, V, gen):
    if kind == "one":
        return torch.full((N, T), V - 1, dtype=torch.int32)
    if kind == "zipf":
        r = torch.exp(torch.rand((N, T), generator=gen, dtype=torch.float64) * np.log(V + 1)).long() - 1
        return r.clamp(0, V - 1).to(torch.int32)
    if kind == "distinct":
        return torch.randperm(V, generator=gen)[:N * T].view(N, T).to(torch.int32)
    return torch.randint(0, V, (N, T), generator=gen, dtype=torch.int32)


def _dev(x):
    return None if x is None else x.cuda()


def _np(x):
    return None if x is None else x.numpy()


def _guarded(shape, dtype):
    """A tensor between two stretches of a sentinel, and a check that they are as they were."""
    n, pad = int(np.prod(shape)), 4096
    base = torch.full((n + 2 * pad,), 3.0, dtype=dtype, device="cuda")
    base[pad:pad + n] = float("nan")
    return base[pad:pad + n].view(shape), lambda: bool((base[:pad] == 3.0).all() and (base[pad + n:] == 3.0).all())


# ------------------------------------------------------------------------------------------------ lookup
FWD = [("bf16", 1, 1, 8, 1, "none"), ("bf16", 3, 5, 64, 11, "ragged"), ("bf16", 7, 33, 520, 300, "holes"), ("bf16", 2, 700, 1536, 5000, "ragged"),
       ("bf16", 4, 9, 8, 77, "empty"), ("bf16", 300, 60, 24, 100, "holes"), ("bf16", 40, 513, 1032, 999, "ragged"), ("bf16", 2, 3, 16384, 7, "none"),
       ("f32", 1, 1, 1, 1, "none"), ("f32", 5, 17, 3, 9, "holes"), ("f32", 6, 50, 63, 20, "ragged"), ("f32", 9, 40, 256, 4096, "ragged"),
       ("f32", 33, 600, 101, 50, "holes"), ("f32", 20, 900, 132, 70, "ragged")]


@pytest.mark.parametrize("dtype,N,T,d,V,mask", FWD)
@pytest.mark.parametrize("scale", [1.0, -2.7])
def test_lookup(rb, dtype, N, T, d, V, mask, scale):
    gen = torch.Generator().manual_seed(N * 1000 + T + d)
    table = torch.randn((V, d), generator=gen).to(TYPES[dtype])
    tokens, m = _ids("uniform", N, T, V, gen), _mask(mask, N, T, gen)
    out, untouched = _guarded((N, T, d), TYPES[dtype])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = rb.rapid_embedding_fwd(table.cuda(), tokens.cuda(), _dev(m), scale=scale, out=out, dev_status=status)
    ref = orc.embedding_fwd(_f64(table), tokens.numpy(), _np(m), float(np.float32(scale)))
    assert got is out and untouched() and status.item() == 0
    bound = 0.0 if scale == 1.0 else (2.0 ** -24 + HALF[dtype] * (1 + 2.0 ** -20)) * np.abs(ref)
    assert np.all(np.abs(_f64(out) - ref) <= bound)


def test_lookup_ids_out_of_range(rb):
    table = torch.randn(6, 8).bfloat16().cuda()
    tokens = torch.tensor([[0, 6, -1, 5], [2 ** 31 - 1, 1, -2 ** 31, 3]], dtype=torch.int32).cuda()
    mask = torch.tensor([[1, 1, 1, 1], [1, 1, 0, 1]], dtype=torch.uint8).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = rb.rapid_embedding_fwd(table, tokens, mask, dev_status=status)
    assert np.array_equal(_f64(got), orc.embedding_fwd(_f64(table), tokens.cpu().numpy(), mask.cpu().numpy(), 1.0))
    assert status.item() == rb.STATUS_BAD_TOKEN
    status.zero_()
    rb.rapid_embedding_fwd(table, tokens.clamp(0, 5), mask, dev_status=status)
    assert status.item() == 0
    rb.rapid_embedding_fwd(table, tokens, mask)          # without a word to flag it in
    assert torch.isnan(rb.rapid_embedding_fwd(torch.full_like(table, float("nan")), tokens, mask)[0, 0]).all()


def test_lookup_offsets_past_32_bits(rb):
    """Output, table and their offsets of more than 2^32 elements: the last rows, and samples in between."""
    V, d, T = 70000, 65536, 66000
    table = torch.empty((V, d), dtype=torch.bfloat16, device="cuda")
    rows = torch.arange(V, device="cuda", dtype=torch.float32)
    table[:] = (rows % 251)[:, None].bfloat16()
    table[:, -8:] = (rows % 241)[:, None].bfloat16()
    tokens = (V - 1 - torch.arange(T, dtype=torch.int32, device="cuda")).view(1, T)
    out = rb.rapid_embedding_fwd(table, tokens)
    want = tokens[0].float()
    assert torch.equal(out[0, :, 0].float(), want % 251) and torch.equal(out[0, :, -1].float(), want % 241)
    assert torch.equal(out[0, :, 32768].float(), want % 251)
    dt = torch.full((V, d), 7.0, dtype=torch.bfloat16, device="cuda")
    rb.rapid_embedding_bwd(out, tokens, None, V, dtable=dt)
    assert torch.equal(dt[tokens[0].long()[:300]], out[0, :300]) and torch.equal(dt[tokens[0].long()[-300:]], out[0, -300:])
    assert torch.equal(dt[tokens[0].long(), 0], out[0, :, 0]) and torch.equal(dt[tokens[0].long(), -1], out[0, :, -1])
    assert not dt[:V - T].any()


# ---------------------------------------------------------------------------------------------- gradient
BWD = [  # dtype, N, T, d, V, ids, mask, dw
    ("bf16", 1, 1, 8, 1, "one", "none", "f32"), ("bf16", 1, 1, 64, 300, "uniform", "none", "bf16"), ("bf16", 2, 9, 8, 5, "zipf", "empty", "f32"),
    ("bf16", 4, 300, 136, 2, "uniform", "ragged", "f32"), ("bf16", 3, 500, 520, 700, "zipf", "holes", "bf16"),
    ("bf16", 8, 1000, 64, 513, "one", "none", "f32"), ("bf16", 1, 4096, 16, 4096, "distinct", "none", "f32"),
    ("bf16", 1, 4097, 1536, 512, "zipf", "none", "bf16"), ("bf16", 50, 700, 72, 300000, "zipf", "ragged", "f32"),
    ("bf16", 64, 700, 264, 5000, "zipf", "holes", "f32"), ("bf16", 270, 1000, 24, 151, "zipf", "none", "f32"),
    ("bf16", 2, 40, 4104, 30, "zipf", "ragged", "f32"),
    ("f32", 1, 1, 1, 1, "one", "none", "f32"), ("f32", 5, 40, 3, 7, "zipf", "holes", "bf16"), ("f32", 3, 900, 256, 4096, "zipf", "ragged", "f32"),
    ("f32", 70, 500, 63, 1000, "uniform", "holes", "f32"), ("f32", 9, 1000, 132, 40, "one", "ragged", "bf16"), ("f32", 2, 30, 2050, 9, "zipf", "none", "f32"),
    ("f32", 6, 11, 20, 262145, "uniform", "none", "f32"),
    # one pass over up to 12 bits of the id: sizes and vocabularies at its ends, runs over many stretches
    ("bf16", 1, 8193, 8, 513, "uniform", "none", "f32"), ("f32", 32, 1024, 20, 4096, "zipf", "none", "f32"), ("bf16", 32, 1024, 16, 4097, "zipf", "holes", "f32"),
    ("f32", 40, 500, 7, 1024, "one", "holes", "f32"), ("bf16", 30, 1000, 136, 3000, "zipf", "ragged", "bf16"), ("bf16", 1, 32769, 8, 2048, "zipf", "none", "f32"),
    ("bf16", 9, 1000, 8, 4000, "zipf", "empty", "f32"), ("f32", 25, 1300, 5, 600, "one", "none", "bf16"),
]


def _check_gradient(got, old, ref, size, terms, dw):
    want = ref if old is None else _f64(old) + ref
    bound = (terms[:, None] + 2) * 2.0 ** -24 * size + HALF[dw] * (1 + 2.0 ** -12) * np.abs(want)
    if old is not None:
        bound[terms == 0] = 0.0
    assert np.all(np.abs(_f64(got) - want) <= bound)


@pytest.mark.parametrize("dtype,N,T,d,V,ids,mask,dw", BWD)
def test_gradient(rb, dtype, N, T, d, V, ids, mask, dw):
    gen = torch.Generator().manual_seed(N * 1000 + T + d)
    tokens, m = _ids(ids, N, T, V, gen), _mask(mask, N, T, gen)
    dh = torch.randn((N, T, d), generator=gen).to(TYPES[dtype])
    scale = float(np.float32(1.3))
    ref, size, terms = orc.embedding_bwd(_f64(dh), tokens.numpy(), _np(m), V, scale)
    dev = dh.cuda()
    if m is not None:
        dev[m.cuda() == 0] = float("nan")           # masked rows are not read
    out, untouched = _guarded((V, d), TYPES[dw])
    print(f"gradient {dtype} {N}x{T} d={d} V={V} {ids} {mask}", flush=True)
    got = rb.rapid_embedding_bwd(dev, tokens.cuda(), _dev(m), V, scale=scale, dtable=out)
    assert got is out and untouched()
    _check_gradient(out, None, ref, size, terms, dw)
    again = rb.rapid_embedding_bwd(dev, tokens.cuda(), _dev(m), V, scale=scale, dw_dtype=TYPES[dw])
    assert torch.equal(out, again)                   # the same bits
    if dw == "f32":
        old = torch.randn((V, d), generator=gen)
        acc = old.cuda()
        rb.rapid_embedding_bwd(dev, tokens.cuda(), _dev(m), V, scale=scale, dtable=acc, accumulate=True)
        _check_gradient(acc, old, ref, size, terms, dw)


def test_gradient_ids_out_of_range_add_nothing(rb):
    tokens = torch.tensor([[0, 9, -1, 5, 5, -2 ** 31, 2 ** 31 - 1]], dtype=torch.int32)
    dh = torch.randn(1, 7, 16)
    ref, size, terms = orc.embedding_bwd(_f64(dh), tokens.numpy(), None, 9, 1.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = rb.rapid_embedding_bwd(dh.cuda(), tokens.cuda(), None, 9, dev_status=status)
    _check_gradient(got, None, ref, size, terms, "f32")
    assert status.item() == rb.STATUS_BAD_TOKEN


def test_gradient_keeps_infinities_where_they_are(rb):
    """A gradient that is not finite reaches its own id's entry and no other."""
    dh = torch.ones(1, 300, 8)
    dh[0, 7, 3] = float("inf")
    dh[0, 200, 5] = float("nan")
    tokens = (torch.arange(300, dtype=torch.int32) % 10).view(1, 300)
    got = rb.rapid_embedding_bwd(dh.cuda(), tokens.cuda(), None, 12).cpu()
    assert got[7, 3] == float("inf") and torch.isnan(got[0, 5])
    got[7, 3] = got[0, 5] = 30.0
    assert torch.equal(got[:10], torch.full((10, 8), 30.0)) and not got[10:].any()


# ------------------------------------------------------------------------------------------------ 8 bits
def _check_8_bits(q, W):
    values, e = orc.quantize(W)
    scales = np.full((W.shape[0], -(-e.shape[1] // 4) * 4), 127)
    scales[:, :e.shape[1]] = e + 127
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(_f64(q.values), values, equal_nan=True)


@pytest.mark.parametrize("dtype,V,d", [("bf16", 1, 8), ("bf16", 3, 128), ("bf16", 129, 136), ("bf16", 1000, 520), ("bf16", 257, 1536), ("f32", 1, 1), ("f32", 5, 127),
                                       ("f32", 131, 129), ("f32", 640, 260), ("f32", 77, 1001), ("f32", 128, 513)])
@pytest.mark.parametrize("layout", ["vd", "dv"])
def test_quantize(rb, dtype, V, d, layout):
    gen = torch.Generator().manual_seed(V + d)
    W = torch.randn((V, d), generator=gen) * torch.exp(3 * torch.randn((V, 1), generator=gen))
    W[torch.rand((V, d), generator=gen) < 0.1] = 0.0
    W[V // 2] = 0.0
    W = W.to(TYPES[dtype])
    stored = (W if layout == "vd" else W.t()).contiguous().cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = rb.rapid_quantize_fp8(stored, w_layout=rb.W_VD if layout == "vd" else rb.W_DV, dev_status=status)
    _check_8_bits(q, _f64(W))
    assert status.item() == 0
    q.values.view(torch.uint8).fill_(0x7f); q.scales.fill_(255)          # every byte is written
    assert rb.rapid_quantize_fp8(stored, w_layout=rb.W_VD if layout == "vd" else rb.W_DV, out=q) is q
    _check_8_bits(q, _f64(W))


@pytest.mark.parametrize("layout", ["vd", "dv"])
def test_quantize_edges(rb, layout):
    """Blocks whose largest value lies on, just above and far from 448 times a power of two, subnormal ones, ties, values that are not finite."""
    d = 128
    rows = [torch.full((d,), v) for v in (448.0, 448.0000305, 447.99997, 1.75, 1.7500001, 3.4e38, 2.0 ** -126, 1e-45, 3e-40, 0.0, -1e-30)]
    ties = torch.arange(d, dtype=torch.float32) * 0.0625 + 440.0 / 128                # midpoints and their neighbours under scale 1
    ties[0] = 448.0
    rows.append(ties)
    rows.append(torch.nextafter(ties, torch.zeros(d)).index_fill(0, torch.tensor([0]), 448.0))
    W = torch.stack(rows)
    put = lambda x: (x if layout == "vd" else x.t()).contiguous().cuda()
    lay = rb.W_VD if layout == "vd" else rb.W_DV
    _check_8_bits(rb.rapid_quantize_fp8(put(W), w_layout=lay), _f64(W))
    W[2, 5], W[3, 0], W[4, 127] = float("nan"), float("inf"), float("-inf")
    W[5] = float("nan")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    _check_8_bits(rb.rapid_quantize_fp8(put(W), w_layout=lay, dev_status=status), _f64(W))
    assert status.item() == rb.STATUS_NONFINITE_VALUE


# ------------------------------------------------------------------------------------- log-probs in 8 bits
LOGP = [  # dtype, N, T, d, V, mask, temperature
    ("bf16", 1, 1, 8, 1, "ragged", 1.0), ("bf16", 1, 1, 1536, 1000, "ragged", 1.0), ("bf16", 16, 1, 256, 3000, "ragged", 0.7), ("bf16", 3, 5, 128, 255, "holes", 1.0),
    ("bf16", 2, 9, 136, 256, "empty", 1.0), ("bf16", 5, 13, 520, 257, "ragged", 1.0), ("bf16", 2, 31, 896, 2050, "ragged", 2.0), ("bf16", 4, 16, 640, 511, "none", 1.0),
    ("bf16", 5, 13, 264, 70, "ragged", 1.0), ("bf16", 1, 129, 384, 400, "none", 1.0), ("bf16", 3, 300, 200, 700, "holes", 0.5), ("bf16", 9, 1000, 64, 130, "ragged", 1.0),
    ("bf16", 2, 4200, 72, 300, "holes", 1.0), ("bf16", 1, 17000, 16, 90, "none", 1.0),
    ("f32", 1, 1, 1, 2, "none", 1.0), ("f32", 8, 1, 1001, 600, "none", 1.0), ("f32", 6, 33, 127, 259, "holes", 1.0), ("f32", 2, 70, 515, 1300, "ragged", 0.9),
    ("f32", 1, 257, 2049, 300, "none", 1.0), ("bf16", 32, 1, 136, 256, "none", 1.0), ("bf16", 33, 1, 136, 256, "none", 1.0), ("bf16", 8, 8, 264, 385, "holes", 1.0),
    ("bf16", 5, 13, 264, 384, "ragged", 1.0), ("bf16", 4, 250, 520, 3001, "holes", 1.0), ("bf16", 17, 1000, 136, 300, "ragged", 1.0), ("f32", 2, 16, 4500, 1031, "none", 1.0),
    ("bf16", 1, 1100, 256, 5000, "holes", 1.0),
]


def _check_logp(logp, lse, hidden, W, tokens, m, temp):
    ref_p, ref_s, size, top, cut = orc.logprob_fp8(_f64(hidden), _f64(W), tokens.numpy(), m.numpy(), float(np.float32(temp)))
    for got, ref in ((logp, ref_p), (lse, ref_s)):
        bound = 7 * 2.0 ** -13 * cut + 2 * hidden.shape[2] * 2.0 ** -23 * size + 2.0 ** -16 + 2.0 ** -21 * (1 + top + np.abs(ref))
        bound[m.numpy() == 0] = 0.0
        assert np.all(np.abs(_f64(got) - ref) <= bound)
    assert np.all(_f64(logp) <= 0.0)


def _head(V, d, gen, dtype):
    return (torch.randn((V, d), generator=gen) * torch.exp(0.5 * torch.randn((V, 1), generator=gen)) / np.sqrt(d) * 2).to(TYPES[dtype])


@pytest.mark.parametrize("dtype,N,T,d,V,mask,temp", LOGP)
def test_logprob(rb, dtype, N, T, d, V, mask, temp):
    gen = torch.Generator().manual_seed(N * 1000 + T + d)
    W = _head(V, d, gen, dtype)
    hidden, tokens = torch.randn((N, T, d), generator=gen).to(TYPES[dtype]), _ids("zipf", N, T, V, gen)
    m = _mask(mask, N, T, gen)
    m = torch.ones((N, T), dtype=torch.uint8) if m is None else m
    dev = hidden.cuda()
    dev[m.cuda() == 0] = float("nan")               # masked states are not read
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    W8 = rb.rapid_quantize_fp8(W.cuda(), w_layout=rb.W_VD)
    ws = rb.alloc_workspace(rb.rapid_workspace_bytes(rb.OP_LOGPROB_FWD_FP8, N, T, d, V, 1, 0))
    ws.fill_(0xff)
    print(f"logprob {dtype} {N}x{T} d={d} V={V} {mask}", flush=True)
    logp, lse = rb.rapid_logprob_fwd_fp8(dev, W8, tokens.cuda(), m.cuda(), temperature=temp, want_lse=True, workspace=ws, dev_status=status)
    _check_logp(logp, lse, hidden, W, tokens, m, temp)
    assert status.item() == 0
    only, none = rb.rapid_logprob_fwd_fp8(dev, W8, tokens.cuda(), m.cuda(), temperature=temp, workspace=ws)
    assert none is None and torch.equal(only, logp)  # the same bits, and the workspace needs no clearing


def test_logprob_needs_no_order_of_sizes(rb):
    """Blocks of very different size within a row on both sides, zero rows among them."""
    gen = torch.Generator().manual_seed(3)
    V, d = 300, 640
    spread = torch.exp2(torch.randint(-30, 1, (V, 5), generator=gen).float()).repeat_interleave(128, 1)
    W, hidden = torch.randn((V, d), generator=gen) * spread, torch.randn((4, 20, d), generator=gen)
    hidden *= torch.exp2(torch.randint(-25, 2, (4, 20, 5), generator=gen).float()).repeat_interleave(128, 2)
    hidden[1, 3] = 0.0
    W[17] = 0.0
    tokens, m = _ids("uniform", 4, 20, V, gen), torch.ones((4, 20), dtype=torch.uint8)
    logp, lse = rb.rapid_logprob_fwd_fp8(hidden.cuda(), rb.rapid_quantize_fp8(W.cuda(), w_layout=rb.W_VD), tokens.cuda(), m.cuda(), want_lse=True)
    _check_logp(logp, lse, hidden, W, tokens, m, 1.0)


@pytest.mark.parametrize("N,T", [(2, 8), (3, 100), (2, 5000)])
def test_logprob_flags(rb, N, T):
    """Ids out of range count as token 0; a state that is not finite spoils its own row alone, a weight that is not finite every row."""
    gen = torch.Generator().manual_seed(5)
    V, d = 700, 256
    W = _head(V, d, gen, "bf16").cuda()
    hidden, tokens, m = torch.randn((N, T, d), generator=gen).bfloat16().cuda(), _ids("uniform", N, T, V, gen).cuda(), torch.ones((N, T), dtype=torch.uint8, device="cuda")
    W8, status = rb.rapid_quantize_fp8(W, w_layout=rb.W_VD), torch.zeros(1, dtype=torch.int32, device="cuda")
    good, good_lse = rb.rapid_logprob_fwd_fp8(hidden, W8, tokens, m, want_lse=True, dev_status=status)
    assert status.item() == 0 and torch.isfinite(good).all()
    bad, zero = tokens.clone(), tokens.clone()
    bad[0, 1], bad[1, 2], zero[0, 1], zero[1, 2] = V, -1, 0, 0
    assert torch.equal(rb.rapid_logprob_fwd_fp8(hidden, W8, bad, m, dev_status=status)[0], rb.rapid_logprob_fwd_fp8(hidden, W8, zero, m)[0])
    assert status.item() == rb.STATUS_BAD_TOKEN
    status.zero_()
    h = hidden.clone()
    h[0, 0, 7], h[1, 4, 200] = float("nan"), float("inf")
    p, s = rb.rapid_logprob_fwd_fp8(h, W8, tokens, m, want_lse=True, dev_status=status)
    assert status.item() == rb.STATUS_NONFINITE_VALUE
    hit = torch.zeros_like(m, dtype=torch.bool)
    hit[0, 0] = hit[1, 4] = True
    assert not torch.isfinite(p[hit]).any() and not torch.isfinite(s[hit]).any()
    assert torch.equal(p[~hit], good[~hit]) and torch.equal(s[~hit], good_lse[~hit])
    W[123, 50] = float("nan")
    p, s = rb.rapid_logprob_fwd_fp8(hidden, rb.rapid_quantize_fp8(W, w_layout=rb.W_VD), tokens, m, want_lse=True)
    assert not torch.isfinite(p).any() and not torch.isfinite(s).any()


def test_layouts_and_types_agree(rb):
    """One head as [d,V] and [V,d], and a bf16 batch handed over in fp32: the same bits."""
    gen = torch.Generator().manual_seed(8)
    W = _head(333, 264, gen, "bf16")
    a, b = rb.rapid_quantize_fp8(W.cuda(), w_layout=rb.W_VD), rb.rapid_quantize_fp8(W.t().contiguous().cuda(), w_layout=rb.W_DV)
    c = rb.rapid_quantize_fp8(W.float().cuda(), w_layout=rb.W_VD)
    for o in (b, c):
        assert torch.equal(a.values.view(torch.uint8), o.values.view(torch.uint8)) and torch.equal(a.scales, o.scales)
    hidden, tokens, m = torch.randn((3, 40, 264), generator=gen).bfloat16().cuda(), _ids("uniform", 3, 40, 333, gen).cuda(), torch.ones((3, 40), dtype=torch.uint8, device="cuda")
    assert torch.equal(rb.rapid_logprob_fwd_fp8(hidden, a, tokens, m)[0], rb.rapid_logprob_fwd_fp8(hidden.float(), b, tokens, m)[0])


# ---------------------------------------------------------------------------------- streams, graphs, together
def _calls(rb, gen, N, T, d, V):
    """The four calls on one set of buffers, and the tensors that they fill."""
    s = dict(table=_head(V, d, gen, "bf16").cuda(), tokens=_ids("zipf", N, T, V, gen).cuda(), mask=_mask("holes", N, T, gen).cuda(),
             dh=torch.randn((N, T, d), generator=gen).bfloat16().cuda(), dtable=torch.zeros((V, d), device="cuda"))
    s["hidden"] = torch.empty((N, T, d), dtype=torch.bfloat16, device="cuda")
    s["W8"] = rb.rapid_quantize_fp8(s["table"], w_layout=rb.W_VD)
    return s


def _run_calls(rb, s, ws):
    rb.rapid_embedding_fwd(s["table"], s["tokens"], s["mask"], scale=1.5, out=s["hidden"])
    rb.rapid_embedding_bwd(s["dh"], s["tokens"], s["mask"], s["table"].shape[0], dtable=s["dtable"], workspace=ws)
    rb.rapid_embedding_bwd(s["hidden"], s["tokens"], s["mask"], s["table"].shape[0], dtable=s["dtable"], accumulate=True, workspace=ws)
    rb.rapid_quantize_fp8(s["table"], w_layout=rb.W_VD, out=s["W8"])
    s["logp"], s["lse"] = rb.rapid_logprob_fwd_fp8(s["hidden"], s["W8"], s["tokens"], s["mask"], want_lse=True, workspace=ws)


def _results(s):
    return [s[k].clone() for k in ("hidden", "dtable", "logp", "lse")] + [s["W8"].values.view(torch.uint8).clone(), s["W8"].scales.clone()]


def _workspace(rb, *sizes):
    return rb.alloc_workspace(max(rb.rapid_workspace_bytes(op, *z, 1, rb.DTYPE_BF16) for op in (rb.OP_EMBEDDING_BWD, rb.OP_LOGPROB_FWD_FP8) for z in sizes))


def test_on_another_stream(rb):
    gen = torch.Generator().manual_seed(11)
    s = _calls(rb, gen, 6, 500, 264, 900)
    ws = _workspace(rb, (6, 500, 264, 900))
    _run_calls(rb, s, ws)
    want = _results(s)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for k in ("hidden", "dtable"):
            s[k].fill_(3.0)
        _run_calls(rb, s, ws)
        got = _results(s)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_graphs_that_share_a_workspace(rb):
    """Two captured runs of all calls, of different sizes, on one workspace: replays in turn with new inputs, eager work in between, give what
    eager calls give."""
    gen = torch.Generator().manual_seed(12)
    sizes = [(5, 700, 264, 900), (3, 20, 136, 4000)]
    ws = _workspace(rb, *sizes)
    states = [_calls(rb, gen, *z) for z in sizes]
    graphs = []
    for s in states:
        _run_calls(rb, s, ws)                        # the first call of a kernel is not a captured one
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _run_calls(rb, s, ws)
        graphs.append(g)
    captured = [(s["logp"], s["lse"]) for s in states]
    for turn in range(3):
        for s, g, z, (logp, lse) in zip(states, graphs, sizes, captured):
            N, T, d, V = z
            s["tokens"].copy_(_ids("zipf", N, T, V, gen)); s["mask"].copy_(_mask("ragged" if turn else "holes", N, T, gen))
            s["table"].copy_(_head(V, d, gen, "bf16"))
            g.replay()
            torch.cuda.synchronize()
            s["logp"], s["lse"] = logp, lse
            got = _results(s)
            _run_calls(rb, s, ws)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, _results(s))), (turn, z)


# ------------------------------------------------------------------------------------------- one update of a tied table
def _tied(rb, dtype, **kw):
    from paper_2510_03515_amd import iw_grpg as ig
    from paper_2510_03515_amd import workloads as wl
    spec = wl.small_spec("tied", dtype, **dict(dict(d=72, V=301, prompts=4, G=4, len_lo=2, len_hi=21, reward="bernoulli"), **kw))
    return ig, wl.make_tied_workload(spec, seed=3, device="cuda", scale=spec.d ** 0.5, as_served=ig.served_in_8_bits)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tied_step_against_the_formula_and_differences(rb, dtype):
    """The table's gradient of one loss step through both uses: against the loss oracle's dHidden and dW, put together by the table oracle, and (fp32) against
    central differences of the objective, in float64, along random directions."""
    from oracle import rapid_oracle as loss_orc
    ig, w = _tied(rb, dtype)
    E, scale, N = w["table"], float(np.float32(w["scale"])), w["tokens"].shape[0]
    inputs, tokens, mask = w["inputs"], w["tokens"], w["mask"]
    hidden = rb.rapid_embedding_fwd(E, inputs, mask, scale=scale)
    W8 = rb.rapid_quantize_fp8(E, w_layout=rb.W_VD)
    logp_b, _ = rb.rapid_logprob_fwd_fp8(hidden, W8, tokens, mask)
    out = rb.rapid_iw_pg_loss_fwd_bwd(hidden, E, tokens, mask, logp_b, w["rewards"], w["group_ids"], w["K"], w_layout=rb.W_VD)
    head = out.dW.clone()
    rb.rapid_embedding_bwd(out.dhidden, inputs, mask, E.shape[0], scale=scale, dtable=out.dW, accumulate=True)
    # the lookup's share, from the states' gradient as the loss step returned it
    ref, size, terms = orc.embedding_bwd(_f64(out.dhidden), inputs.cpu().numpy(), mask.cpu().numpy(), E.shape[0], scale)
    _check_gradient(out.dW, head, ref, size, terms, "f32")
    # all of it, from the definition; the loss step's own bounds (1e-5 of a tensor in fp32, 2e-2 in bf16) hold for the sum of its two parts
    h64, E64 = _f64(hidden), _f64(E)
    want = loss_orc.iw_pg_loss_fwd_bwd(h64, E64.T.copy(), tokens.cpu().numpy(), mask.cpu().numpy(), _f64(logp_b), _f64(w["rewards"]), w["group_ids"].cpu().numpy(), w["K"])
    both = want["dW"].T + orc.embedding_bwd(want["dH"], inputs.cpu().numpy(), mask.cpu().numpy(), E.shape[0], scale)[0]
    parts = np.linalg.norm(want["dW"]) + np.linalg.norm(both - want["dW"].T)
    assert np.linalg.norm(_f64(out.dW) - both) <= (1e-5 if dtype == "f32" else 2e-2) * parts
    if dtype != "f32":
        return
    m, x, y, adv = mask.cpu().numpy(), inputs.cpu().numpy(), tokens.cpu().numpy(), np.asarray(want["adv"])

    def objective(table):       # advantages held: the gradient acts on the ratios alone
        total = 0.0
        for n in range(N):
            at = np.nonzero(m[n])[0]
            z = scale * table[x[n, at]] @ table.T
            lp = z[np.arange(len(at)), y[n, at]] - np.log(np.exp(z - z.max(axis=1, keepdims=True)).sum(axis=1)) - z.max(axis=1)
            total -= np.exp(np.sum(lp - _f64(logp_b)[n, at])) * adv[n] / N
        return total

    rng = np.random.default_rng(1)
    for _ in range(4):
        along = rng.standard_normal(E64.shape)
        along /= np.linalg.norm(along)
        step = 1e-5                                  # truncation ~ step^2, cancellation 2^-53 / step: 1e-10 each, far below 1e-5 of the gradient
        slope = (objective(E64 + step * along) - objective(E64 - step * along)) / (2 * step)
        assert abs(slope - np.sum(_f64(out.dW) * along)) <= 1e-5 * parts + 1e-8


@pytest.mark.parametrize("optimizer,cache", [("sgd", False), ("adamw", True)])
def test_tied_inner_loop_runs(rb, optimizer, cache):
    """The command's path: every step's calls together, and a behaviour policy in 8 bits that is close to, and not, the table's own."""
    ig, w = _tied(rb, "bf16", d=136, V=700, prompts=8)
    before = w["table"].clone()
    log, summary, E = ig.iw_grpg_tied(w, inner_steps=4, lr=2e-4 if optimizer == "sgd" else 2e-6, optimizer=optimizer, logits_cache=cache)
    assert len(log) == 4 and all(np.isfinite(list(r.values())).all() for r in log)
    assert 0.0 < log[0]["max_abs_s"] < 1.0
    assert np.isfinite(summary["reward_final_is_estimate"]) and abs(summary["reward_behaviour"] - w["rewards"].mean().item()) < 1e-5
    assert torch.equal(w["table"], before) and not torch.equal(E, before) and torch.isfinite(E.float()).all()


def test_another_current_device_is_refused(rb, monkeypatch):
    """Every call looks where its tensors lie; nothing is launched."""
    s = _calls(rb, torch.Generator().manual_seed(2), 2, 5, 8, 9)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    calls = [lambda **kw: rb.rapid_embedding_fwd(s["table"], s["tokens"], s["mask"], **kw), lambda **kw: rb.rapid_embedding_bwd(s["dh"], s["tokens"], s["mask"], 9, **kw),
             lambda **kw: rb.rapid_quantize_fp8(s["table"], w_layout=rb.W_VD, **kw),
             lambda **kw: rb.rapid_logprob_fwd_fp8(s["hidden"], s["W8"], s["tokens"], s["mask"], **kw)]
    for call in calls:
        for word in (status.cpu(), status.float(), status[:0]):
            with pytest.raises(TypeError):
                call(dev_status=word)
        call(dev_status=status)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: torch.cuda.device_count())
    for call in calls:
        with pytest.raises(TypeError, match="current device"):
            call(dev_status=status)


@pytest.mark.parametrize("key,values", [(10, (0, 1, 3, 8, 1024)), (13, (1, 2))])
def test_logprob_tile_order_changes_nothing(rb, key, values):
    """The order of the 8-bit logits' tiles and the row tiles of a launch: the same bits."""
    gen = torch.Generator().manual_seed(21)
    N, T, d, V = 4, 290, 264, 70001
    W8 = rb.rapid_quantize_fp8(_head(V, d, gen, "bf16").cuda(), w_layout=rb.W_VD)
    hidden, tokens, m = torch.randn((N, T, d), generator=gen).bfloat16().cuda(), _ids("zipf", N, T, V, gen).cuda(), _mask("holes", N, T, gen).cuda()
    want, want_lse = rb.rapid_logprob_fwd_fp8(hidden, W8, tokens, m, want_lse=True)
    try:
        for value in values:
            assert rb.load().rapid_set_tuning(key, value) == 0
            p, s = rb.rapid_logprob_fwd_fp8(hidden, W8, tokens, m, want_lse=True)
            assert torch.equal(p, want) and torch.equal(s, want_lse), value
    finally:
        rb.load().rapid_set_tuning(key, {10: 4, 13: 64}[key])


@pytest.mark.parametrize("N,T,d", [(64, 1030, 1021), (64, 1030, 1024), (3, 7, 5), (3, 7, 6), (900, 70, 7), (2, 20000, 2), (16, 4000, 1049)])
def test_fp32_rows_of_any_length_past_the_caches(rb, N, T, d):
    """fp32 lookups of rows off 16-byte boundaries, outputs on both sides of 256 MB: the table's rows, and nothing beside them; their gradient sums to as much."""
    V = 901
    table = torch.randn(V, d, device="cuda")
    tokens = torch.randint(0, V, (N, T), dtype=torch.int32, device="cuda")
    mask = (torch.rand(N, T, device="cuda") < 0.9).to(torch.uint8)
    out, untouched = _guarded((N, T, d), torch.float32)
    rb.rapid_embedding_fwd(table, tokens, mask, out=out)
    assert untouched() and torch.equal(out, table[tokens.long()] * (mask[:, :, None] != 0))
    count = torch.bincount(tokens[mask != 0].long(), minlength=V).float()
    grad = rb.rapid_embedding_bwd(torch.ones_like(out), tokens, mask, V)
    assert torch.equal(grad, count[:, None].expand(V, d))        # small whole numbers: exact in fp32
