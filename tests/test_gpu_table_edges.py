"""The calls on a tied model's table with inputs that leave a kernel no room: sums that are exact in any order, so that one column, row or scale out of
place shows.

Coded heads.  W[v] is a random row of +-2^u (u 0 or 1 per block of 128), times 2^-s of the block; a hidden row is aligned with one row of W, m = 1, 2 or 3
times its signs and 2^t (t 0, 1 or 2 per row and block), times 2^s of the block.  Values of a block keep their 4 bits in e4m3, products are whole numbers (times
1, 2 or 4, the same in a group of eight), so nothing is cut off and every logit is a whole number below 2^24.  What is left
of the bound is the log-sum-exp: roundings of the scaled exponent (a few 2^-24 of the largest |logit|), of its fp32 additions (128 at most in a slot) and
of the exponentials (2^-16 in all), and of the results: 2^-16 + 2^-21 (1 + top + |ref|).
The temperature is such that the aligned entry of the vocabulary has about half of the probability: counting it twice or not at all moves the
log-sum-exp by some 0.4.
"""
import numpy as np
import pytest
import torch

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def rb():
    from paper_2510_03515_amd import binding
    binding.load()
    assert torch.cuda.is_available()
    return binding


def _edges(V):
    """Entries at the ends of 32-wide blocks, tiles of 128 and 256, and of the last tiles, which begin where they end with the vocabulary."""
    at = [V - 1, V - 256, 256 * (V // 256) - 1, 256 * (V // 256), V - 128, 128 * (V // 128) - 1, 128 * (V // 128), 0, V - 2, V - 32, V - 33, V - 64, V - 65, V - 129,
          V - 257, 31, 32, 127, 128, 255, 256, V // 2]
    return [v for v in dict.fromkeys(at) if 0 <= v < V]


def _coded(dtype, N, T, d, V, spread=20):
    """hidden [N,T,d], W [V,d], targets, tokens [N,T], temperature; and the whole logits [N T, V] in float64."""
    gen = torch.Generator().manual_seed(N * 7919 + T * 31 + d + V)
    M, blocks = N * T, -(-d // 128)
    per = lambda x: x.repeat_interleave(128, -1)[..., :d]
    s = per(torch.randint(-spread, spread + 1, (blocks,), generator=gen).double())
    if spread > 100:                                                # the largest scale of one side meets the smallest of the other
        s = per(torch.where(torch.arange(blocks) % 2 == 0, float(spread), -float(spread) + 8).double())
    sign = torch.randint(0, 2, (V, d), generator=gen).double() * 2 - 1
    W = sign * torch.exp2(per(torch.randint(0, 2, (V, blocks), generator=gen).double()))
    edges = _edges(V)
    target = torch.randint(0, V, (M,), generator=gen)
    target[:len(edges)] = torch.tensor(edges[:M])
    size = torch.randint(1, 4, (M, d), generator=gen).double()
    size[:, ::128] = 3.0                                            # (the largest of a block does not hang on the draw)
    hidden = sign[target] * size * torch.exp2(per(torch.randint(0, 3, (M, blocks), generator=gen).double()))
    z = (hidden @ W.t()).numpy()
    temp = float(np.float32(z[np.arange(M), target.numpy()].mean() / (np.log(V) + 2.0)))
    tokens = torch.where(torch.rand(M, generator=gen) < 0.7, target, torch.randint(0, V, (M,), generator=gen))
    cast = lambda x, e: (x * torch.exp2(e)).to(torch.float32).to(TYPES[dtype])
    return cast(hidden, s).view(N, T, d), cast(W, -s), tokens.to(torch.int32).view(N, T), temp, z


def _log_probs(z, tokens, temp, weight=None):
    """(logp, lse, bound) of logits; weight: how often an entry of the vocabulary is counted."""
    z = z / temp
    top = np.abs(z).max(axis=1)
    zy, most = z[np.arange(len(z)), tokens.reshape(-1).numpy()], z.max(axis=1)
    z -= most[:, None]
    np.exp(z, out=z)
    lse = np.log(z.sum(axis=1) if weight is None else z @ weight) + most
    bound = lambda ref: 2.0 ** -16 + 2.0 ** -21 * (1 + top + np.abs(ref))
    return zy - lse, lse, bound


HEADS = {   # by the kernel that the sizes choose: dtype, N, T, d, V
    "small head": [("bf16", 5, 13, 520, 70), ("bf16", 5, 13, 1032, 255), ("bf16", 2, 40, 1536, 255), ("bf16", 3, 50, 128, 257), ("bf16", 2, 30, 72, 513),
                   ("bf16", 1, 300, 1024, 200), ("bf16", 3, 400, 512, 129), ("f32", 2, 20, 513, 129)],
    "32 rows": [("bf16", 4, 8, 520, 256), ("bf16", 1, 32, 1032, 257), ("bf16", 8, 4, 264, 385), ("bf16", 1, 32, 1536, 511), ("bf16", 31, 1, 512, 255 + 128),
                ("f32", 3, 7, 1001, 640), ("bf16", 2, 16, 136, 33000), ("bf16", 2, 16, 264, 70001)],
    "64 rows": [("bf16", 8, 8, 520, 513), ("bf16", 1, 33, 1024, 383), ("bf16", 1, 64, 1536, 257), ("f32", 5, 9, 515, 1023), ("bf16", 4, 16, 136, 66049)],
    "few row tiles": [("bf16", 1, 65, 520, 256), ("bf16", 5, 100, 1032, 257), ("bf16", 3, 300, 1536, 511), ("bf16", 2, 512, 264, 1025), ("bf16", 4, 64, 512, 300),
                      ("f32", 4, 40, 1001, 769), ("bf16", 1, 290, 136, 50021)],
    "row tiles": [("bf16", 2, 700, 520, 300), ("bf16", 1, 1100, 1536, 257), ("bf16", 3, 500, 1032, 511), ("bf16", 2, 1000, 1024, 768), ("bf16", 4, 300, 136, 2049),
                  ("f32", 2, 600, 1001, 513), ("bf16", 1, 1025, 512, 256), ("bf16", 11, 100, 136, 70001)],
}
CASES = [c for cases in HEADS.values() for c in cases]


@pytest.mark.parametrize("dtype,N,T,d,V", [c for c in CASES if c[1] * c[2] * c[4] <= 3000000])
def test_oracle_sees_one_column(dtype, N, T, d, V):
    """On the CPU: an entry left out, or the entries that the last two tiles share counted twice, is far outside of the bound of some row."""
    _, _, tokens, temp, z = _coded(dtype, N, T, d, V)
    assert np.abs(z).max() < 2 ** 24
    _, lse, bound = _log_probs(z, tokens, temp)
    wrong = [np.where(np.arange(V) == V - 1, 0.0, 1.0), np.where(np.arange(V) >= V - 32, 0.0, 1.0), np.where(np.arange(V) == 0, 0.0, 1.0)]
    for tile in (128, 256):
        if V > tile and V % tile:
            shared = (np.arange(V) >= V - tile) & (np.arange(V) < tile * (V // tile))
            if shared.any():
                wrong += [np.where(shared, 2.0, 1.0), np.where(shared, 0.0, 1.0)]
    for weight in wrong:
        off = np.abs(_log_probs(z, tokens, temp, weight)[1] - lse)
        assert (off > 100 * bound(lse)).any()


def _scored(rb, hidden, W, tokens, temp, exact=True):
    q = rb.rapid_quantize_fp8(W.cuda(), w_layout=rb.W_VD)
    if exact:                                                        # nothing was rounded
        blocks = q.values.shape[1] // 128
        back = (q.values.double().view(W.shape[0], blocks, 128) * torch.exp2(q.scales[:, :blocks].double() - 127)[:, :, None]).view(W.shape[0], -1)
        assert torch.equal(back[:, :W.shape[1]].cpu(), W.double()) and not back[:, W.shape[1]:].any()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mask = torch.ones(tokens.shape, dtype=torch.uint8, device="cuda")
    logp, lse = rb.rapid_logprob_fwd_fp8(hidden.cuda(), q, tokens.cuda(), mask, temperature=temp, want_lse=True, dev_status=status)
    return logp.double().cpu().numpy().reshape(-1), lse.double().cpu().numpy().reshape(-1), status.item()


def _check_coded(rb, dtype, N, T, d, V, **kw):
    hidden, W, tokens, temp, z = _coded(dtype, N, T, d, V, **kw)
    print(f"coded head {dtype} {N}x{T} d={d} V={V} {kw}", flush=True)
    logp, lse, status = _scored(rb, hidden, W, tokens, temp)
    want_p, want_s, bound = _log_probs(z, tokens, temp)
    assert status == 0
    assert np.all(np.abs(lse - want_s) <= bound(want_s))
    assert np.all(np.abs(logp - want_p) <= bound(want_p)) and np.all(logp <= 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,T,d,V", CASES)
def test_every_column_counts_once(rb, dtype, N, T, d, V):
    _check_coded(rb, dtype, N, T, d, V)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,T,d,V", [("bf16", 2, 9, 264, 70), ("bf16", 4, 8, 520, 257), ("f32", 3, 20, 1001, 300), ("bf16", 3, 90, 264, 300), ("f32", 2, 600, 520, 511)])
def test_scales_of_opposite_size(rb, dtype, N, T, d, V):
    """Blocks of 2^118 against 2^-118: the block's product alone is out of fp32's range before the second scale, the logit is not."""
    _check_coded(rb, dtype, N, T, d, V, spread=118)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [16, 64])
def test_log_sum_exp_does_not_drift_over_the_tiles(rb, rows):
    """One entry of the first tile holds all the probability, and 15 or more further tiles of the same workgroup follow it.  Its logit Z and the temperature
    1 are exact, so the log-sum-exp is Z but for the rounding of Z log2(e), once (2^-24 of Z), of the sum of one term and of the result (2^-24 of
    Z again): 2^-23 Z + 2^-21."""
    V, d = 128 * 256 * 16 + 1, 136
    Z = [(a, w) for a in range(8, 16) for w in range(8, 16) if 512 <= 8 * a * w < 1024][:rows]
    Z = (Z * rows)[:rows]
    hidden, W = torch.zeros(1, rows, d), torch.zeros((V, d), dtype=torch.bfloat16)
    for j, (a, w) in enumerate(Z):
        hidden[0, j, 2 * j], W[j, 2 * j] = float(a), 8.0 * w
    tokens = torch.arange(rows, dtype=torch.int32).view(1, rows)
    logp, lse, status = _scored(rb, hidden.bfloat16(), W, tokens, 1.0, exact=False)
    want = np.array([8.0 * a * w for a, w in Z])
    assert status == 0 and np.all(np.abs(lse - want) <= 2.0 ** -23 * want + 2.0 ** -21)
    assert np.all(np.abs(logp) <= 2.0 ** -23 * want + 2.0 ** -21) and np.all(logp <= 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("N,T,d,V", [(1, 3, 16, 90), (2, 8, 264, 700), (1, 40, 136, 300), (2, 100, 264, 300), (2, 600, 136, 513)])
def test_logits_next_to_the_end_of_fp32(rb, N, T, d, V):
    """A logit of 2.6e38 times log2(e) is beyond fp32: results are the formula's (whose log-probs are 0 and -2.6e38) or not finite, never a finite other value."""
    hidden, W = torch.zeros(N, T, d), torch.zeros(V, d)
    hidden[0, 0, 5], W[V - 1, 5] = 1.75 * 2.0 ** 63, 1.75 * 2.0 ** 63
    hidden[0, 1, 5], W[0, 6] = 1.75 * 2.0 ** 63, 1.0
    hidden[0, 2, 6] = 3.0
    tokens = torch.zeros((N, T), dtype=torch.int32)
    tokens[0, 0] = V - 1
    logp, lse, _ = _scored(rb, hidden, W, tokens, 1.0, exact=False)
    z = 3.0625 * 2.0 ** 126
    for got, want in ((lse[0], z), (lse[1], z), (logp[0], 0.0), (logp[1], -z)):
        assert not np.isfinite(got) or abs(got - want) <= 2.0 ** -22 * abs(want), (got, want)
    rest = np.log(V - 1 + np.exp(3.0))
    assert abs(lse[2] - rest) < 1e-4 and abs(logp[2] - (3.0 - rest)) < 1e-4      # the other rows are as they would be alone
    assert np.all(np.abs(lse[3:] - np.log(V)) < 1e-4)


@pytest.mark.gpu
@pytest.mark.parametrize("N,T,d,V", [(1, 20, 128, 200), (4, 8, 520, 3000), (1, 50, 1536, 700), (2, 200, 1024, 3000), (2, 700, 264, 2000)])
def test_confident_tokens(rb, N, T, d, V):
    """Sampled tokens with nearly all of the probability, logits 12 to 25: in every group of eight the aligned entry has one product of 448^2 and seven of 2^2, which the
    matrix unit leaves out (each is below 2^-13 of the largest).  The log-sum-exp may be lower than the formula's by 28 / 448^2 of its
    logit, never higher; the sampled logit is summed with all of it, and the log-prob is 0 where that comes out above."""
    gen = torch.Generator().manual_seed(d + V)
    M = N * T
    groups = torch.where(torch.arange(d) % 8 == 0, 448.0, 2.0)
    hidden = (groups * torch.where(torch.rand(M, 1, generator=gen) < 0.5, 1.0, 0.5)).view(N, T, d)       # powers of two: the same bits in e4m3
    W = torch.zeros(V, d)
    target = int(torch.randint(0, V, (1,), generator=gen))
    W[target] = groups
    tokens = torch.full((N, T), target, dtype=torch.int32)
    top = float((groups * groups).sum())
    temp = float(np.float32(top / 25.0))
    logp, lse, status = _scored(rb, hidden.bfloat16(), W.bfloat16(), tokens, temp)
    z = hidden[:, :, 0].double().numpy().reshape(-1) / 448.0 * top / temp
    want = z + np.log1p((V - 1) * np.exp(-z))
    cut = z * 28 / 448.0 ** 2
    fp32 = 2.0 ** -16 + 2.0 ** -21 * (1 + 2 * z) + d * 2.0 ** -22 * z / 8
    assert status == 0
    assert np.all(lse <= want + fp32) and np.all(lse >= want - cut - fp32)
    assert np.all(np.abs(logp - (z - want)) <= cut + fp32) and np.all(logp <= 0.0)
    above = lse < z - fp32
    assert above.any() and np.all(logp[above] == 0.0)


# ------------------------------------------------------------------------------ lookup and gradient of very many positions
def _whole_rows(N, T, d, dtype):
    """Gradient rows of small whole numbers that depend on position and column: every sum is exact in fp32."""
    p, c = torch.arange(N * T, device="cuda")[:, None], torch.arange(d, device="cuda")[None, :]
    return ((p * 31 + p // 64 * 5 + c * 17) % 7 - 3).to(TYPES[dtype]).view(N, T, d)


def _zipf(N, T, V, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = torch.exp(torch.rand((N, T), generator=gen, device="cuda", dtype=torch.float64) * np.log(V + 1)).long() - 1
    return r.clamp(0, V - 1).to(torch.int32), (torch.rand((N, T), generator=gen, device="cuda") < 0.8).to(torch.uint8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,T,d,V", [
    ("bf16", 1300, 1000, 8, 5000), ("bf16", 1100, 2000, 8, 300000), ("f32", 1100, 1000, 5, 600),        # sorts with two and three rounds a block, one to three passes
    ("f32", 64, 1030, 1021, 901), ("f32", 64, 1030, 1024, 901), ("bf16", 64, 2100, 1024, 5000)])         # gradient rows of more than 256 MB
def test_gradient_of_many_positions(rb, dtype, N, T, d, V):
    print(f"many positions {dtype} {N}x{T} d={d} V={V}", flush=True)
    tokens, mask = _zipf(N, T, V, d)
    dh = _whole_rows(N, T, d, dtype)
    at = mask.view(-1).nonzero()[:, 0]
    want = torch.zeros((V, d), dtype=torch.float64, device="cuda")
    for part in at.split(1 << 18):
        want.index_add_(0, tokens.view(-1)[part].long(), dh.view(-1, d)[part].double())
    assert want.abs().max().item() < 2 ** 24
    assert torch.equal(rb.rapid_embedding_bwd(dh, tokens, mask, V).double(), want)
    old = (torch.arange(V * d, device="cuda") % 11).float().view(V, d)
    got = rb.rapid_embedding_bwd(dh, tokens, mask, V, dtable=old.clone(), accumulate=True)
    assert torch.equal(got.double(), want + old)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,N,T,d", [("bf16", 1, (1 << 25) + 5, 8), ("f32", 5, ((1 << 25) + 35) // 5, 3), ("f32", 1, (1 << 25) + 1, 5)])
def test_lookup_of_many_positions(rb, dtype, N, T, d):
    """More than 2^25 positions, where a wave takes 64 of them."""
    V = 1013
    table = torch.randn((V, d), device="cuda").to(TYPES[dtype])
    tokens, mask = _zipf(N, T, V, d)
    out = rb.rapid_embedding_fwd(table, tokens, mask)
    for i in range(0, N * T, 1 << 22):
        at = slice(i, i + (1 << 22))
        assert torch.equal(out.view(-1, d)[at], table[tokens.view(-1)[at].long()] * (mask.view(-1)[at, None] != 0))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,positions,d,V", [
    ("bf16", 2560, 16, 4096), ("bf16", 2561, 16, 4096), ("f32", 2561, 6, 513), ("bf16", 2561, 24, 512), ("f32", 3000, 8, 2), ("bf16", 2561, 8, 4097),
    ("bf16", 6144, 16, 4097), ("bf16", 6145, 16, 4097), ("f32", 6145, 5, 300000), ("bf16", 6145, 8, 300), ("bf16", 32768, 8, 4096), ("bf16", 32769, 8, 4096)])
@pytest.mark.parametrize("kept", [1.0, 0.5, 0.0])
def test_gradient_on_both_sides_of_the_sorts(rb, dtype, positions, d, V, kept):
    """The one-block sort, one wide pass and passes of many blocks, next to where one takes over from the other; few or no valid positions among them."""
    print(f"sorts {dtype} {positions} d={d} V={V} {kept}", flush=True)
    tokens, mask = _zipf(1, positions, V, positions + d)
    mask *= (torch.rand((1, positions), generator=torch.Generator().manual_seed(d)) < kept).cuda()
    if kept == 1.0:
        tokens[0, 5], tokens[0, positions - 1] = V, -1               # ids without a row
    dh = _whole_rows(1, positions, d, dtype)
    good = (mask != 0) & (tokens >= 0) & (tokens < V)
    want = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, tokens[good].long(), dh[good].double())
    assert torch.equal(rb.rapid_embedding_bwd(dh, tokens, mask, V).double(), want)
    assert torch.equal(rb.rapid_embedding_bwd(dh, tokens, mask, V, dtable=torch.ones((V, d), device="cuda"), accumulate=True).double(), want + 1.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("bf16", 200), ("bf16", 1032), ("f32", 3), ("f32", 100), ("f32", 257)])
def test_lookup_on_both_sides_of_several_rows_a_wave(rb, dtype, d):
    table = torch.randn((333, d), device="cuda").to(TYPES[dtype])
    for positions in (2047, 2048, 2049, 2112):
        tokens, mask = _zipf(1, positions, 333, positions)
        assert torch.equal(rb.rapid_embedding_fwd(table, tokens, mask), table[tokens.long()] * (mask[:, :, None] != 0))
