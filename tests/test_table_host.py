"""CPU checks of the calls on a tied model's table: the oracle against independent legs, sizes, and every refusal (no kernel is
launched: the pointers are never dereferenced)."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import table_oracle as orc

F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def rb():
    from paper_2510_03515_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2510_03515_amd import build
        build.build(verbose=False)
    binding.load()
    return binding


def test_oracle_rounds_as_torch_casts():
    """Every e4m3 value, every midpoint between two and its neighbours on both sides."""
    every = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (every[1:] + every[:-1]) / 2
    x = np.concatenate([every, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e3)])
    x = np.concatenate([x, -x])
    assert np.array_equal(orc.round_e4m3(every), every)
    near = np.abs(x[:, None] - np.concatenate([every, -every])[None, :])
    assert np.array_equal(np.abs(orc.round_e4m3(x) - x), near.min(axis=1))                       # nearest
    f = x.astype(np.float32)
    f = f[f.astype(np.float64) == x]                                                               # (torch casts from fp32)
    assert np.array_equal(orc.round_e4m3(f), torch.from_numpy(f).to(torch.float8_e4m3fn).double().numpy())   # and ties to even


@pytest.mark.parametrize("most,e", [(448.0, 0), (448.0000305, 1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.875, -9), (3.4e38, 120),
                                    (2.0 ** -126, -126), (1e-45, -126), (0.0, 0)])
def test_oracle_exponents(most, e):
    x = np.zeros((1, 130))
    x[0, 5] = -most
    x[0, 128] = 448.0
    values, exponents = orc.quantize(x)
    assert values.shape == (1, 256) and list(exponents[0]) == [e, 0]
    assert np.all(np.abs(values) <= 448) and (e == -126 or most == 0 or np.abs(values[0, 5]) > 216)


def test_oracle_gradient_against_differences():
    """The lookup is linear in the table: differences of <G, lookup(E)> along every entry are the gradient."""
    rng = np.random.default_rng(0)
    table, tokens = rng.standard_normal((5, 3)), rng.integers(-1, 6, (2, 4))
    mask = (rng.random((2, 4)) < 0.7).astype(np.uint8)
    G = rng.standard_normal((2, 4, 3))
    grad, size, terms = orc.embedding_bwd(G, tokens, mask, 5, 2.5)
    for v in range(5):
        for k in range(3):
            moved = [table.copy(), table.copy()]
            moved[0][v, k] += 0.5
            moved[1][v, k] -= 0.5
            up, down = (np.sum(G * orc.embedding_fwd(m, tokens, mask, 2.5)) for m in moved)
            assert abs((up - down) - grad[v, k]) < 1e-12
    assert terms.sum() == np.sum((mask != 0) & (tokens >= 0) & (tokens < 5)) and np.all(size >= np.abs(grad) - 1e-12)


def test_sizes(rb):
    lib = rb.load()
    for d, values, scales in ((1, 128, 4), (128, 128, 4), (129, 256, 4), (512, 512, 4), (513, 640, 8), (896, 896, 8), (1536, 1536, 12), (2048, 2048, 16)):
        assert lib.rapid_fp8_value_bytes(d) == values and lib.rapid_fp8_scale_bytes(d) == scales
    assert lib.rapid_fp8_value_bytes(0) == 0 and lib.rapid_fp8_scale_bytes(-5) == 0
    for op in (rb.OP_EMBEDDING_BWD, rb.OP_LOGPROB_FWD_FP8):
        args = (op, 4, 100, 64, 1000)
        assert rb.rapid_workspace_bytes(*args, 1, F32) == rb.rapid_workspace_bytes(*args, 9, BF16, minimum=True) > 0
        assert rb.rapid_workspace_bytes(*args, 1, F32, max_tokens=7) == rb.rapid_workspace_bytes(*args, 1, F32)
        assert rb.rapid_workspace_bytes(op, 0, 1, 64, 100, 1, F32) == 0 and rb.rapid_workspace_bytes(op, 1, 1, 64, 100, 1, 5) == 0
        assert rb.rapid_workspace_bytes(op, 1 << 40, 1 << 40, 64, 100, 1, F32) == 0
    assert rb.rapid_workspace_bytes(rb.OP_LOGPROB_FWD_FP8, 2, 1 << 25, 64, 100, 1, F32) == 0      # 2^25 positions at most


one = C.c_void_p(256)
odd = C.c_void_p(264)


def test_refusals_embedding_fwd(rb):
    f = rb.load().rapid_embedding_fwd
    good = dict(table=one, tokens=one, mask=one, N=2, T=3, d=8, V=9, dtype=BF16, scale=1.0, out=one, status=None, stream=None)
    call = lambda **kw: f(*dict(good, **kw).values())
    for p in ("table", "tokens", "out"):
        assert call(**{p: None}) == -1
    assert call(dtype=2) == -3
    for kw in (dict(N=0), dict(T=-1), dict(d=0), dict(V=0), dict(d=12), dict(d=65544), dict(V=4000001), dict(N=1 << 33, T=1 << 33), dict(N=50000, T=50000),
               dict(table=odd), dict(out=odd), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert call(**kw) == -2, kw


def test_refusals_embedding_bwd(rb):
    f = rb.load().rapid_embedding_bwd
    good = dict(dh=one, tokens=one, mask=None, N=2, T=3, d=8, V=9, dtype=BF16, scale=1.0, dw=F32, acc=0, out=one, status=None, ws=one, bytes=1 << 30, stream=None)
    call = lambda **kw: f(*dict(good, **kw).values())
    for p in ("dh", "tokens", "out"):
        assert call(**{p: None}) == -1
    assert call(dtype=7) == -3 and call(dw=3) == -3 and call(dw=BF16, acc=1) == -3
    for kw in (dict(N=0), dict(d=4), dict(V=4000001), dict(dh=odd), dict(out=odd), dict(scale=float("nan"))):
        assert call(**kw) == -2, kw
    need = rb.rapid_workspace_bytes(rb.OP_EMBEDDING_BWD, 2, 3, 8, 9, 1, BF16)
    for kw in (dict(ws=None), dict(ws=odd), dict(bytes=need - 1), dict(bytes=0)):
        assert call(**kw) == -4, kw
    assert b"minimum" in rb.load().rapid_last_error()


def test_refusals_quantize(rb):
    f = rb.load().rapid_quantize_fp8
    good = dict(W=one, d=8, V=9, dtype=BF16, layout=0, values=one, scales=one, status=None, stream=None)
    call = lambda **kw: f(*dict(good, **kw).values())
    for p in ("W", "values", "scales"):
        assert call(**{p: None}) == -1
    assert call(dtype=2) == -3 and call(layout=2) == -3
    for kw in (dict(d=0), dict(V=0), dict(d=9), dict(V=4000001), dict(W=odd), dict(values=odd), dict(scales=C.c_void_p(258))):
        assert call(**kw) == -2, kw


def test_refusals_logprob(rb):
    f = rb.load().rapid_logprob_fwd_fp8
    good = dict(hidden=one, values=one, scales=one, tokens=one, mask=one, N=2, T=3, d=8, V=9, dtype=BF16, temp=1.0, logp=one, lse=None, status=None, ws=one,
                bytes=1 << 30, stream=None)
    call = lambda **kw: f(*dict(good, **kw).values())
    for p in ("hidden", "values", "scales", "tokens", "mask", "logp"):
        assert call(**{p: None}) == -1
    assert call(dtype=2) == -3
    for kw in (dict(N=0), dict(d=9), dict(V=4000001), dict(hidden=odd), dict(values=odd), dict(scales=C.c_void_p(258)), dict(temp=0.0), dict(temp=float("inf")),
               dict(temp=float("nan")), dict(N=1 << 13, T=1 << 13)):
        assert call(**kw) == -2, kw
    need = rb.rapid_workspace_bytes(rb.OP_LOGPROB_FWD_FP8, 2, 3, 8, 9, 1, BF16)
    for kw in (dict(ws=None), dict(ws=odd), dict(bytes=need - 1)):
        assert call(**kw) == -4, kw


def test_binding_refuses_cpu_tensors_and_shapes(rb):
    tokens = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(TypeError):
        rb.rapid_embedding_fwd(torch.zeros(5, 8), tokens)
    with pytest.raises(TypeError):
        rb.rapid_quantize_fp8(torch.zeros(5, 8))
    with pytest.raises(TypeError):
        rb.rapid_embedding_bwd(torch.zeros(2, 3, 8), tokens, None, 5)
    with pytest.raises(TypeError):
        rb.Fp8Weight(torch.zeros(5, 128), torch.zeros(5, 4, dtype=torch.uint8), 8)


def test_binding_refuses_other_devices_status_words_and_workspaces(rb, monkeypatch):
    """What every one of the calls checks last, with tensors that only claim to lie on a GPU."""
    class On:
        def __init__(self, device, dtype=torch.int32, n=1, contiguous=True):
            self.device, self.dtype, self.n, self.is_cuda, self.contiguous = f"cuda:{device}", dtype, n, device >= 0, contiguous
        def get_device(self): return int(self.device[5:])
        def is_contiguous(self): return self.contiguous
        def view(self, *_): return torch.zeros(self.n)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    rb._here((On(1), None), None)
    rb._here((On(1),), On(1), On(1, torch.uint8, 4096))
    for args in (((On(0),), None), ((On(1), On(2)), None), ((On(1),), On(0)), ((On(1),), On(-1)), ((On(1),), On(1, torch.uint8)), ((On(1),), On(1, n=0)),
                 ((On(1),), None, On(0, torch.uint8)), ((On(1),), None, On(1, torch.float32)), ((On(1),), None, On(1, torch.uint8, contiguous=False))):
        with pytest.raises(TypeError):
            rb._here(*args)


def test_sizes_of_calls_that_are_refused(rb):
    """bf16 rows that are no multiple of 8 columns, shorter than one piece among them: no size, and no fault."""
    for op in (rb.OP_EMBEDDING_BWD, rb.OP_LOGPROB_FWD_FP8):
        for d in (1, 4, 7, 9, 12, 65535):
            for minimum in (False, True):
                assert rb.rapid_workspace_bytes(op, 2, 3, d, 9, 1, BF16, minimum=minimum) == 0
                assert rb.rapid_workspace_bytes(op, 2, 3, d, 9, 1, F32, minimum=minimum) > 0


def test_tied_workload_draws_from_its_policy():
    """Tokens of the tied workload by the previous token against softmax(scale E[x] . E): chi-squared over the ids, and the inputs are the tokens before."""
    from paper_2510_03515_amd import workloads as wl
    spec = wl.small_spec("tied", "f32", d=16, V=12, prompts=40, G=16, len_lo=30, len_hi=30)
    w = wl.make_tied_workload(spec, seed=1, scale=4.0)
    x, y, E = w["inputs"].long(), w["tokens"].long(), w["table"].double()
    assert torch.equal(x[:, 1:], y[:, :-1]) and len(x[:, 0].unique()) > 5
    p = torch.softmax(4.0 * E @ E.t(), dim=1)
    seen = torch.zeros(12, 12, dtype=torch.float64)
    seen.index_put_((x.reshape(-1), y.reshape(-1)), torch.ones(x.numel(), dtype=torch.float64), accumulate=True)
    want = seen.sum(1, keepdim=True) * p
    assert want.min() > 5                                             # enough in every cell for the statistic to be near its distribution
    # 132 degrees of freedom: mean 132, standard deviation 16.2; 6 of them
    assert ((seen - want) ** 2 / want).sum() < 132 + 6 * 16.2
