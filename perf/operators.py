"""Operators around the one table W of a tied model: the calls of an update besides the loss step, over the sizes they come in.

Kinds of call (`kind`):
  embed   hidden states of a batch's input tokens, looked up in the table [V, d] and scaled; masked positions are zero
  grad    the table's gradient from the gradient of those states: rows of the same token are added up, into a fresh gradient or
          (`accumulate`) into the one that the loss step left in the tied head
  quant   the table to 8 bits (e4m3) with a power of two as the scale of every 128 values of a row; given as [V, d] ("vd") or [d, V] ("dv")
  score   log-probs of sampled tokens under a policy whose head is kept in 8 bits

A batch is N generations with lengths uniform in [len_lo, len_hi], padded to len_hi; with `holes` a fifth of the valid positions is masked too.
Token ids follow Zipf's law over a shuffled vocabulary, as in text.
"""
import math

import numpy as np
import torch

own = False

V_QWEN = 151936


def listed():
    bf16 = dict(dtype="bf16", d=1536, V=V_QWEN, holes=False)
    f32 = dict(dtype="f32", d=256, V=4096, holes=False)
    return [
        # input of one decoding step of 8 sequences: a launch
        dict(bf16, name="embed_decode", kind="embed", N=8, len_lo=1, len_hi=1, scale=1.0),
        # the synthetic bandit's inference batch in fp32, with the square root of d as the scale
        dict(f32, name="embed_bandit_f32", kind="embed", N=512, len_lo=8, len_hi=48, scale=16.0),
        # the headline mini-batch: 32 x 8 generations of up to 2048 tokens
        dict(bf16, name="embed_1.5b", kind="embed", N=256, len_lo=256, len_hi=2048, scale=1.0),
        # gradient of the bandit's batch in fp32
        dict(f32, name="grad_bandit_f32", kind="grad", N=512, len_lo=8, len_hi=48, scale=16.0, dw="f32", accumulate=False),
        # micro-batch of gradient accumulation: one prompt's 4 generations, added to the tied head's fp32 gradient
        dict(bf16, name="grad_micro_accumulate", kind="grad", N=4, len_lo=64, len_hi=1024, scale=1.0, dw="f32", accumulate=True),
        # the headline mini-batch's gradient for a bf16 optimiser
        dict(bf16, name="grad_1.5b", kind="grad", N=256, len_lo=256, len_hi=2048, scale=1.0, dw="bf16", accumulate=False),
        # fp32 master weights of a 0.5B-shaped head to 8 bits, rows as checkpoints store them
        dict(name="quant_0.5b_f32", kind="quant", dtype="f32", d=896, V=V_QWEN, layout="vd"),
        # 1.5B-shaped head in the library's other layout, whose blocks run down the columns
        dict(name="quant_1.5b_dv", kind="quant", dtype="bf16", d=1536, V=V_QWEN, layout="dv"),
        # the tokens that 16 sequences just drew: the table is read once for next to no products
        dict(bf16, name="score_16_tokens", kind="score", N=16, len_lo=1, len_hi=1, temp=1.0),
        # a serving loop scores a few short generations
        dict(bf16, name="score_few", kind="score", N=8, len_lo=8, len_hi=64, temp=1.0),
        # sizes that end inside tiles and blocks, fp32 states, a sampling temperature, masked positions in between
        dict(name="score_odd_f32", kind="score", dtype="f32", d=1001, V=50021, holes=True, N=23, len_lo=16, len_hi=301, temp=0.7),
        # behaviour or reference log-probs of an inference batch
        dict(bf16, name="score_batch", kind="score", N=64, len_lo=1024, len_hi=1024, temp=1.0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["embed", "grad", "grad", "quant", "score", "score", "score"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    V = _log_int(rng, 500, V_QWEN)
    d = 8 * _log_int(rng, 8, 256) if dtype == "bf16" else _log_int(rng, 17, 2000)
    if kind == "quant":
        return dict(kind=kind, dtype=dtype, d=d if dtype == "bf16" else min(d, 900), V=V, layout=rng.choice(["vd", "dv"]))
    while True:
        hi = _log_int(rng, 1, 2048)
        c = dict(kind=kind, dtype=dtype, d=d, V=V, holes=rng.random() < 0.3, N=_log_int(rng, 1, 512),
                 len_lo=max(1, int(hi * rng.uniform(0.05, 0.6))), len_hi=hi)
        positions = c["N"] * hi
        if kind == "score":
            c.update(temp=rng.choice([1.0, 1.0, 0.7]))
            if positions <= 65536 and positions * d * V <= 65536 * 1536 * V_QWEN:
                return c
        else:
            c.update(scale=rng.choice([1.0, math.sqrt(d)]))
            if kind == "grad":
                c.update(dw=rng.choice(["f32", "f32", "bf16"]), accumulate=False)
                c["accumulate"] = c["dw"] == "f32" and rng.random() < 0.5
            if positions * d * (2 if dtype == "bf16" else 4) <= 256 * 2048 * 1536 * 2:
                return c


_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _randn(shape, gen, std, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(_TYPES[dtype])


def _table(case, gen):
    # rows of a head differ in size by more than the entries of one row
    size = torch.exp(0.3 * torch.randn((case["V"], 1), generator=gen, device="cuda"))
    return (torch.randn((case["V"], case["d"]), generator=gen, device="cuda") * 0.02 * size).to(_TYPES[case["dtype"]])


def _batch(case, gen):
    N, T, V = case["N"], case["len_hi"], case["V"]
    length = torch.randint(case["len_lo"], T + 1, (N, 1), generator=gen, device="cuda")
    mask = torch.arange(T, device="cuda")[None, :] < length
    if case["holes"]:
        mask &= torch.rand((N, T), generator=gen, device="cuda") < 0.8
    rank = torch.exp(torch.rand((N, T), generator=gen, device="cuda", dtype=torch.float64) * math.log(V + 1)).long() - 1
    tokens = torch.randperm(V, generator=gen, device="cuda")[rank.clamp(0, V - 1)].to(torch.int32)
    return tokens, mask.to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] == "quant":
        W = _table(case, gen)
        return dict(case=case, W=W.t().contiguous() if case["layout"] == "dv" else W)
    tokens, mask = _batch(case, gen)
    s = dict(case=case, tokens=tokens, mask=mask)
    if case["kind"] == "embed":
        return dict(s, table=_table(case, gen))
    shape = (case["N"], case["len_hi"], case["d"])
    if case["kind"] == "grad":
        s["dhidden"] = _randn(shape, gen, 1e-3, case["dtype"])
        s["dtable"] = torch.empty((case["V"], case["d"]), dtype=_TYPES[case["dw"]], device="cuda")
        if case["accumulate"]:
            s["dtable"].normal_(0.0, 1e-3, generator=gen)
        return s
    # hidden states as the final norm leaves them
    values, exponents = _to_8_bits(_table(case, gen).float())
    return dict(s, hidden=_randn(shape, gen, 1.0, case["dtype"]), values=values, scales=_scales(exponents))


def _scales(exponents):
    """Scales as the head keeps them: a byte e + 127 a block, and whole words a row."""
    return torch.nn.functional.pad((exponents + 127).to(torch.uint8), (0, -exponents.shape[1] % 4), value=127)


def _power(e):
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _to_8_bits(x):
    """Rows [R, d] in fp32 as e4m3 values [R, d up to whole blocks of 128] and the exponents of their blocks."""
    R, d = x.shape
    x = torch.nn.functional.pad(x, (0, -d % 128)).view(R, -1, 128)
    fraction, exponent = torch.frexp(x.abs().amax(2))       # largest = fraction 2^exponent, fraction in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(fraction == 0, 0, (exponent - 9 + (fraction > 0.875).int()).clamp(min=-126))
    return (x * _power(-e)[:, :, None]).view(R, -1).to(torch.float8_e4m3fn), e


def _from_8_bits(values, exponents):
    R = values.shape[0]
    return (values.float().view(R, -1, 128) * _power(exponents)[:, :, None]).view(R, -1)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2510_03515_amd import binding as rb
    case = s["case"]
    if case["kind"] == "embed":
        return rb.rapid_embedding_fwd(s["table"], s["tokens"], s["mask"], scale=case["scale"])
    if case["kind"] == "grad":
        return rb.rapid_embedding_bwd(s["dhidden"], s["tokens"], s["mask"], case["V"], scale=case["scale"],
                                      dtable=s["dtable"], accumulate=case["accumulate"])
    if case["kind"] == "quant":
        q = rb.rapid_quantize_fp8(s["W"], w_layout=rb.W_DV if case["layout"] == "dv" else rb.W_VD)
        return dict(values=q.values, scales=q.scales)
    W8 = rb.Fp8Weight(s["values"], s["scales"], case["d"])
    logp, lse = rb.rapid_logprob_fwd_fp8(s["hidden"], W8, s["tokens"], s["mask"], temperature=case["temp"], want_lse=True)
    return dict(logp=logp, lse=lse)


def _run_plain(s):
    case = s["case"]
    if case["kind"] == "quant":
        W = s["W"].t() if case["layout"] == "dv" else s["W"]
        values, exponents = _to_8_bits(W.float())
        return dict(values=values, scales=_scales(exponents))
    valid = s["mask"].bool()
    tokens = s["tokens"][valid].long()
    if case["kind"] == "embed":
        out = torch.zeros((*valid.shape, case["d"]), dtype=s["table"].dtype, device="cuda")
        out[valid] = (s["table"][tokens].float() * case["scale"]).to(out.dtype)
        return out
    if case["kind"] == "grad":
        rows = s["dhidden"][valid].float() * case["scale"]
        if case["accumulate"]:
            return s["dtable"].index_add_(0, tokens, rows)
        return torch.zeros(s["dtable"].shape, device="cuda").index_add_(0, tokens, rows).to(s["dtable"].dtype)
    W = _from_8_bits(s["values"], s["scales"][:, :s["values"].shape[1] // 128].int() - 127)
    h = _from_8_bits(*_to_8_bits(s["hidden"][valid].float()))
    z = (h @ W.t()) / case["temp"]
    zy = z.gather(1, tokens[:, None])[:, 0]
    largest = z.amax(1, keepdim=True)
    lse = largest[:, 0] + z.sub_(largest).exp_().sum(1).log()
    out = dict(logp=torch.zeros(valid.shape, device="cuda"), lse=torch.zeros(valid.shape, device="cuda"))
    out["logp"][valid], out["lse"][valid] = zy - lse, lse
    return out


def _round_e4m3(x):
    """x (64 bits, at most 448 in size) to the nearest of: 4 significant bits from 2^-6 on, multiples of 2^-9 below; ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _blocks64(x):
    """Rows in 64 bits: rounded values of their blocks of 128 and the blocks' scales, the smallest 2^e, e >= -126, with 448 2^e >= every value."""
    R, d = x.shape
    blocks = -(-d // 128)
    padded = torch.zeros((R, blocks * 128), dtype=torch.float64, device="cuda")
    padded[:, :d] = x
    padded = padded.view(R, blocks, 128)
    most = padded.abs().amax(2)
    e = torch.ceil(torch.log2(most.clamp(min=2.0 ** -200) / 448)).clamp(min=-126)
    e = torch.where(most > 448 * torch.exp2(e), e + 1, torch.where((most <= 448 * torch.exp2(e - 1)) & (e > -126), e - 1, e))
    e = torch.where(most == 0, torch.zeros_like(e), e)
    return _round_e4m3(padded * torch.exp2(-e)[:, :, None]), e


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quant":
        W = s["W"].t() if case["layout"] == "dv" else s["W"]
        values, scales = [], []
        for part in W.split(8192):
            q, e = _blocks64(part.double())
            values.append(q.view(part.shape[0], -1).float())
            scales.append(torch.full((part.shape[0], -(-e.shape[1] // 4) * 4), 127, dtype=torch.uint8, device="cuda"))
            scales[-1][:, :e.shape[1]] = (e + 127).to(torch.uint8)
        return dict(values=torch.cat(values).double(), scales=torch.cat(scales))
    N, T, d = case["N"], case["len_hi"], case["d"]
    where = s["mask"].reshape(-1).nonzero()[:, 0]
    tokens = s["tokens"].reshape(-1)[where].long()
    if case["kind"] == "embed":
        out = torch.zeros((N * T, d), dtype=torch.float64, device="cuda")
        for at, tok in zip(where.split(65536), tokens.split(65536)):
            out[at] = s["table"][tok].double() * case["scale"]
        return out.view(N, T, d)
    if case["kind"] == "grad":
        flat = s["dhidden"].view(N * T, d)
        out = s["dtable"].double() if case["accumulate"] else torch.zeros((case["V"], d), dtype=torch.float64, device="cuda")
        for at, tok in zip(where.split(65536), tokens.split(65536)):
            out.index_add_(0, tok, flat[at].double() * case["scale"])
        return out
    W = s["values"].double().view(case["V"], -1, 128)
    W = W * torch.exp2(s["scales"][:, :W.shape[1]].double() - 127)[:, :, None]
    W = W.view(case["V"], -1)
    flat = s["hidden"].view(N * T, d)
    logp, lse = (torch.zeros(N * T, dtype=torch.float64, device="cuda") for _ in range(2))
    for at, tok in zip(where.split(4096), tokens.split(4096)):
        q, e = _blocks64(flat[at].double())
        z = (q * torch.exp2(e)[:, :, None]).view(at.numel(), -1) @ W.t() / case["temp"]
        lse[at] = torch.logsumexp(z, 1)
        logp[at] = z.gather(1, tok[:, None])[:, 0] - lse[at]
    return dict(logp=logp.view(N, T), lse=lse.view(N, T))


def _tokens(case):
    return case["N"] * (case["len_lo"] + case["len_hi"]) / 2 * (0.8 if case["holes"] else 1.0)


def _distinct(case):
    """Expected number of different ids in a batch of Zipf's law."""
    rank = np.arange(1, case["V"] + 1)
    return float((1.0 - (1.0 - np.log((rank + 1) / rank) / math.log(case["V"] + 1)) ** _tokens(case)).sum())


def work(case):
    d, V, e = case["d"], case["V"], 2 if case["dtype"] == "bf16" else 4
    blocks = -(-d // 128)
    in_8_bits = V * (blocks * 128 + -(-blocks // 4) * 4)
    if case["kind"] == "quant":     # the table in, values and scales out
        return dict(bytes=V * d * e + in_8_bits, flops=3 * V * d)
    M, positions = _tokens(case), case["N"] * case["len_hi"]
    if case["kind"] == "embed":     # the rows of the ids that occur and the ids in; every position out
        return dict(bytes=_distinct(case) * d * e + positions * (d * e + 5), flops=M * d)
    if case["kind"] == "grad":      # valid gradient rows and ids in; the table out, or the rows of the ids that occur in and out
        table = 8 * _distinct(case) * d if case["accumulate"] else V * d * (2 if case["dw"] == "bf16" else 4)
        return dict(bytes=M * d * e + positions * 5 + table, flops=2 * M * d)
    return dict(bytes=M * d * e + in_8_bits + positions * 13, flops=2 * M * d * V)
