"""The rest of a layer and of its head around the scan, as cases that can be timed and checked.

A case is one pass through an operator as a program makes it: the normalisation at the entry of a
sublayer, which adds the sublayer before onto the residual stream (its output for products in
bf16, in fp32, or in 8 bits with scales), and its gradient; the gated product of an MLP, act(x Wg^T) * (x Wu^T),
and its gradient; and the head of an evaluation or of a sampler that weighs alternatives: the
log-probability of a given token of each row, the entropy, and the most probable tokens.

Widths are those of the layers that the rest of the benchmark runs (1024 with 2048 and 4096, the
paper's 448 and 832) and odd ones between them; vocabularies are generic sizes of 1,000 to 131,072.

Row counts: a single token; a denoising step of 16 rows of 32 tokens; the paper's blocks of
256 tokens; training windows of up to 16,384 tokens.
"""
import math

import torch

own = False   # False: the plain form in torch operations; True: this library's kernels

EPS = 1e-5
E4M3_MAX = 448.0


def _norm(rows, width, *, x="bf16", residual="none", out="bf16", block=0, **name):
    return dict(kind="norm", rows=rows, width=width, x=x, residual=residual, out=out, block=block, **name)


def _norm_grad(rows, width, *, dy="bf16", s="bf16", stream=True, **name):
    return dict(kind="norm_grad", rows=rows, width=width, dy=dy, s=s, stream=stream, **name)


def _gated(kind, rows, k, n, *, dtype="bf16", act="silu", bias=False, keep=False, **name):
    return dict(kind=kind, rows=rows, k=k, n=n, dtype=dtype, act=act, bias=bias, keep=keep, **name)


def _logprobs(rows, k, n, *, dtype="bf16", top=0, given=True, exclude=False, **name):
    return dict(kind="logprobs", rows=rows, k=k, n=n, dtype=dtype, top=top, given=given, exclude=exclude, **name)


def listed():
    return [
        # the smallest call: one token enters a sublayer, launch and host latency
        _norm(1, 1024, residual="bf16", name="norm_token"),
        # a denoising step of 16 sequences with blocks of 32 tokens, for products in 8 bits
        _norm(512, 1024, residual="bf16", out="e4m3", name="norm_step_e4m3"),
        # a training window of the 350M layer shape with an fp32 residual stream
        _norm(16384, 1024, residual="fp32", name="norm_train"),
        # its gradient, with what arrives on the stream from behind
        _norm_grad(16384, 1024, s="fp32", name="norm_grad_train"),
        # one token through the MLP's gated product: the weights' bytes are the whole of it
        _gated("gated", 1, 1024, 4096, name="gated_token"),
        # the same for a denoising step
        _gated("gated", 512, 1024, 4096, name="gated_step"),
        # training: both pre-activations kept
        _gated("gated", 16384, 1024, 4096, keep=True, name="gated_train"),
        # its gradient: input and both weights
        _gated("gated_grad", 16384, 1024, 4096, name="gated_grad_train"),
        # a ragged fp32 gradient with GELU and biases at the paper's small width
        _gated("gated_grad", 1003, 448, 1934, dtype="fp32", act="gelu", bias=True, name="gated_grad_fp32"),
        # a sampler's token with its alternatives
        _logprobs(1, 1024, 32768, top=8, given=False, name="logprobs_token"),
        # a denoising step that orders its positions by entropy and margin: what the drafted tokens
        # have, and five alternatives, the mask token ruled out
        _logprobs(512, 1024, 50257, top=5, exclude=True, name="logprobs_step"),
        # an evaluation of held-out text at the paper's width, ragged
        _logprobs(4003, 832, 32003, name="logprobs_eval"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case: the kinds and ranges of the listed ones."""
    kind = rng.choice(["norm", "norm", "norm_grad", "gated", "gated", "gated_grad", "gated_grad", "logprobs", "logprobs",
                       "logprobs"])
    rows = rng.choice([_log(rng, 1, 16384), _log(rng, 1, 16384), _log(rng, 1, 64),
                       min(16384, rng.randint(1, 128) * rng.choice([16, 32, 64, 256]))])
    if kind.startswith("norm"):
        width = rng.choice([448, 832, 1024, 1664, 2048, 4096, _log(rng, 33, 12000), 8 * _log(rng, 8, 1200)])
        rows = max(1, min(rows, 16384 * 1024 // width))
        if kind == "norm_grad":
            return _norm_grad(rows, width, dy=rng.choice(["bf16", "bf16", "fp32"]), s=rng.choice(["bf16", "fp32"]),
                              stream=rng.random() < 0.7)
        out = rng.choice(["bf16", "bf16", "fp32", "e4m3", "e4m3"])
        return _norm(rows, width, x=rng.choice(["bf16", "bf16", "fp32"]), residual=rng.choice(["none", "bf16", "fp32"]),
                     out=out, block=128 if out == "e4m3" and rng.random() < 0.5 else 0)
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    share = 16 if dtype == "fp32" else 1
    k = rng.choice([448, 832, 1024, 1024, 1664, 2048, _log(rng, 33, 2500), 8 * _log(rng, 8, 300)])
    if kind.startswith("gated"):
        n = rng.choice([832, 1024, 1934, 2048, 4096, 4096, _log(rng, 33, 5000), 8 * _log(rng, 8, 600)])
        rows = max(1, min(rows, 16384 * 1024 * 4096 // share // (k * n)))
        return _gated(kind, rows, k, n, dtype=dtype, act=rng.choice(["silu", "silu", "gelu", "none"]),
                      bias=rng.random() < 0.4, keep=kind == "gated" and rng.random() < 0.5)
    k = min(k, 2048)
    n = rng.choice([32768, 50257, _log(rng, 1000, 131072), _log(rng, 1000, 131072), 64 * _log(rng, 16, 2048)])
    rows = max(1, min(rows, 4096 * 832 * 32003 // share // (k * n)))
    return _logprobs(rows, k, n, dtype=dtype, top=rng.choice([0, 1, 2, 5, 8, 16]), given=rng.random() < 0.7,
                     exclude=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=g.device, dtype=torch.float32)


def _stream(M, N, g):
    """A residual stream: tokens of different size, and a few channels far larger than the others."""
    size = 1.0 + 3.0 * torch.rand((M, 1), generator=g, device=g.device)
    large = torch.where(torch.rand((N,), generator=g, device=g.device) < 0.01, 20.0, 1.0)
    return _randn((M, N), g) * size * large


def _grid(v, step, most):
    """Multiples of `step` up to 255 of them: bf16 holds them, and sums of their products are exact in fp32 whatever
    their order, so that which of two tokens is the more probable does not hang on it."""
    return (v / step).round().clamp(-most, most) * step


def prepare(case, seed):
    g = torch.Generator(device="cuda" if torch.cuda.is_available() else "cpu")
    g.manual_seed(int(seed))
    kind, M = case["kind"], case["rows"]
    s = {"case": case}
    if kind.startswith("norm"):
        N = case["width"]
        s["w"] = 1.0 + 0.1 * _randn((N,), g)
        if kind == "norm":
            stream = _stream(M, N, g)
            if case["residual"] == "none":
                s["x"], s["residual"] = stream.to(TYPES[case["x"]]), None
            else:
                s["x"], s["residual"] = _randn((M, N), g).to(TYPES[case["x"]]), stream.to(TYPES[case["residual"]])
        else:
            s["s"] = _stream(M, N, g).to(TYPES[case["s"]])
            s["dy"] = (_randn((M, N), g) / M).to(TYPES[case["dy"]])
            s["dsum"] = (_randn((M, N), g) / M).to(TYPES[case["s"]]) if case["stream"] else None
        return s
    K, N, ty = case["k"], case["n"], TYPES[case["dtype"]]
    if kind == "logprobs":
        s["w"] = _grid(_randn((N, K), g) / math.sqrt(K), 2.0 ** -10, 255).to(ty)
        # a head that knows something: each row leans towards one token, by a margin of its own
        lean = torch.randint(0, N - 1, (M,), generator=g, device=g.device)
        by = 4.0 + 10.0 * torch.rand((M, 1), generator=g, device=g.device)
        s["x"] = _grid(_randn((M, K), g) + by * s["w"][lean].float(), 2.0 ** -4, 127).to(ty)
        s["exclude"] = N - 1 if case["exclude"] else -1
        s["tokens"] = None
        if case["given"]:
            # most of the given tokens are the ones that the rows lean to; a few are padding
            u = torch.rand((M,), generator=g, device=g.device)
            other = torch.randint(0, N - 1, (M,), generator=g, device=g.device)
            s["tokens"] = torch.where(u < 0.05, torch.full_like(lean, -100), torch.where(u < 0.4, other, lean))
        return s
    # normalised activations, weights that keep their scale
    s["x"] = _randn((M, K), g).to(ty)
    s["wg"] = (_randn((N, K), g) / math.sqrt(K)).to(ty)
    s["wu"] = (_randn((N, K), g) / math.sqrt(K)).to(ty)
    s["bg"] = 0.1 * _randn((N,), g) if case["bias"] else None
    s["bu"] = 0.1 * _randn((N,), g) if case["bias"] else None
    if kind == "gated_grad":
        s["dh"] = (_randn((M, N), g) / M).to(ty)
        s["pre"] = (_randn((M, N), g).to(ty), _randn((M, N), g).to(ty))
    return s


# ------------------------------------------------------------------ the plain form
def _act(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return z


def _act_grad(z, act):
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    return torch.ones_like(z)


def _blocks(v, block):
    """[rows, width] as [rows, blocks, columns], zeros past the width."""
    if block == 0:
        return v[:, None]
    M, N = v.shape
    n = (N + block - 1) // block
    full = torch.zeros((M, n * block), dtype=v.dtype, device=v.device)
    full[:, :N] = v
    return full.view(M, n, block)


def _plain_norm(s):
    case, x, w = s["case"], s["x"].float(), s["w"]
    r = s["residual"]
    v = x if r is None else x + r.float()
    y = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * w
    total = None if r is None else v.to(r.dtype)
    if case["out"] != "e4m3":
        return y.to(TYPES[case["out"]]), total
    y = _blocks(y, case["block"])
    top = y.abs().amax(2, keepdim=True)
    scale = torch.where(top > 0, top / E4M3_MAX, torch.ones_like(top))
    q = (y / scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    q = q.reshape(case["rows"], -1)[:, :case["width"]]
    return q, scale[:, :, 0], total


def _plain_norm_grad(s):
    v, dy, w = s["s"].float(), s["dy"].float(), s["w"]
    rstd = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    n, dn = v * rstd, dy * w
    ds = rstd * (dn - n * (n * dn).mean(1, keepdim=True))
    if s["dsum"] is not None:
        ds = ds + s["dsum"].float()
    return ds.to(s["s"].dtype), (dy * n).sum(0)


def _plain_gated(s):
    case, x, ty = s["case"], s["x"].float(), s["x"].dtype
    wg, wu = s["wg"].float(), s["wu"].float()
    if case["kind"] == "gated_grad":
        gate, up = s["pre"][0].float(), s["pre"][1].float()
        dh = s["dh"].float()
        dg, du = dh * up * _act_grad(gate, case["act"]), dh * _act(gate, case["act"])
        dx = dg @ wg + du @ wu
        db = (dg.sum(0), du.sum(0)) if case["bias"] else (None, None)
        return (dx.to(ty), (dg.t() @ x).to(ty), (du.t() @ x).to(ty), *db)
    gate, up = x @ wg.t(), x @ wu.t()
    if case["bias"]:
        gate, up = gate + s["bg"], up + s["bu"]
    h = (_act(gate, case["act"]) * up).to(ty)
    return (h, gate.to(ty), up.to(ty)) if case["keep"] else h


def _plain_logprobs(s):
    case = s["case"]
    logits = s["x"].float() @ s["w"].float().t() + 0.0
    if s["exclude"] >= 0:
        logits[:, s["exclude"]] = -math.inf
    if case["top"] == 0:
        token = logits.max(1, keepdim=True).indices
    else:
        # values in order as whole numbers, and behind them the column from the last to the first
        bits = logits.view(torch.int32)
        last = case["n"] - 1
        at = torch.arange(case["n"], device=logits.device)
        key = (bits ^ ((bits >> 31) & 0x7fffffff)).to(torch.int64) << 32 | (last - at)
        token = last - (key.topk(case["top"], 1).values & 0xffffffff)
    d = logits - logits.gather(1, token[:, :1])
    # the top token's 1 is kept apart: a log-probability near 0 is the others' sum
    e = torch.exp(d).scatter(1, token[:, :1], 0.0)
    others = e.sum(1, keepdim=True)
    rest = torch.log1p(others)
    slope = torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True)
    entropy = (rest - slope / (1 + others))[:, 0]
    logprob = None
    if s["tokens"] is not None:
        given = s["tokens"] >= 0
        logprob = torch.where(given, (d.gather(1, s["tokens"].clamp(min=0)[:, None]) - rest)[:, 0], 0.0)
    if case["top"] == 0:
        return logprob, entropy, None, None
    return logprob, entropy, token, d.gather(1, token) - rest


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "logprobs": _plain_logprobs}
        return plain.get(kind, _plain_gated)(s)
    import paper_2607_02805_amd as bd
    if kind == "norm":
        out, total, scale = bd.add_rmsnorm(s["x"], s["w"], s["residual"], eps=EPS, scale_block=case["block"],
                                           out_dtype=torch.float8_e4m3fn if case["out"] == "e4m3" else TYPES[case["out"]])
        return (out, scale, total) if case["out"] == "e4m3" else (out, total)
    if kind == "norm_grad":
        return bd.add_rmsnorm_backward(s["dy"], s["s"], s["w"], s["dsum"], eps=EPS)
    if kind == "gated":
        got = bd.gated_projection(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=case["act"],
                                  pre=True if case["keep"] else None)
        return (got[0], *got[1]) if case["keep"] else got
    if kind == "gated_grad":
        db = True if case["bias"] else None
        return bd.gated_projection_backward(s["dh"], s["x"], s["wg"], s["wu"], s["pre"], act=case["act"], dbg=db, dbu=db)
    return bd.head_logprobs(s["x"], s["w"], s["tokens"], top=case["top"], exclude=s["exclude"])


# ------------------------------------------------------------------ what a pass needs
SIZE = {"none": 0, "e4m3": 1, "bf16": 2, "fp32": 4}


def work(case):
    kind, M = case["kind"], case["rows"]
    if kind == "norm":
        N = case["width"]
        scales = 0 if case["out"] != "e4m3" else (N + 127) // 128 if case["block"] else 1
        return {"bytes": M * N * (SIZE[case["x"]] + 2 * SIZE[case["residual"]] + SIZE[case["out"]]) + 4 * N + 4 * M * scales,
                "flops": 6 * M * N}
    if kind == "norm_grad":
        N = case["width"]
        return {"bytes": M * N * (SIZE[case["dy"]] + SIZE[case["s"]] * (2 + case["stream"])) + 8 * N, "flops": 14 * M * N}
    K, N, e = case["k"], case["n"], SIZE[case["dtype"]]
    if kind == "gated":
        return {"bytes": e * (M * K + 2 * N * K + M * N * (3 if case["keep"] else 1)) + 8 * N * case["bias"],
                "flops": 4 * M * N * K}
    if kind == "gated_grad":
        return {"bytes": e * (2 * M * K + 4 * N * K + 3 * M * N) + 8 * N * case["bias"], "flops": 8 * M * N * K}
    return {"bytes": e * (M * K + N * K) + M * (4 + 12 * case["given"] + 12 * case["top"]), "flops": 2 * M * N * K}


# ------------------------------------------------------------------ in 64 bits
def _value64(z, act):
    return z * torch.sigmoid(z) if act == "silu" else z * torch.special.ndtr(z) if act == "gelu" else z


def _derivative64(z, act):
    if act == "silu":
        return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) * 0.3989422804014326779
    return torch.ones_like(z)


def _exact_norm(s):
    case, w = s["case"], s["w"].double()
    v = s["x"].double() if s["residual"] is None else s["x"].double() + s["residual"].double()
    total = None if s["residual"] is None else v
    y = w * v * torch.rsqrt(v.square().sum(1, keepdim=True) / case["width"] + EPS)
    if case["out"] != "e4m3":
        return y, total
    step = case["block"] or case["width"]
    scale = torch.stack([c.abs().max(1).values for c in y.split(step, 1)], 1) / E4M3_MAX
    scale = torch.where(scale > 0, scale, 1.0)
    return y / scale.repeat_interleave(step, 1)[:, :case["width"]], scale, total


def _exact_norm_grad(s):
    # of sum(dy * w * v * q), q = (mean v^2 + eps)^-1/2: by v directly, and through q
    v, dy, w = s["s"].double(), s["dy"].double(), s["w"].double()
    q = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    through = -(dy * w * v).sum(1, keepdim=True) * q.pow(3) / v.shape[1]
    ds = dy * w * q + through * v
    return (ds if s["dsum"] is None else ds + s["dsum"].double()), torch.einsum("ij,ij,ik->j", dy, v, q)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(s)
    if kind == "norm_grad":
        return _exact_norm_grad(s)
    x = s["x"].double()
    if kind == "gated":
        z = torch.mm(x, torch.cat([s["wg"], s["wu"]]).double().t().contiguous())
        if case["bias"]:
            z += torch.cat([s["bg"], s["bu"]]).double()
        gate, up = z.chunk(2, 1)
        h = _value64(gate, case["act"]) * up
        return (h, gate, up) if case["keep"] else h
    if kind == "gated_grad":
        gate, up, dh = s["pre"][0].double(), s["pre"][1].double(), s["dh"].double()
        dz = torch.cat([dh * up * _derivative64(gate, case["act"]), dh * _value64(gate, case["act"])], 1)
        dw = torch.mm(dz.t().contiguous(), x).chunk(2)
        db = dz.sum(0).chunk(2) if case["bias"] else (None, None)
        return torch.mm(dz, torch.cat([s["wg"], s["wu"]]).double()), *dw, *db
    w, got = s["w"].double().t().contiguous(), []
    step = max(1, (1 << 28) // case["n"])     # rows at a time
    for r in range(0, case["rows"], step):
        logp = torch.mm(x[r:r + step], w)
        if s["exclude"] >= 0:
            logp[:, s["exclude"]] = -math.inf
        logp -= torch.logsumexp(logp, 1, keepdim=True)
        entropy = torch.special.entr(logp.exp()).sum(1)
        given = None
        if s["tokens"] is not None:
            t = s["tokens"][r:r + step]
            given = torch.where(t >= 0, logp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        got.append((given, entropy, logp.topk(case["top"], 1).values if case["top"] else None))
    given, entropy, top = ([p for p in part if p is not None] for part in zip(*got))
    return (torch.cat(given) if given else None, torch.cat(entropy), None, torch.cat(top) if top else None)
