"""The dense work around the scan, as cases that can be timed and checked.

A case is one pass through an operator as a program makes it: a projection of a Mamba-H layer
(the mixer's input and output projections, the MLP's two products) with its bias, activation
and residual; its gradient; the language-model head of a denoising step, which picks a token
and says how sure it is; and the masked training loss over the vocabulary with its gradient.

Widths are those of the layers that the rest of the benchmark runs (d_model 1024 with d_inner
2048, the paper's 448 and 832 with 896 and 1664) and odd ones between them; vocabularies are
generic sizes of 1,000 to 131,072.  Activations and weights are bf16 or fp32, bias fp32.

Row counts: a single token; a denoising step of 16 rows of 32 tokens; the paper's blocks of
256 tokens; training windows of up to 16,384 tokens.
"""
import math

import torch

own = False   # False: the plain form in torch operations; True: this library's kernels

MASKED = -100     # a label that leaves its row out of the loss


def _case(kind, rows, k, n, *, dtype="bf16", act="none", bias=False, residual=False, keep=False,
          exclude=False, out=0.0, **name):
    return dict(kind=kind, rows=rows, k=k, n=n, dtype=dtype, act=act, bias=bias, residual=residual,
                keep=keep, exclude=exclude, out=out, **name)


def listed():
    return [
        # the smallest call: one token through a small fp32 projection, launch and host latency
        _case("project", 1, 256, 512, dtype="fp32", act="silu", bias=True, name="project_tiny_fp32"),
        # one token through the mixer's input projection (z, x, B, C, dt of the 350M layer):
        # the weights' bytes are the whole of it
        _case("project", 1, 1024, 4384, name="project_in_token"),
        # the same for a denoising step of 16 sequences with blocks of 32 tokens
        _case("project", 512, 1024, 4384, name="project_in_step"),
        # the mixer's output projection at the paper's width and block length, adding onto the
        # residual stream
        _case("project", 4096, 1664, 832, residual=True, name="project_out_paper"),
        # the MLP's first product in training: bias and GELU, the pre-activation kept
        _case("project", 16384, 1024, 4096, act="gelu", bias=True, keep=True, name="project_mlp_train"),
        # its gradient: input, weights and bias
        _case("project_grad", 16384, 1024, 4096, act="gelu", bias=True, name="project_grad_mlp"),
        # a ragged fp32 gradient at the paper's small width
        _case("project_grad", 1003, 448, 1934, dtype="fp32", act="silu", bias=True,
              name="project_grad_fp32"),
        # the head for one token
        _case("select", 1, 1024, 32768, name="select_token"),
        # the head of a denoising step: every position's most probable token, the mask token
        # ruled out
        _case("select", 512, 1024, 50257, exclude=True, name="select_step"),
        # perplexity of held-out text at the paper's width in fp32: the loss alone
        _case("loss", 1500, 832, 16001, dtype="fp32", name="loss_eval_fp32"),
        # the training loss of a ragged batch with its gradient
        _case("loss_grad", 777, 832, 32003, exclude=True, out=0.3, name="loss_grad_ragged"),
        # the masked objective of a training window: half of the tokens are clean and left out
        _case("loss_grad", 8192, 1024, 50257, exclude=True, out=0.5, name="loss_grad_train"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """One more case: the kinds and ranges of the listed ones."""
    kind = rng.choice(["project", "project", "project", "project_grad", "project_grad", "select",
                       "select", "loss", "loss_grad", "loss_grad"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    share = 16 if dtype == "fp32" else 1
    rows = rng.choice([_log(rng, 1, 16384), _log(rng, 1, 16384), _log(rng, 1, 64),
                       min(16384, rng.randint(1, 128) * rng.choice([16, 32, 64, 256]))])
    k = rng.choice([448, 832, 896, 1024, 1024, 1664, 2048, 4096, _log(rng, 33, 2500), 8 * _log(rng, 8, 400)])
    if kind.startswith("project"):
        n = rng.choice([448, 832, 1024, 1934, 3610, 4096, 4384, _log(rng, 33, 5000), 8 * _log(rng, 8, 600)])
        rows = max(1, min(rows, 16384 * 1024 * 4096 // share // (k * n)))
        act = rng.choice(["none", "none", "silu", "gelu"])
        return _case(kind, rows, k, n, dtype=dtype, act=act, bias=rng.random() < 0.5,
                     residual=kind == "project" and rng.random() < 0.4,
                     keep=kind == "project" and act != "none" and rng.random() < 0.5)
    k = min(k, 2048)
    n = rng.choice([32768, 50257, _log(rng, 1000, 131072), _log(rng, 1000, 131072), 64 * _log(rng, 16, 2048)])
    most = {"select": 512 * 1024 * 50257, "loss": 4096 * 1024 * 50257, "loss_grad": 8192 * 1024 * 50257}[kind]
    rows = max(1, min(rows, most // share // (k * n)))
    return _case(kind, rows, k, n, dtype=dtype, exclude=rng.random() < 0.5,
                 out=0.0 if kind == "select" else rng.choice([0.0, 0.15, 0.5, 0.85]))


# ------------------------------------------------------------------ inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=g.device, dtype=torch.float32)


def prepare(case, seed):
    g = torch.Generator(device="cuda" if torch.cuda.is_available() else "cpu")
    g.manual_seed(int(seed))
    M, K, N, ty = case["rows"], case["k"], case["n"], _dtype(case)
    # normalised activations, weights that keep their scale
    x = _randn((M, K), g)
    w = (_randn((N, K), g) / math.sqrt(K)).to(ty)
    s = {"case": case, "w": w}
    if case["kind"].startswith("project"):
        s["x"] = x.to(ty)
        s["bias"] = 0.1 * _randn((N,), g) if case["bias"] else None
        s["residual"] = _randn((M, N), g).to(ty) if case["residual"] else None
        if case["kind"] == "project_grad":
            s["dy"] = (_randn((M, N), g) / M).to(ty)
            s["pre"] = _randn((M, N), g).to(ty) if case["act"] != "none" else None
        return s
    # a head that knows something: each row leans towards one token, by a margin of its own
    lean = torch.randint(0, N, (M,), generator=g, device=g.device)
    s["exclude"] = N - 1 if case["exclude"] else -1
    if case["exclude"]:
        lean = lean % (N - 1)
    by = 8.0 + 8.0 * torch.rand((M, 1), generator=g, device=g.device)
    if case["kind"] != "select":
        by = by * 0.6
    s["x"] = (x + by * w[lean].float()).to(ty)
    if case["kind"] != "select":
        out = torch.rand((M,), generator=g, device=g.device) < case["out"]
        s["labels"] = torch.where(out, torch.full_like(lean, MASKED), lean)
        # the weight of a block noised at time t is 1 / t, over the tokens of the window
        s["dloss"] = 1.0 / (0.1 + 0.9 * torch.rand((M,), generator=g, device=g.device)) / M
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


def _logits(s):
    logits = s["x"].float() @ s["w"].float().t()
    if s["exclude"] >= 0:
        logits[:, s["exclude"]] = -math.inf
    return logits


def _plain(s):
    case = s["case"]
    kind, x, w, ty = case["kind"], s["x"], s["w"], _dtype(case)
    if kind == "project":
        z = x.float() @ w.float().t()
        if s["bias"] is not None:
            z = z + s["bias"]
        out = _act(z, case["act"])
        if s["residual"] is not None:
            out = out + s["residual"].float()
        return (out.to(ty), z.to(ty)) if case["keep"] else out.to(ty)
    if kind == "project_grad":
        dz = s["dy"].float()
        if s["pre"] is not None:
            dz = dz * _act_grad(s["pre"].float(), case["act"])
        db = dz.sum(0) if case["bias"] else None
        return (dz @ w.float()).to(ty), (dz.t() @ x.float()).to(ty), db
    logits = _logits(s)
    top = logits.max(1, keepdim=True).values
    at = torch.arange(case["n"], device=x.device).expand_as(logits)
    token = torch.where(logits == top, at, case["n"]).min(1, keepdim=True).values
    e = torch.exp(logits - top)
    # the top token's 1 is kept apart: a log-probability near 0 is the others' sum
    others = e.scatter(1, token, 0.0).sum(1, keepdim=True)
    rest = torch.log1p(others)
    if kind == "select":
        return token[:, 0], -rest[:, 0]
    labels = s["labels"]
    counts = labels >= 0
    safe = labels.clamp(min=0)[:, None]
    zero = torch.zeros_like(rest[:, 0])
    loss = torch.where(counts, (rest + (top - logits.gather(1, safe)))[:, 0], zero)
    lse = torch.where(counts, (top + rest)[:, 0], zero)
    if kind == "loss":
        return loss, lse
    # probability less one of the label: minus the sum of the others
    p = (e / (1 + others)).scatter_(1, safe, 0.0)
    p.scatter_(1, safe, -p.sum(1, keepdim=True))
    p = p * torch.where(counts, s["dloss"], zero)[:, None]
    return loss, lse, (p @ w.float()).to(ty), (p.t() @ x.float()).to(ty)


# ------------------------------------------------------------------ one pass
def run(s):
    if not own:
        return _plain(s)
    import paper_2607_02805_amd as bd
    case = s["case"]
    kind, x, w, act = case["kind"], s["x"], s["w"], case["act"]
    if kind == "project":
        return bd.projection(x, w, s["bias"], act=act, residual=s["residual"],
                             pre=True if case["keep"] else None)
    if kind == "project_grad":
        return bd.projection_backward(s["dy"], x, w, pre=s["pre"], act=act,
                                      db=True if case["bias"] else None)
    if kind == "select":
        return bd.head_select(x, w, exclude=s["exclude"])
    loss, lse = bd.head_loss(x, w, s["labels"], exclude=s["exclude"])
    if kind == "loss":
        return loss, lse
    dx, dw = bd.head_loss_backward(s["dloss"], x, w, s["labels"], loss, lse,
                                   exclude=s["exclude"])
    return loss, lse, dx, dw


# ------------------------------------------------------------------ what a pass needs
def work(case):
    M, K, N, kind = case["rows"], case["k"], case["n"], case["kind"]
    e = 4 if case["dtype"] == "fp32" else 2
    if kind == "project":
        nbytes = e * (M * K + N * K + M * N * (1 + case["residual"] + case["keep"])) + 4 * N * case["bias"]
        return {"bytes": nbytes, "flops": 2 * M * N * K}
    if kind == "project_grad":
        nbytes = e * (2 * M * K + 2 * N * K + M * N * (1 + (case["act"] != "none"))) + 4 * N * case["bias"]
        return {"bytes": nbytes, "flops": 4 * M * N * K}
    if kind == "select":
        return {"bytes": e * (M * K + N * K) + 12 * M, "flops": 2 * M * N * K}
    rows = M * (1 - case["out"])     # the rows that count: the others' results are zeros
    if kind == "loss":
        return {"bytes": e * (rows * K + N * K) + 16 * M, "flops": 2 * rows * N * K}
    # the logits, then both products of the gradient
    return {"bytes": e * (rows * K + M * K + 2 * N * K) + 20 * M, "flops": 6 * rows * N * K}


# ------------------------------------------------------------------ in 64 bits
def _derivative64(z, act):
    """d act / dz from the definitions, in 64 bits."""
    if act == "silu":
        return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) * 0.3989422804014326779
    return torch.ones_like(z)


def _value64(z, act):
    return z * torch.sigmoid(z) if act == "silu" else z * torch.special.ndtr(z) if act == "gelu" else z


def exact(case, seed):
    s = prepare(case, seed)
    kind, x, w = case["kind"], s["x"].double(), s["w"].double()
    if kind == "project":
        z = torch.mm(x, w.t().contiguous())
        z = z if s["bias"] is None else z + s["bias"].double()
        out = _value64(z, case["act"])
        out = out if s["residual"] is None else out + s["residual"].double()
        return (out, z) if case["keep"] else out
    if kind == "project_grad":
        dz = s["dy"].double()
        dz = dz if s["pre"] is None else dz * _derivative64(s["pre"].double(), case["act"])
        return torch.mm(dz, w), torch.mm(dz.t().contiguous(), x), dz.sum(0) if case["bias"] else None
    allowed = torch.ones(case["n"], dtype=torch.bool, device=x.device)
    if s["exclude"] >= 0:
        allowed[s["exclude"]] = False
    losses, lses, dxs, picked = [], [], [], []
    dw = torch.zeros_like(w) if kind == "loss_grad" else None
    step = max(1, (1 << 28) // case["n"])     # rows at a time
    for r in range(0, case["rows"], step):
        xr = x[r:r + step]
        logp = torch.mm(xr, w.t().contiguous()).masked_fill_(~allowed, -math.inf)
        lse = torch.logsumexp(logp, 1)
        logp -= lse[:, None]
        if kind == "select":
            picked.append(logp.max(1).values)
            continue
        lab = s["labels"][r:r + step]
        keep = lab >= 0
        losses.append(torch.where(keep, -logp.gather(1, lab.clamp(min=0)[:, None])[:, 0], 0.0))
        lses.append(torch.where(keep, lse, 0.0))
        if kind == "loss_grad":
            p = logp.exp_()
            at = torch.arange(len(lab), device=x.device)[keep]
            p[at, lab[keep]] -= 1.0
            p *= torch.where(keep, s["dloss"][r:r + step].double(), 0.0)[:, None]
            dxs.append(torch.mm(p, w))
            dw += torch.mm(p.t().contiguous(), xr)
    if kind == "select":
        return None, torch.cat(picked)
    got = [torch.cat(losses), torch.cat(lses)]
    return tuple(got) if kind == "loss" else (*got, torch.cat(dxs), dw)
