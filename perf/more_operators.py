"""What stands before, between and behind the layers of libtng's simulated workers, as measurable cases: embedding tables and their
gradients, root-mean-square norms with a residual into 8-bit codes, and the orthogonalised update of a matrix.

A case is a dict of plain values.  kind:
  "embed"       tokens to rows of a table, times a scale (lowbit.embed)
  "embed_step"  the same, and from the gradient of its result the table's, one for each worker (lowbit.embed_grad)
  "norm"        h = x + residual, and the rows of h normalised, in x's type or in 8-bit codes (lowbit.rms_norm, rms_norm_codes)
  "norm_step"   the same, and from the gradient of its result, and the one that comes along the residual, those of x and the weights
                (lowbit.rms_norm_grad)
  "update"      matrices orthogonalised by five products' polynomials (update.orthogonalize)

Formulas:
  embed:   y[m][t] = scale table[id[m][t]]; a token outside the table (padding) is a row of zeros and has no gradient
           dtable[m][v] = scale sum of dy[m][t] over the t with id[m][t] = v
  norm:    h = x + residual, rounded to x's type; s = 1 / sqrt(mean h^2 + eps); y = h s w
           coded: R = max |y| of the row, t = clamp(y (1 / R), -1, 1) 127 rounded to nearest even; value R / 127 code
           dx = s (w dy - h s^2 mean(w dy h)) + dresidual; dw[m] = sum of dy h s over a worker's rows
  update:  X = x / (||x|| + eps); five times A = X X^T, X = a X + (b A + c A A) X; y = scale X
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
TINY = 2.0 ** -126
NORM_EPS, UPDATE_EPS = 1e-6, 1e-7
QUINTIC = (3.4445, -4.775, 2.0315)  # a, b, c of the Muon optimiser's polynomial
STEPS = 5


def listed():
    return [
        # a minibatch of the smallest token networks: launches and latency
        dict(name="embed_step_small", kind="embed_step", M=4, T=33, V=1000, C=256, table="f32", type="f32", ids="zipf"),
        # four workers, 2048 tokens each, a vocabulary of 32000: the gradient's 1 GB
        dict(name="embed_step_large", kind="embed_step", M=4, T=2048, V=32000, C=2048, table="f32", type="bf16", ids="zipf"),
        # padded batches of odd sizes with one token that is most of the rest: long sums of one row
        dict(name="embed_step_padded", kind="embed_step", M=3, T=20011, V=4099, C=1003, table="f32", type="f16", ids="padded"),
        # a long prompt's rows
        dict(name="embed_prompt", kind="embed", M=1, T=32768, V=50000, C=4096, table="bf16", type="bf16", ids="zipf"),
        # a sequence asks for one token: latency
        dict(name="norm_token", kind="norm", M=1, T=1, C=4096, type="bf16", codes=True, residual=True),
        # a prompt on the way into a layer of 8-bit codes
        dict(name="norm_prompt", kind="norm", M=1, T=8192, C=4096, type="bf16", codes=True, residual=True),
        # a training step of four workers
        dict(name="norm_step", kind="norm_step", M=4, T=2048, C=4096, type="bf16", codes=True, residual=True),
        # a small one of odd sizes
        dict(name="norm_step_odd", kind="norm_step", M=3, T=111, C=1003, type="f32", codes=False, residual=True),
        # rows that no wavefront holds
        dict(name="norm_step_wide", kind="norm_step", M=1, T=1537, C=20011, type="f16", codes=False, residual=False),
        # the smallest matrices of a network, together
        dict(name="update_small", kind="update", M=16, R=64, C=256, type="f32"),
        # tall matrices that no tile divides
        dict(name="update_ragged", kind="update", M=4, R=2053, C=1003, type="bf16"),
        # the largest matrix
        dict(name="update_large", kind="update", M=1, R=4096, C=4096, type="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi, unit=160):
    """Any length, or (half of the time) a multiple of `unit` where the length allows it."""
    n = _log_int(rng, lo, hi)
    return n // unit * unit if n >= unit and rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(["embed", "embed_step", "norm", "norm_step", "update"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind in ("embed", "embed_step"):
        M, C = _log_int(rng, 1, 8), _size(rng, 64, 8192)
        V = max(16, min(_size(rng, 64, 65536), (1 << 28) // ((M if kind == "embed_step" else 1) * C)))
        T = max(1, min(_size(rng, 1, 32768), (1 << 26) // (M * C)))
        return dict(kind=kind, M=M, T=T, V=V, C=C, table=rng.choice(["f32", dtype]), type=dtype, ids=rng.choice(["zipf", "zipf", "even", "padded"]))
    if kind in ("norm", "norm_step"):
        M, C = _log_int(rng, 1, 8), _size(rng, 64, 20000)
        T = max(1, min(_size(rng, 1, 8192), (1 << 25) // (M * C)))
        return dict(kind=kind, M=M, T=T, C=C, type=dtype, codes=dtype != "f32" and rng.random() < 0.6, residual=rng.random() < 0.7)
    R, C = _size(rng, 32, 4096), _size(rng, 32, 4096)
    n = min(R, C)
    M = max(1, min(_log_int(rng, 1, 16), 4 * 4096 ** 3 // (3 * n * R * C + n ** 3)))
    return dict(kind=kind, M=M, R=R, C=C, type=dtype)


# ---- inputs

def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device=DEVICE)


def _activations(gen, *shape):
    """Normal numbers with a few channels that are much larger than the rest, as hidden states have them."""
    return _randn(gen, *shape) * torch.exp(0.75 * _randn(gen, shape[-1]))


def _tokens(gen, M, T, V, ids):
    """Tokens as text has them ("zipf": the chance of the k-th most frequent falls as 1 / k), evenly drawn, or in batches whose ends are padding
    (-1) and half of whose tokens are one."""
    u = torch.rand((M, T), generator=gen, device=DEVICE, dtype=torch.float64)
    if ids == "even":
        return (u * V).long().clamp(max=V - 1)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1).long().clamp(0, V - 1)
    out = torch.randperm(V, generator=gen, device=DEVICE)[rank]
    if ids == "padded":
        out = torch.where(torch.rand((M, T), generator=gen, device=DEVICE) < 0.5, V // 2, out)
        ends = (T * (0.75 + 0.25 * torch.rand((M, 1), generator=gen, device=DEVICE))).ceil()
        out = torch.where(torch.arange(T, device=DEVICE) < ends, out, -1)
    return out


def prepare(case, seed):
    gen, kind, dtype = _gen(seed), case["kind"], TYPES[case["type"]]
    st = dict(kind=kind, type=dtype)
    if kind in ("embed", "embed_step"):
        M, T, V, C = (case[k] for k in "MTVC")
        st.update(ids=_tokens(gen, M, T, V, case["ids"]), table=(_randn(gen, V, C) / math.sqrt(C)).to(TYPES[case["table"]]), scale=math.sqrt(C))
        if kind == "embed_step":
            st["dy"] = (1e-2 * _randn(gen, M, T, C)).to(dtype)
    elif kind in ("norm", "norm_step"):
        shape = tuple(case[k] for k in "MTC")
        st.update(codes=case["codes"], x=_activations(gen, *shape).to(dtype), residual=None, weight=1 + 0.2 * _randn(gen, shape[-1]))
        if case["residual"]:
            st["residual"] = _activations(gen, *shape).to(dtype)
        if kind == "norm_step":
            st["dy"] = (1e-2 * _randn(gen, *shape)).to(dtype)
            st["dresidual"] = (1e-2 * _randn(gen, *shape)).to(dtype) if case["residual"] else None
    else:
        # the average of gradients: a few directions that all samples share, and noise
        M, R, C = case["M"], case["R"], case["C"]
        few = min(8, R, C)
        x = torch.bmm(_randn(gen, M, R, few), _randn(gen, M, few, C)) / math.sqrt(few) + _randn(gen, M, R, C)
        st["x"] = (1e-3 * x).to(dtype)
    return st


# ---- the plain form

def _plain_embed(st):
    ids, table = st["ids"], st["table"]
    V, C = table.shape
    inside = ((ids >= 0) & (ids < V))[..., None]
    at = ids.clamp(0, V - 1)
    y = (torch.where(inside, table[at].float(), 0.0) * st["scale"]).to(st["type"])
    if st["kind"] == "embed":
        return y
    M = ids.shape[0]
    rows = (at + V * torch.arange(M, device=DEVICE)[:, None]).view(-1)
    dtable = torch.zeros((M * V, C), device=DEVICE).index_add_(0, rows, torch.where(inside, st["dy"].float(), 0.0).view(-1, C))
    return {"y": y, "dtable": (dtable * st["scale"]).view(M, V, C)}


def _plain_norm(st):
    x, w = st["x"].float(), st["weight"]
    h = x if st["residual"] is None else (x + st["residual"].float()).to(st["type"]).float()
    s = 1.0 / torch.sqrt((h * h).mean(-1, keepdim=True) + NORM_EPS)
    y = h * s * w
    if st["codes"]:
        r = y.abs().amax(-1, keepdim=True)
        r = torch.where(r < TINY, 0.0, r)
        y = torch.round((y * torch.where(r > 0, 1.0 / r, 0.0)).clamp(-1, 1) * 127) * (r / 127)
    out = {"y": y.to(st["type"])}
    if st["residual"] is not None:
        out["h"] = h.to(st["type"])
    if st["kind"] == "norm":
        return out
    dy = st["dy"].float()
    g = dy * w
    dx = s * (g - h * (s * s * (g * h).mean(-1, keepdim=True)))
    if st["dresidual"] is not None:
        dx = dx + st["dresidual"].float()
    out.update(dx=dx.to(st["type"]), dw=(dy * h * s).sum(1))
    return out


def _update_scale(st):
    return max(1.0, st["x"].shape[1] / st["x"].shape[2]) ** 0.5


def _plain_update(st):
    x = st["x"].float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x.double() ** 2).sum((1, 2), keepdim=True)) + UPDATE_EPS).float()
    a, b, c = QUINTIC
    for _ in range(STEPS):
        gram = torch.matmul(x, x.transpose(1, 2))
        x = a * x + torch.matmul(b * gram + c * torch.matmul(gram, gram), x)
    x = _update_scale(st) * x
    return (x.transpose(1, 2).contiguous() if tall else x).to(st["type"])


# ---- a pass

def _run_norm(lowbit, st):
    x, w, r = st["x"], st["weight"], st["residual"]
    out = {}
    if st["codes"]:
        n = lowbit.rms_norm_codes(x, w, residual=r, eps=NORM_EPS)
        out["y"] = torch.mul(n.q, n.scale[..., None], out=torch.empty_like(x))  # (the values that the codes stand for)
        h = n.h
    elif r is not None:
        out["y"], h = lowbit.rms_norm(x, w, residual=r, eps=NORM_EPS)
    else:
        out["y"], h = lowbit.rms_norm(x, w, eps=NORM_EPS), x
    if r is not None:
        out["h"] = h
    if st["kind"] == "norm_step":
        out["dx"], out["dw"] = lowbit.rms_norm_grad(st["dy"], h, w, dresidual=st["dresidual"], eps=NORM_EPS)
    return out


def run(st):
    kind = st["kind"]
    if not own:
        return (_plain_embed if kind in ("embed", "embed_step") else _plain_norm if kind in ("norm", "norm_step") else _plain_update)(st)
    from paper_1901_08227_amd import lowbit, update

    if kind in ("norm", "norm_step"):
        return _run_norm(lowbit, st)
    if kind == "update":
        return update.orthogonalize(st["x"], coefficients=(QUINTIC,) * STEPS, eps=UPDATE_EPS, scale=_update_scale(st))
    y = lowbit.embed(st["ids"], st["table"], scale=st["scale"], dtype=st["type"])
    if kind == "embed":
        return y
    return {"y": y, "dtable": lowbit.embed_grad(st["ids"], st["dy"], st["table"].shape[0], scale=st["scale"])}


def work(case):
    size = SIZE[case["type"]]
    if case["kind"] in ("embed", "embed_step"):
        M, T, V, C = (case[k] for k in "MTVC")
        # rows of the table that are asked for (of drawn tokens: a chance of 1 / (k ln V) for the k-th), the tokens, the result
        hits = M * T if case["ids"] != "padded" else M * T // 2
        if case["ids"] == "even":
            read = V * (1 - (1 - 1 / V) ** hits)
        else:
            edge = hits / math.log(V + 1)
            read = min(V, hits, edge * (1 + max(0.0, math.log(V / max(1.0, edge)))))
        n = read * C * SIZE[case["table"]] + 8 * M * T + M * T * C * size
        if case["kind"] == "embed":
            return {"bytes": int(n), "flops": M * T * C}
        return {"bytes": int(n + M * T * C * size + 4 * M * V * C), "flops": 3 * M * T * C}
    if case["kind"] in ("norm", "norm_step"):
        n = case["M"] * case["T"] * case["C"]
        moved = n * (size * (3 if case["residual"] else 1) + (1 if case["codes"] else size))
        if case["kind"] == "norm":
            return {"bytes": moved, "flops": 6 * n}
        return {"bytes": moved + n * size * (4 if case["residual"] else 3) + 4 * case["C"] * (case["M"] + 1), "flops": 18 * n}
    M, R, C = case["M"], case["R"], case["C"]
    n, m = min(R, C), max(R, C)
    return {"bytes": 2 * M * R * C * size, "flops": M * STEPS * (3 * n * n * m + n ** 3)}


# ---- 64 bits

def _exact_embed(case, st):
    M, T, V, C = (case[k] for k in "MTVC")
    ids, table, y = st["ids"], st["table"].double(), torch.zeros((M, T, C), dtype=torch.float64, device=DEVICE)
    dtable = torch.zeros((M, V, C), dtype=torch.float64, device=DEVICE) if case["kind"] == "embed_step" else None
    for m in range(M):
        t = torch.nonzero((ids[m] >= 0) & (ids[m] < V)).view(-1)
        y[m, t] = table[ids[m, t]] * st["scale"]
        if dtable is not None:
            dtable[m].index_put_((ids[m, t],), st["dy"][m, t].double() * st["scale"], accumulate=True)
    return y if dtable is None else {"y": y, "dtable": dtable}


def _exact_norm(case, st):
    h, w = st["x"].double(), st["weight"].double()
    if case["residual"]:
        h = (st["x"].float() + st["residual"].float()).to(st["type"]).double()  # (h's rounding is part of the definition)
    mean_square = torch.linalg.vector_norm(h, dim=-1, keepdim=True) ** 2 / case["C"]
    unit = h * torch.rsqrt(mean_square + NORM_EPS)
    out = {"y": unit * w}
    if case["codes"]:
        step = out["y"].abs().amax(-1, keepdim=True) / 127
        out["y"] = torch.round(out["y"] / step).clamp(-127, 127) * step
    if case["residual"]:
        out["h"] = st["x"].double() + st["residual"].double()
    if case["kind"] == "norm_step":
        g = st["dy"].double() * w
        dx = torch.rsqrt(mean_square + NORM_EPS) * (g - unit * (g * unit).sum(-1, keepdim=True) / case["C"])
        out["dx"] = dx + st["dresidual"].double() if case["residual"] else dx
        out["dw"] = torch.stack([(st["dy"][m].double() * unit[m]).sum(0) for m in range(case["M"])])
    return out


def _exact_update(st):
    out = []
    for x in st["x"]:
        wide = x.shape[0] <= x.shape[1]
        v = x.double() if wide else x.double().t()
        v = v / (torch.linalg.matrix_norm(v) + UPDATE_EPS)
        for _ in range(STEPS):
            gram = v @ v.t()
            p = QUINTIC[0] * torch.eye(len(v), dtype=torch.float64, device=DEVICE) + QUINTIC[1] * gram + QUINTIC[2] * (gram @ gram)
            v = p @ v
        out.append((v if wide else v.t()) * _update_scale(st))
    return torch.stack(out)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("embed", "embed_step"):
        return _exact_embed(case, st)
    return _exact_norm(case, st) if case["kind"] in ("norm", "norm_step") else _exact_update(st)
