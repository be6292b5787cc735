"""The gated feed-forward block and the norm of all gradients, as cases that can be timed and whose outputs can be compared.

  fwd    Y = (act(X Wg) * (X Wu)) Wd (ht_ffn_fwd)
  bwd    gradients of X and of the three weights; the projections are made again (ht_ffn_bwd)
  train  both, the backward pass with the projections that the forward pass kept
  norm   the norm of all gradients of a model together (ht_grad_norm)
  clip   the norm, and the gradients scaled so that it is at most max_norm (ht_grad_clip)

Values are fp32, as everywhere in the library.  Rows of X are N(0, 1), weights are such that the projections have a standard
deviation of 1.5 and 1, so that gates are open and closed; gradients of Y are small.  A model's gradients are the tensors of `layers`
blocks (a square matrix, the three weights of a gated block, two vectors), a table, and their magnitudes differ by orders.
"""
import math

import torch

own = False


def listed():
    return [
        # A single row, as a serving loop has it: reading the weights is all there is.
        dict(name="fwd_1", kind="fwd", n=1, d=1_024, f=4_096, e=1_024, act="silu", form="out_in"),
        # A few requests at a time, the weights of a narrower model.
        dict(name="fwd_24", kind="fwd", n=24, d=512, f=2_048, e=512, act="silu", form="in_out"),
        # Odd sizes all over, another width behind the block than before it.
        dict(name="fwd_odd", kind="fwd", n=1_003, d=301, f=1_213, e=172, act="gelu", form="in_out"),
        # Scoring a large batch with wide layers.
        dict(name="fwd_16k", kind="fwd", n=16_384, d=1_024, f=4_096, e=1_024, act="silu", form="in_out"),
        # The gradients of a handful of rows: those of the weights are nearly all that is written.
        dict(name="bwd_40", kind="bwd", n=40, d=256, f=1_024, e=256, act="silu", form="in_out"),
        # An ordinary training batch beside the layers that the library trains.
        dict(name="bwd_2k", kind="bwd", n=2_048, d=256, f=1_024, e=256, act="gelu_tanh", form="in_out"),
        # Every vertex of a full graph, behind a layer of 256 columns.
        dict(name="bwd_233k", kind="bwd", n=232_965, d=256, f=1_024, e=256, act="silu", form="in_out"),
        # The largest training batch, forward and backward.
        dict(name="train_8k", kind="train", n=8_192, d=1_024, f=4_096, e=1_024, act="silu", form="out_in"),
        # The gradients of two narrow layers: launches are all there is.
        dict(name="norm_small", kind="norm", layers=2, d=64, f=172, vocab=1_000, ratio=0.5),
        # Those of a deep model with a large table.
        dict(name="norm_460M", kind="norm", layers=24, d=1_024, f=4_096, vocab=131_072, ratio=0.5),
        # Many small tensors of odd sizes, clipped.
        dict(name="clip_odd", kind="clip", layers=40, d=99, f=301, vocab=5_003, ratio=0.3),
        # An ordinary model, clipped.
        dict(name="clip_100M", kind="clip", layers=12, d=768, f=2_048, vocab=50_003, ratio=0.7),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "bwd", "train", "norm", "clip"])
    if kind in ("norm", "clip"):
        layers, d, f = _log_uniform(rng, 1, 40), _log_uniform(rng, 16, 1_024), _log_uniform(rng, 32, 4_096)
        f = min(f, max(32, 300_000_000 // (3 * d * layers)))
        vocab = _log_uniform(rng, 100, 131_072)
        if kind == "clip":                                   # no more work than the largest listed case
            layers, vocab = min(layers, 12), min(vocab, 50_003)
            f = min(f, 2_048)
            d = min(d, 768)
        return dict(kind=kind, layers=layers, d=d, f=f, vocab=vocab, ratio=rng.choice([0.1, 0.5, 2.0]))
    d, f = _log_uniform(rng, 16, 1_024), _log_uniform(rng, 32, 4_096)
    e = d if rng.random() < 0.7 else _log_uniform(rng, 16, 1_024)
    most = {"fwd": 16_384 * 6, "bwd": 3_600 * 16, "train": 8_192 * 18}[kind] / {"fwd": 6, "bwd": 16, "train": 18}[kind] * 1_024 * 4_096
    rows = min(232_965, int(most / (max(d, e) * f)))
    return dict(kind=kind, n=_log_uniform(rng, 1, rows), d=d, f=f, e=e, act=rng.choice(["silu", "gelu", "gelu_tanh", "sigmoid"]),      # (relu's slope has a border)
                form=rng.choice(["in_out", "out_in"]))


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 23)
    return g


def _matrix(rows, cols):
    """Zeros of [rows x cols] whose rows start on 16 bytes, as the library wants its tensors."""
    return torch.zeros(rows, (cols + 3) // 4 * 4, device="cuda")


def _normal(rows, cols, g, std=1.0):
    m = _matrix(rows, cols)
    m[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * std
    return m


def _shapes(case):
    """A model's gradients: [rows x columns] of each; vectors are single rows."""
    d, f = case["d"], case["f"]
    shapes = [(case["vocab"], d)]
    for _ in range(case["layers"]):
        shapes += [(d, d), (d, f), (d, f), (f, d), (1, d), (1, d)]
    return shapes


def _flat(case, dtype=torch.float32):
    """Room for all gradients in one block, as programs keep them, and its parts as matrices whose rows start on 16 bytes."""
    shapes = [(rows, (cols + 3) // 4 * 4) for rows, cols in _shapes(case)]
    flat = torch.zeros(sum(rows * ld for rows, ld in shapes), dtype=dtype, device="cuda")
    return flat, [part.view(shape) for part, shape in zip(flat.split([rows * ld for rows, ld in shapes]), shapes)]


def _inputs(case, seed):
    g = _generator(seed)
    if case["kind"] in ("norm", "clip"):
        grads, total = [], 0.0
        for k, (rows, cols) in enumerate(_shapes(case)):
            std = 1e-2 * 10.0 ** (-3.0 * ((k * 7) % 11) / 10.0)
            t = _normal(rows, cols, g, std)
            share = 1.0
            if k == 0 and rows > 1_000:                      # of the table most rows' ids did not occur
                share = 0.25
                t *= (torch.rand(rows, 1, generator=g, device="cuda") < share)
            grads.append(t)
            total += rows * cols * share * std * std
        return {"grads": grads, "max_norm": case["ratio"] * math.sqrt(total)}
    n, d, f, e = case["n"], case["d"], case["f"], case["e"]
    x = {"X": _normal(n, d, g)}
    for name, rows, cols, std in (("Wg", d, f, 1.5 / math.sqrt(d)), ("Wu", d, f, 1.0 / math.sqrt(d)), ("Wd", f, e, 1.0 / math.sqrt(f))):
        x[name] = _normal(rows, cols, g, std) if case["form"] == "in_out" else _normal(cols, rows, g, std)
    if case["kind"] != "fwd":
        x["dY"] = _normal(n, e, g, 1e-3)
    return x


class State:
    def __init__(self, case):
        self.case = case
        self.ctx = None

    def __del__(self):
        if self.ctx is not None:
            self.B.ht_ctx_destroy(self.ctx)
            self.ctx = None


def prepare(case, seed):
    s = State(case)
    s.x = _inputs(case, seed)
    if case["kind"] == "clip":
        s.flat, s.out = _flat(case)
    if own:
        from paper_2311_14898_amd import binding as B
        s.B = B
        s.ctx = B.ht_ctx_create(0)
        if case["kind"] in ("norm", "clip"):
            s.norm = torch.zeros(1, device="cuda")
            s.cols = [cols for _, cols in _shapes(case)]
        else:
            n = case["n"]
            s.act = {"silu": B.HT_GATE_SILU, "gelu": B.HT_GATE_GELU, "gelu_tanh": B.HT_GATE_GELU_TANH, "relu": B.HT_GATE_RELU,
                     "sigmoid": B.HT_GATE_SIGMOID}[case["act"]]
            s.form = B.HT_W_IN_OUT if case["form"] == "in_out" else B.HT_W_OUT_IN
            s.Y = _matrix(n, case["e"]) if case["kind"] != "bwd" else None
            s.kept = {k: _matrix(n, case["f"]) for k in ("gate", "up")} if case["kind"] == "train" else {}
            s.grads = {"d" + k: torch.zeros_like(s.x[k]) for k in ("X", "Wg", "Wu", "Wd")} if case["kind"] != "fwd" else {}
        torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _data(case, name, t):
    """The columns of t that are data."""
    in_out = case["form"] == "in_out"
    cols = {"X": case["d"], "Y": case["e"], "Wg": case["f"] if in_out else case["d"], "Wd": case["e"] if in_out else case["f"]}
    cols["Wu"] = cols["Wg"]
    return t[:, :cols[name]]


def _run_own(s):
    B, case, x = s.B, s.case, s.x
    if case["kind"] == "norm":
        B.ht_grad_norm(s.ctx, x["grads"], s.norm, cols=s.cols, sync=False)
        return {"norm": s.norm}
    if case["kind"] == "clip":
        B.ht_grad_clip(s.ctx, x["grads"], x["max_norm"], out=s.out, norm=s.norm, cols=s.cols, sync=False)
        return {"norm": s.norm, "out": s.flat}
    sizes, weights, out = (case["d"], case["f"], case["e"]), (x["X"], x["Wg"], x["Wu"], x["Wd"]), {}
    if case["kind"] != "bwd":
        B.ht_ffn_fwd(s.ctx, *sizes, *weights, s.Y, act=s.act, w_form=s.form, **s.kept, sync=False)
        out["Y"] = _data(case, "Y", s.Y)
    if case["kind"] != "fwd":
        B.ht_ffn_bwd(s.ctx, *sizes, *weights, x["dY"], **s.grads, act=s.act, w_form=s.form, **s.kept, sync=False)
        out.update({k: _data(case, k[1:], t) for k, t in s.grads.items()})
    return out


def _plain_act(a, act, slope):
    """act(a), and with `slope` its derivative."""
    if act == "relu":
        return a.clamp(min=0.0), (a > 0).to(a.dtype) if slope else None
    if act in ("silu", "sigmoid"):
        t = 1.0 / (1.0 + torch.exp(-a))
        if act == "sigmoid":
            return t, t * (1.0 - t) if slope else None
        return a * t, t * (1.0 + a * (1.0 - t)) if slope else None
    if act == "gelu":
        t = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * t, t + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi)) if slope else None
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (a + 0.044715 * a * a * a))
    s = 0.5 * (1.0 + t) + 0.5 * a * (1.0 - t * t) * (c * (1.0 + 3.0 * 0.044715 * a * a)) if slope else None
    return 0.5 * a * (1.0 + t), s


def _run_plain(s):
    case, x = s.case, s.x
    if case["kind"] in ("norm", "clip"):
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for t in x["grads"]:
            total += (t * t).sum(dtype=torch.float64)        # (pad columns are zeros)
        norm = total.sqrt()
        out = {"norm": norm.float().reshape(1)}
        if case["kind"] == "clip":
            c = torch.clamp(x["max_norm"] / norm, max=1.0).float()
            for t, o in zip(x["grads"], s.out):
                torch.mul(t, c, out=o)
            out["out"] = s.flat
        return out
    X = _data(case, "X", x["X"])
    Wg, Wu, Wd = (_data(case, k, x[k]) if case["form"] == "in_out" else _data(case, k, x[k]).t() for k in ("Wg", "Wu", "Wd"))
    A, U = X @ Wg, X @ Wu
    value, slope = _plain_act(A, case["act"], case["kind"] != "fwd")
    H = value * U
    out = {}
    if case["kind"] != "bwd":
        out["Y"] = H @ Wd
    if case["kind"] != "fwd":
        dY = _data(case, "Y", x["dY"])
        G = dY @ Wd.t()
        dU = G * value
        dA = G.mul_(U).mul_(slope)
        out["dX"] = dA @ Wg.t() + dU @ Wu.t()
        if case["form"] == "in_out":
            out.update(dWg=X.t() @ dA, dWu=X.t() @ dU, dWd=H.t() @ dY)
        else:
            out.update(dWg=dA.t() @ X, dWu=dU.t() @ X, dWd=dY.t() @ H)
    return out


# ---------------------------------------------------------------- from the definitions, in 64 bits

def _exact_act(a, act):
    """act(a) and its derivative, from the sigmoid and the normal distribution."""
    if act == "relu":
        return torch.where(a > 0, a, torch.zeros_like(a)), torch.where(a > 0, torch.ones_like(a), torch.zeros_like(a))
    if act == "gelu":
        phi = torch.special.ndtr(a)
        return a * phi, phi + a * torch.exp(-a.square() / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":                                   # (1 + tanh u) / 2 = sigmoid(2 u)
        u2 = 2 * math.sqrt(2 / math.pi) * (a + 0.044715 * a.pow(3))
        s = torch.sigmoid(u2)
        return a * s, s + a * s * torch.sigmoid(-u2) * (2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * a.square()))
    s = torch.sigmoid(a)
    ds = s * torch.sigmoid(-a)
    return (s, ds) if act == "sigmoid" else (a * s, s + a * ds)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["kind"] in ("norm", "clip"):
        parts = torch.stack([torch.linalg.vector_norm(t.flatten(), dtype=torch.float64) for t in x["grads"]])
        norm = torch.linalg.vector_norm(parts)
        out = {"norm": norm.reshape(1)}
        if case["kind"] == "clip":
            factor = x["max_norm"] / norm if float(norm) > x["max_norm"] else torch.ones((), dtype=torch.float64, device="cuda")
            out["out"], parts = _flat(case, torch.float64)
            for part, t in zip(parts, x["grads"]):
                part.copy_(t.double() * factor)
        return out
    n, d, f, e, turned = case["n"], case["d"], case["f"], case["e"], case["form"] == "out_in"
    w = {}
    for name, rows, cols in (("Wg", d, f), ("Wu", d, f), ("Wd", f, e)):
        t = x[name].double()
        w[name] = t[:cols, :rows].t().contiguous() if turned else t[:rows, :cols].contiguous()
    out = {}
    if case["kind"] != "bwd":
        out["Y"] = torch.empty(n, e, dtype=torch.float64, device="cuda")
    if case["kind"] != "fwd":
        out["dX"] = torch.empty(n, d, dtype=torch.float64, device="cuda")
        sums = {k: torch.zeros_like(w[k]) for k in w}
    step = max(1, (1 << 26) // f)
    for r in range(0, n, step):
        h = x["X"][r:r + step, :d].double()
        gate, up = torch.mm(h, w["Wg"]), torch.mm(h, w["Wu"])
        value, slope = _exact_act(gate, case["act"])
        if "Y" in out:
            out["Y"][r:r + step] = torch.mm(value * up, w["Wd"])
        if case["kind"] == "fwd":
            continue
        dy = x["dY"][r:r + step, :e].double()
        back = torch.mm(dy, w["Wd"].t().contiguous())
        d_gate, d_up = back * up * slope, back * value
        out["dX"][r:r + step] = torch.mm(d_gate, w["Wg"].t().contiguous()) + torch.mm(d_up, w["Wu"].t().contiguous())
        ht = h.t().contiguous()
        sums["Wg"] += torch.mm(ht, d_gate)
        sums["Wu"] += torch.mm(ht, d_up)
        sums["Wd"] += torch.mm((value * up).t().contiguous(), dy)
    if case["kind"] != "fwd":
        out.update({"d" + k: t.t() if turned else t for k, t in sums.items()})
    return out


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    """Inputs read once and outputs written once; of the products, their multiply-adds."""
    kind = case["kind"]
    if kind in ("norm", "clip"):
        values = sum(rows * cols for rows, cols in _shapes(case))
        return {"bytes": 4 * values * (1 if kind == "norm" else 2), "flops": 2 * values if kind == "norm" else 3 * values}
    n, d, f, e = case["n"], case["d"], case["f"], case["e"]
    weights, there, back = 2 * d * f + f * e, n * (d + e), n * d
    if kind == "fwd":
        return {"bytes": 4 * (weights + there), "flops": 4 * n * d * f + 2 * n * f * e}
    if kind == "bwd":
        return {"bytes": 4 * (2 * weights + there + back), "flops": 12 * n * d * f + 4 * n * f * e}
    return {"bytes": 4 * (2 * weights + there + back + n * e), "flops": 12 * n * d * f + 6 * n * f * e}
