"""The operators at the two ends of a model over ids, as cases that can be timed and whose outputs can be compared.

  embed_fwd  rows of a table by id, scaled (ht_embed_fwd)
  embed_bwd  the table's gradient: the rows' gradients summed by id (ht_embed_bwd)
  head       softmax cross entropy of a linear layer over many classes, with the gradients of its input and of its
             weights, or the loss alone; the logits are not kept (ht_head_loss)
  distill    distillation from a teacher's top logits: loss, and gradient of the student's logits (ht_distill_loss)

Values are fp32 and ids int32, as everywhere in the library.  Ids and labels are drawn from a power law (the k-th most
frequent one has a share of about 1 / k), hidden rows are N(0, 1), weights give logits of standard deviation 2.
"""
import math

import torch

own = False

EMBED_SCALE_OF = math.sqrt      # lookups are scaled by the square root of the width


def listed():
    return [
        # A single id: what a serving loop asks for between two steps.
        dict(name="embed_fwd_1", kind="embed_fwd", n=1, V=65_536, d=256),
        # A full graph whose vertices carry ids of a smaller set (types, words), at an odd width.
        dict(name="embed_fwd_233k", kind="embed_fwd", n=232_965, V=50_003, d=301),
        # The gradient of a small batch over a small table.
        dict(name="embed_bwd_1k", kind="embed_bwd", n=1_000, V=10_000, d=64),
        # The gradient of a large batch over a large table: hot ids have tens of thousands of rows.
        dict(name="embed_bwd_500k", kind="embed_bwd", n=500_000, V=131_072, d=256),
        # Scoring one row over a large vocabulary: reading the weights is all there is.
        dict(name="head_score_1", kind="head", n=1, d=256, C=131_072, form="out_in", grad=False, unlabelled=0.0),
        # An ordinary training batch, weights as the library's layers have them.
        dict(name="head_2k_32k", kind="head", n=2_048, d=256, C=32_768, form="in_out", grad=True, unlabelled=0.0),
        # Odd sizes all over, most rows without a label.
        dict(name="head_odd", kind="head", n=7_001, d=602, C=50_003, form="in_out", grad=True, unlabelled=0.7),
        # The last layer of a full graph with labels on one vertex in a hundred.
        dict(name="head_1M_172", kind="head", n=1_000_000, d=256, C=172, form="in_out", grad=True, unlabelled=0.99),
        # The largest training batch over the largest vocabulary, the weights tied to a table of embeddings.
        dict(name="head_8k_131k", kind="head", n=8_192, d=256, C=131_072, form="out_in", grad=True, unlabelled=0.0),
        # A single row of distillation.
        dict(name="distill_1", kind="distill", n=1, C=131_072, K=32, T=2.0, grad=True),
        # Students of a graph's classes: short rows, many of them, some without a teacher.
        dict(name="distill_100k_172", kind="distill", n=100_003, C=172, K=8, T=4.0, grad=True),
        # A batch over a large vocabulary.
        dict(name="distill_4k_131k", kind="distill", n=4_096, C=131_072, K=64, T=1.0, grad=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed_fwd", "embed_bwd", "head", "head", "distill"])
    if kind in ("embed_fwd", "embed_bwd"):
        return dict(kind=kind, n=_log_uniform(rng, 1, 500_000), V=_log_uniform(rng, 100, 131_072), d=_log_uniform(rng, 16, 256))
    if kind == "head":
        d, C = _log_uniform(rng, 32, 1_024), _log_uniform(rng, 100, 131_072)
        most = min(1_000_000, int(8_192 * 256 * 131_072 / (d * C)))      # no more work than the largest listed case
        unlabelled = rng.choice([0.0, 0.0, 0.1, 0.7])
        return dict(kind=kind, n=_log_uniform(rng, 1, most), d=d, C=C, form=rng.choice(["in_out", "out_in"]),
                    grad=rng.random() < 0.75, unlabelled=unlabelled)
    C = _log_uniform(rng, 100, 131_072)
    return dict(kind=kind, n=_log_uniform(rng, 1, min(1_000_000, 4_096 * 131_072 // C)), C=C, K=_log_uniform(rng, 1, min(C, 100)),
                T=rng.choice([1.0, 2.0, 4.0]), grad=rng.random() < 0.75)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 11)
    return g


def _ids(n, V, g):
    """n ids below V, the k-th most frequent one with a share of about 1 / k; frequent ids are spread over the range."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    step = next(s for s in range(int(0.618 * V) | 1, 2 * V + 3, 2) if math.gcd(s, V) == 1)
    return ((rank * step) % V).to(torch.int32)


def _matrix(rows, cols):
    """Zeros of [rows x cols] whose rows start on 16 bytes, as the library wants its tensors."""
    return torch.zeros(rows, (cols + 3) // 4 * 4, device="cuda")


def _normal(rows, cols, g, std=1.0):
    m = _matrix(rows, cols)
    m[:, :cols] = torch.randn(rows, cols, generator=g, device="cuda") * std
    return m


def _inputs(case, seed):
    g, kind = _generator(seed), case["kind"]
    x = {}
    if kind == "embed_fwd":
        x["table"] = _normal(case["V"], case["d"], g)
        x["ids"] = _ids(case["n"], case["V"], g)
    elif kind == "embed_bwd":
        x["dH"] = _normal(case["n"], case["d"], g, 1e-2)
        x["ids"] = _ids(case["n"], case["V"], g)
    elif kind == "head":
        n, d, C = case["n"], case["d"], case["C"]
        x["H"] = _normal(n, d, g)
        shape = (d, C) if case["form"] == "in_out" else (C, d)
        x["W"] = _normal(*shape, g, 2.0 / math.sqrt(d))
        y = _ids(n, C, g)
        if case["unlabelled"] > 0:
            y[torch.rand(n, generator=g, device="cuda") < case["unlabelled"]] = -1
            y[n // 2] = C // 2                             # one label at least
        x["y"] = y
    else:
        n, C, K = case["n"], case["C"], case["K"]
        x["X"] = _normal(n, C, g, 2.0)
        x["top_ids"] = torch.empty(n, K, dtype=torch.int32, device="cuda")
        x["top"] = torch.empty(n, K, device="cuda")
        rows = max(1, (1 << 27) // C)
        for r in range(0, n, rows):                        # a teacher that agrees with the student in part
            part = x["X"][r:r + rows, :C]
            part = part + torch.randn(part.shape, generator=g, device="cuda") * 2.0
            v, i = torch.topk(part, K, dim=1)
            x["top"][r:r + rows] = v
            x["top_ids"][r:r + rows] = i.to(torch.int32)
        lot = torch.rand(n, generator=g, device="cuda")
        lot[n // 2] = 1.0                                  # one whole row at least
        x["top_ids"][lot < 0.02] = -1                      # no teacher for these rows
        x["top_ids"][(lot < 0.12).nonzero()[:, 0], K // 2:] = -1     # short lists
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
    if own:
        from paper_2311_14898_amd import binding as B
        s.B = B
        s.ctx = B.ht_ctx_create(0)
        kind = case["kind"]
        if kind == "embed_fwd":
            s.H = _matrix(case["n"], case["d"])
        elif kind == "embed_bwd":
            s.dT = _matrix(case["V"], case["d"])
        elif kind == "head":
            n, d, C = case["n"], case["d"], case["C"]
            s.loss, s.row_loss, s.row_lse = (torch.zeros(k, device="cuda") for k in (1, n, n))
            s.dH = _matrix(n, d) if case["grad"] else None
            s.dW = _matrix(*((d, C) if case["form"] == "in_out" else (C, d))) if case["grad"] else None
        else:
            s.loss, s.row_loss = torch.zeros(1, device="cuda"), torch.zeros(case["n"], device="cuda")
            s.dX = _matrix(case["n"], case["C"]) if case["grad"] else None
        torch.cuda.synchronize()
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    return _run_own(s) if own else _run_plain(s.case, s.x)


def _run_own(s):
    B, case, x, kind = s.B, s.case, s.x, s.case["kind"]
    if kind == "embed_fwd":
        B.ht_embed_fwd(s.ctx, case["d"], x["table"], x["ids"], s.H, scale=EMBED_SCALE_OF(case["d"]), sync=False)
        return {"H": s.H[:, :case["d"]]}
    if kind == "embed_bwd":
        B.ht_embed_bwd(s.ctx, case["d"], x["dH"], x["ids"], s.dT, scale=EMBED_SCALE_OF(case["d"]), sync=False)
        return {"dT": s.dT[:, :case["d"]]}
    if kind == "head":
        form = B.HT_W_IN_OUT if case["form"] == "in_out" else B.HT_W_OUT_IN
        B.ht_head_loss(s.ctx, case["d"], case["C"], x["H"], x["W"], x["y"], s.loss, row_loss=s.row_loss, row_lse=s.row_lse,
                       dH=s.dH, dW=s.dW, w_form=form, sync=False)
        out = {"loss": s.loss, "row_loss": s.row_loss, "row_lse": s.row_lse}
        if case["grad"]:
            out.update(dH=s.dH[:, :case["d"]], dW=s.dW[:, :case["C"] if case["form"] == "in_out" else case["d"]])
        return out
    B.ht_distill_loss(s.ctx, case["C"], x["X"], x["top_ids"], x["top"], s.loss, temperature=case["T"], row_loss=s.row_loss,
                      dlogits=s.dX, sync=False)
    out = {"loss": s.loss, "row_loss": s.row_loss}
    if case["grad"]:
        out["dX"] = s.dX[:, :case["C"]]
    return out


def _run_plain(case, x):
    kind = case["kind"]
    if kind == "embed_fwd":
        return {"H": x["table"][x["ids"].long(), :case["d"]] * EMBED_SCALE_OF(case["d"])}
    if kind == "embed_bwd":
        dT = torch.zeros(case["V"], case["d"], device="cuda")
        dT.index_add_(0, x["ids"].long(), x["dH"][:, :case["d"]])
        return {"dT": dT.mul_(EMBED_SCALE_OF(case["d"]))}
    if kind == "head":
        return _plain_head(case, x)
    return _plain_distill(case, x)


def _plain_head(case, x):
    n, d, C = case["n"], case["d"], case["C"]
    rows = (x["y"] >= 0).nonzero()[:, 0] if case["unlabelled"] > 0 else None
    H = x["H"][:, :d] if rows is None else x["H"][rows, :d]
    y = x["y"].long() if rows is None else x["y"][rows].long()
    W = x["W"][:, :C] if case["form"] == "in_out" else x["W"][:, :d].t()
    z = H @ W
    at = torch.arange(z.shape[0], device="cuda")
    xy = z[at, y]
    m = z.max(dim=1, keepdim=True).values
    z = z.sub_(m).exp_()
    total = z.sum(dim=1, keepdim=True)
    lse = (total.log() + m)[:, 0]
    l = lse - xy
    out = {"loss": l.sum().reshape(1) / z.shape[0]}
    for name, value in (("row_loss", l), ("row_lse", lse)):       # rows without a label: 0
        out[name] = value if rows is None else torch.zeros(n, device="cuda").index_copy_(0, rows, value)
    if not case["grad"]:
        return out
    z = z.div_(total)
    z[at, y] -= 1.0
    z = z.div_(z.shape[0])
    dH = z @ W.t()
    dH = dH if rows is None else torch.zeros(n, d, device="cuda").index_copy_(0, rows, dH)
    dW = H.t() @ z if case["form"] == "in_out" else z.t() @ H
    return dict(out, dH=dH, dW=dW)


def _plain_distill(case, x):
    n, C, T = case["n"], case["C"], case["T"]
    valid = x["top_ids"] >= 0
    has = valid.any(dim=1)
    ids = x["top_ids"].clamp(min=0).long()
    t = torch.where(valid, x["top"] / T, torch.full_like(x["top"], -math.inf))
    t = t - torch.where(has, t.max(dim=1).values, torch.zeros_like(t[:, 0]))[:, None]
    e = t.exp()
    q = e / torch.where(has, e.sum(dim=1), torch.ones_like(e[:, 0]))[:, None]
    logq = torch.where(q > 0, q, torch.ones_like(q)).log()
    z = x["X"][:, :C] / T
    m = z.max(dim=1, keepdim=True).values
    z_top = z.gather(1, ids)
    z = z.sub_(m).exp_()
    total = z.sum(dim=1, keepdim=True)
    logp = z_top - (m + total.log())
    l = torch.where(q > 0, q * (logq - logp), torch.zeros_like(q)).sum(dim=1) * (T * T)
    count = has.sum().float()
    out = {"loss": (l.sum() / count).reshape(1), "row_loss": l}
    if case["grad"]:
        z = z.div_(total).scatter_add_(1, ids, -q)
        out["dX"] = z.mul_((has.float() * (T / count))[:, None])
    return out


# ---------------------------------------------------------------- from the definitions, in 64 bits

def exact(case, seed):
    x, kind = _inputs(case, seed), case["kind"]
    if kind == "embed_fwd":
        d = case["d"]
        one_hot_free = torch.index_select(x["table"].double(), 0, x["ids"].long())[:, :d]
        return {"H": one_hot_free * EMBED_SCALE_OF(d)}
    if kind == "embed_bwd":
        d, V = case["d"], case["V"]
        order = torch.argsort(x["ids"].long(), stable=True)
        sums = torch.cumsum(x["dH"][order, :d].double(), dim=0)
        ends = torch.cumsum(torch.bincount(x["ids"].long(), minlength=V), dim=0)
        upto = torch.cat([torch.zeros(1, d, dtype=torch.float64, device="cuda"), sums])[ends]
        return {"dT": torch.diff(upto, dim=0, prepend=torch.zeros(1, d, dtype=torch.float64, device="cuda")) * EMBED_SCALE_OF(d)}
    if kind == "head":
        return _exact_head(case, x)
    return _exact_distill(case, x)


def _exact_head(case, x):
    n, d, C = case["n"], case["d"], case["C"]
    W = x["W"][:, :C].double() if case["form"] == "in_out" else x["W"][:, :d].double().t().contiguous()
    Wt = W.t().contiguous()
    y = x["y"].long()
    count = int((y >= 0).sum())
    row_loss, row_lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dH = torch.zeros(n, d, dtype=torch.float64, device="cuda") if case["grad"] else None
    dW = torch.zeros(d, C, dtype=torch.float64, device="cuda") if case["grad"] else None
    mine = torch.nonzero(y >= 0)[:, 0]
    for part in torch.split(mine, max(1, (1 << 27) // C)):
        h, t = x["H"][part, :d].double(), y[part]
        logits = h @ W
        row_lse[part] = torch.logsumexp(logits, dim=1)
        logp = torch.log_softmax(logits, dim=1)
        row_loss[part] = -logp.gather(1, t[:, None])[:, 0]
        if case["grad"]:
            p = logp.exp_()
            p.scatter_add_(1, t[:, None], torch.full((len(t), 1), -1.0, dtype=torch.float64, device="cuda"))
            dH[part] = p @ Wt / count
            dW += h.t().contiguous() @ p / count
    out = {"loss": row_loss.sum().reshape(1) / count, "row_loss": row_loss, "row_lse": row_lse}
    if case["grad"]:
        out.update(dH=dH, dW=dW if case["form"] == "in_out" else dW.t())
    return out


def _exact_distill(case, x):
    n, C, T = case["n"], case["C"], case["T"]
    there = x["top_ids"] >= 0
    whole = there.sum(dim=1) > 0
    count = int(whole.sum())
    row_loss = torch.zeros(n, dtype=torch.float64, device="cuda")
    dX = torch.zeros(n, C, dtype=torch.float64, device="cuda") if case["grad"] else None
    for part in torch.split(torch.nonzero(whole)[:, 0], max(1, (1 << 26) // C)):
        logp = torch.log_softmax(x["X"][part, :C].double() / T, dim=1)
        teacher = (x["top"][part].double() / T).masked_fill(~there[part], -math.inf)
        logq = torch.log_softmax(teacher, dim=1)
        q = logq.exp()
        at = x["top_ids"][part].long().clamp(min=0)
        terms = torch.nan_to_num(q * (logq - logp.gather(1, at)), nan=0.0)          # 0 * -inf of absent entries
        row_loss[part] = terms.sum(dim=1) * T * T
        if case["grad"]:
            dX[part] = logp.exp_().scatter_add_(1, at, -q) * (T / count)
    out = {"loss": row_loss.sum().reshape(1) / count, "row_loss": row_loss}
    if case["grad"]:
        out["dX"] = dX
    return out


# ---------------------------------------------------------------- what a pass cannot do without

def _distinct(n, V):
    """Ids among n draws from the power law, as many as are expected."""
    share = torch.log1p(1.0 / torch.arange(1, V + 1, dtype=torch.float64)) / math.log(V + 1.0)
    return float((1.0 - torch.exp(n * torch.log1p(-share))).sum())


def work(case):
    """Inputs read once and outputs written once; of the products, the multiply-adds of the loss (2 n d C) and of each gradient."""
    kind, n = case["kind"], case["n"]
    if kind == "embed_fwd":
        d = case["d"]
        return {"bytes": 4 * (n + _distinct(n, case["V"]) * d + n * d), "flops": n * d}
    if kind == "embed_bwd":
        d = case["d"]
        return {"bytes": 4 * (n + n * d + case["V"] * d), "flops": 2 * n * d}
    if kind == "head":
        d, C = case["d"], case["C"]
        rows = max(1, round(n * (1.0 - case["unlabelled"])))
        there = 4 * (n + rows * d + C * d + 2 * n)
        if not case["grad"]:
            return {"bytes": there, "flops": 2 * rows * d * C}
        return {"bytes": there + 4 * (n * d + C * d), "flops": 6 * rows * d * C}
    C, K = case["C"], case["K"]
    return {"bytes": 4 * (n * C * (2 if case["grad"] else 1) + 2 * n * K + n), "flops": 5 * n * C}
