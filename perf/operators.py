"""The operators that tune the query side of an index that stands, with their plain forms.

The vectors of an index are embeddings that a model learned.  They stay; what is tuned is how a
query reaches them.  A batch holds rows of many tenants: each row goes through a projection that
all share and a low-rank adapter of its own (`project`), the result is what the index is searched
with, and the adapters learn from the log probabilities of items under a softmax over the inner
products with a table of vectors (`logprob`, with its entropy and its most probable items).  Both
have their backward pass.

    project            y = W x + s_a B_a (A_a x), a the row's adapter (-1: none)
    project_backward   gradients of x and of every adapter's A and B (W is shared and stays)
    logprob            l_v = scale <q, t_v> over the live rows v of the table; log p of the row's
                       target, log sum exp, entropy, the `top` most probable rows
    logprob_backward   gradients of the queries and of the table

A case is a dict of plain values; `listed()` gives the fixed ones, `draw(rng)` another one of the
same ranges, `prepare(case, seed)` the tensors, `run(state)` one pass.  With `own` false a pass is
elementary torch operations, with `own` true it is the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

F32, BF16 = "float32", "bfloat16"
TYPES = {F32: torch.float32, BF16: torch.bfloat16, "uint8": torch.uint8}
WIDTH = {F32: 4, BF16: 2, "uint8": 1}


def _project(name, n, d_in, d_out, rank, adapters, dtype, op="project", out=F32, mix="many"):
    # mix: how a batch's rows share the adapters ("many": any order; "runs": a few long runs)
    return dict(name=name, op=op, n=n, d_in=d_in, d_out=d_out, rank=rank, adapters=adapters, dtype=dtype,
                out=out, mix=mix)


def _logprob(name, n, v, d, dtype, op="logprob", table=None, top=10, live=1.0, padded=0.0, entropy=True,
             table_grad=False):
    # live: share of the table's rows that a query may see; padded: share of rows without a target
    return dict(name=name, op=op, n=n, v=v, d=d, dtype=dtype, table=table or dtype, top=top, live=live,
                padded=padded, entropy=entropy, table_grad=table_grad)


def listed():
    return [
        # the smallest call: one query of one tenant on its way into a 128-dimensional index; latency counts
        _project("project_one_query", 1, 768, 128, 8, 4, F32),
        # what a server gathers in a few milliseconds, every row another tenant
        _project("project_100_tenants", 100, 1024, 960, 16, 64, BF16),
        # the throughput batch of the 1M x 128 index
        _project("project_10000", 10_000, 1024, 128, 16, 250, F32),
        # an encoder's wide layer with adapters, a ragged batch of a few long runs
        _project("project_wide", 8_191, 4096, 4096, 64, 7, BF16, out=BF16, mix="runs"),
        # the adapters' training step for the 960-dimensional index
        _project("project_backward_960", 2_999, 1024, 960, 8, 32, F32, op="project_backward"),
        # the same at an encoder's width
        _project("project_backward_wide", 8_191, 2048, 2048, 32, 7, BF16, op="project_backward", mix="runs"),
        # one query against a million vectors: the table is read once
        _logprob("logprob_one_query", 1, 1_000_000, 128, F32),
        # a few queries over a table of learned vectors, an odd number of rows, some of them deleted
        _logprob("logprob_16_queries", 16, 131_071, 1024, BF16, top=5, live=0.9),
        # the throughput batch against the byte vectors of the 1M x 128 index
        _logprob("logprob_10000_bytes", 10_000, 1_000_000, 128, F32, table="uint8", entropy=False),
        # a training batch over a large table, a tenth of its rows padding
        _logprob("logprob_4096", 4_096, 128_000, 1024, BF16, top=20, padded=0.1),
        # in-batch negatives: the table is the batch's own items, both sides learn
        _logprob("logprob_backward_in_batch", 1_000, 1_024, 96, F32, op="logprob_backward", table_grad=True),
        # the gradient of the training batch, table included
        _logprob("logprob_backward_4095", 4_095, 65_537, 1024, BF16, op="logprob_backward", padded=0.1,
                 table_grad=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("project", "project", "project_backward", "logprob", "logprob", "logprob_backward"))
    dtype = rng.choice((F32, BF16))
    if op.startswith("project"):
        d_in, d_out = (rng.choice((96, 128, 257, 384, 768, 960, 1000, 1024, 2048, 4096)) for _ in range(2))
        n = _log_uniform(rng, 1, 10_000)
        # no dearer than the wide listed case
        n = max(1, min(n, int(8_191 * 4096 * 4096 / (d_in * d_out) / (8 if dtype == F32 else 2))))
        rank = rng.choice((1, 4, 8, 8, 16, 16, 24, 32, 64))
        c = _project("", n, d_in, d_out, rank, _log_uniform(rng, 1, min(256, max(1, 4096 // rank))), dtype, op=op,
                     out=rng.choice((F32, dtype)), mix=rng.choice(("many", "runs")))
    else:
        d = rng.choice((32, 96, 100, 128, 128, 255, 384, 768, 960, 1024))
        v = _log_uniform(rng, 1_000, 200_000)
        n = _log_uniform(rng, 1, 4_096)
        n = max(1, min(n, int(4_095 * 65_537 * 1024 / (v * d) / (4 if dtype == F32 else 1))))
        back = op == "logprob_backward"
        bytes_table = not back and dtype == F32 and rng.random() < 0.3
        c = _logprob("", n, v, d, dtype, op=op, table="uint8" if bytes_table else dtype,
                     top=0 if back else rng.choice((0, 1, 5, 10, 20, 50)),
                     live=rng.choice((1.0, 1.0, 0.9, 0.3)), padded=rng.choice((0.0, 0.0, 0.2)),
                     entropy=rng.random() < 0.7, table_grad=back and rng.random() < 0.5)
    del c["name"]
    return c


# ---- data ----------------------------------------------------------------------------------------


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _unit(x):
    return x / x.norm(dim=1, keepdim=True).clamp_(min=1e-12)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["op"].startswith("project"):
        return _prepare_project(case, g)
    return _prepare_logprob(case, g)


def _prepare_project(case, g):
    n, d_in, d_out, rank, adapters = (case[k] for k in ("n", "d_in", "d_out", "rank", "adapters"))
    t = TYPES[case["dtype"]]
    s = dict(case, x=_normal(g, n, d_in).to(t), w=(_normal(g, d_out, d_in) / math.sqrt(d_in)).to(t),
             a=(_normal(g, adapters, rank, d_in) / math.sqrt(d_in)).to(t),
             b=(_normal(g, adapters, d_out, rank) * 0.3 / math.sqrt(rank)).to(t),
             scale=torch.rand(adapters, generator=g, device="cuda") + 0.5)
    # one row in eight has no adapter
    ids = torch.randint(0, adapters, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[torch.rand(n, generator=g, device="cuda") < 0.125] = -1
    s["adapter"] = ids.sort().values if case["mix"] == "runs" else ids
    if case["op"] == "project_backward":
        s["dy"] = (_normal(g, n, d_out) / math.sqrt(n)).to(t)
    return s


def _prepare_logprob(case, g):
    n, v, d = case["n"], case["v"], case["d"]
    t = TYPES[case["dtype"]]
    targets = torch.randint(0, v, (n,), generator=g, device="cuda")
    if case["table"] == "uint8":
        # byte vectors as the 1M x 128 workload's: many small components, a few large ones
        table = (_normal(g, v, d).abs_() * 40.0).round_().clamp_(0.0, 255.0).to(torch.uint8)
        q = (table[targets].float() + 25.0 * _normal(g, n, d)).round_().clamp_(0.0, 255.0)
        scale = 8.0 / (40.0 * 40.0 * math.sqrt(d))
    else:
        # unit vectors, a query near its target: a temperature of 0.05
        table = _unit(_normal(g, v, d)).to(t)
        q = _unit(table[targets].float() + 1.5 / math.sqrt(d) * _normal(g, n, d)).to(t)
        scale = 20.0
    live = None
    if case["live"] < 1.0:
        # a bit per row of the table, 32 to a word, set where a query may see the row
        live = torch.rand(v, generator=g, device="cuda") < case["live"]
        live[targets[: max(1, n - n // 8)]] = True        # a few targets stay masked
    if case["padded"] > 0.0:
        targets = torch.where(torch.rand(n, generator=g, device="cuda") < case["padded"], -1, targets)
    s = dict(case, q=q, table=table, targets=targets, scale=scale, live=None if live is None else _pack_bits(live))
    if case["op"] == "logprob_backward":
        s["dlogp"] = -torch.rand(n, generator=g, device="cuda") / n
        s["dentropy"] = _normal(g, n) * (0.1 / n) if case["entropy"] else None
        # what the forward pass left
        s["lse"], s["h"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        alive = _live_bits(s["live"], v)
        for lo, hi in _chunks(n, v):
            z = _logits(s, alive, lo, hi)
            lse = torch.logsumexp(z, 1)
            p = torch.exp(z - lse[:, None])
            s["lse"][lo:hi] = lse
            s["h"][lo:hi] = lse - torch.where(p > 0, p * z, 0.0).sum(1)
    return s


def _pack_bits(live):
    v = live.numel()
    bits = torch.zeros((v + 31) // 32 * 32, dtype=torch.int64, device=live.device)
    bits[:v] = live
    words = (bits.view(-1, 32) << torch.arange(32, device=live.device)).sum(1)
    return (words - ((words >> 31) << 32)).to(torch.int32)


def _live_bits(words, v):
    if words is None:
        return None
    return ((words[:, None] >> torch.arange(32, device=words.device, dtype=torch.int32)) & 1).view(-1)[:v].bool()


# ---- one pass ------------------------------------------------------------------------------------


def run(s):
    if own:
        return _run_own(s)
    return dict(project=_plain_project, project_backward=_plain_project_backward, logprob=_plain_logprob,
                logprob_backward=_plain_logprob_backward)[s["op"]](s)


def _run_own(s):
    from paper_2601_07183_amd import binding

    if s["op"] == "project":
        p = binding.Projection(s["w"], s["a"], s["b"], s["scale"])
        return dict(y=p.project(s["x"], s["adapter"], out_dtype=TYPES[s["out"]]))
    if s["op"] == "project_backward":
        p = binding.Projection(s["w"], s["a"], s["b"], s["scale"])
        dx, da, db = p.backward(s["x"], s["adapter"], s["dy"])
        return dict(dx=dx, da=da, db=db)
    if s["op"] == "logprob":
        r = binding.logprob(s["q"], s["table"], s["targets"], scale=s["scale"], top=s["top"], live=s["live"],
                            entropy=s["entropy"])
        out = dict(logp=r.logp, lse=r.lse)
        if s["entropy"]:
            out["entropy"] = r.entropy
        if s["top"]:
            out.update(top_ids=r.top_ids, top_logp=r.top_logp)
        return out
    dq, dtable = binding.logprob_backward(s["q"], s["table"], s["targets"], s["lse"], s["dlogp"], scale=s["scale"],
                                          live=s["live"], entropy=s["h"], dentropy=s["dentropy"],
                                          table_grad=s["table_grad"])
    return dict(dq=dq, dtable=dtable) if s["table_grad"] else dict(dq=dq)


def _own_columns(s, width):
    """[n][adapters * width] truth values: the columns of a row's own adapter."""
    n, adapters = s["n"], s["adapters"]
    mine = s["adapter"].long()[:, None] == torch.arange(adapters, device="cuda")
    return mine[:, :, None].expand(n, adapters, width).reshape(n, adapters * width)


def _plain_project(s):
    # all adapters' products for all rows, the other tenants' columns set to zero
    r, k = s["rank"], s["adapters"] * s["rank"]
    x, w = s["x"].float(), s["w"].float()
    u = torch.where(_own_columns(s, r), x @ s["a"].float().view(k, -1).t(), 0.0)
    b = (s["b"].float() * s["scale"][:, None, None]).permute(1, 0, 2).reshape(s["d_out"], k)
    return dict(y=(x @ w.t() + u @ b.t()).to(TYPES[s["out"]]))


def _plain_project_backward(s):
    r, k = s["rank"], s["adapters"] * s["rank"]
    x, w, dy = s["x"].float(), s["w"].float(), s["dy"].float()
    a = s["a"].float().view(k, -1)
    b = (s["b"].float() * s["scale"][:, None, None]).permute(1, 0, 2).reshape(s["d_out"], k)
    mine = _own_columns(s, r)
    u = torch.where(mine, x @ a.t(), 0.0)
    du = torch.where(mine, dy @ b, 0.0)
    t = TYPES[s["dtype"]]
    db = (dy.t() @ u).view(s["d_out"], s["adapters"], r).permute(1, 0, 2) * s["scale"][:, None, None]
    return dict(dx=(dy @ w + du @ a).to(t), da=(du.t() @ x).view(s["adapters"], r, -1).to(t), db=db.to(t))


def _chunks(n, v):
    # rows at a time: about 2 GB of logits
    step = max(1, (1 << 29) // v)
    return [(lo, min(n, lo + step)) for lo in range(0, n, step)]


def _logits(s, alive, lo, hi):
    z = (s["q"][lo:hi].float() @ s["table"].float().t()) * s["scale"]
    return z if alive is None else z.masked_fill_(~alive, -math.inf)


def _plain_logprob(s):
    n, v, top = s["n"], s["v"], s["top"]
    alive = _live_bits(s["live"], v)
    out = dict(logp=torch.zeros(n, device="cuda"), lse=torch.empty(n, device="cuda"))
    if s["entropy"]:
        out["entropy"] = torch.empty(n, device="cuda")
    if top:
        out["top_ids"] = torch.empty((n, top), dtype=torch.int64, device="cuda")
        out["top_logp"] = torch.empty((n, top), device="cuda")
    for lo, hi in _chunks(n, v):
        z = _logits(s, alive, lo, hi)
        t = s["targets"][lo:hi]
        m = z.max(1, keepdim=True).values
        if top:
            # values next to each other are told apart in 64 bits
            ids = z.topk(min(v, top + 24), dim=1).indices
            ids = ids.sort(1).values
            near = (s["table"][ids].double() * s["q"][lo:hi, None].double()).sum(2)
            if alive is not None:
                near = near.masked_fill(~alive[ids], -math.inf)
            near, order = near.sort(dim=1, descending=True, stable=True)
            out["top_ids"][lo:hi] = ids.gather(1, order)[:, :top]
            best = near[:, :top] * s["scale"]
        zt = z.gather(1, t.clamp(min=0)[:, None])
        z.sub_(m)
        e = z.exp()
        total = e.sum(1, keepdim=True)
        logs = total.log()
        out["lse"][lo:hi] = (m + logs)[:, 0]
        out["logp"][lo:hi] = torch.where(t >= 0, (zt - m - logs)[:, 0], 0.0)
        if s["entropy"]:
            out["entropy"][lo:hi] = (logs - e.mul_(z.clamp_(min=-1e4)).sum(1, keepdim=True) / total)[:, 0]
        if top:
            out["top_logp"][lo:hi] = (best - m.double() - logs.double()).float()
    return out


def _plain_logprob_backward(s):
    n, v, d = s["n"], s["v"], s["d"]
    alive = _live_bits(s["live"], v)
    table = s["table"].float()
    dq = torch.empty((n, d), device="cuda")
    dtable = torch.zeros((v, d), device="cuda") if s["table_grad"] else None
    for lo, hi in _chunks(n, v):
        z = _logits(s, alive, lo, hi) - s["lse"][lo:hi, None]
        p = z.exp()
        t = s["targets"][lo:hi]
        seen = t >= 0
        if alive is not None:
            seen = seen & alive[t.clamp(min=0)]
        g = torch.where(seen, s["dlogp"][lo:hi], 0.0)[:, None]
        grad = -g * p
        if s["dentropy"] is not None:
            z.clamp_(min=-1e4)
            grad -= s["dentropy"][lo:hi, None] * p * (z + s["h"][lo:hi, None])
        grad.scatter_add_(1, t.clamp(min=0)[:, None], g)
        grad *= s["scale"]
        dq[lo:hi] = grad @ table
        if dtable is not None:
            dtable += grad.t() @ s["q"][lo:hi].float()
    t = TYPES[s["dtype"]]
    return dict(dq=dq.to(t), dtable=dtable.to(t)) if s["table_grad"] else dict(dq=dq.to(t))


# ---- from the definition, in 64 bits ---------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "project":
        y = s["x"].double() @ s["w"].double().t()
        for a, rows in _rows_of(s):
            y[rows] += float(s["scale"][a]) * (s["x"][rows].double() @ s["a"][a].double().t()) @ s["b"][a].double().t()
        return dict(y=y)
    if case["op"] == "project_backward":
        dx = s["dy"].double() @ s["w"].double()
        da, db = torch.zeros_like(s["a"], dtype=torch.float64), torch.zeros_like(s["b"], dtype=torch.float64)
        for a, rows in _rows_of(s):
            x, dy, f = s["x"][rows].double(), s["dy"][rows].double(), float(s["scale"][a])
            du = f * dy @ s["b"][a].double()
            dx[rows] += du @ s["a"][a].double()
            da[a] = du.t() @ x
            db[a] = f * dy.t() @ (x @ s["a"][a].double().t())
        return dict(dx=dx, da=da, db=db)
    parts = []
    table = s["table"].double()
    dead = None
    if s["live"] is not None:
        v = torch.arange(case["v"], device="cuda")
        dead = ((s["live"][v // 32] >> (v % 32).int()) & 1) == 0
    dtable = torch.zeros_like(table) if case["table_grad"] else None
    step = max(1, (1 << 28) // case["v"])
    for lo in range(0, case["n"], step):
        q, t = s["q"][lo:lo + step].double(), s["targets"][lo:lo + step]
        rows = torch.arange(len(t), device="cuda")
        ip = q @ table.t()
        if dead is not None:
            ip[:, dead] = -math.inf
        z = ip * s["scale"]
        lse = z.logsumexp(1)
        z -= lse[:, None]                                  # log p
        if case["op"] == "logprob":
            part = dict(logp=torch.where(t >= 0, z[rows, t.clamp(min=0)], 0.0), lse=lse)
            if case["top"]:
                vals, ids = ip.topk(min(case["v"], case["top"] + 8), dim=1)
                # among equal products the lower index first
                ids, order = ids.sort(1)
                order = vals.gather(1, order).sort(dim=1, descending=True, stable=True).indices
                part["top_ids"] = ids.gather(1, order)[:, :case["top"]]
                part["top_logp"] = z.gather(1, part["top_ids"])
            if case["entropy"]:
                part["entropy"] = -torch.special.xlogy(z.exp(), z.exp()).sum(1)
            parts.append(part)
            continue
        p = z.exp()
        to = torch.where(t >= 0, s["dlogp"][lo:lo + step].double(), 0.0)
        if dead is not None:
            to = torch.where(dead[t.clamp(min=0)], 0.0, to)
        grad = -to[:, None] * p
        grad[rows, t.clamp(min=0)] += to
        if s["dentropy"] is not None:
            plogp = torch.special.xlogy(p, p)
            h = -plogp.sum(1)
            grad -= s["dentropy"][lo:lo + step, None].double() * (plogp + p * h[:, None])
        grad *= s["scale"]
        parts.append(dict(dq=grad @ table))
        if dtable is not None:
            dtable += grad.t() @ q
    order = ("logp", "lse", "entropy", "top_ids", "top_logp", "dq")
    out = {k: torch.cat([p[k] for p in parts]) for k in order if k in parts[0]}
    if dtable is not None:
        out["dtable"] = dtable
    return out


def _rows_of(s):
    for a in range(s["adapters"]):
        rows = (s["adapter"] == a).nonzero()[:, 0]
        if len(rows):
            yield a, rows


# ---- what a pass cannot do without -----------------------------------------------------------------


def work(case):
    e, n = WIDTH[case["dtype"]], case["n"]
    if case["op"].startswith("project"):
        d_in, d_out, r = case["d_in"], case["d_out"], case["rank"]
        used = min(case["adapters"], n)
        weights = e * (float(d_in) * d_out + used * r * (d_in + d_out))
        if case["op"] == "project":
            return {"bytes": weights + n * (e * d_in + WIDTH[case["out"]] * d_out + 4),
                    "flops": 2.0 * n * (d_in * d_out + r * (d_in + d_out))}
        # read x, dy; write dx and every adapter's gradients
        grads = e * case["adapters"] * r * (d_in + d_out)
        return {"bytes": weights + grads + n * (e * (2 * d_in + d_out) + 4),
                "flops": 2.0 * n * (d_in * d_out + r * (3 * d_in + 2 * d_out))}
    v, d = case["v"], case["d"]
    read = n * e * d + float(WIDTH[case["table"]]) * v * d + 8 * n
    if case["op"] == "logprob":
        return {"bytes": read + n * (12 + 12 * case["top"]), "flops": 2.0 * n * v * d}
    return {"bytes": read + 16 * n + e * d * (n + (v if case["table_grad"] else 0)),
            "flops": 2.0 * n * v * d * (3 if case["table_grad"] else 2)}
