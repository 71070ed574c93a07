"""The operators on sparse routing matrices as they are timed: what a layer that sends tokens to experts, or to
low-rank adapters, calls in one pass, over the sizes it meets.

The assignment of T tokens to E experts is a T x E matrix R in CSR with a few entries a row.  A case is one pass through

  op "route"     topk_route: R from the logits; with grad the gradient of the logits from that of R's values
  op "exchange"  Routing(R): R transposed, that is the tokens sorted by expert; dispatch: their rows in that order;
                 combine: the experts' rows summed back with R's values; with grad both gradients
  op "experts"   Routing(R) and matmul: every expert's matrix times its rows; with grad the gradients of rows and matrices
  op "adapters"  base + sum over a token's adapters of value * B (A x), S being the tokens x adapters matrix in CSR

Fields: T tokens, E experts, k experts a token, H or K and N the lengths of rows, L adapters of rank r, requests of
consecutive tokens; ragged: some tokens have fewer entries, some none; normalize: weights sum to one over the chosen.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one new token chooses its experts: latency
        {"name": "route_token", "op": "route", "T": 1, "E": 64, "k": 8, "dtype": "f32", "normalize": True, "grad": False},
        # a prompt's tokens, few experts, their number no power of two; values are shares of all experts
        {"name": "route_prompt", "op": "route", "T": 4099, "E": 60, "k": 4, "dtype": "bf16", "normalize": False, "grad": True},
        # a training batch over many experts
        {"name": "route_train", "op": "route", "T": 65537, "E": 256, "k": 8, "dtype": "f32", "normalize": True, "grad": True},
        # one step of a batch of requests: a few rows to many experts and back
        {"name": "exchange_step", "op": "exchange", "T": 33, "H": 2048, "E": 64, "k": 8, "dtype": "bf16", "ragged": False,
         "grad": False},
        # prompts of several requests: eight copies of long rows
        {"name": "exchange_prompt", "op": "exchange", "T": 8191, "H": 4096, "E": 64, "k": 8, "dtype": "bf16", "ragged": False,
         "grad": False},
        # a training step in 32 bits, tokens dropped, both directions
        {"name": "exchange_train", "op": "exchange", "T": 16385, "H": 2048, "E": 257, "k": 4, "dtype": "f32", "ragged": True,
         "grad": True},
        # one step of six requests: the met experts' matrices are read for a row or two each
        {"name": "experts_step", "op": "experts", "T": 6, "E": 64, "k": 4, "K": 2048, "N": 1024, "dtype": "bf16", "grad": False},
        # prompts through a few wide experts
        {"name": "experts_prompt", "op": "experts", "T": 4099, "E": 8, "k": 2, "K": 2048, "N": 8192, "dtype": "bf16",
         "grad": False},
        # a training step: the product and both gradients
        {"name": "experts_train", "op": "experts", "T": 8192, "E": 32, "k": 4, "K": 2048, "N": 2048, "dtype": "bf16",
         "grad": True},
        # the same for a small model whose sizes no tile divides
        {"name": "experts_odd", "op": "experts", "T": 1001, "E": 17, "k": 3, "K": 1000, "N": 1003, "dtype": "f16", "grad": True},
        # one step of 48 requests, each with an adapter of its own choice or none
        {"name": "adapters_step", "op": "adapters", "T": 48, "requests": 48, "L": 64, "r": 16, "K": 4096, "N": 4096,
         "dtype": "bf16"},
        # prompts of 12 requests
        {"name": "adapters_prompt", "op": "adapters", "T": 8191, "requests": 12, "L": 16, "r": 32, "K": 4096, "N": 2048,
         "dtype": "f16"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _length(rng, lo, hi):
    """The length of a row: two of three are multiples of 16, as widths of models are; the others are any number."""
    n = _log(rng, lo, hi)
    return max(lo, n - n % 16) + (16 if n // 16 == 192 else 0) if rng.random() < 2 / 3 else n + (1 if n == 3072 else 0)


def draw(rng):
    while True:
        op = rng.choice(["route", "exchange", "experts", "experts", "adapters"])
        c = {"op": op}
        if op == "route":
            c.update(T=_log(rng, 1, 65537), E=_log(rng, 2, 512), dtype=rng.choice(list(_DT)), normalize=rng.random() < 0.5)
        elif op == "exchange":
            c.update(T=_log(rng, 1, 16385), H=_length(rng, 16, 8192), E=_log(rng, 2, 512), dtype=rng.choice(list(_DT)),
                     ragged=rng.random() < 0.5)
        elif op == "experts":
            c.update(T=_log(rng, 1, 16385), E=_log(rng, 1, 64), K=_length(rng, 16, 4096), N=_length(rng, 16, 8192),
                     dtype=rng.choice(["bf16", "f16"]))
        else:
            T = _log(rng, 1, 8191)
            c.update(T=T, requests=min(T, _log(rng, 1, 256)), L=_log(rng, 1, 64), r=rng.choice([4, 8, 16, 16, 32, 64]),
                     K=_length(rng, 16, 4096), N=_length(rng, 16, 8192), dtype=rng.choice(["bf16", "f16"]))
        if op != "adapters":
            c.update(k=min(c["E"], rng.randint(1, 8)), grad=rng.random() < 0.5)
        w = work(c)
        if w["bytes"] < 1.2e9 and w["flops"] < 8e11 and (op != "experts" or c["E"] * c["K"] * c["N"] < 2 ** 28):
            return c


# ------------------------------------------------------------------ inputs


def _gen(seed, part):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 16 + part)
    return gen


def _normal(shape, dt, gen, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda") * scale).to(dt)


def _lengths(T, k, ragged):
    """Entries of every row: k, or where ragged none in one row of 16, half in one of 4.  Not by the seed: outputs keep their sizes."""
    i = torch.arange(T, device="cuda")
    n = torch.full((T,), k, device="cuda")
    if ragged:
        n = torch.where(i % 4 == 1, (k + 1) // 2, n)
        n = torch.where(i % 16 == 5, 0, n)
    return n


def _routing(T, E, k, ragged, gen):
    """R as a router makes it: distinct columns in ascending order, some columns in more demand than others, weights
    that sum to one over the chosen."""
    scores = torch.randn((T, E), generator=gen, device="cuda") + 0.3 * torch.randn(E, generator=gen, device="cuda")
    cols = torch.topk(scores, k, dim=1).indices.sort(1).values
    weight = torch.softmax(torch.gather(scores, 1, cols), 1)
    n = _lengths(T, k, ragged)
    keep = torch.arange(k, device="cuda")[None, :] < n[:, None]
    rowptr = torch.zeros(T + 1, dtype=torch.int64, device="cuda")
    rowptr[1:] = torch.cumsum(n, 0)
    return {"rowptr": rowptr, "colidx": cols[keep].to(torch.int32), "vals": weight[keep]}


def _requests(T, requests):
    """The request of every token: consecutive tokens, lengths in the ratio 1 : 2 : ... : 5 again and again."""
    w = torch.tensor([1 + (3 * j) % 5 for j in range(requests)], dtype=torch.float64)
    ends = torch.floor(torch.cumsum(w, 0) / w.sum() * (T - requests) + 0.5).to(torch.int64) + torch.arange(1, requests + 1)
    return torch.searchsorted(ends.cuda(), torch.arange(T, device="cuda"), right=True)


def prepare(case, seed):
    c, gen = dict(case), _gen(seed, 0)
    T, dt, s = c["T"], _DT[c["dtype"]], {"case": c}
    if c["op"] == "route":
        logits = torch.randn((T, c["E"]), generator=gen, device="cuda") * 2
        # experts that a token may not choose; in one row of 64 none is left
        shut = torch.rand((T, c["E"]), generator=gen, device="cuda") < 0.02
        shut |= (torch.arange(T, device="cuda") % 64 == 37)[:, None]
        s["logits"] = logits.masked_fill(shut, -math.inf).to(dt)
        s["gvals"] = _normal(T * c["k"], torch.float32, gen)
        return s
    if c["op"] == "adapters":
        L, r, K, N = c["L"], c["r"], c["K"], c["N"]
        of = _requests(T, c["requests"])
        has = of % 8 != 7  # one request of eight has no adapter
        rowptr = torch.zeros(T + 1, dtype=torch.int64, device="cuda")
        rowptr[1:] = torch.cumsum(has, 0)
        which = torch.randint(0, L, (c["requests"],), generator=gen, device="cuda")
        share = torch.rand(L, generator=gen, device="cuda") * 1.5 + 0.5  # an adapter's own scale
        col = which[of[has]]
        s.update(rowptr=rowptr, colidx=col.to(torch.int32), vals=share[col], x=_normal((T, K), dt, gen),
                 A=_normal((L, r, K), dt, gen, 1 / math.sqrt(K)), B=_normal((L, N, r), dt, gen, 1 / math.sqrt(r)),
                 base=_normal((T, N), dt, gen))
        return s
    s.update(_routing(T, c["E"], c["k"], c.get("ragged", False), gen))
    Z = s["colidx"].numel()
    if c["op"] == "exchange":
        s.update(x=_normal((T, c["H"]), dt, gen), ys=_normal((Z, c["H"]), dt, gen))
        if c["grad"]:
            s.update(gy=_normal((T, c["H"]), dt, gen), gxs=_normal((Z, c["H"]), dt, gen))
    else:
        s.update(xs=_normal((Z, c["K"]), dt, gen), W=_normal((c["E"], c["N"], c["K"]), dt, gen, 1 / math.sqrt(c["K"])))
        if c["grad"]:
            s["gys"] = _normal((Z, c["N"]), dt, gen)
    return s


# ------------------------------------------------------------------ one pass


def run(state):
    return (_own if own else _plain)[state["case"]["op"]](state, state["case"])


def _csr(s, cols):
    from paper_2606_20855_gb300 import DeviceCSR
    return DeviceCSR(s["case"]["T"], cols, s["rowptr"], s["colidx"], s["vals"])


def _own_route(s, c):
    from paper_2606_20855_gb300 import topk_route, topk_route_backward
    R = topk_route(s["logits"], c["k"], normalize=c["normalize"])
    out = {"rowptr": R.rowptr, "colidx": R.colidx, "vals": R.vals}
    if c["grad"]:
        out["glogits"] = topk_route_backward(s["logits"], R, s["gvals"], normalize=c["normalize"])
    return out


def _own_exchange(s, c):
    from paper_2606_20855_gb300 import Routing
    plan = Routing(_csr(s, c["E"]))
    out = {"offsets": plan.offsets, "rows": plan.rows, "entries": plan.entries, "slots": plan.slots,
           "xs": plan.dispatch(s["x"]), "y": plan.combine(s["ys"])}
    if c["grad"]:
        out["gys"], out["gvals"] = plan.combine_backward(s["gy"], s["ys"])
        out["gx"] = plan.dispatch_backward(s["gxs"])
    return out


def _own_experts(s, c):
    from paper_2606_20855_gb300 import Routing
    plan = Routing(_csr(s, c["E"]))
    out = {"ys": plan.matmul(s["xs"], s["W"])}
    if c["grad"]:
        out["gxs"], out["gW"] = plan.matmul_backward(s["gys"], s["xs"], s["W"])
    return out


def _own_adapters(s, c):
    from paper_2606_20855_gb300 import adapters
    return {"y": adapters(s["x"], s["A"], s["B"], _csr(s, c["L"]), s["base"])}


_own = {"route": _own_route, "exchange": _own_exchange, "experts": _own_experts, "adapters": _own_adapters}


def _plain_route(s, c):
    x, k = s["logits"].float(), c["k"]
    T = x.shape[0]
    chosen = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k].sort(1).values
    top = x.max(1, keepdim=True).values
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))  # zero in a row where every expert is shut
    picked = torch.gather(e, 1, chosen)
    total = (picked if c["normalize"] else e).sum(1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)
    v = picked / total
    out = {"rowptr": torch.arange(T + 1, device=x.device) * k, "colidx": chosen.to(torch.int32).reshape(-1), "vals": v.reshape(-1)}
    if c["grad"]:
        g = s["gvals"].view(T, k)
        mean = (v * g).sum(1, keepdim=True)
        if c["normalize"]:
            grad = torch.zeros_like(x).scatter(1, chosen, v * (g - mean))
        else:
            grad = e / total * (torch.zeros_like(x).scatter(1, chosen, g) - mean)
        out["glogits"] = grad.to(s["logits"].dtype)
    return out


def _transposed(s, E):
    """Offsets of the columns, and for every slot in their order its row and entry; the slot of every entry."""
    T, Z = s["rowptr"].numel() - 1, s["colidx"].numel()
    row = torch.repeat_interleave(torch.arange(T, device="cuda"), s["rowptr"][1:] - s["rowptr"][:-1], output_size=Z)
    col, entries = torch.sort(s["colidx"], stable=True)
    offsets = torch.searchsorted(col, torch.arange(E + 1, dtype=torch.int32, device="cuda"))
    slots = torch.empty_like(entries)
    slots[entries] = torch.arange(Z, device="cuda")
    return offsets, row[entries], entries, slots, col.long()


def _plain_exchange(s, c):
    offsets, rows, entries, slots, _ = _transposed(s, c["E"])
    dt, shape = s["x"].dtype, s["x"].shape
    v = s["vals"][entries][:, None]
    ys = s["ys"].float()
    out = {"offsets": offsets, "rows": rows.to(torch.int32), "entries": entries.to(torch.int32), "slots": slots.to(torch.int32),
           "xs": s["x"][rows], "y": torch.zeros(shape, device="cuda").index_add_(0, rows, ys * v).to(dt)}
    if c["grad"]:
        gy = s["gy"].float()[rows]
        out["gys"] = (gy * v).to(dt)
        out["gvals"] = (gy * ys).sum(1)[slots]
        out["gx"] = torch.zeros(shape, device="cuda").index_add_(0, rows, s["gxs"].float()).to(dt)
    return out


def _plain_experts(s, c):
    offsets, _, _, _, col = _transposed(s, c["E"])
    dt, W = s["xs"].dtype, s["W"].float()
    most = int((offsets[1:] - offsets[:-1]).max())  # every expert's rows in a block of the longest's size
    at = torch.arange(col.numel(), device="cuda") - offsets[col]

    def block(rows):
        b = torch.zeros((c["E"], most, rows.shape[1]), device="cuda")
        b[col, at] = rows.float()
        return b

    xs = block(s["xs"])
    out = {"ys": torch.matmul(xs, W.transpose(1, 2))[col, at].to(dt)}
    if c["grad"]:
        gys = block(s["gys"])
        out["gxs"] = torch.matmul(gys, W)[col, at].to(dt)
        out["gW"] = torch.matmul(gys.transpose(1, 2), xs).to(dt)
    return out


def _plain_adapters(s, c):
    T, L, r = c["T"], c["L"], c["r"]
    Z = s["colidx"].numel()
    row = torch.repeat_interleave(torch.arange(T, device="cuda"), s["rowptr"][1:] - s["rowptr"][:-1], output_size=Z)
    S = torch.zeros((T, L), device="cuda")
    S[row, s["colidx"].long()] = s["vals"]
    inner = torch.matmul(s["x"].float(), s["A"].float().view(L * r, -1).T).view(T, L, r) * S[:, :, None]
    y = s["base"].float() + torch.matmul(inner.view(T, L * r), s["B"].float().transpose(1, 2).reshape(L * r, -1))
    return {"y": y.to(s["base"].dtype)}


_plain = {"route": _plain_route, "exchange": _plain_exchange, "experts": _plain_experts, "adapters": _plain_adapters}


# ------------------------------------------------- the same results in 64 bits


def _by_expert(rowptr, colidx, E):
    """For every expert the rows and entries that name it, in order."""
    Z = colidx.numel()
    row = torch.searchsorted(rowptr, torch.arange(Z, device="cuda"), right=True) - 1
    picked = [torch.nonzero(colidx == e).flatten() for e in range(E)]
    return [(row[p], p) for p in picked]


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "route":
        x, T, E, k = s["logits"].double(), c["T"], c["E"], c["k"]
        # columns by value, then by index, from the place of every logit among its row's: rows in blocks
        on = torch.zeros((T, E), dtype=torch.bool, device="cuda")
        col = torch.arange(E, device="cuda")
        step = max(1, (1 << 25) // (E * E))
        for a in range(0, T, step):
            b = x[a:a + step]
            before = (b[:, None, :] > b[:, :, None]) | ((b[:, None, :] == b[:, :, None]) & (col[None, None, :] < col[None, :, None]))
            on[a:a + step] = before.sum(2) < k
        z = torch.where(on, x, -math.inf) if c["normalize"] else x
        p = torch.nan_to_num(torch.exp(x - torch.logsumexp(z, 1, keepdim=True)), nan=0.0)
        out = {"rowptr": k * torch.arange(T + 1, device="cuda"), "colidx": on.nonzero()[:, 1].to(torch.int32), "vals": p[on]}
        if c["grad"]:
            g = torch.zeros_like(x)
            g[on] = s["gvals"].double()
            q = torch.where(on, p, 0.0) if c["normalize"] else p
            out["glogits"] = q * (g - (torch.where(on, p, 0.0) * g).sum(1, keepdim=True))
        return out
    if c["op"] == "adapters":
        y = s["base"].double()
        for a, (rows, entries) in enumerate(_by_expert(s["rowptr"], s["colidx"], c["L"])):
            inner = s["x"][rows].double() @ s["A"][a].double().T
            y[rows] += s["vals"][entries].double()[:, None] * (inner @ s["B"][a].double().T)
        return {"y": y}
    lists = _by_expert(s["rowptr"], s["colidx"], c["E"])
    if c["op"] == "exchange":
        x, ys = s["x"].double(), s["ys"].double()
        rows, entries = (torch.cat([pair[i] for pair in lists]) for i in (0, 1))
        ends = torch.cumsum(torch.tensor([0] + [p[0].numel() for p in lists], device="cuda"), 0)
        slots = torch.argsort(entries)
        out = {"offsets": ends, "rows": rows.to(torch.int32), "entries": entries.to(torch.int32),
               "slots": slots.to(torch.int32), "xs": x[rows], "y": torch.zeros_like(x)}
        if c["grad"]:
            gy, gxs = s["gy"].double(), s["gxs"].double()
            out.update(gys=torch.zeros_like(ys), gvals=torch.zeros(slots.numel(), dtype=torch.float64, device="cuda"),
                       gx=torch.zeros_like(x))
        at = 0
        for r, e in lists:  # one expert's rows are distinct
            v, part = s["vals"][e].double()[:, None], slice(at, at + r.numel())
            out["y"][r] += v * ys[part]
            if c["grad"]:
                out["gys"][part] = v * gy[r]
                out["gvals"][e] = torch.einsum("ih,ih->i", gy[r], ys[part])
                out["gx"][r] += gxs[part]
            at += r.numel()
        return out
    xs, gys, at = s["xs"].double(), s["gys"].double() if c["grad"] else None, 0
    out = {"ys": []}
    if c["grad"]:
        out.update(gxs=[], gW=[])
    for e, (r, _) in enumerate(lists):
        part, W = slice(at, at + r.numel()), s["W"][e].double()
        out["ys"].append(xs[part] @ W.T)
        if c["grad"]:
            out["gxs"].append(gys[part] @ W)
            out["gW"].append(gys[part].T @ xs[part])
        at += r.numel()
    return {name: torch.stack(v) if name == "gW" else torch.cat(v) for name, v in out.items()}


# ------------------------------------------------------------- what a pass needs


def _entries(T, k, ragged):
    if not ragged:
        return T * k
    none, half = (T + 10) // 16, (T + 2) // 4  # rows 5, 21, ... and 1, 5, 9, ...
    return T * k - none * k - (half - none) * (k - (k + 1) // 2)


def work(case):
    """Inputs read once, outputs written once; of the experts' matrices and the adapters those that are met (as many as
    even chances give)."""
    c, T = case, case["T"]
    s = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "adapters":
        L, r, K, N, q = c["L"], c["r"], c["K"], c["N"], c["requests"]
        used, Z = q - q // 8, T * (q - q // 8) / q
        met = L * (1 - (1 - 1 / L) ** used)
        return {"bytes": s * (T * (K + 2 * N) + met * r * (K + N)) + 8 * Z + 8 * (T + 1), "flops": 2 * Z * r * (K + N)}
    E = c["E"]
    Z = _entries(T, c["k"], c.get("ragged", False))
    if c["op"] == "route":
        back = s * T * E + 4 * Z if c["grad"] else 0
        return {"bytes": s * T * E + 8 * Z + 8 * (T + 1) + back, "flops": T * E * (8 if c["grad"] else 4)}
    if c["op"] == "exchange":
        H = c["H"]
        n = (T + Z + Z + T) + (T + Z + Z + T if c["grad"] else 0)
        return {"bytes": s * H * n + 8 * (T + 1) + 8 * (E + 1) + 20 * Z + (4 * Z if c["grad"] else 0),
                "flops": Z * H * (6 if c["grad"] else 2)}
    K, N = c["K"], c["N"]
    met = E * (1 - (1 - c["k"] / E) ** T)
    b = Z * (K + N) + met * N * K + (Z * (K + N) + E * N * K if c["grad"] else 0)
    return {"bytes": s * b + 8 * (T + 1) + 8 * Z, "flops": 2 * Z * N * K * (3 if c["grad"] else 1)}
