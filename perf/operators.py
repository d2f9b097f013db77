"""Timed cases of the operators with which discovered networks answer and learn.

  sample  drawing indices from rows of scores with given random numbers, under a temperature, top-k,
          top-p and min-p: the answers of networks with several outputs, the parents of a
          generation from their fitness
  loss    negative log-likelihood of the drawn answers under the scores' softmax, with the gradient of
          the scores
  keep    activation of a population's networks that keeps the state of every step in 8 bits
  back    gradients of the edges' weights (and of the patterns) from those 8-bit states

`run` computes them in plain torch, or, where `own` is true, with the library.

The definition of `sample`. A score that is NaN is taken as -inf, one above the largest float32 as that.
Of a row with maximum m and temperature T, entry i weighs q_i = floor(2^31 exp((x_i - m) (1/T))), a whole
number, so every later sum is exact in any order; an entry of -inf weighs 0, and a temperature below the
least normal float32 leaves the first maximum only. top-k leaves the k largest scores, top-p of those
the ones before which (by falling score) less than top_p of the sum lies, min-p of those the ones with
q_i >= 2^31 min_p; equal scores rank by index. With total weight S of what is left, the number u in
[0, 1) draws the first index at which the running sum by index exceeds floor(u S). A row in which
nothing is left gives index -1 and log-probability -inf.
"""

import math

import numpy as np
import torch

own = False

FLT_MAX = float(np.finfo(np.float32).max)
TINY = float(np.finfo(np.float32).tiny)
ONE = 2.0 ** 31
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


# ----------------------------------------------------------------------------- cases

def _sample(name, rows, n, type, draws=1, t=1.0, k=0, p=1.0, min_p=0.0, per_row=False, pad=0):
    return {"name": name, "op": "sample", "rows": rows, "n": n, "type": type, "draws": draws, "t": t,
            "k": k, "p": p, "min_p": min_p, "per_row": per_row, "pad": pad}


def _loss(name, rows, n, type, t=1.0):
    return {"name": name, "op": "loss", "rows": rows, "n": n, "type": type, "t": t}


def _nets(name, op, genomes, lo, hi, inputs, outputs, deg_in, deg_h, patterns, steps, grad_in=False):
    return {"name": name, "op": op, "genomes": genomes, "lo": lo, "hi": hi, "inputs": inputs,
            "outputs": outputs, "deg_in": deg_in, "deg_h": deg_h, "patterns": patterns, "steps": steps,
            "grad_in": grad_in}


def listed():
    return [
        # the answers of a population of 1000 to the four XOR patterns, among 8 outputs: latency
        _sample("sample_answers_pop1000", 4000, 8, "f32", t=0.5),
        # the parents of the next generation: as many draws as genomes, from the best fifth
        _sample("sample_parents_pop1000", 1, 1000, "f32", draws=1000, t=0.05, k=200),
        # one of the nodes of every network of a batch, each row with its own settings
        _sample("sample_rows256_n2485", 256, 2485, "bf16", t=0.8, k=300, p=0.9, min_p=0.01, per_row=True),
        # a few long rows, all filters
        _sample("sample_rows16_n50001", 16, 50001, "f16", t=0.7, k=50, p=0.9, min_p=0.02),
        # many long rows, the nucleus alone
        _sample("sample_rows256_n131072", 256, 131072, "f32", t=1.0, p=0.95),
        # the losses of a data set's answers: many rows of few scores
        _loss("loss_rows150000_n10", 150000, 10, "f32", t=0.5),
        # long rows in 16 bits
        _loss("loss_rows2047_n32001", 2047, 32001, "bf16"),
        # XOR: a population of 1000 on four patterns, feedforward substrates: latency
        _nets("keep_pop1000_rows4", "keep", 1000, 2, 120, 3, 1, 3, 0, 4, 4),
        # a data set's rows through networks with hidden nodes among themselves
        _nets("keep_pop150_rows1000", "keep", 150, 4, 773, 32, 4, 16, 60, 1000, 4),
        # the gradients of both, and of one network larger than a workgroup's memory
        _nets("back_pop1000_rows4", "back", 1000, 2, 120, 3, 1, 3, 0, 4, 4),
        _nets("back_pop150_rows1000", "back", 150, 4, 773, 32, 4, 16, 60, 1000, 4, grad_in=True),
        _nets("back_large3_rows61", "back", 3, 5000, 9000, 5, 2, 5, 40, 61, 6),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "loss", "keep", "back"])
    type = rng.choice(["f32", "bf16", "f16"])
    if op == "sample":
        filters = {"t": round(math.exp(rng.uniform(-3.0, 1.0)), 3)}
        if rng.random() < 0.5:
            filters["k"] = _log(rng, 1, 1000)
        if rng.random() < 0.6:
            filters["p"] = round(rng.uniform(0.3, 0.99), 3)
        if rng.random() < 0.4:
            filters["min_p"] = round(math.exp(rng.uniform(-6.0, -1.0)), 4)
        if rng.random() < 0.3:  # parents: one row, many draws
            n = _log(rng, 100, 300000)
            return {k: v for k, v in _sample("", 1, n, "f32", draws=_log(rng, 100, 300000),
                                             **filters).items() if k != "name"}
        n = _log(rng, 2, 131072)
        rows = _log(rng, 1, min(20000, 256 * 131072 // n))
        c = _sample("", rows, n, type, per_row=rng.random() < 0.4, pad=rng.choice([0, 0, 1, 7, 64]),
                    **filters)
    elif op == "loss":
        n = _log(rng, 2, 65536)
        rows = _log(rng, 16, max(16, min(150000, 2047 * 32001 // n)))
        c = _loss("", rows, n, type, round(math.exp(rng.uniform(-1.0, 1.0)), 3))
    else:
        hi = _log(rng, 40, 4000)
        genomes = _log(rng, 1, max(1, min(500, 60000 // hi)))
        c = _nets("", op, genomes, _log(rng, 1, hi), hi, _log(rng, 1, 32), rng.choice([1, 2, 4, 9]),
                  _log(rng, 1, 16), rng.choice([0, 3, 20, 50]), 1, rng.randint(1, 8),
                  op == "back" and rng.random() < 0.5)
        most = 1.0e9 if op == "keep" else 5.0e8
        c["patterns"] = _log(rng, 1, int(max(1, min(1000, most / (c["steps"] * sum(_edges(c)))))))
    return {k: v for k, v in c.items() if k != "name"}


# ----------------------------------------------------------------------------- inputs

def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _hidden(case):
    """Hidden nodes of each genome: spread over [lo, hi] in the logarithm."""
    g = case["genomes"]
    if g == 1:
        return [case["hi"]]
    a, b = math.log(case["lo"]), math.log(case["hi"])
    return [int(round(math.exp(a + (b - a) * i / (g - 1)))) for i in range(g)]


def _edges(case):
    """(edges from inputs, edges from hidden nodes) of all genomes."""
    k, o = min(case["deg_in"], case["inputs"]), case["outputs"]
    return (sum((m + o) * k for m in _hidden(case)),
            sum(m * min(case["deg_h"], m) + o * m for m in _hidden(case)))


def _picks(rng, rows, k, n):
    """[rows, k] distinct numbers below n in rising order: steps coprime to n from a random start."""
    step = rng.integers(1, max(n, 2), size=rows)
    while n > 1:
        bad = np.gcd(step, n) != 1
        if not bad.any():
            break
        step[bad] = rng.integers(1, n, size=int(bad.sum()))
    return np.sort((rng.integers(0, n, size=(rows, 1)) + step[:, None] * np.arange(k)) % n, axis=1)


def _networks(case, seed):
    """Host arrays of a population's networks. A genome's nodes are its inputs, its outputs and its hidden
    nodes; a hidden node has edges from inputs and from hidden nodes, an output from inputs and
    from every hidden node."""
    rng = np.random.default_rng([int(seed), 7])
    n_in, n_out = case["inputs"], case["outputs"]
    k = min(case["deg_in"], n_in)
    node_offset, degrees, src = [0], [], []
    for m in _hidden(case):
        base, h = node_offset[-1], min(case["deg_h"], m)
        degrees.append(np.concatenate([np.zeros(n_in, np.int64), np.full(n_out, k + m, np.int64),
                                       np.full(m, k + h, np.int64)]))
        hid = base + n_in + n_out
        src.append(np.concatenate([base + _picks(rng, n_out, k, n_in),
                                   np.broadcast_to(hid + np.arange(m), (n_out, m))], axis=1).reshape(-1))
        src.append(np.concatenate([base + _picks(rng, m, k, n_in), hid + _picks(rng, m, h, m)],
                                  axis=1).reshape(-1))
        node_offset.append(hid + m)
    degrees = np.concatenate(degrees)
    in_offset = np.concatenate([[0], np.cumsum(degrees)]).astype(np.int64)
    src = np.concatenate(src).astype(np.uint32)
    dst = np.repeat(np.arange(len(degrees)), degrees)
    w = rng.standard_normal(len(src)) * 2.0 / np.sqrt(degrees[dst])
    return {"node_offset": np.array(node_offset, np.int64), "in_offset": in_offset, "src": src,
            "dst": dst, "w": w.astype(np.float32)}


def _prepare_nets(case, seed):
    nets = _networks(case, seed)
    g = _gen(seed, 11)
    nodes, G, P = int(nets["node_offset"][-1]), case["genomes"], case["patterns"]
    s = {"case": case, "x": torch.rand((P, case["inputs"]), generator=g, device="cuda") * 2 - 1}
    if case["op"] == "back":
        # states as they come out of the sigmoids, in 8 bits: code c stands for c / 255
        planes = case["steps"] - 1
        codes = torch.randn((planes, nodes, P), generator=g, device="cuda").mul_(2).sigmoid_()
        codes = codes.mul_(255).round_().to(torch.uint8)
        s["out"] = (torch.randn((G, P, case["outputs"]), generator=g, device="cuda") * 1.5).sigmoid()
        s["grad_out"] = torch.randn((G, P, case["outputs"]), generator=g, device="cuda") / P
    if own:
        from paper_2608_27612_amd import emr
        subs = [(2.0 * i / max(1, case["inputs"]) - 1, -1.0, emr.EMR_DIR_OUT) for i in range(case["inputs"])]
        subs += [(2.0 * i / max(1, case["outputs"]) - 1, 1.0, emr.EMR_DIR_IN) for i in range(case["outputs"])]
        s["net"] = emr.emr_load_networks(subs, nets["node_offset"], nets["in_offset"], nets["src"],
                                         nets["w"])
        if case["op"] == "back":
            s["kept"] = emr.kept_from_codes(codes)
    else:
        first = nets["node_offset"][:-1]
        at = first[:, None] + np.arange(case["inputs"] + case["outputs"])
        s["src"] = torch.from_numpy(nets["src"].astype(np.int64)).cuda()
        s["dst"] = torch.from_numpy(nets["dst"]).cuda()
        s["w"] = torch.from_numpy(nets["w"]).cuda()
        s["in_nodes"] = torch.from_numpy(at[:, :case["inputs"]].reshape(-1)).cuda()
        s["out_nodes"] = torch.from_numpy(at[:, case["inputs"]:].reshape(-1)).cuda()
        s["nodes"] = nodes
        if case["op"] == "back":
            s["codes"] = codes
    return s


def prepare(case, seed):
    if case["op"] in ("keep", "back"):
        return _prepare_nets(case, seed)
    g = _gen(seed, 3)
    rows, n = case["rows"], case["n"]
    width = n + case.get("pad", 0)
    x = torch.randn((rows, width), generator=g, device="cuda") * 3.0
    if case["op"] == "sample" and case["draws"] > 1:
        x = torch.rand((rows, width), generator=g, device="cuda")  # fitness
    elif n > 4:
        # masked scores, a few as the type's lowest value; every 64th row from the 8th on masked whole
        mask = torch.rand((rows, width), generator=g, device="cuda")
        x[mask < 0.05] = -math.inf
        x[mask > 0.995] = torch.finfo(TYPES[case["type"]]).min
        x[7::64] = -math.inf
    x = x.to(TYPES[case["type"]])[:, :n]
    s = {"case": case, "x": x}
    if case["op"] == "loss":
        index = torch.randint(0, n, (rows,), generator=g, device="cuda", dtype=torch.int32)
        best = x.float().argmax(1).to(torch.int32)  # (an answer that a row could have given)
        at = x.float().gather(1, index.long()[:, None])[:, 0]
        index = torch.where(at > -1e4, index, best)
        index[3::97] = -1  # rows without an answer
        s["index"] = index
        s["scale"] = torch.randn((rows,), generator=g, device="cuda")
        return s
    s["u"] = torch.rand((rows, case["draws"]), generator=g, device="cuda")
    for key, value, kind in (("t", case["t"], torch.float32), ("k", case["k"], torch.int32),
                             ("p", case["p"], torch.float32), ("min_p", case["min_p"], torch.float32)):
        if case["per_row"] and key in ("t", "k", "p"):
            f = torch.rand((rows,), generator=g, device="cuda") + 0.5
            if key == "t":
                f[::50] = 0.0  # rows that take their maximum
            if key == "p":
                f = f.clamp(max=1.0)
            s[key] = (value * f).to(kind)
        else:
            s[key] = value
    return s


# ----------------------------------------------------------------------------- plain forms

def _plain_sample(s):
    x, u = s["x"].float(), s["u"]
    rows, n = x.shape
    col = lambda v, kind: (v if torch.is_tensor(v)  # noqa: E731
                           else torch.full((rows,), v, device=x.device)).to(kind)[:, None]
    t, k, p, min_p = (col(s["t"], torch.float32), col(s["k"], torch.int64),
                      col(s["p"], torch.float32), col(s["min_p"], torch.float32))
    x = torch.where(torch.isnan(x), -math.inf, x).clamp(max=FLT_MAX)
    m, first = x.max(1, keepdim=True)
    first = torch.where(x == m, torch.arange(n, device=x.device), n).amin(1, keepdim=True)
    live = x > -math.inf
    y = torch.where(live, (x - m) * (1.0 / t.clamp(min=TINY, max=FLT_MAX)), -math.inf)
    greedy = ~(t >= TINY)
    here = torch.arange(n, device=x.device) == first
    y = torch.where(greedy, torch.where(here & live, 0.0, -math.inf), y)
    q = (torch.exp(y) * ONE).to(torch.int64)
    if torch.is_tensor(s["k"]) or torch.is_tensor(s["p"]) or s["k"] > 0 or s["p"] < 1:
        order = x.sort(dim=1, descending=True, stable=True)[1]
        qs = q.gather(1, order)
        rank = torch.arange(n, device=x.device)
        qs = torch.where((k <= 0) | (rank < k), qs, 0)
        total = qs.sum(1, keepdim=True)
        before = qs.cumsum(1) - qs
        on = (p < 1)
        qs = torch.where(~on | (before == 0) | (before.double() < p.double() * total.double()), qs, 0)
        q = torch.zeros_like(q).scatter_(1, order, qs)
    q = torch.where(q.double() >= min_p.double().clamp(max=1.0) * ONE, q, 0)
    run = q.cumsum(1)
    total = run[:, -1:]
    target = torch.minimum((u.double() * total.double()).to(torch.int64), total - 1)
    index = torch.searchsorted(run, target, right=True)
    some = (total > 0).expand_as(index)
    at = y.gather(1, index.clamp(max=n - 1))
    logp = torch.where(some, at - torch.log(total.float() / ONE), -math.inf)
    return {"index": torch.where(some, index, -1).to(torch.int32), "logp": logp}


def _plain_loss(s):
    x, index, c = s["x"].float(), s["index"].long(), s["scale"]
    inv = 1.0 / s["case"]["t"]
    n = x.shape[1]
    m = x.amax(1, keepdim=True)
    some = ((index >= 0) & (index < n) & (m[:, 0] > -math.inf))[:, None]
    y = torch.where(some, (x - m) * inv, 0.0)
    e = torch.exp(y)
    total = e.sum(1, keepdim=True)
    at = index.clamp(0, n - 1)[:, None]
    loss = torch.where(some, (torch.log(total) - y.gather(1, at)) * c[:, None], 0.0)[:, 0]
    p = e / total
    p.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
    grad = torch.where(some, p * (c[:, None] * inv), 0.0)
    return {"loss": loss, "grad": grad.to(s["x"].dtype)}


def _spread(out, to, weight, values, at):
    """out[to] += weight values[at], in pieces of columns that bound the temporaries."""
    step = max(1, (1 << 28) // max(1, len(to)))
    for a in range(0, out.shape[1], step):
        out[:, a:a + step].index_add_(0, to, weight[:, None] * values[:, a:a + step][at])
    return out


def _plain_keep(s):
    case = s["case"]
    x = s["x"].t().repeat(case["genomes"], 1)
    state = torch.zeros((s["nodes"], case["patterns"]), device="cuda")
    state[s["in_nodes"]] = x
    kept = []
    for t in range(case["steps"]):
        z = _spread(torch.zeros_like(state), s["dst"], s["w"], state, s["src"])
        state = 1.0 / (1.0 + torch.exp(-z))
        state[s["in_nodes"]] = x
        if t + 1 < case["steps"]:
            codes = torch.round(state * 255.0)
            codes[s["in_nodes"]] = 0
            kept.append(codes.mul_(1.0 / 255.0).to(torch.float16))
    out = state[s["out_nodes"]].reshape(case["genomes"], case["outputs"], -1).transpose(1, 2)
    return {"outputs": out.contiguous(), "kept": torch.stack(kept) if kept else []}


def _plain_back(s):
    case = s["case"]
    G, P = case["genomes"], case["patterns"]
    x = s["x"].t().repeat(G, 1)
    out = s["out"].transpose(1, 2).reshape(-1, P)
    gz = torch.zeros((s["nodes"], P), device="cuda")
    gz[s["out_nodes"]] = s["grad_out"].transpose(1, 2).reshape(-1, P) * out * (1.0 - out)
    grad_w = torch.zeros_like(s["w"])
    grad_x = torch.zeros_like(x)
    step = max(1, (1 << 28) // max(1, len(s["w"])))
    for t in range(case["steps"] - 1, -1, -1):
        if t > 0:
            state = s["codes"][t - 1].float() * (1.0 / 255.0)
        else:
            state = torch.zeros((s["nodes"], P), device="cuda")
        state[s["in_nodes"]] = x
        for a in range(0, P, step):
            grad_w += (gz[:, a:a + step][s["dst"]] * state[:, a:a + step][s["src"]]).sum(1)
        delta = _spread(torch.zeros_like(gz), s["src"], s["w"], gz, s["dst"])
        grad_x += delta[s["in_nodes"]]
        gz = delta * state * (1.0 - state)
        gz[s["in_nodes"]] = 0.0
    if not case["grad_in"]:
        return {"grad_w": grad_w}
    return {"grad_w": grad_w, "grad_x": grad_x.reshape(G, -1, P).transpose(1, 2).contiguous()}


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"sample": _plain_sample, "loss": _plain_loss, "keep": _plain_keep,
                "back": _plain_back}[op](s)
    from paper_2608_27612_amd import emr
    if op == "sample":
        index, logp = emr.emr_sample(s["x"], s["u"], temperature=s["t"], top_k=s["k"], top_p=s["p"],
                                     min_p=s["min_p"])
        return {"index": index, "logp": logp}
    if op == "loss":
        loss, grad = emr.emr_answer_loss(s["x"], s["index"], scale=s["scale"], temperature=case["t"])
        return {"loss": loss, "grad": grad}
    if op == "keep":
        outputs, kept = s["net"].activate_keep(s["x"], case["steps"])
        return {"outputs": outputs, "kept": kept.values(torch.float16) if case["steps"] > 1 else []}
    grad_w, grad_x = s["net"].activate_backward(s["x"], case["steps"], s["out"], s["kept"], s["grad_out"],
                                                grad_inputs=case["grad_in"])
    return {"grad_w": grad_w, "grad_x": grad_x} if case["grad_in"] else {"grad_w": grad_w}


# ----------------------------------------------------------------------------- work

def work(case):
    op = case["op"]
    if op == "sample":
        cells, draws = case["rows"] * case["n"], case["rows"] * case["draws"]
        # a subtraction, a product, an exponential and a sum for each score
        return {"bytes": cells * SIZE[case["type"]] + draws * 12, "flops": 4 * cells}
    if op == "loss":
        cells = case["rows"] * case["n"]
        return {"bytes": 2 * cells * SIZE[case["type"]] + case["rows"] * 12, "flops": 7 * cells}
    e_in, e_hid = _edges(case)
    G, P, T = case["genomes"], case["patterns"], case["steps"]
    hidden = sum(_hidden(case))
    nodes = hidden + G * (case["inputs"] + case["outputs"])
    edges, outs = e_in + e_hid, G * P * case["outputs"]
    rows = P * case["inputs"]
    # The inputs hold still: their edges count once, whatever the steps. Hidden states are 0 before the
    # first step, so the other edges count T - 1 times. A multiplication and an addition each, two
    # products in the backward direction. The states of hidden and output nodes are what is kept.
    kept = (T - 1) * P * (nodes - G * case["inputs"])
    if op == "keep":
        return {"bytes": edges * 8 + nodes * 8 + (rows + outs) * 4 + kept,
                "flops": 2 * P * (e_in + (T - 1) * e_hid) + 4 * P * T * (nodes - G * case["inputs"])}
    grads = edges + (G * rows if case["grad_in"] else 0)
    return {"bytes": edges * 8 + nodes * 8 + (rows + 2 * outs + grads) * 4 + kept,
            "flops": 2 * P * ((2 if case["grad_in"] else 1) * e_in + 2 * (T - 1) * e_hid)}


# ----------------------------------------------------------------------------- 64 bits

def _exact_sample(s):
    """Log-probabilities of the draws; row by row, by thresholds found among the sorted scores."""
    x = s["x"].double().cpu().numpy()
    u = s["u"].double().cpu().numpy()
    rows, n = x.shape
    of = lambda v, r: float(v[r]) if torch.is_tensor(v) else float(np.float32(v))  # noqa: E731
    logp = np.full(u.shape, -np.inf)
    for r in range(rows):
        v = np.minimum(np.where(np.isnan(x[r]), -np.inf, x[r]), FLT_MAX)
        m = v.max()
        if m == -np.inf:
            continue
        t = of(s["t"], r)
        if not t >= TINY:
            logp[r] = 0.0
            continue
        y = (v - m) / min(t, FLT_MAX)
        q = np.floor(np.exp(y) * ONE)
        k, p = int(of(s["k"], r)), of(s["p"], r)
        if k > 0 or p < 1:
            order = np.argsort(-v, kind="stable")
            kept = order[:k] if k > 0 else order
            if p < 1:
                c = np.cumsum(q[kept])
                kept = kept[:1 + int(np.searchsorted(c, p * c[-1], side="left"))]
            left = np.zeros(n)
            left[kept] = q[kept]
            q = left
        q[q < min(of(s["min_p"], r), 1.0) * ONE] = 0
        c = np.cumsum(q)
        i = np.searchsorted(c, np.minimum(np.floor(u[r] * c[-1]), c[-1] - 1), side="right")
        logp[r] = y[i] - np.log(c[-1] / ONE)
    return {"index": None, "logp": torch.from_numpy(logp)}


def _exact_loss(s):
    x, index, c = s["x"].double(), s["index"].long(), s["scale"].double()
    n = x.shape[1]
    some = (index >= 0) & (index < n) & torch.isfinite(x).any(1)
    x = torch.where(some[:, None], x / s["case"]["t"], 0.0)
    logp = x - torch.logsumexp(x, 1, keepdim=True)
    hot = torch.zeros_like(x).scatter_(1, index.clamp(0, n - 1)[:, None], 1.0)
    loss = -logp.gather(1, index.clamp(0, n - 1)[:, None])[:, 0] * c
    grad = (torch.exp(logp) - hot) * (c / s["case"]["t"])[:, None]
    return {"loss": torch.where(some, loss, 0.0), "grad": torch.where(some[:, None], grad, 0.0)}


def _dense(nets, g):
    """Genome g's first node, edge range and [nodes, nodes] matrix of weights, rows by destination."""
    a, b = (int(v) for v in nets["node_offset"][g:g + 2])
    e0, e1 = int(nets["in_offset"][a]), int(nets["in_offset"][b])
    dst = torch.from_numpy(nets["dst"][e0:e1] - a).cuda()
    src = torch.from_numpy(nets["src"][e0:e1].astype(np.int64) - a).cuda()
    m = torch.zeros((b - a, b - a), dtype=torch.float64, device="cuda")
    m[dst, src] = torch.from_numpy(nets["w"][e0:e1]).cuda().double()
    return a, b, e0, e1, dst, src, m


def _exact_keep(case, seed, s):
    nets = _networks(case, seed)
    x = s["x"].double().t()
    G, P, n_in, n_out = case["genomes"], case["patterns"], case["inputs"], case["outputs"]
    out = torch.zeros((G, P, n_out), dtype=torch.float64, device="cuda")
    kept = torch.zeros((case["steps"] - 1, int(nets["node_offset"][-1]), P), dtype=torch.float64,
                       device="cuda") if case["steps"] > 1 else []
    for g in range(G):
        a, b, _, _, _, _, m = _dense(nets, g)
        state = torch.zeros((b - a, P), dtype=torch.float64, device="cuda")
        state[:n_in] = x
        for t in range(case["steps"]):
            state = torch.sigmoid(m @ state)
            state[:n_in] = x
            if t + 1 < case["steps"]:
                kept[t, a + n_in:b] = torch.round(255 * state[n_in:]) / 255
        out[g] = state[n_in:n_in + n_out].t()
    return {"outputs": out, "kept": kept}


def _exact_back(case, seed, s, codes):
    nets = _networks(case, seed)
    x = s["x"].double().t()
    G, P, n_in, n_out, T = (case[k] for k in ("genomes", "patterns", "inputs", "outputs", "steps"))
    grad_w = torch.zeros(len(nets["w"]), dtype=torch.float64, device="cuda")
    grad_x = torch.zeros((G, P, n_in), dtype=torch.float64, device="cuda")
    for g in range(G):
        a, b, e0, e1, dst, src, m = _dense(nets, g)
        gm = torch.zeros_like(m)
        delta = torch.zeros((b - a, P), dtype=torch.float64, device="cuda")
        delta[n_in:n_in + n_out] = s["grad_out"][g].double().t()
        after = torch.zeros_like(delta)
        after[n_in:n_in + n_out] = s["out"][g].double().t()
        for t in range(T, 0, -1):
            before = codes[t - 2, a:b].double() / 255 if t > 1 else torch.zeros_like(delta)
            before[:n_in] = x
            d = delta * after * (1 - after)
            d[:n_in] = 0
            gm += d @ before.t()
            delta = m.t() @ d
            grad_x[g] += delta[:n_in].t()
            after = before
        grad_w[e0:e1] = gm[dst, src]
    return {"grad_w": grad_w, "grad_x": grad_x} if case["grad_in"] else {"grad_w": grad_w}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "sample":
        return _exact_sample(s)
    if case["op"] == "loss":
        return _exact_loss(s)
    if max(_hidden(case)) > 20000:
        return None
    return _exact_keep(case, seed, s) if case["op"] == "keep" else _exact_back(case, seed, s, s["codes"])
