"""Learned inputs, normalised layers and a teacher's logits: what training has the framework do beside its graph layers.

Three operators, each with its gradient:

  norm      y = (x - mean) / sqrt(var + eps) gamma + beta, by rows; backward: gx, and the sums over the rows ggamma and gbeta
  embed     out[i] = scale table[t_i]; backward: gtable[v] = scale sum of g[i] over the i with t_i = v.  A token that pads is a row of
            zeros and has no gradient
  distill   a loss between logits z and the k largest logits t of a teacher, with its gradient:  p = softmax(t / T) over these k,
            q = softmax(z / T), a row's loss is (1 - h) T^2 KL(p || q) + h CE(softmax(z), label), and the gradient that of their mean; an id
            of -1 is no entry, a label of -1 no label

Rows are fp32, bf16 or fp16, their stride a multiple of 16 bytes; parameters and their gradients are fp32.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


def listed():
    return [
        # hidden rows of a unit-test sized network: launches and host time count
        dict(op="norm", name="norm-tiny", back=False, type="f32", rows=2048, d=16),
        # hidden layer of the large co-purchase graph
        dict(op="norm", name="norm-large", back=False, type="f32", rows=612257, d=256),
        # backward on a small graph, a width that is no multiple of anything
        dict(op="norm", name="norm-grad-odd", back=True, type="f32", rows=6000, d=50),
        # backward on the co-purchase graph
        dict(op="norm", name="norm-grad-large", back=True, type="f32", rows=612257, d=256),
        # backward of a wide text layer in 16 bits, a batch of 16 sequences of 1024 tokens
        dict(op="norm", name="norm-grad-text", back=True, type="bf16", rows=16384, d=4096),
        # inputs of a text batch, padded sequences
        dict(op="embed", name="embed-text", back=False, type="bf16", tokens="text", n=32768, vocabulary=32000, d=2048),
        # gradient of learned node types: a handful of rows that every node shares
        dict(op="embed", name="embed-grad-types", back=True, type="f32", tokens="types", n=2048, vocabulary=16, d=32),
        # gradient of a word table from a text batch: few words make up most of it, most words do not occur
        dict(op="embed", name="embed-grad-text", back=True, type="bf16", tokens="text", n=65536, vocabulary=131072, d=1024),
        # gradient of learned node inputs, from the inner rows of all partitions and their halo rows
        dict(op="embed", name="embed-grad-nodes", back=True, type="f32", tokens="nodes", n=1300000, vocabulary=612257, d=100),
        # objective of a unit-test sized network
        dict(op="distill", name="distill-tiny", type="f32", rows=2048, classes=7, k=3, temperature=2.0, hard=0.5),
        # objective of the co-purchase graph: the teacher's eight best classes and the labels
        dict(op="distill", name="distill-nodes", type="f32", rows=612257, classes=47, k=8, temperature=2.0, hard=0.5),
        # a text model's objective, from a stored file of the teacher's 64 best words alone
        dict(op="distill", name="distill-text", type="bf16", rows=8192, classes=50001, k=64, temperature=1.5, hard=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: one row to the nodes of a large graph, narrow layers to wide ones, a few classes to a vocabulary."""
    op = rng.choice(["norm", "norm", "embed", "embed", "distill"])
    back = rng.random() < 0.6
    most = {k: max(work(c)[k] for c in listed() if c["op"] == op and c.get("back", back) == back) for k in ("bytes", "flops")}
    while True:
        case = dict(op=op, type=rng.choice(list(TYPES)))
        if op == "norm":
            case.update(back=back, rows=_log(rng, 1, 610000), d=rng.choice([_log(rng, 8, 8192), rng.randint(16, 640), 64 * rng.randint(1, 16)]))
        elif op == "embed":
            tokens = rng.choice(["types", "text", "nodes"])
            case.update(back=back, tokens=tokens, d=rng.choice([_log(rng, 8, 4096), rng.randint(16, 640), 64 * rng.randint(1, 16)]))
            case["vocabulary"] = _log(rng, 2, 512) if tokens == "types" else _log(rng, 500, 610000)
            case["n"] = case["vocabulary"] + _log(rng, 1, 700000) if tokens == "nodes" else _log(rng, 1, 1000000)
        else:
            classes = rng.choice([rng.randint(3, 112), rng.randint(3, 112), _log(rng, 100, 131072)])
            case.update(rows=_log(rng, 1, 610000), classes=classes, k=min(classes, _log(rng, 1, 128)),
                        temperature=rng.choice([1.0, 1.5, 2.0, 4.0]), hard=rng.choice([0.0, 0.1, 0.5]))
        w = work(case)
        if all(w[k] <= most[k] for k in w):
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------------------
def _padded(rows, d, dtype):
    step = 16 // torch.empty((), dtype=dtype).element_size()
    return torch.zeros((rows, (d + step - 1) // step * step), device="cuda", dtype=dtype)[:, :d]


def _normal(rows, d, dtype, gen, spread):
    """Normal numbers, rows of sizes whose logarithms differ by `spread`."""
    x = _padded(rows, d, dtype)
    x.normal_(generator=gen)
    return x.mul_(torch.exp(spread * torch.randn((rows, 1), device="cuda", generator=gen)).to(dtype))


def _tokens(case, gen):
    n, v = case["n"], case["vocabulary"]
    u = torch.rand(n, device="cuda", generator=gen, dtype=torch.float64)
    if case["tokens"] == "types":
        return (u * v).long().clamp(max=v - 1).int(), -1
    if case["tokens"] == "nodes":           # every node once, partition by partition, then the halo rows: nodes of high degree many times
        few = (v * u[v:] ** 3).long().clamp(max=v - 1)
        return torch.cat([torch.randperm(v, device="cuda", generator=gen), few]).int(), -1
    words = torch.exp(u * math.log(v)).long().clamp(max=v - 1)                  # the i-th word about as often as 1 / i; word 0 pads
    length = min(n, 1024)
    ends = torch.randint(length // 2, length + 1, ((n + length - 1) // length,), device="cuda", generator=gen)
    at = torch.arange(n, device="cuda")
    return torch.where(at % length < ends[at // length], words, 0).int(), 0


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dtype, s = TYPES[case["type"]], dict(case=case)
    if case["op"] == "norm":
        rows, d = case["rows"], case["d"]
        s["x"] = _normal(rows, d, dtype, gen, 0.5)
        s["x"].add_(0.3 * torch.randn((rows, 1), device="cuda", generator=gen).to(dtype))
        s["gamma"] = 1 + 0.1 * torch.randn(d, device="cuda", generator=gen)
        s["beta"] = 0.1 * torch.randn(d, device="cuda", generator=gen)
        if case["back"]:                                                        # the forward pass has left the rows' statistics
            s["g"] = _normal(rows, d, dtype, gen, 1.0)
            s["mean"] = torch.empty(rows, device="cuda")
            s["rstd"] = torch.empty(rows, device="cuda")
            for i in range(0, rows, 65536):
                x = s["x"][i:i + 65536].double()
                s["mean"][i:i + 65536] = x.mean(1)
                s["rstd"][i:i + 65536] = 1 / torch.sqrt(x.var(1, unbiased=False) + EPS)
    elif case["op"] == "embed":
        s["tokens"], s["padding"] = _tokens(case, gen)
        s["scale"] = math.sqrt(case["d"]) if case["tokens"] == "text" else 1.0
        if case["back"]:
            s["g"] = _normal(case["n"], case["d"], dtype, gen, 1.0)
        else:
            s["table"] = _normal(case["vocabulary"], case["d"], dtype, gen, 0.0).mul_(case["d"] ** -0.5)
    else:
        rows, classes, k = case["rows"], case["classes"], case["k"]
        s["z"] = _normal(rows, classes, dtype, gen, 0.3)
        step = classes // k                                                     # k different classes a row
        first = torch.randint(0, classes, (rows, 1), device="cuda", generator=gen)
        at = torch.arange(k, device="cuda") * step
        s["ids"] = ((first + at + torch.randint(0, step, (rows, k), device="cuda", generator=gen)) % classes).int()
        s["logits"] = 2 * torch.randn((rows, k), device="cuda", generator=gen).sort(1, descending=True)[0]
        s["ids"][torch.rand(rows, device="cuda", generator=gen) < 0.01, k // 2:] = -1   # some rows came with fewer (k = 1: with none)
        s["labels"] = None
        if case["hard"] > 0:
            s["labels"] = s["ids"][:, 0].clamp(min=0).clone()
            s["labels"][torch.rand(rows, device="cuda", generator=gen) < 0.3] = -1      # nodes without a label
    return s


def _weight(case):
    """Of a row: the mean, times what a training run in fp16 scales its loss by."""
    return (2.0 ** 14 if case["type"] == "f16" else 1.0) / case["rows"]


# ---- one pass ---------------------------------------------------------------------------------------------------------------
_handle = None


def _library():
    """The binding and a context on the current stream, kept as a program keeps them."""
    global _handle
    import paper_2308_13466_b200.binding as B
    if _handle is None:
        _handle = B.sat_create(0, torch.cuda.current_stream().cuda_stream)
    return B, _handle


def _run_own(s):
    B, ctx = _library()
    case = s["case"]
    if case["op"] == "norm":
        if not case["back"]:
            if "y" not in s:
                s["y"] = _padded(*s["x"].shape, s["x"].dtype)
                s["mean"], s["rstd"] = (torch.empty(case["rows"], device="cuda") for _ in range(2))
            B.sat_layernorm_fwd(ctx, s["x"], s["gamma"], s["beta"], EPS, s["y"], s["mean"], s["rstd"])
            return dict(y=s["y"], mean=s["mean"], rstd=s["rstd"])
        if "gx" not in s:
            s["gx"] = _padded(*s["x"].shape, s["x"].dtype)
            s["ggamma"], s["gbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["beta"])
        B.sat_layernorm_bwd(ctx, s["x"], s["g"], s["gamma"], s["mean"], s["rstd"], s["gx"], s["ggamma"], s["gbeta"])
        return dict(gx=s["gx"], ggamma=s["ggamma"], gbeta=s["gbeta"])
    if case["op"] == "embed":
        if not case["back"]:
            if "out" not in s:
                s["out"] = _padded(case["n"], case["d"], s["table"].dtype)
            B.sat_embed_fwd(ctx, s["tokens"], s["table"], s["scale"], s["padding"], s["out"])
            return s["out"]
        if "order" not in s:                                                    # room for the order, which every pass works out anew
            s["order"] = B.new_token_order(case["n"], case["vocabulary"])
            s["gtable"] = _padded(case["vocabulary"], case["d"], torch.float32)
        B.sat_token_sort(ctx, s["tokens"], s["padding"], s["order"])
        B.sat_embed_bwd(ctx, s["order"], s["g"], s["scale"], s["gtable"])
        return s["gtable"]
    if "gz" not in s:
        s["gz"], s["loss"] = _padded(*s["z"].shape, s["z"].dtype), torch.empty(case["rows"], device="cuda")
    B.sat_distill_grad(ctx, s["z"], s["ids"], s["logits"], case["temperature"], case["hard"], s["labels"], None, _weight(case), None, s["gz"], s["loss"])
    return dict(loss=s["loss"], g=s["gz"])


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    if case["op"] == "norm":
        x = s["x"].float()
        if not case["back"]:
            mean = x.mean(1, keepdim=True)
            x = x - mean
            rstd = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
            return dict(y=(x * rstd * s["gamma"] + s["beta"]).to(s["x"].dtype), mean=mean[:, 0], rstd=rstd[:, 0])
        xh = (x - s["mean"][:, None]) * s["rstd"][:, None]
        g = s["g"].float()
        ggamma, gbeta = (g * xh).sum(0), g.sum(0)
        u = g * s["gamma"]
        gx = s["rstd"][:, None] * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
        return dict(gx=gx.to(s["x"].dtype), ggamma=ggamma, gbeta=gbeta)
    if case["op"] == "embed":
        there = s["tokens"] != s["padding"]
        if not case["back"]:
            rows = s["table"][s["tokens"].long()].float() * s["scale"]
            return torch.where(there[:, None], rows, 0.0).to(s["table"].dtype)
        rows = torch.where(there[:, None], s["g"].float() * s["scale"], 0.0)
        return torch.zeros((case["vocabulary"], case["d"]), device="cuda").index_add_(0, s["tokens"].long(), rows)
    return _distill(s)


def _distill(s):
    case, T, h = s["case"], s["case"]["temperature"], s["case"]["hard"]
    z, ids, t = s["z"].float(), s["ids"].long(), s["logits"]
    there = ids >= 0
    some = there.any(1, keepdim=True).float()                                   # without an entry there is nothing to learn from the teacher
    at = ids.clamp(min=0)
    v = z - z.amax(1, keepdim=True)
    t = t - torch.where(there, t, -math.inf).amax(1, keepdim=True)
    e = torch.where(there, torch.exp(t / T), 0.0)
    total = e.sum(1, keepdim=True) + (1 - some)
    p = e / total
    q = torch.exp(v / T)
    sq = q.sum(1, keepdim=True)
    logs = torch.where(there, t - v.gather(1, at), 0.0) / T
    loss = (1 - h) * T * T * ((p * logs).sum(1) + some[:, 0] * torch.log(sq[:, 0]) - torch.log(total[:, 0]))
    g = (1 - h) * T * some * (q / sq)
    g.scatter_add_(1, at, -(1 - h) * T * p)
    if h > 0:
        labelled = s["labels"] >= 0
        y = s["labels"].long().clamp(min=0)[:, None]
        q = torch.exp(v)
        sq = q.sum(1, keepdim=True)
        loss = loss + torch.where(labelled, h * (torch.log(sq) - v.gather(1, y))[:, 0], 0.0)
        g += torch.where(labelled[:, None], h * q / sq, 0.0)
        g.scatter_add_(1, y, torch.where(labelled[:, None], -h, 0.0))
    return dict(loss=loss, g=(g * _weight(case)).to(s["z"].dtype))


def work(case):
    """Inputs once and outputs once; of a table that is looked up, what a batch can touch of it."""
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "norm":
        rows, d = case["rows"], case["d"]
        if case["back"]:
            return {"bytes": 3 * size * rows * d + 8 * rows + 12 * d, "flops": 14 * rows * d}
        return {"bytes": 2 * size * rows * d + 8 * rows + 8 * d, "flops": 8 * rows * d}
    if case["op"] == "embed":
        n, v, d = case["n"], case["vocabulary"], case["d"]
        if case["back"]:
            return {"bytes": 4 * n + size * n * d + 4 * v * d, "flops": n * d}
        return {"bytes": 4 * n + size * (n + min(n, v)) * d, "flops": n * d}
    rows, c, k = case["rows"], case["classes"], case["k"]
    return {"bytes": rows * (2 * size * c + 8 * k + (4 if case["hard"] > 0 else 0)), "flops": rows * ((12 if case["hard"] > 0 else 6) * c + 10 * k)}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"].double()
        if not case["back"]:
            var, mean = torch.var_mean(x, 1, unbiased=False)
            rstd = (var + EPS) ** -0.5
            return dict(y=torch.addcmul(s["beta"].double(), (x - mean[:, None]) * rstd[:, None], s["gamma"].double()), mean=mean, rstd=rstd)
        g, mean, rstd = s["g"].double(), s["mean"].double()[:, None], s["rstd"].double()[:, None]
        x = (x - mean).mul_(rstd)
        ggamma, gbeta = torch.einsum("rd,rd->d", g, x), torch.ones(len(g), dtype=torch.float64, device="cuda") @ g
        g.mul_(s["gamma"].double())
        along = torch.einsum("rd,rd->r", g, x)[:, None] / case["d"]
        g.sub_(g.sum(1, keepdim=True) / case["d"]).sub_(x.mul_(along)).mul_(rstd)
        return dict(gx=g, ggamma=ggamma, gbeta=gbeta)
    if case["op"] == "embed":
        tokens = s["tokens"].long()
        if not case["back"]:
            keep = (tokens != s["padding"]).double() * s["scale"]
            return torch.index_select(s["table"].double(), 0, tokens).mul_(keep[:, None])
        order = torch.argsort(tokens, stable=True)                              # sums by token as differences of running sums
        sums = torch.cumsum(s["g"].double()[order] * s["scale"], 0)
        sums = torch.cat([torch.zeros_like(sums[:1]), sums])
        ends = torch.searchsorted(tokens[order].contiguous(), torch.arange(case["vocabulary"] + 1, device="cuda"))
        got = sums[ends[1:]] - sums[ends[:-1]]
        got[torch.diff(ends) == 0] = 0.0
        if s["padding"] >= 0:
            got[s["padding"]] = 0.0
        return got
    T, h, rows = case["temperature"], case["hard"], case["rows"]
    loss, g = [], []
    step = max(1, 2 ** 28 // case["classes"])
    for i in range(0, rows, step):
        z = s["z"][i:i + step].double().requires_grad_()
        ids = s["ids"][i:i + step].long()
        t = torch.where(ids >= 0, s["logits"][i:i + step].double() / T, -1e9).log_softmax(1)    # (rows without an entry: any numbers)
        logq = (z / T).log_softmax(1).gather(1, ids.clamp(min=0))
        part = (1 - h) * T * T * torch.where(ids >= 0, t.exp() * (t - logq), 0.0).sum(1)
        if h > 0:
            y = s["labels"][i:i + step].long()
            part = part + h * torch.where(y >= 0, -z.log_softmax(1).gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
        (part.sum() * _weight(case)).backward()
        loss.append(part.detach())
        g.append(z.grad)
    return dict(loss=torch.cat(loss), g=torch.cat(g))
