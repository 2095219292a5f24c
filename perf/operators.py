"""Cases for timing the learned-policy operators: distillation from the exact placement rule's best
hosts, the load-balance loss with per-host counts, and sampling hosts from a policy's logits.

A policy scores every host for every request: logits [rows, hosts], -inf where the host cannot take the
request. `run` goes through one operator, in plain torch operations (32 bits, rounded once at the end)
or, with `own` set, through the library's entry points.
"""
import math

import torch

own = False

NEG_INF = float("-inf")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEMENT_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
WEIGHT_ONE = 2.0 ** 31        # sampling weight of a row's best host
UNIFORM_STEPS = 2 ** 24       # steps of a random number or a top-p share
MIN_TEMPERATURE = 2.0 ** -20  # at and below it the best host is taken


def listed():
    return [
        # one small decision batch on a tiny cluster, trained on as it arrives: latency
        dict(name="distill_step_1024x32_f32", op="distill", mode="step", groups=1, rows=1024, hosts=32,
             k=3, temperature=1.0, dtype="f32"),
        # the ordinary training step: a medium cluster's batch, the rule's three best as teacher
        dict(name="distill_step_16384x256_bf16", op="distill", mode="step", groups=1, rows=16384, hosts=256,
             k=3, temperature=2.0, dtype="bf16"),
        # a day's requests against the heavily oversubscribed cluster: bandwidth
        dict(name="distill_step_262144x1024_bf16", op="distill", mode="step", groups=1, rows=262144, hosts=1024,
             k=3, temperature=1.0, dtype="bf16"),
        # held-out loss on a cluster of an odd size, a larger policy's 32 best logits as teacher, no gradient
        dict(name="distill_eval_8191x4099_f16", op="distill", mode="eval", groups=1, rows=8191, hosts=4099,
             k=32, temperature=1.5, dtype="f16"),
        # few requests, very large cluster, through autograd (forward, then backward with the saved statistics)
        dict(name="distill_autograd_48x65536_f32", op="distill", mode="autograd", groups=1, rows=48, hosts=65536,
             k=16, temperature=1.0, dtype="f32"),
        # the balance term of the tiny cluster's step: latency
        dict(name="balance_step_1x1024x32_f32", op="balance", mode="step", groups=1, rows=1024, hosts=32,
             k=3, temperature=1.0, dtype="f32"),
        # odd sizes, rows that start at any 2-byte offset
        dict(name="balance_step_1x16385x257_f16", op="balance", mode="step", groups=1, rows=16385, hosts=257,
             k=3, temperature=1.0, dtype="f16"),
        # watching the load of a large cluster: loss, counts and mean shares, no gradient
        dict(name="balance_eval_1x65536x4096_bf16", op="balance", mode="eval", groups=1, rows=65536, hosts=4096,
             k=3, temperature=1.0, dtype="bf16"),
        # the what-if sweep: 256 independent clusters in one call, each with its own balance
        dict(name="balance_step_256x4096x1024_bf16", op="balance", mode="step", groups=256, rows=4096, hosts=1024,
             k=3, temperature=1.0, dtype="bf16"),
        # one request at a time against the largest cluster: latency of a long row
        dict(name="sample_1x65536_f32", op="sample", mode="all", groups=1, rows=1, hosts=65536,
             k=3, temperature=0.8, dtype="f32"),
        # three replicas for each of a medium batch, all filters at once, a setting of its own for every row
        dict(name="sample_16384x4096_bf16", op="sample", mode="all", groups=1, rows=16384, hosts=4096,
             k=3, temperature=0.9, dtype="bf16"),
        # exploration over the oversubscribed cluster: no top-k, a wide nucleus, one draw
        dict(name="sample_nucleus_262144x1024_bf16", op="sample", mode="nucleus", groups=1, rows=262144, hosts=1024,
             k=1, temperature=1.0, dtype="bf16"),
    ]


def draw(rng):
    op = rng.choice(["distill", "distill", "balance", "balance", "sample", "sample"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    most = {"distill": 2 ** 28, "balance": 2 ** 29, "sample": 2 ** 27}[op]

    def spread(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.4:
            v -= v % 32 if v >= 64 else 0
        return max(lo, min(hi, v))

    hosts = spread(32, 65536)
    groups = spread(1, 256) if op == "balance" and rng.random() < 0.5 else 1
    rows = spread(1, max(1, min(262144, most // (hosts * groups))))
    if op == "distill":
        mode, k = rng.choice(["step", "step", "eval", "autograd"]), rng.choice([1, 3, 3, 8, 32, 64])
    elif op == "balance":
        mode, k = rng.choice(["step", "step", "eval"]), rng.choice([1, 2, 3, 3, 8])
    else:
        mode, k = rng.choice(["all", "nucleus", "plain"]), rng.choice([1, 3, 3])
    return dict(op=op, mode=mode, groups=groups, rows=rows, hosts=hosts, k=min(k, hosts),
                temperature=rng.choice([0.7, 1.0, 1.0, 1.5, 2.0]), dtype=dtype)


def grad_scale(case):
    """What the gradient is multiplied by: the mean over the rows for distillation, 1 for the balance loss; in
    f16 with the loss scale that training in that type keeps, so that gradients stay among its normal numbers."""
    if case["dtype"] == "f16":
        return 1024.0 if case["op"] == "distill" else 1024.0 * case["rows"] / case["hosts"]
    return 1.0 / case["rows"] if case["op"] == "distill" else 1.0


def work(case):
    rows = case["groups"] * case["rows"]
    table = rows * case["hosts"] * ELEMENT_BYTES[case["dtype"]]
    elements = rows * case["hosts"]
    if case["op"] == "sample":
        # logits and random numbers in, four settings per row in, hosts and their number out
        return {"bytes": table + rows * (4 * case["k"] + 16 + 4 * case["k"] + 4), "flops": 4 * elements}
    gradient = case["mode"] != "eval"
    if case["op"] == "distill":
        # logits, ids and teacher logits in, loss out, gradient out
        return {"bytes": table * (2 if gradient else 1) + rows * (8 * case["k"] + 4),
                "flops": elements * (7 if gradient else 4)}
    # logits and ids in, loss, counts and mean shares out, gradient out
    return {"bytes": table * (2 if gradient else 1) + rows * 4 * case["k"] + case["groups"] * (8 * case["hosts"] + 4),
            "flops": elements * (9 if gradient else 5)}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _logits(gen, case):
    """A policy's scores: about a tenth of the hosts cannot take a request (-inf), about one request in
    200 fits nowhere."""
    rows, hosts = case["groups"] * case["rows"], case["hosts"]
    out = torch.empty((rows, hosts), dtype=DTYPES[case["dtype"]], device="cuda")
    step = max(1, min(rows, 2 ** 27 // hosts))
    for r in range(0, rows, step):
        part = out[r:r + step]
        x = torch.randn(part.shape, generator=gen, device="cuda").mul_(2.5)
        x.masked_fill_(torch.rand(part.shape, generator=gen, device="cuda") < 0.1, NEG_INF)
        if rows > 1:
            x.masked_fill_(torch.rand((part.shape[0], 1), generator=gen, device="cuda") < 0.005, NEG_INF)
        part.copy_(x)
    return out


def _chosen(gen, logits, k):
    """k distinct hosts per row, some hosts chosen far more often than others, -1 where the host is out."""
    rows, hosts = logits.shape
    first = (torch.rand((rows, 1), generator=gen, device="cuda").square_() * hosts).long().clamp_(max=hosts - 1)
    ids = (first + torch.arange(k, device="cuda") * max(1, hosts // k)) % hosts
    return torch.where(logits.gather(1, ids) == NEG_INF, -1, ids).int()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    groups, rows, hosts, k = case["groups"], case["rows"], case["hosts"], case["k"]
    total = groups * rows
    s = {"case": case, "logits": _logits(gen, case)}
    if case["op"] == "sample":
        s["uniforms"] = torch.rand((total, k), generator=gen, device="cuda")
        s["temperature"] = torch.rand(total, generator=gen, device="cuda").mul_(0.4).add_(case["temperature"] - 0.2)
        s["top_k"] = s["top_p"] = s["min_p"] = None
        if case["mode"] != "plain":
            s["top_p"] = torch.rand(total, generator=gen, device="cuda").mul_(0.2).add_(0.79)
        if case["mode"] == "all":
            s["top_k"] = torch.randint(1, 101, (total,), generator=gen, device="cuda", dtype=torch.int32)
            s["min_p"] = torch.rand(total, generator=gen, device="cuda").mul_(0.05)
        s["out_hosts"] = torch.empty((total, k), dtype=torch.int32, device="cuda")
        s["out_found"] = torch.empty((total,), dtype=torch.int32, device="cuda")
        return s
    s["hosts"] = _chosen(gen, s["logits"], k)
    if case["op"] == "distill":
        # the teacher's scores fall from its best host to its last
        s["teacher"] = torch.randn((total, k), generator=gen, device="cuda").abs_().cumsum_(1).neg_().add_(4.0)
        s["loss"] = torch.empty((total,), device="cuda")
        if case["mode"] == "autograd":
            s["logits"].requires_grad_(True)
    else:
        s["logits"] = s["logits"].view(groups, rows, hosts)
        s["hosts"] = s["hosts"].view(groups, rows, k)
        s["loss"] = torch.empty((groups,), device="cuda")
        s["counts"] = torch.empty((groups, hosts), dtype=torch.int32, device="cuda")
        s["shares"] = torch.empty((groups, hosts), device="cuda")
    if case["mode"] == "step":
        s["grad"] = torch.empty_like(s["logits"])
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _plain_distill(s):
    case = s["case"]
    temperature, dtype = case["temperature"], s["logits"].dtype
    x = s["logits"].detach().float()
    rows, hosts = x.shape
    inside = (s["hosts"] >= 0) & (s["hosts"] < hosts)
    ids = torch.where(inside, s["hosts"], 0).long()
    at = x.gather(1, ids)
    there = inside & (at > NEG_INF) & (s["teacher"] > NEG_INF)
    some = there.any(1, keepdim=True)

    t = torch.where(there, s["teacher"] / temperature, NEG_INF)
    t = t - torch.where(some, t.amax(1, keepdim=True), 0.0)
    total = torch.where(some, t.exp().sum(1, keepdim=True), 1.0)
    q = t.exp() / total

    top = x.amax(1, keepdim=True)
    alive = top > NEG_INF
    top = torch.where(alive, top, 0.0)
    e = ((x - top) / temperature).exp()
    sum_e = torch.where(alive, e.sum(1, keepdim=True), 1.0)
    log_ratio = (t - total.log()) - ((at - top) / temperature - sum_e.log())
    loss = temperature ** 2 * torch.where(there, q * log_ratio, 0.0).sum(1)
    if case["mode"] == "eval":
        return {"loss": loss}
    grad = e.div_(sum_e).mul_(some.float())
    grad.scatter_add_(1, ids, torch.where(there, -q, 0.0))
    return {"loss": loss, "grad": grad.mul_(temperature * grad_scale(case)).to(dtype)}


def _plain_balance(s):
    case = s["case"]
    x = s["logits"].float()
    groups, rows, hosts = x.shape
    inside = (s["hosts"] >= 0) & (s["hosts"] < hosts)
    counts = torch.zeros((groups, hosts), dtype=torch.int32, device=x.device)
    ids = torch.where(inside, s["hosts"], 0).long()
    counts.scatter_add_(1, ids.view(groups, -1), inside.int().view(groups, -1))
    live = inside.any(2, keepdim=True).float()
    n_live = live.sum(1, keepdim=True).clamp(min=1.0)
    f = counts.float() / counts.sum(1, keepdim=True).clamp(min=1).float()

    top = x.amax(2, keepdim=True)
    alive = top > NEG_INF
    e = (x - torch.where(alive, top, 0.0)).exp()
    p = e.div_(torch.where(alive, e.sum(2, keepdim=True), 1.0)).mul_(live)
    shares = (p / n_live).sum(1)
    loss = hosts * (f * shares).sum(1)
    out = {"loss": loss, "counts": counts, "shares": shares}
    if case["mode"] == "step":
        dot = (p * f[:, None, :]).sum(2, keepdim=True)
        out["grad"] = (f[:, None, :] - dot).mul_(p).mul_(grad_scale(case) * hosts / n_live).to(s["logits"].dtype)
    return out


def _steps(total, share):
    """floor(total * share / 2^24) for a whole-numbered share of 2^24, without leaving 63 bits."""
    return share * (total >> 24) + ((share * (total & (UNIFORM_STEPS - 1))) >> 24)


def _plain_sample(s):
    x = s["logits"].float()
    rows, hosts = x.shape
    x = torch.where(torch.isnan(x), NEG_INF, x).clamp(max=torch.finfo(torch.float32).max)
    top = x.amax(1, keepdim=True)
    alive = top > NEG_INF
    greedy = ~(s["temperature"][:, None] > MIN_TEMPERATURE)
    temperature = torch.where(greedy, 1.0, s["temperature"][:, None])
    scale = torch.full_like(temperature, math.log2(math.e)) / temperature
    weight = (torch.exp2((x - torch.where(alive, top, 0.0)) * scale) * WEIGHT_ONE).long()

    # best first, ties to the lowest index; what stays is a first part of that order
    _, order = x.sort(dim=1, descending=True, stable=True)
    place = torch.arange(hosts, device=x.device)
    weight = weight.gather(1, order)
    stays = ~greedy | (place == 0)
    if s["top_k"] is not None:
        k = s["top_k"][:, None].long()
        stays &= (place < k) | (k <= 0)
    weight *= stays
    if s["top_p"] is not None:
        p = s["top_p"][:, None]
        share = (p.clamp(0.0, 1.0) * UNIFORM_STEPS).long()
        limit = _steps(weight.sum(1, keepdim=True), share).clamp(min=1)
        stays = (weight.cumsum(1) - weight < limit) | ~(p < 1.0)
    if s["min_p"] is not None:
        stays &= weight >= (s["min_p"][:, None].clamp(0.0, 1.0) * WEIGHT_ONE).long()
    weight = torch.empty_like(weight).scatter_(1, order, weight * stays)

    drawn = []
    steps = (s["uniforms"].clamp(0.0, 1.0) * UNIFORM_STEPS).long().clamp(max=UNIFORM_STEPS - 1)
    for d in range(steps.shape[1]):
        running = weight.cumsum(1)
        left = running[:, -1:]
        host = (running <= _steps(left, steps[:, d:d + 1])).sum(1, keepdim=True)
        host = torch.where(left > 0, host, -1)
        drawn.append(host)
        weight.scatter_(1, host.clamp(min=0), 0)
    hosts_out = torch.cat(drawn, 1).int()
    return {"hosts": hosts_out, "found": (hosts_out >= 0).sum(1).int()}


# ---- the library's calls --------------------------------------------------------------------------------------------
def _own(s):
    from paper_2503_20591_b200 import binding, policy

    case = s["case"]
    if case["op"] == "sample":
        binding.nbos_policy_sample(s["logits"], s["uniforms"], s["out_hosts"], s["out_found"],
                                   temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return {"hosts": s["out_hosts"], "found": s["out_found"]}
    if case["op"] == "balance":
        grad = s.get("grad")
        binding.nbos_policy_balance(s["logits"], s["hosts"], s["loss"], s["counts"], s["shares"],
                                    grad_scale=grad_scale(case), out_grad=grad)
        out = {"loss": s["loss"], "counts": s["counts"], "shares": s["shares"]}
        return out if grad is None else dict(out, grad=grad)
    if case["mode"] == "autograd":
        loss = policy.distill_loss(s["logits"], s["hosts"], s["teacher"], temperature=case["temperature"])
        grad, = torch.autograd.grad(loss.sum() * grad_scale(case), s["logits"])
        return {"loss": loss.detach(), "grad": grad}
    grad = s.get("grad")
    binding.nbos_policy_distill(s["logits"], s["hosts"], s["teacher"], s["loss"], temperature=case["temperature"],
                                grad_scale=grad_scale(case), out_grad=grad)
    return {"loss": s["loss"]} if grad is None else {"loss": s["loss"], "grad": grad}


def run(state):
    if own:
        return _own(state)
    return {"distill": _plain_distill, "balance": _plain_balance, "sample": _plain_sample}[state["case"]["op"]](state)


# ---- 64 bits --------------------------------------------------------------------------------------------------------
def _softmax64(x):
    """Row softmax and its logarithm in 64 bits; a row without a finite entry has neither."""
    lse = torch.logsumexp(x, -1, keepdim=True)
    log_p = torch.where(lse == NEG_INF, NEG_INF, x - lse)
    return log_p.exp(), log_p


def _exact_distill(case, s, a, b):
    x = s["logits"].detach()[a:b].double() / case["temperature"]
    ids = s["hosts"][a:b].long()
    inside = (ids >= 0) & (ids < case["hosts"])
    ids = ids * inside
    p, log_p = _softmax64(x)
    at = log_p.gather(1, ids)
    there = inside & (at != NEG_INF)
    q, log_q = _softmax64(torch.where(there, s["teacher"][a:b].double() / case["temperature"], NEG_INF))
    loss = case["temperature"] ** 2 * torch.where(q > 0, q * (log_q - at), 0.0).sum(1)
    if case["mode"] == "eval":
        return loss, None
    p = p * there.any(1, keepdim=True)
    p.scatter_add_(1, ids, -q)
    return loss, p * (case["temperature"] * grad_scale(case))


def _exact_balance(case, s, g):
    x, ids, n = s["logits"][g].double(), s["hosts"][g].long(), case["hosts"]
    inside = (ids >= 0) & (ids < n)
    counts = torch.bincount(ids[inside], minlength=n)
    live = inside.any(1)
    n_live, f = max(1, int(live.sum())), counts.double() / max(1, int(counts.sum()))
    p = _softmax64(x)[0] * live[:, None]
    shares = p.sum(0) / n_live
    grad = None
    if case["mode"] == "step":
        grad = (grad_scale(case) * n / n_live) * p * (f - (p @ f)[:, None])
    return n * (f @ shares), counts.int(), shares, grad


def exact(case, seed):
    # sampling answers in whole numbers; the largest sweep's gradient does not fit the time in 64 bits
    if case["op"] == "sample" or case["groups"] * case["rows"] * case["hosts"] > 2 ** 28:
        return None
    s = prepare(case, seed)
    if case["op"] == "distill":
        step = max(1, 2 ** 26 // case["hosts"])
        parts = [_exact_distill(case, s, a, min(a + step, case["rows"])) for a in range(0, case["rows"], step)]
        out = {"loss": torch.cat([p[0] for p in parts])}
        if case["mode"] != "eval":
            out["grad"] = torch.cat([p[1] for p in parts])
        return out
    parts = [_exact_balance(case, s, g) for g in range(case["groups"])]
    out = {k: torch.stack([p[i] for p in parts]) for i, k in enumerate(("loss", "counts", "shares"))}
    if case["mode"] == "step":
        out["grad"] = torch.stack([p[3] for p in parts])
    return out
