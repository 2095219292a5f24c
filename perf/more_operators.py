"""Cases for timing the operators of a two-tower policy's training step: distillation on the scores of two towers
without the table of scores, the norms around a tower's residual block, and clipping by the global gradient norm.

A two-tower policy scores host h for request r as the product of two vectors, -inf where the request does not
fit the host (four whole-numbered asks against four of room). `run` goes through one operator, in plain torch
operations (32 bits, rounded once at the end) or, with `own` set, through the library's entry points.
"""
import math

import torch

own = False

NEG_INF = float("-inf")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEMENT_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6   # of the norms, and beside the gradient norm


def listed():
    return [
        # the small policy's ordinary step: 16 snapshots of 256 hosts, 512 requests each, vectors of 64: latency
        dict(name="towers_step_16x512x256_w64_bf16", op="towers", mode="step", groups=16, rows=512, hosts=256,
             width=64, k=3, temperature=1.0, mask=True, dtype="bf16"),
        # few requests against the largest cluster: one long row of hosts for each, through autograd
        dict(name="towers_autograd_1x48x65536_w128_f16", op="towers", mode="autograd", groups=1, rows=48, hosts=65536,
             width=128, k=16, temperature=1.0, mask=False, dtype="f16"),
        # held-out loss: odd sizes, rows that no wide load can start at, a larger policy's 32 best as teacher
        dict(name="towers_eval_1x4099x10007_w301_f16", op="towers", mode="eval", groups=1, rows=4099, hosts=10007,
             width=301, k=32, temperature=1.5, mask=True, dtype="f16"),
        # a day's requests against the medium cluster: matrix products and exponentials weigh the same
        dict(name="towers_step_1x65536x4096_w256_bf16", op="towers", mode="step", groups=1, rows=65536, hosts=4096,
             width=256, k=3, temperature=2.0, mask=True, dtype="bf16"),
        # a vocabulary's worth of hosts and wide vectors, one label a row: matrix products
        dict(name="towers_step_1x8192x65536_w1024_bf16", op="towers", mode="step", groups=1, rows=8192, hosts=65536,
             width=1024, k=1, temperature=1.0, mask=False, dtype="bf16"),
        # one request is served: a single row between two blocks
        dict(name="block_eval_1x1_w4096_bf16", op="block", mode="eval", groups=1, rows=1, width=4096, gate="width",
             dtype="bf16"),
        # a block of the small policy's request tower, each snapshot with its gate
        dict(name="block_step_16x512_w64_f32", op="block", mode="step", groups=16, rows=512, width=64, gate="group",
             dtype="f32"),
        # odd sizes, every row with a gate of its own
        dict(name="block_step_1x4099_w2050_f16", op="block", mode="step", groups=1, rows=4099, width=2050, gate="row",
             dtype="f16"),
        # a large batch through autograd: bandwidth
        dict(name="block_autograd_8x8192_w2048_bf16", op="block", mode="autograd", groups=8, rows=8192, width=2048,
             gate="group", dtype="bf16"),
        # the small policy's sixteen weights and biases: latency
        dict(name="clip_16_tensors_w64_f32", op="clip", tensors=16, largest=4096, clip=True, dtype="f32"),
        # a mixed model: weights in bf16, norms and biases in f32, sizes from one value to millions
        dict(name="clip_400_tensors_mixed", op="clip", tensors=400, largest=2 ** 22 + 3, clip=True, dtype="mixed"),
        # a large model's gradients: far more than the caches hold
        dict(name="clip_48_tensors_bf16", op="clip", tensors=48, largest=2 ** 26, clip=True, dtype="bf16"),
    ]


def draw(rng):
    op = rng.choice(["towers", "towers", "block", "block", "clip"])

    def spread(lo, hi):
        v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
        if rng.random() < 0.5:
            v -= v % 32 if v >= 64 else 0
        return max(lo, min(hi, v))

    if op == "towers":
        width, hosts = spread(16, 1024), spread(32, 65536)
        groups = spread(1, 16) if rng.random() < 0.4 else 1
        most = min(2 ** 39 // (hosts * width * groups), 2 ** 29 // (hosts * groups), 262144)
        rows = spread(1, max(1, most))
        return dict(op=op, mode=rng.choice(["step", "step", "eval", "autograd"]), groups=groups, rows=rows,
                    hosts=hosts, width=width, k=min(hosts, rng.choice([1, 3, 3, 16, 32])),
                    temperature=rng.choice([0.7, 1.0, 1.0, 2.0]), mask=rng.random() < 0.5,
                    dtype=rng.choice(["bf16", "bf16", "f16"]))
    if op == "block":
        width = spread(16, 8192)
        groups = spread(1, 64) if rng.random() < 0.6 else 1
        rows = spread(1, max(1, 2 ** 27 // (width * groups)))
        return dict(op=op, mode=rng.choice(["step", "step", "eval", "autograd"]), groups=groups, rows=rows, width=width,
                    gate=rng.choice(["none", "width", "group", "row"]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
    tensors = spread(1, 500)
    return dict(op=op, tensors=tensors, largest=spread(64, max(64, min(2 ** 26, 2 ** 30 // tensors))),
                clip=rng.random() < 0.8, dtype=rng.choice(["f32", "bf16", "f16", "mixed"]))


def grad_scale(case):
    """What the loss is multiplied by: its mean over the rows, in f16 the loss scale that training in that type keeps."""
    return 1024.0 if case["dtype"] == "f16" else 1.0 / (case["groups"] * case["rows"])


def _sizes(case):
    """(numel, type) of each tensor of a clipping case: a large one, then ever smaller ones, and small ones between."""
    out = []
    for i in range(case["tensors"]):
        small = i % 3 == 2
        n = max(1, case["largest"] // (61 + 7 * i) if small else case["largest"] // (1 + i // 12))
        dtype = case["dtype"] if case["dtype"] != "mixed" else ("f32" if small else "bf16")
        out.append((n, dtype))
    return out


def work(case):
    if case["op"] == "clip":
        total = sum(n * ELEMENT_BYTES[t] for n, t in _sizes(case))
        return {"bytes": 2 * total + 4, "flops": 3 * sum(n for n, _ in _sizes(case))}
    e, rows, width = ELEMENT_BYTES[case["dtype"]], case["groups"] * case["rows"], case["width"]
    gradient = case["mode"] != "eval"
    if case["op"] == "block":
        table, gates = rows * width * e, {"none": 0, "width": 1, "group": case["groups"], "row": rows}[case["gate"]] * width * e
        # residual, branch, gate and two weights in, both results out; then the two gradients in, those of all five out
        step = 4 * table + 2 * gates + 16 * width if gradient else 0
        return {"bytes": 4 * table + gates + 8 * width + step, "flops": rows * width * (30 if gradient else 10)}
    vectors = (rows + case["groups"] * case["hosts"]) * width * e
    mask = 16 * (rows + case["groups"] * case["hosts"]) if case["mask"] else 0
    # both towers' vectors, ids and teacher logits in, loss out; both gradients out
    return {"bytes": vectors * (2 if gradient else 1) + mask + rows * (8 * case["k"] + 4),
            "flops": 2 * rows * case["hosts"] * width * (3 if gradient else 1)}


# ---- inputs ---------------------------------------------------------------------------------------------------------
def _normal(gen, shape, dtype, scale=1.0):
    out = torch.empty(shape, dtype=DTYPES[dtype], device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 2 ** 27):
        part = flat[a:a + 2 ** 27]
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda").mul_(scale))
    return out


def _ints(gen, lo, hi, shape):
    return torch.randint(lo, hi, shape, generator=gen, device="cuda", dtype=torch.int32)


def _prepare_towers(case, s, gen):
    groups, rows, hosts, width, k = (case[i] for i in ("groups", "rows", "hosts", "width", "k"))
    s["requests"] = _normal(gen, (groups, rows, width), case["dtype"])
    s["vectors"] = _normal(gen, (groups, hosts, width), case["dtype"], 2.5 / math.sqrt(width))
    s["asks"] = s["room"] = None
    if case["mask"]:
        # GPUs, VRAM, millicpus, memory; one request in 200 asks for more GPUs than any host has, some hosts are full
        gpus = 2 ** _ints(gen, 0, 4, (groups, rows))
        gpus[torch.rand((groups, rows), generator=gen, device="cuda") < 0.005] = 64
        s["asks"] = torch.stack([gpus, 16 * gpus, _ints(gen, 1000, 16001, (groups, rows)),
                                 _ints(gen, 1024, 65537, (groups, rows))], dim=-1).int().contiguous()
        s["room"] = torch.stack([_ints(gen, 0, 17, (groups, hosts)), _ints(gen, 64, 641, (groups, hosts)),
                                 _ints(gen, 8000, 128001, (groups, hosts)),
                                 _ints(gen, 32768, 1048577, (groups, hosts))], dim=-1).contiguous()
    # k distinct hosts a row, some far more often than others, now and then fewer
    first = (torch.rand((groups, rows, 1), generator=gen, device="cuda").square_() * hosts).long().clamp_(max=hosts - 1)
    ids = (first + torch.arange(k, device="cuda") * max(1, hosts // k)) % hosts
    ids[torch.rand((groups, rows, k), generator=gen, device="cuda") < 0.02] = -1
    s["hosts"] = ids.int()
    # the teacher's scores fall from its best host to its last
    s["teacher"] = torch.randn((groups, rows, k), generator=gen, device="cuda").abs_().cumsum_(-1).neg_().add_(4.0)
    s["loss"] = torch.empty((groups, rows), device="cuda")
    if case["mode"] == "step":
        s["stats"] = torch.empty((groups, rows, 2 + k), device="cuda")
        s["grad_requests"], s["grad_vectors"] = torch.empty_like(s["requests"]), torch.empty_like(s["vectors"])
    elif case["mode"] == "autograd":
        s["requests"].requires_grad_(True)
        s["vectors"].requires_grad_(True)


def _prepare_block(case, s, gen):
    groups, rows, width, dtype = (case[i] for i in ("groups", "rows", "width", "dtype"))
    shape = (groups, rows, width)
    s["residual"], s["branch"] = _normal(gen, shape, dtype, 2.0), _normal(gen, shape, dtype, 0.5)
    gate = {"none": None, "width": (width,), "group": (groups, 1, width), "row": shape}[case["gate"]]
    s["gate"] = None if gate is None else _normal(gen, gate, dtype, 0.5)
    s["post"] = 1.0 + 0.1 * torch.randn(width, generator=gen, device="cuda")
    s["pre"] = 1.0 + 0.1 * torch.randn(width, generator=gen, device="cuda")
    s["alpha"] = 0.9
    if case["mode"] != "eval":
        s["grad_out"], s["grad_normed"] = _normal(gen, shape, dtype, 0.1), _normal(gen, shape, dtype, 0.1)
    leaves = [t for t in ("residual", "branch", "gate", "post", "pre") if s[t] is not None]
    if case["mode"] == "autograd":
        for t in leaves:
            s[t].requires_grad_(True)
    else:
        s["out"], s["normed"] = torch.empty(shape, dtype=DTYPES[dtype], device="cuda"), torch.empty(shape, dtype=DTYPES[dtype], device="cuda")
    if case["mode"] == "step":
        s["stats"] = torch.empty((groups, rows, 2), device="cuda")
        s["grads"] = {t: torch.empty_like(s[t]) for t in leaves}


def _prepare_clip(case, s, gen):
    # a few tensors of far larger gradients than the others, as early and late layers have
    s["tensors"] = [_normal(gen, (n,), t, 10.0 ** -(i % 4)) for i, (n, t) in enumerate(_sizes(case))]
    # the clipped ones go to flat buffers, one a type, in which each tensor starts on a 16-byte boundary
    spans, ends = [], {}
    for t in s["tensors"]:
        per16 = 16 // t.element_size()
        spans.append((t.dtype, ends.get(t.dtype, 0), t.numel()))
        ends[t.dtype] = spans[-1][1] + (t.numel() + per16 - 1) // per16 * per16
    s["flat"] = {t: torch.zeros(n, dtype=t, device="cuda") for t, n in ends.items()}
    s["outs"] = [s["flat"][t][a:a + n] for t, a, n in spans]
    s["norm"] = torch.empty((), device="cuda")
    size = math.sqrt(sum(n * 10.0 ** (-2 * (i % 4)) for i, (n, _) in enumerate(_sizes(case))))
    s["max_norm"] = 0.3 * size if case["clip"] else 4.0 * size


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    {"towers": _prepare_towers, "block": _prepare_block, "clip": _prepare_clip}[case["op"]](case, s, gen)
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------
def _fits(asks, room):
    """[G, R, H]: which requests fit which hosts."""
    out = None
    for i in range(4):
        one = asks[:, :, None, i] <= room[:, None, :, i]
        out = one if out is None else out.logical_and_(one)
    return out


def _plain_towers(s):
    case, T = s["case"], s["case"]["temperature"]
    a, b = s["requests"].detach().float(), s["vectors"].detach().float()
    x = a @ b.transpose(1, 2)
    if case["mask"]:
        x.masked_fill_(~_fits(s["asks"], s["room"]), NEG_INF)
    inside = (s["hosts"] >= 0) & (s["hosts"] < case["hosts"])
    ids = torch.where(inside, s["hosts"], 0).long()
    at = x.gather(2, ids)
    there = inside & (at > NEG_INF) & (s["teacher"] > NEG_INF)
    some = there.any(2, keepdim=True)
    t = torch.where(there, s["teacher"] / T, NEG_INF)
    t = t - torch.where(some, t.amax(2, keepdim=True), 0.0)
    total = torch.where(some, t.exp().sum(2, keepdim=True), 1.0)
    q = t.exp() / total

    top = x.amax(2, keepdim=True)
    alive = top > NEG_INF
    top = torch.where(alive, top, 0.0)
    e = x.sub_(top).div_(T).exp_()
    sum_e = torch.where(alive, e.sum(2, keepdim=True), 1.0)
    log_ratio = (t - total.log()) - ((at - top) / T - sum_e.log())
    loss = T ** 2 * torch.where(there, q * log_ratio, 0.0).sum(2)
    if case["mode"] == "eval":
        return {"loss": loss}
    g = e.div_(sum_e).mul_(some.float())
    g.scatter_add_(2, ids, torch.where(there, -q, 0.0))
    g.mul_(T * grad_scale(case))
    return {"loss": loss, "grad_requests": (g @ b).to(s["requests"].dtype),
            "grad_vectors": (g.transpose(1, 2) @ a).to(s["vectors"].dtype)}


def _plain_block(s):
    case = s["case"]
    dtype = s["residual"].dtype
    x, y, post, pre = (s[t].detach().float() for t in ("residual", "branch", "post", "pre"))
    gate = None if s["gate"] is None else s["gate"].detach().float()
    rstd_y = (y.square().mean(-1, keepdim=True) + EPS).rsqrt()
    y_hat = y * rstd_y
    n = y_hat * post
    r = s["alpha"] * x + (n if gate is None else gate * n)
    rstd_r = (r.square().mean(-1, keepdim=True) + EPS).rsqrt()
    r_hat = r * rstd_r
    out = {"out": r.to(dtype), "normed": (r_hat * pre).to(dtype)}
    if case["mode"] == "eval":
        return out
    dh = s["grad_normed"].float()
    out["grad_pre"] = (dh * r_hat).sum((0, 1))
    dr = dh * pre
    dr = s["grad_out"].float() + rstd_r * (dr - r_hat * (dr * r_hat).mean(-1, keepdim=True))
    out["grad_residual"] = (s["alpha"] * dr).to(dtype)
    if gate is not None:
        dg = dr * n
        if case["gate"] == "group":
            dg = dg.sum(1, keepdim=True)
        elif case["gate"] == "width":
            dg = dg.sum((0, 1))
        out["grad_gate"] = dg.to(dtype)
        dr = dr * gate
    out["grad_post"] = (dr * y_hat).sum((0, 1))
    dy = dr * post
    out["grad_branch"] = (rstd_y * (dy - y_hat * (dy * y_hat).mean(-1, keepdim=True))).to(dtype)
    return out


def _plain_clip(s):
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    for t in s["tensors"]:
        total = total + t.float().square().sum(dtype=torch.float64)
    norm = total.sqrt().float()
    factor = (s["max_norm"] / (norm + EPS)).clamp(max=1.0)
    for t, out in zip(s["tensors"], s["outs"]):
        out.copy_(t.float() * factor)
    return _clipped(s, norm)


def _clipped(s, norm):
    return dict({"clipped_" + str(t)[6:]: flat for t, flat in s["flat"].items()}, norm=norm)


# ---- the library's calls --------------------------------------------------------------------------------------------
def _own_towers(s):
    from paper_2503_20591_b200 import binding, policy

    case = s["case"]
    T, fit = case["temperature"], dict(asks=s["asks"], room=s["room"])
    if case["mode"] == "autograd":
        loss = policy.tower_distill_loss(s["requests"], s["vectors"], s["hosts"], s["teacher"], temperature=T, **fit)
        da, db = torch.autograd.grad(loss.sum() * grad_scale(case), (s["requests"], s["vectors"]))
        return {"loss": loss.detach(), "grad_requests": da, "grad_vectors": db}
    binding.nbos_policy_towers(s["requests"], s["vectors"], s["hosts"], s["teacher"], s["loss"], s.get("stats"),
                               temperature=T, **fit)
    if case["mode"] == "eval":
        return {"loss": s["loss"]}
    binding.nbos_policy_towers_backward(s["requests"], s["vectors"], s["hosts"], s["teacher"], s["stats"],
                                        s["grad_requests"], s["grad_vectors"], grad_scale=grad_scale(case),
                                        temperature=T, **fit)
    return {"loss": s["loss"], "grad_requests": s["grad_requests"], "grad_vectors": s["grad_vectors"]}


def _own_block(s):
    from paper_2503_20591_b200 import binding, policy

    case = s["case"]
    inputs = [s[t] for t in ("residual", "branch", "gate", "post", "pre")]
    if case["mode"] == "autograd":
        out, normed = policy.block_norm(*inputs, residual_scale=s["alpha"], eps=EPS)
        names = [t for t in ("residual", "branch", "gate", "post", "pre") if s[t] is not None]
        grads = torch.autograd.grad((out, normed), [s[t] for t in names], (s["grad_out"], s["grad_normed"]))
        out = {"out": out.detach(), "normed": normed.detach()}
        return dict(out, **{"grad_" + t: g for t, g in zip(names, grads)})
    binding.nbos_policy_block_norm(*inputs, s["out"], s["normed"], s.get("stats"), residual_scale=s["alpha"], eps=EPS)
    out = {"out": s["out"], "normed": s["normed"]}
    if case["mode"] == "eval":
        return out
    g = s["grads"]
    binding.nbos_policy_block_norm_backward(*inputs, s["stats"], s["grad_out"], s["grad_normed"], g["residual"],
                                            g["branch"], g.get("gate"), g["post"], g["pre"], residual_scale=s["alpha"])
    return dict(out, **{"grad_" + t: v for t, v in g.items()})


def _own_clip(s):
    from paper_2503_20591_b200 import binding

    binding.nbos_policy_clip(s["tensors"], s["max_norm"], s["norm"], s["outs"])
    return _clipped(s, s["norm"])


def run(state):
    if own:
        out = {"towers": _own_towers, "block": _own_block, "clip": _own_clip}[state["case"]["op"]](state)
    else:
        out = {"towers": _plain_towers, "block": _plain_block, "clip": _plain_clip}[state["case"]["op"]](state)
    return {k: out[k] for k in sorted(out)}   # both sides in the same order


# ---- 64 bits --------------------------------------------------------------------------------------------------------
def _log_softmax64(x):
    lse = torch.logsumexp(x, -1, keepdim=True)
    return torch.where(lse == NEG_INF, NEG_INF, x - lse)


def _exact_towers(case, s):
    T, hosts = case["temperature"], case["hosts"]
    losses, grads_a, grads_b = [], [], []
    step = max(1, 2 ** 26 // hosts)
    for n in range(case["groups"]):
        b = s["vectors"][n].detach().double()
        grad_b = torch.zeros_like(b)
        for r in range(0, case["rows"], step):
            a = s["requests"][n, r:r + step].detach().double()
            x = (a @ b.T) / T
            if case["mask"]:
                asks, room = s["asks"][n, r:r + step], s["room"][n]
                x[(asks[:, None, :] > room[None, :, :]).any(2)] = NEG_INF
            ids = s["hosts"][n, r:r + step].long()
            inside = (ids >= 0) & (ids < hosts)
            ids = ids * inside
            log_p = _log_softmax64(x)
            at = log_p.gather(1, ids)
            there = inside & (at != NEG_INF)
            log_q = _log_softmax64(torch.where(there, s["teacher"][n, r:r + step].double() / T, NEG_INF))
            q = log_q.exp()
            losses.append(T * T * torch.where(q > 0, q * (log_q - at), 0.0).sum(1))
            if case["mode"] == "eval":
                continue
            g = log_p.exp_() * there.any(1, keepdim=True)
            g.scatter_add_(1, ids, -q)
            g.mul_(T * grad_scale(case))
            grads_a.append(g @ b)
            grad_b += g.T @ a
        grads_b.append(grad_b)
    shape = (case["groups"], case["rows"])
    out = {"loss": torch.cat(losses).view(shape)}
    if case["mode"] != "eval":
        out["grad_requests"] = torch.cat(grads_a).view(*shape, -1)
        out["grad_vectors"] = torch.stack(grads_b)
    return out


def _exact_block(case, s):
    """Forward in 64 bits; the gradients by autograd on it."""
    names = [t for t in ("residual", "branch", "gate", "post", "pre") if s[t] is not None]
    leaf = {t: s[t].detach().double().requires_grad_(case["mode"] != "eval") for t in names}

    def normed(v, weight):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS) * weight

    n = normed(leaf["branch"], leaf["post"])
    r = s["alpha"] * leaf["residual"] + (leaf["gate"] * n if "gate" in leaf else n)
    h = normed(r, leaf["pre"])
    out = {"out": r.detach(), "normed": h.detach()}
    if case["mode"] != "eval":
        grads = torch.autograd.grad((r, h), list(leaf.values()), (s["grad_out"].double(), s["grad_normed"].double()))
        out.update({"grad_" + t: g for t, g in zip(names, grads)})
    return out


def _exact_clip(case, s):
    norm = torch.sqrt(sum(torch.linalg.vector_norm(t.double()) ** 2 for t in s["tensors"]))
    factor = min(1.0, s["max_norm"] / (float(norm) + EPS))
    flat = {t: torch.zeros(f.numel(), dtype=torch.float64, device="cuda") for t, f in s["flat"].items()}
    for t, out in zip(s["tensors"], s["outs"]):
        at = out.storage_offset()
        flat[t.dtype][at:at + t.numel()] = t.double() * factor
    return dict({"clipped_" + str(t)[6:]: f for t, f in flat.items()}, norm=norm)


def exact(case, seed):
    s = prepare(case, seed)
    out = {"towers": _exact_towers, "block": _exact_block, "clip": _exact_clip}[case["op"]](case, s)
    return {k: out[k] for k in sorted(out)}
