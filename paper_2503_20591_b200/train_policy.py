"""Trains a small placement policy on the exact rule's decisions and lets it place requests.

    python -m paper_2503_20591_b200.train_policy [--hosts 256] [--snapshots 16] [--batch 512] [--steps 150]
                                                 [--blocks 0] [--max-norm X] [--no-table]

One step: a batch of requests is placed by nbos_place_batch on every snapshot (the teacher); the policy scores every
host for every request and answers by sampling three distinct hosts; the distillation loss pulls it to the teacher's
three hosts, the balance loss moves probability away from hosts that its own answers load more than others. Afterwards
both ways of placing are compared.

--blocks gives either tower residual blocks, --max-norm clips the gradients by their global norm, --no-table trains on the
two towers' vectors (in bfloat16) without the table of scores: for clusters whose table does not fit. There is no balance loss
then, which needs the table; what is reported is measured on pieces of it.
"""
from __future__ import annotations

import argparse

import torch

from . import binding, policy, workloads

BALANCE_WEIGHT = 0.01
TEACHER_LOGITS = (2.0, 1.0, 0.0)   # best, second, third host
PIECE = 1 << 22                    # scores that are looked at together when the policy is measured
ANSWER = dict(temperature=0.7, top_k=16, top_p=0.95, min_p=0.01)   # how the policy is asked


class ResidualBlocks(torch.nn.Module):
    """Blocks x + gate * norm(branch(norm(x))) behind a tower, with the norms around each branch in one kernel."""

    def __init__(self, width: int, blocks: int):
        super().__init__()
        self.branches = torch.nn.ModuleList(torch.nn.Sequential(torch.nn.Linear(width, width), torch.nn.ReLU(), torch.nn.Linear(width, width))
                                            for _ in range(blocks))
        self.gates = torch.nn.ParameterList(torch.full((width,), 0.1) for _ in range(blocks))
        self.post = torch.nn.ParameterList(torch.ones(width) for _ in range(blocks))
        self.pre = torch.nn.ParameterList(torch.ones(width) for _ in range(blocks))

    def forward(self, x):
        normed = x
        for branch, gate, post, pre in zip(self.branches, self.gates, self.post, self.pre):
            x, normed = policy.block_norm(x, branch(normed), gate, post, pre)
        return normed


class TwoTowerPolicy(torch.nn.Module):
    """logits[n, b, h] = request vector . host vector."""

    def __init__(self, request_features: int, host_features: int, width: int = 64, blocks: int = 0):
        super().__init__()
        self.request = torch.nn.Sequential(torch.nn.Linear(request_features, width), torch.nn.ReLU(),
                                           torch.nn.Linear(width, width))
        self.host = torch.nn.Sequential(torch.nn.Linear(host_features, width), torch.nn.ReLU(),
                                        torch.nn.Linear(width, width))
        if blocks:
            self.request.append(ResidualBlocks(width, blocks))
            self.host.append(ResidualBlocks(width, blocks))

    def vectors(self, requests, hosts):
        return self.request(requests), self.host(hosts)

    def forward(self, requests, hosts, fits):
        request, host = self.vectors(requests, hosts)
        logits = request @ host.transpose(1, 2)
        return logits.masked_fill(~fits, float("-inf"))


class Cluster:
    """Host state of a workload on the device: a snapshot for the exact rule, features for the policy."""

    def __init__(self, w):
        self.snapshot = binding.snapshot_from_workload(w)
        self.state = {k: torch.from_numpy(getattr(w, k)).cuda() for k in w.HOST_FIELDS}
        self.limit = [torch.from_numpy(a).long().cuda()[:, None, None] for a in (w.limit_num * w.replicas_R, w.limit_den)]
        s = {k: v.float() for k, v in self.state.items()}
        self.features = torch.stack([(s["gpus_total"] - s["gpus_committed"]) / 8, s["gpus_subscribed"] / 16, s["gpus_total"] / 8,
                                     s["vram_gb"] / 640, s["millicpus"] / 128_000, s["mem_mb"] / 1_048_576], dim=-1)
        # what a request may ask for at most, [N, H, 4]: GPUs within the host and within its subscription limit, then the capacities
        total, held = self.state["gpus_total"].long(), self.state["gpus_subscribed"].long()
        by_limit = torch.div(total * self.limit[0][:, 0], self.limit[1][:, 0], rounding_mode="floor") - held
        gpus = torch.where(total >= 1, torch.minimum(total, by_limit), -1).clamp(min=-1)
        self.room = torch.stack([gpus.int(), self.state["vram_gb"], self.state["millicpus"], self.state["mem_mb"]], dim=-1).contiguous()

    def teacher(self, requests):
        """requests [N, B, 4] int32: the exact rule's hosts [N, B, 3], -1 where fewer fit."""
        out = torch.empty((*requests.shape[:2], 3), dtype=torch.int32, device="cuda")
        binding.nbos_place_batch(self.snapshot, requests, out)
        return out

    def fits(self, requests, snapshots=slice(None)):
        """[N, B, H]: which hosts can take which request (capacities and subscription limit)."""
        s = {k: v[snapshots, None, :] for k, v in self.state.items()}
        limit = [v[snapshots] for v in self.limit]
        g, v, c, m = (requests[..., i, None] for i in range(4))
        return ((s["gpus_total"] >= 1) & (g <= s["gpus_total"]) & (v <= s["vram_gb"]) & (c <= s["millicpus"])
                & (m <= s["mem_mb"]) & ((s["gpus_subscribed"] + g) * limit[1] <= s["gpus_total"] * limit[0]))

    def close(self):
        binding.nbos_snapshot_destroy(self.snapshot)


def request_features(requests):
    return requests.float() / torch.tensor([8.0, 128.0, 16_000.0, 65_536.0], device=requests.device)


def train(hosts: int = 256, snapshots: int = 16, batch: int = 512, steps: int = 150, seed: int = 0, report=print,
          blocks: int = 0, max_norm: float | None = None, table: bool = True) -> dict:
    torch.manual_seed(seed)
    cluster = Cluster(workloads.what_if_sweep(snapshots, hosts, batch))
    try:
        net = TwoTowerPolicy(4, cluster.features.shape[-1], blocks=blocks).cuda()
        optimizer = torch.optim.Adam(net.parameters(), lr=3e-3)
        teacher_logits = torch.tensor(TEACHER_LOGITS, device="cuda")
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def draw():
            g = 2 ** torch.randint(0, 4, (snapshots, batch), generator=gen, device="cuda")
            c = torch.randint(1000, 16001, (snapshots, batch), generator=gen, device="cuda")
            m = torch.randint(1024, 65537, (snapshots, batch), generator=gen, device="cuda")
            return torch.stack([g, 16 * g, c, m], dim=-1).int()

        def agrees(logits, wanted):
            """(requests whose best host by the policy is one of the rule's three, requests that can be placed)"""
            best = logits.argmax(-1, keepdim=True).int()
            there = wanted[..., :1] >= 0
            return ((best == wanted).any(-1, keepdim=True) & there).sum(), there.sum()

        def draw_answers():
            return torch.rand((snapshots, batch, 3), generator=gen, device="cuda")

        def answer(logits, uniforms):
            """Three distinct hosts a request, drawn from the policy, and how many were there."""
            return policy.sample_hosts(logits.detach(), uniforms, **ANSWER)

        def measure(requests, wanted):
            """The policy's answers to all requests and what they are like, in pieces of snapshots and requests: the table of all
            scores is never there."""
            uniforms = draw_answers()
            n_step = max(1, min(snapshots, PIECE // hosts))
            b_step = max(1, min(batch, PIECE // (hosts * n_step)))
            total = dict(hits=0, there=0, found=0, infeasible=0, repeated=0)
            even, used, used_by_rule = [], 0, 0
            with torch.no_grad():
                request, host = net.vectors(request_features(requests), cluster.features)
                for n in range(0, snapshots, n_step):
                    ns = slice(n, n + n_step)
                    live = counts = rule_counts = shares = 0
                    for b in range(0, batch, b_step):
                        bs = slice(b, b + b_step)
                        fits = cluster.fits(requests[ns, bs], ns)
                        logits = (request[ns, bs] @ host[ns].transpose(1, 2)).masked_fill(~fits, float("-inf"))
                        rule = wanted[ns, bs].contiguous()
                        placed, found = answer(logits, uniforms[ns, bs].contiguous())
                        chosen = placed >= 0
                        hits, there = agrees(logits, rule)
                        total["hits"] += hits
                        total["there"] += there
                        total["found"] += found.sum()
                        total["infeasible"] += (~fits.gather(2, placed.clamp(min=0).long()) & chosen).sum()
                        total["repeated"] += sum(((placed[..., i] == placed[..., j]) & chosen[..., i] & chosen[..., j]).sum()
                                                 for i, j in ((0, 1), (0, 2), (1, 2)))
                        _, own, share = policy.balance_loss(logits, placed)
                        rows = chosen.any(-1).sum(1, keepdim=True)
                        live, counts, shares = live + rows, counts + own, shares + share.double() * rows
                        rule_counts = rule_counts + policy.balance_loss(logits, rule)[1]
                    load = counts.double() / counts.sum(1, keepdim=True).clamp(min=1)
                    even.append(hosts * (load * shares / live.clamp(min=1)).sum(1))
                    used += (counts > 0).sum()
                    used_by_rule += (rule_counts > 0).sum()
            total = {k: int(v) for k, v in total.items()}
            return dict(agreement=total["hits"] / max(1, total["there"]), feasible=total["infeasible"] == 0, distinct=total["repeated"] == 0,
                        found=total["found"] / (snapshots * batch), even=float(torch.cat(even).mean()), hosts_used=int(used) / snapshots,
                        hosts_used_by_rule=int(used_by_rule) / snapshots)

        history = []
        for step in range(steps):
            requests = draw()
            wanted = cluster.teacher(requests)
            reported = step % max(1, steps // 5) == 0 or step == steps - 1
            if table:
                logits = net(request_features(requests), cluster.features, cluster.fits(requests))
                distill = policy.distill_loss(logits, wanted, teacher_logits)
                even, _, _ = policy.balance_loss(logits, answer(logits, draw_answers())[0])   # the load is the policy's own, not the rule's
                loss = distill.mean() + BALANCE_WEIGHT * even.mean()
            else:
                request, host = (v.bfloat16() for v in net.vectors(request_features(requests), cluster.features))
                distill = policy.tower_distill_loss(request, host, wanted, teacher_logits, asks=requests, room=cluster.room)
                loss = distill.mean()
                if reported:
                    seen = measure(requests, wanted)
                    shown = seen["even"], seen["agreement"]
            optimizer.zero_grad(set_to_none=True)
            loss.backward()
            if max_norm is not None:
                policy.clip_gradients(net.parameters(), max_norm)
            optimizer.step()
            if reported:
                if not table and binding.nbos_policy_towers_status() != binding.NBOS_OK:
                    raise RuntimeError("a two-tower kernel gave up on a wait: the last steps' gradients are undefined")
                if table:
                    hits, there = agrees(logits.detach(), wanted)
                    shown = even.mean().item(), float(hits / there)
                history.append((distill.mean().item(), *shown))
                report(f"step {step}: distillation {history[-1][0]:.4f}, balance {history[-1][1]:.2f}, "
                       f"best host among the rule's three {history[-1][2]:.3f}")

        requests = draw()
        result = measure(requests, cluster.teacher(requests))
        del result["even"]
        result = dict(history=history, **result)
        report(f"sampled: {result['found']:.2f} hosts a request, all feasible: {result['feasible']}, distinct: {result['distinct']}; "
               f"{result['hosts_used']:.0f} hosts of a snapshot used ({result['hosts_used_by_rule']:.0f} by the rule)")
        return result
    finally:
        cluster.close()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("hosts", 256), ("snapshots", 16), ("batch", 512), ("steps", 150), ("seed", 0), ("blocks", 0)):
        parser.add_argument(f"--{name}", type=int, default=value)
    parser.add_argument("--max-norm", type=float, default=None)
    parser.add_argument("--no-table", dest="table", action="store_false")
    train(**vars(parser.parse_args()))
