"""Trains a small placement policy on the exact rule's decisions and lets it place requests.

    python -m paper_2503_20591_b200.train_policy [--hosts 256] [--snapshots 16] [--batch 512] [--steps 150]

One step: a batch of requests is placed by nbos_place_batch on every snapshot (the teacher); the policy scores every
host for every request and answers by sampling three distinct hosts; the distillation loss pulls it to the teacher's
three hosts, the balance loss moves probability away from hosts that its own answers load more than others. Afterwards
both ways of placing are compared.
"""
from __future__ import annotations

import argparse

import torch

from . import binding, policy, workloads

BALANCE_WEIGHT = 0.01
TEACHER_LOGITS = (2.0, 1.0, 0.0)   # best, second, third host
ANSWER = dict(temperature=0.7, top_k=16, top_p=0.95, min_p=0.01)   # how the policy is asked


class TwoTowerPolicy(torch.nn.Module):
    """logits[n, b, h] = request vector . host vector."""

    def __init__(self, request_features: int, host_features: int, width: int = 64):
        super().__init__()
        self.request = torch.nn.Sequential(torch.nn.Linear(request_features, width), torch.nn.ReLU(),
                                           torch.nn.Linear(width, width))
        self.host = torch.nn.Sequential(torch.nn.Linear(host_features, width), torch.nn.ReLU(),
                                        torch.nn.Linear(width, width))

    def forward(self, requests, hosts, fits):
        logits = self.request(requests) @ self.host(hosts).transpose(1, 2)
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

    def teacher(self, requests):
        """requests [N, B, 4] int32: the exact rule's hosts [N, B, 3], -1 where fewer fit."""
        out = torch.empty((*requests.shape[:2], 3), dtype=torch.int32, device="cuda")
        binding.nbos_place_batch(self.snapshot, requests, out)
        return out

    def fits(self, requests):
        """[N, B, H]: which hosts can take which request (capacities and subscription limit)."""
        s = {k: v[:, None, :] for k, v in self.state.items()}
        g, v, c, m = (requests[..., i, None] for i in range(4))
        return ((s["gpus_total"] >= 1) & (g <= s["gpus_total"]) & (v <= s["vram_gb"]) & (c <= s["millicpus"])
                & (m <= s["mem_mb"]) & ((s["gpus_subscribed"] + g) * self.limit[1] <= s["gpus_total"] * self.limit[0]))

    def close(self):
        binding.nbos_snapshot_destroy(self.snapshot)


def request_features(requests):
    return requests.float() / torch.tensor([8.0, 128.0, 16_000.0, 65_536.0], device=requests.device)


def train(hosts: int = 256, snapshots: int = 16, batch: int = 512, steps: int = 150, seed: int = 0, report=print) -> dict:
    torch.manual_seed(seed)
    cluster = Cluster(workloads.what_if_sweep(snapshots, hosts, batch))
    try:
        net = TwoTowerPolicy(4, cluster.features.shape[-1]).cuda()
        optimizer = torch.optim.Adam(net.parameters(), lr=3e-3)
        teacher_logits = torch.tensor(TEACHER_LOGITS, device="cuda")
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def draw():
            g = 2 ** torch.randint(0, 4, (snapshots, batch), generator=gen, device="cuda")
            c = torch.randint(1000, 16001, (snapshots, batch), generator=gen, device="cuda")
            m = torch.randint(1024, 65537, (snapshots, batch), generator=gen, device="cuda")
            return torch.stack([g, 16 * g, c, m], dim=-1).int()

        def agreement(logits, wanted):
            """Share of placeable requests whose best host by the policy is one of the rule's three."""
            best = logits.argmax(-1, keepdim=True).int()
            there = wanted[..., :1] >= 0
            return float(((best == wanted).any(-1, keepdim=True) & there).sum() / there.sum())

        def answer(logits):
            """Three distinct hosts a request, drawn from the policy, and how many were there."""
            return policy.sample_hosts(logits.detach(), torch.rand((snapshots, batch, 3), generator=gen, device="cuda"), **ANSWER)

        history = []
        for step in range(steps):
            requests = draw()
            wanted = cluster.teacher(requests)
            logits = net(request_features(requests), cluster.features, cluster.fits(requests))
            distill = policy.distill_loss(logits, wanted, teacher_logits)
            even, _, _ = policy.balance_loss(logits, answer(logits)[0])   # the load is the policy's own, not the rule's
            loss = distill.mean() + BALANCE_WEIGHT * even.mean()
            optimizer.zero_grad(set_to_none=True)
            loss.backward()
            optimizer.step()
            if step % max(1, steps // 5) == 0 or step == steps - 1:
                history.append((distill.mean().item(), even.mean().item(), agreement(logits.detach(), wanted)))
                report(f"step {step}: distillation {history[-1][0]:.4f}, balance {history[-1][1]:.2f}, "
                       f"best host among the rule's three {history[-1][2]:.3f}")

        requests = draw()
        fits = cluster.fits(requests)
        with torch.no_grad():
            logits = net(request_features(requests), cluster.features, fits)
        placed, found = answer(logits)
        chosen = placed >= 0
        feasible = fits.gather(2, placed.clamp(min=0).long()) | ~chosen
        distinct = all(((placed[..., i] != placed[..., j]) | ~chosen[..., i] | ~chosen[..., j]).all().item()
                       for i, j in ((0, 1), (0, 2), (1, 2)))
        rule = cluster.teacher(requests)
        _, rule_counts, _ = policy.balance_loss(logits, rule)
        _, own_counts, _ = policy.balance_loss(logits, placed)
        result = dict(history=history, agreement=agreement(logits, rule), feasible=bool(feasible.all()), distinct=distinct,
                      found=float(found.float().mean()), hosts_used=float((own_counts > 0).float().sum(1).mean()),
                      hosts_used_by_rule=float((rule_counts > 0).float().sum(1).mean()))
        report(f"sampled: {result['found']:.2f} hosts a request, all feasible: {result['feasible']}, distinct: {distinct}; "
               f"{result['hosts_used']:.0f} hosts of a snapshot used ({result['hosts_used_by_rule']:.0f} by the rule)")
        return result
    finally:
        cluster.close()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("hosts", 256), ("snapshots", 16), ("batch", 512), ("steps", 150), ("seed", 0)):
        parser.add_argument(f"--{name}", type=int, default=value)
    train(**vars(parser.parse_args()))
