"""One mixture-of-experts sublayer of a decode step on one GPU, from compressed experts to its output:

    residual += x;  h = norm(residual)         zipmoe_add_rmsnorm   (bf16 rows, and 8-bit rows with scales beside them)
    ids, weights = top-k of h @ gate^T         zipmoe_route
    y = sum of the chosen experts' FFNs        zipmoe_expert_ffn on the experts that are recovered (the planner's pool F), or, for a
                                               prompt of more than 256 tokens, the grouped products (zipmoe_group_tokens,
                                               zipmoe_grouped_matmul, zipmoe_combine_rows; they round the activations between the
                                               products to 8 significant bits, zipmoe_expert_ffn to 16);
                                               zipmoe_decode_expert_ffn on those that stay compressed

A layer may keep some of its experts recovered and the others compressed.  The call on recovered experts takes -1 for a choice
that is not its own.  The call on compressed experts wants every id in range, so each choice is a row of its own there, those
that are not its own run with an expert that is wanted anyway, and their results are dropped before the rest is weighed.

    python examples/expert_sublayer.py [--tokens 4] [--experts 8] [--resident 4] [--hidden 2048] [--inter 1536] [--k 2]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2601_21198_b200 import binding as zb, inputs  # noqa: E402


class ExpertSublayer:
    """norm_weight [hidden], gate [n_experts, hidden]: device bf16; blobs[3 * e + j]: encoded w1, w3, w2 (blocked layout);
    the first `resident` experts are recovered when the layer is built, the others are run as they are."""

    def __init__(self, norm_weight, gate, k, blobs, hidden, inter, resident):
        self.norm = zb.RmsNorm(norm_weight)
        self.router = zb.Router(gate, k)
        self.n_resident, self.n_experts = resident, len(blobs) // 3
        self.recovered = self.compressed = None
        if resident:
            plan = zb.DecodePlan(blobs[:3 * resident])
            device = plan.to_device("cuda")
            self.weights = device.new_output()
            device.decode(self.weights)                                   # E-chunks + SM-chunks -> bf16, once
            self.recovered = zb.ResidentExperts.from_decode(plan, self.weights, hidden, inter)
        if resident < self.n_experts:
            self.compressed = zb.DeviceExperts(blobs[3 * resident:], hidden, inter)

    def forward(self, x, residual):
        """x, residual [T, hidden] bf16; residual is updated in place.  Returns (y, q, scales): the sublayer's output and the
        normed rows in 8 bits, for a projection that takes them so."""
        h = torch.empty_like(x)
        q, scales = self.norm.add_norm_8bit(x, residual, residual, out=h)
        ids, weights = self.router.route(h)
        y = torch.zeros(x.shape, device=x.device)
        if self.recovered is not None:
            ffn = self.recovered.ffn if len(h) <= 256 else self.recovered.ffn_prompt
            y += ffn(h, torch.where(ids < self.n_resident, ids, -1), weights)
        if self.compressed is not None:
            T, k = ids.shape
            away = (ids - self.n_resident).reshape(T * k, 1)
            mine = away >= 0
            own = torch.where(mine, away, away.max().clamp(min=0))
            rows = h.view(torch.int16).repeat_interleave(k, dim=0)
            z = torch.cat([self.compressed.ffn(rows[i:i + 64], own[i:i + 64], None) for i in range(0, T * k, 64)])
            z = torch.where(mine, z.view(torch.bfloat16).float(), 0).view(T, k, -1)
            y += (weights.unsqueeze(2) * z).sum(dim=1)
        return y.to(x.dtype), q, scales


def build(n_experts, resident, hidden, inter, k, seed=0):
    ws = [inputs.gaussian((inter, hidden) if j % 3 < 2 else (hidden, inter), 0.02, 1000 * seed + j) for j in range(3 * n_experts)]
    blobs = [zb.zipmoe_encode(w, layout=zb.LAYOUT_BLOCKED, chunk_elems=65536) for w in ws]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    norm_weight = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).to(torch.bfloat16)
    gate = (0.05 * torch.randn(n_experts, hidden, generator=g, device="cuda")).to(torch.bfloat16)
    return ws, ExpertSublayer(norm_weight, gate, k, blobs, hidden, inter, resident)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 4), ("experts", 8), ("resident", 4), ("hidden", 2048), ("inter", 1536), ("k", 2)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    _, layer = build(a.experts, a.resident, a.hidden, a.inter, a.k)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(a.tokens, a.hidden, generator=g, device="cuda").to(torch.bfloat16)
    residual = torch.randn(a.tokens, a.hidden, generator=g, device="cuda").to(torch.bfloat16)
    for _ in range(3):
        layer.forward(x, residual.clone())
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    copies = [residual.clone() for _ in range(20)]
    start.record()
    for r in copies:
        y, q, scales = layer.forward(x, r)
    end.record()
    torch.cuda.synchronize()
    print("%d tokens, %d experts (%d recovered), top-%d: %.1f us per sublayer; output rms %.3g, largest 8-bit scale %.3g" %
          (a.tokens, a.experts, a.resident, a.k, start.elapsed_time(end) * 50, y.float().square().mean().sqrt().item(), scales.max().item()))


if __name__ == "__main__":
    main()
