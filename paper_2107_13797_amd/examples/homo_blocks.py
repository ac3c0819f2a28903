"""One round of homogeneous federated training of the adapters of a block with norms, on synthetic data, and answers of the common model
with weights of eight bits.

    block        h = norm(x),  f = W h + B_1 A_1 h,  r = x + gate norm(f),  logits = H norm(r) + B_2 A_2 norm(r)
    party k      a few steps on its n_k rows: the block, log-probabilities of the labels, the gradients back to its adapters, and updates
                 that are orthogonalised matrix by matrix
    all          the parties' adapters are aggregated through ciphertexts, each weighted by its row count
    party        the common adapters are merged into W and H, these brought to eight bits: the answer of one row, and the loss

The parties of this example share one card, and so their rows one call, each row with its party's adapter. `run_round` returns the
losses, the answer, and the decoded sum beside the same sum in exact integers on the quantised weights.

    python -m paper_2107_13797_amd.examples.homo_blocks [--bits 2048] [--parties 8] [--rows 1024] [--width 2048]
                                                        [--labels 1000] [--rank 16] [--steps 8]
"""
import argparse
import time

import numpy as np
import torch

from .homo_adapters import Adapters, aggregate, exact_sum


class Block:
    """What the parties share and leave as it is: both projections, and the gains of the norms around the block."""

    def __init__(self, normal, width, labels, kind):
        self.w, self.head = normal(width, width, by=width ** -0.5).to(kind), normal(labels, width, by=width ** -0.5).to(kind)
        self.first, self.post, self.last = (1.0 + normal(width, by=0.05) for _ in range(3))
        self.gate = torch.full((width,), 0.5, device="cuda")


def forward(api, block, adapters, x, index):
    """Logits of the rows of x, and what the way back needs."""
    a1, b1, a2, b2 = (v.to(x.dtype) for v in adapters.values)
    _, h, _ = api.haflo_residual_norm(x, pre=block.first)
    f, z1 = api.haflo_adapter_forward(h, block.w, a1, b1, adapters.scale, index)
    _, g, roots = api.haflo_residual_norm(x, f, block.post, block.gate, block.last)
    logits, z2 = api.haflo_adapter_forward(g, block.head, a2, b2, adapters.scale, index)
    return logits, (a1, b1, a2, b2, h, f, z1, g, roots, z2)


def gradients(api, block, adapters, x, label, index, weight):
    """Rows' log-probabilities, and the gradients of the sum of weight times their negatives by each of the adapters' matrices."""
    logits, (a1, b1, a2, b2, h, f, z1, g, roots, z2) = forward(api, block, adapters, x, index)
    logp, entropy, lse, _, _ = api.haflo_label_logprobs(logits, label)
    d = api.haflo_label_logprobs_backward(logits, label, lse, entropy, -weight, out=logits)
    dg, da2, db2 = api.haflo_adapter_backward(d, g, block.head, a2, b2, adapters.scale, index, z2)
    _, df, _, _, _ = api.haflo_residual_norm_backward(dg, None, x, f, block.post, block.gate, block.last, roots, need_dx=False)
    _, da1, db1 = api.haflo_adapter_backward(df, h, block.w, a1, b1, adapters.scale, index, z1, need_dx=False)
    return logp, (da1, db1, da2, db2)


def step(api, block, adapters, x, label, index, weight, rate):
    """One step of every party. The matrices' singular values all become about `rate`, whatever the gradient's were."""
    logp, grads = gradients(api, block, adapters, x, label, index, weight)
    for v, g in zip(adapters.values, grads):
        api.haflo_orthogonal_update(g, v, scale=-rate, out=v)
    return logp


class EightBits:
    """The common model with its adapters merged into the projections, in eight bits."""

    def __init__(self, api, block, common):
        self.block = block
        a1, b1, a2, b2 = (v[0] for v in common.values)
        by = float(common.scale[0])
        self.w, self.head = (api.haflo_quantize_rows(w.float() + by * (b @ a)) for w, a, b in ((block.w, a1, b1), (block.head, a2, b2)))

    def logits(self, api, x):
        b = self.block
        _, h, _ = api.haflo_residual_norm(x, pre=b.first)
        f = api.haflo_int8_forward(h, *self.w)
        _, g, _ = api.haflo_residual_norm(x, f, b.post, b.gate, b.last)
        return api.haflo_int8_forward(g, *self.head)


def run_round(api, pub, own, parties, rows, width, labels, rank, steps, seed=0, rate=0.02, kind=torch.bfloat16, timings=None):
    """pub: public context (the coordinator), own: private context (the parties). Every party has between half of `rows` and
    `rows` rows."""
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, by=1.0):
        return torch.randn(shape, generator=gen, device="cuda") * by

    def timed(name, fn):
        if timings is None:
            return fn()
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        out = fn()
        torch.cuda.synchronize()
        timings[name] = timings.get(name, 0.0) + (time.perf_counter() - t0) * 1e3
        return out

    block = Block(normal, width, labels, kind)
    kinds = normal(labels, width)  # a row is its label's kind and noise
    counts = [int(c) for c in rng.integers(rows // 2, rows + 1, parties)]
    index = torch.repeat_interleave(torch.arange(parties), torch.tensor(counts)).to(torch.int32).cuda()
    label = torch.from_numpy(rng.integers(0, labels, sum(counts)).astype(np.int32)).cuda()
    x = (kinds[label.long()] + 0.5 * normal(sum(counts), width)).to(kind)
    weight = (1.0 / torch.tensor(counts, dtype=torch.float32, device="cuda"))[index.long()]
    first = [normal(rank, width, by=width ** -0.5), torch.zeros((width, rank), device="cuda"), normal(rank, width, by=width ** -0.5),
             torch.zeros((labels, rank), device="cuda")]
    adapters = Adapters(parties, width, labels, rank, [f.expand((parties,) + f.shape).clone() for f in first])

    def loss(logits):
        return float(-api.haflo_label_logprobs(logits, label)[0].mean())

    before = loss(forward(api, block, adapters, x, index)[0])
    for _ in range(steps):
        timed("parties: local steps", lambda: step(api, block, adapters, x, label, index, weight, rate))
    local = loss(forward(api, block, adapters, x, index)[0])
    flat = [adapters.flat(k) for k in range(parties)]
    sum_q, summed = aggregate(api, pub, own, flat, counts, rng, timed)
    common = Adapters.of_flat((summed / sum(counts)).to(torch.float32), width, labels, rank)
    full = loss(forward(api, block, common, x, torch.zeros_like(index))[0])
    model = timed("party: common model to eight bits", lambda: EightBits(api, block, common))
    eight = timed("party: all rows in eight bits", lambda: loss(model.logits(api, x)))
    none = torch.full((1,), -1, dtype=torch.int32, device="cuda")
    _, _, _, top_logp, top_index = timed("party: one row's answer", lambda: api.haflo_label_logprobs(model.logits(api, x[:1]), none, top=5))
    return {
        "sum_q": sum_q.tolist(),
        "want_sum_q": exact_sum(flat, counts),
        "loss": {"before": before, "local": local, "common": full, "eight bits": eight},
        "answer": list(zip(top_index[0].tolist(), top_logp[0].tolist())),
        "label": int(label[0]),
        "weights": flat[0].numel(),
    }


def main():
    ap = argparse.ArgumentParser()
    for name, value in (("bits", 2048), ("parties", 8), ("rows", 1024), ("width", 2048), ("labels", 1000), ("rank", 16), ("steps", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    args = ap.parse_args()
    from paper_2107_13797_amd import api
    p, q = api.haflo_keygen(args.bits, 7)
    own = api.haflo_ctx_create_private(p, q, args.bits)
    pub = api.haflo_ctx_create_public(p * q, args.bits)
    run_round(api, pub, own, 2, 64, 128, 16, 4, 1, seed=1)  # warm-up
    timings = {}
    res = run_round(api, pub, own, args.parties, args.rows, args.width, args.labels, args.rank, args.steps, seed=2, timings=timings)
    assert res["sum_q"] == res["want_sum_q"]
    print("%d-bit key, %d parties, %d weights each: the decoded aggregate equals the exact fixed-point sum"
          % (args.bits, args.parties, res["weights"]))
    for name, ms in timings.items():
        print("  %-34s %9.2f ms" % (name, ms))
    print("  mean loss: %.4f before, %.4f under each party's adapters, %.4f under their average, %.4f with it in eight bits"
          % tuple(res["loss"][k] for k in ("before", "local", "common", "eight bits")))
    print("  one row of label %d: %s" % (res["label"], ", ".join("%d (%.3f)" % a for a in res["answer"])))


if __name__ == "__main__":
    main()
