"""One round of homogeneous federated training of low-rank adapters on synthetic data: the parties share a projection and a head
that stay as they are and train an adapter of each; only the adapters are encrypted, aggregated and sent back.

    party k      a few steps on its n_k rows: projection with adapter, dropout onto the residual, head with adapter,
                 log-probabilities of the labels, and the gradients back to the adapters
    party k      [[w_k]], w_k all weights of its adapters         (encode, encrypt as the key owner)
    coordinator  [[S]] = sum_k n_k [[w_k]]                        (scalar_mul by the row count, add)
    party        w' = D([[S]]) / sum_k n_k                        (decrypt, decode)
    party        one row's answer under w': the most likely labels, with their log-probabilities

The parties of this example share one card, and so their rows one call, each row with its party's adapter. Adapters are kept
in float32 and used in bfloat16. `run_round` returns the losses, the answer, and the decoded sum beside the same sum in exact
integers on the quantised weights.

    python -m paper_2107_13797_amd.examples.homo_adapters [--bits 2048] [--parties 8] [--rows 1024] [--width 2048]
                                                          [--labels 1000] [--rank 16] [--steps 8]
"""
import argparse
import time

import numpy as np
import torch

SCALE_W = 24


class Adapters:
    """The two adapters of several parties: a of the projection, b of it, then the head's."""

    def __init__(self, parties, width, labels, rank, values=None):
        self.shapes = [(rank, width), (width, rank), (rank, width), (labels, rank)]
        self.values = values if values is not None else [torch.zeros((parties,) + s, device="cuda") for s in self.shapes]
        self.scale = torch.full((parties,), 2.0, device="cuda")

    def used(self):
        return [v.to(torch.bfloat16) for v in self.values]

    def flat(self, k):
        return torch.cat([v[k].reshape(-1) for v in self.values])

    @classmethod
    def of_flat(cls, flat, width, labels, rank):
        out = cls(1, width, labels, rank)
        parts = torch.split(flat, [int(np.prod(s)) for s in out.shapes])
        out.values = [p.reshape((1,) + s).contiguous() for p, s in zip(parts, out.shapes)]
        return out


def forward(api, shared, adapters, x, index, p=0.0, seed=0, offset=0):
    """Logits of the rows of x, and what the way back needs; uses three offsets of the generator."""
    a1, b1, a2, b2 = adapters.used()
    y, h1 = api.haflo_adapter_forward(x, shared[0], a1, b1, adapters.scale, index, p, seed, offset)
    z = api.haflo_dropout(y, p, seed, offset + 1, residual=x)
    logits, h2 = api.haflo_adapter_forward(z, shared[1], a2, b2, adapters.scale, index, p, seed, offset + 2)
    return logits, (a1, b1, a2, b2, h1, z, h2)


def step(api, shared, adapters, x, label, index, weight, rate, p, seed, offset):
    """One step of every party by the mean of its rows' losses; `weight`: of each row in its party's mean. Returns the rows'
    log-probabilities before it."""
    logits, (a1, b1, a2, b2, h1, z, h2) = forward(api, shared, adapters, x, index, p, seed, offset)
    logp, entropy, lse, _, _ = api.haflo_label_logprobs(logits, label)
    d = api.haflo_label_logprobs_backward(logits, label, lse, entropy, -weight, out=logits)
    dz, da2, db2 = api.haflo_adapter_backward(d, z, shared[1], a2, b2, adapters.scale, index, h2, p, seed, offset + 2)
    dy = api.haflo_dropout(dz, p, seed, offset + 1)
    _, da1, db1 = api.haflo_adapter_backward(dy, x, shared[0], a1, b1, adapters.scale, index, h1, p, seed, offset, need_dx=False)
    for v, g in zip(adapters.values, (da1, db1, da2, db2)):
        v.sub_(g, alpha=rate)
    return logp


def run_round(api, pub, own, parties, rows, width, labels, rank, steps, seed=0, rate=0.1, p=0.05, timings=None):
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

    bf16 = torch.bfloat16
    shared = normal(width, width, by=width ** -0.5).to(bf16), normal(labels, width, by=width ** -0.5).to(bf16)
    kinds = normal(labels, width)  # a row is its label's kind and noise
    counts = [int(c) for c in rng.integers(rows // 2, rows + 1, parties)]
    index = torch.repeat_interleave(torch.arange(parties), torch.tensor(counts)).to(torch.int32).cuda()
    label = torch.from_numpy(rng.integers(0, labels, sum(counts)).astype(np.int32)).cuda()
    x = (kinds[label.long()] + 0.5 * normal(sum(counts), width)).to(bf16)
    weight = (1.0 / torch.tensor(counts, dtype=torch.float32, device="cuda"))[index.long()]
    first = [normal(rank, width, by=width ** -0.5), torch.zeros((width, rank), device="cuda"), normal(rank, width, by=width ** -0.5),
             torch.zeros((labels, rank), device="cuda")]
    adapters = Adapters(parties, width, labels, rank, [f.expand((parties,) + f.shape).clone() for f in first])

    def loss(of, rows_index):
        logits, _ = forward(api, shared, of, x, rows_index)
        return float(-api.haflo_label_logprobs(logits, label)[0].mean())

    before = loss(adapters, index)
    for n in range(steps):
        timed("parties: local steps", lambda: step(api, shared, adapters, x, label, index, weight, rate, p, seed, 3 * n))
    local = loss(adapters, index)

    total, lp = None, pub.plain_limbs
    flat = [adapters.flat(k) for k in range(parties)]
    for k in range(parties):
        r = rng.integers(0, 2 ** 32, size=(flat[k].numel(), lp), dtype=np.uint32)
        r[:, -1] &= 0x7FFFFFFF
        r = torch.from_numpy(r.view(np.int32)).cuda()
        c = timed("parties: encode + encrypt", lambda: api.haflo_encrypt(own, api.haflo_encode_f32(own, flat[k], SCALE_W), r))
        scaled = timed("coordinator: scalar_mul by n_k", lambda: api.haflo_scalar_mul_i64_bcast(pub, c, counts[k]))
        total = scaled if total is None else timed("coordinator: add", lambda: api.haflo_add(pub, total, scaled))
    sum_q, summed = timed("party: decrypt + decode", lambda: api.haflo_decode(own, api.haflo_decrypt(own, total), SCALE_W))

    common = Adapters.of_flat((summed / sum(counts)).to(torch.float32), width, labels, rank)
    after = loss(common, torch.zeros_like(index))
    none = torch.full((1,), -1, dtype=torch.int32, device="cuda")

    def answer():
        logits, _ = forward(api, shared, common, x[:1], torch.zeros_like(none))
        return api.haflo_label_logprobs(logits, none, top=5)

    _, _, _, top_logp, top_index = timed("party: one row's answer", answer)
    q = [np.rint(f.cpu().numpy().astype(np.float64) * 2.0 ** SCALE_W).astype(np.int64) for f in flat]
    return {
        "sum_q": sum_q.tolist(),
        "want_sum_q": sum(n * qk for n, qk in zip(counts, q)).tolist(),
        "loss": {"before": before, "local": local, "common": after},
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
        print("  %-32s %9.2f ms" % (name, ms))
    print("  mean loss: %.4f before, %.4f under each party's adapters, %.4f under their average"
          % (res["loss"]["before"], res["loss"]["local"], res["loss"]["common"]))
    print("  one row of label %d: %s" % (res["label"], ", ".join("%d (%.3f)" % a for a in res["answer"])))


if __name__ == "__main__":
    main()
