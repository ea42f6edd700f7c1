"""Cases of the language-model operators: embedding lookup and its gradient, products grouped by expert, distillation.

Each case is one call (or one forward / one backward) as a training or serving program makes it.  `run` computes it in
elementary torch operations, or, where `own` is true, through the library's binding.  Token ids follow a Zipf law (the
k-th most frequent id has probability ~ 1/k), as text does; expert shares are uneven, as a router's are.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one decoding step of a small batch: eight tokens looked up, latency counts
        dict(name="lookup_8_tokens", op="lookup", T=8, V=32768, D=1024, src="bf16", dst="bf16", idx="i64"),
        # the tokens of a large training batch, master table in bf16
        dict(name="lookup_64k_tokens", op="lookup", T=65536, V=131072, D=2048, src="bf16", dst="bf16", idx="i64"),
        # a few hundred ids of a table as large as the matrix factorisation's item table (2^14 items, 64 factors)
        dict(name="lookup_grad_512_f64factors", op="lookup_grad", T=512, V=16384, D=64, src="f32", dst="f32", idx="i32"),
        # odd row length (no vector access possible), odd counts
        dict(name="lookup_grad_odd", op="lookup_grad", T=12289, V=50021, D=1001, src="f32", dst="f32", idx="i64"),
        # one large batch, gradient in fp32: the rank buffer that the allreduce combines
        dict(name="lookup_grad_128k", op="lookup_grad", T=131072, V=131072, D=2048, src="bf16", dst="f32", idx="i64"),
        # a short sequence: 16 tokens against a teacher's eight best
        dict(name="distill_step_16", op="distill_step", T=16, V=32768, K=8, src="bf16", tau=1.0, lse=False),
        # loss and gradient of a large batch over a large vocabulary in one pass, teacher's probabilities absolute
        dict(name="distill_step_8k", op="distill_step", T=8192, V=131072, K=64, src="bf16", tau=2.0, lse=True),
        # evaluation: the loss alone, fp32 logits with an odd row length
        dict(name="distill_loss_odd", op="distill_loss", T=2047, V=50021, K=50, src="f32", tau=1.5, lse=False),
        # the gradient alone, as an automatic differentiation calls it with the gradient of every token's loss
        dict(name="distill_grad_4k", op="distill_grad", T=4096, V=32768, K=32, src="bf16", tau=1.0, lse=True),
        # serving: 64 tokens on 32 experts, most of them with a row or two
        dict(name="experts_64_tokens", op="experts", T=64, E=32, N=512, K=1024, dst="bf16"),
        # a large batch after its exchange, uneven shares
        dict(name="experts_32k", op="experts", T=32768, E=16, N=4096, K=2048, dst="bf16"),
        # its backward pass: gradient of the rows and (fp32: rank buffers) of the weights
        dict(name="experts_grad_8k", op="experts_grad", T=8191, E=16, N=1024, K=2048, dst="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["lookup", "lookup_grad", "distill_step", "distill_loss", "distill_grad", "experts", "experts_grad"])
    while True:
        if op in ("lookup", "lookup_grad"):
            c = dict(op=op, T=_log(rng, 8, 131072), V=_log(rng, 4096, 131072), D=_log(rng, 64, 2048),
                     src=rng.choice(["f32", "bf16"]), dst=rng.choice(["f32", "bf16"]), idx=rng.choice(["i32", "i64"]))
            if rng.random() < 0.6:
                c["D"] = max(64, c["D"] // 8 * 8)
        elif op.startswith("distill"):
            c = dict(op=op, T=_log(rng, 16, 8192), V=_log(rng, 8192, 131072), K=_log(rng, 8, 64),
                     src=rng.choice(["f32", "bf16"]), tau=rng.choice([1.0, 1.5, 2.0]), lse=rng.random() < 0.5)
            if rng.random() < 0.6:
                c["V"] = c["V"] // 64 * 64
        else:
            c = dict(op=op, T=_log(rng, 64, 32768), E=_log(rng, 4, 64), N=_log(rng, 64, 512) * 8, K=_log(rng, 64, 256) * 8,
                     dst=rng.choice(["f32", "bf16"]))
        w = work(c)
        if w["bytes"] <= 4.0e9 and w["flops"] <= 5.5e11 and 3 << 10 not in c.values():     # (no case has a size of 3 * 2^10)
            return c


def _gen(seed, k):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + k) % (1 << 62))


def _normal(seed, k, shape, dtype, std=1.0):
    x = torch.empty(shape, dtype=dtype, device="cuda")
    return x.normal_(0.0, std, generator=_gen(seed, k))


def _zipf(seed, T, V):
    """T ids, the frequent ones spread over the vocabulary; one in fifty is padding (-1)."""
    u = torch.rand(T, dtype=torch.float64, device="cuda", generator=_gen(seed, 1))
    rank = (torch.exp(u * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    step = next(s for s in range(int(V * 0.618) | 1, 2 * V + 3, 2) if math.gcd(s, V) == 1)
    ids = rank * step % V
    pad = torch.rand(T, device="cuda", generator=_gen(seed, 2)) < 0.02
    return torch.where(pad, torch.full_like(ids, -1), ids)


def _distinct(T, V):
    """Expected number of distinct ids among T draws of _zipf."""
    n, k = 0.0, 1
    while k <= V:                                   # ranks in blocks of nearly equal probability
        j = min(V, max(k, int(k * 1.02)))
        p = math.log((j + 1.0) / k) / math.log(V + 1.0) / (j - k + 1) * 0.98
        n += (j - k + 1) * -math.expm1(T * math.log1p(-p))
        k = j + 1
    return n


def _shares(seed, T, E):
    """Exclusive prefix sums of the experts' row counts: uneven, one in eight experts empty where there are eight."""
    w = torch.rand(E, dtype=torch.float64, device="cuda", generator=_gen(seed, 3)).square_().add_(0.05)
    if E >= 8:
        w[torch.randperm(E, device="cuda", generator=_gen(seed, 4))[: E // 8]] = 0.0
    cut = torch.zeros(E + 1, dtype=torch.float64, device="cuda")
    cut[1:] = torch.cumsum(w, 0) / w.sum() * T
    displs = cut.round().long()
    displs[E] = T
    return displs


def prepare(case, seed):
    c, s = case, dict(case)
    if c["op"] in ("lookup", "lookup_grad"):
        s["tokens"] = _zipf(seed, c["T"], c["V"]).to(torch.int32 if c["idx"] == "i32" else torch.int64)
        s["scale"] = math.sqrt(c["D"])
        if c["op"] == "lookup":
            s["table"] = _normal(seed, 5, (c["V"], c["D"]), DT[c["src"]], 0.02)
            s["out"] = torch.empty(c["T"], c["D"], dtype=DT[c["dst"]], device="cuda")
        else:
            s["dout"] = _normal(seed, 6, (c["T"], c["D"]), DT[c["src"]], 1e-2)
            s["grad"] = torch.empty(c["V"], c["D"], dtype=DT[c["dst"]], device="cuda")
    elif c["op"].startswith("distill"):
        T, V, K, dt = c["T"], c["V"], c["K"], DT[c["src"]]
        real = V - V // 512                          # the last columns pad the vocabulary: masked with -inf
        s["logits"] = _normal(seed, 7, (T, V), dt, 2.0)
        s["logits"][:, real:] = -math.inf
        width = real // K
        at = torch.randint(real, (T, 1), device="cuda", generator=_gen(seed, 8)) + torch.arange(K, device="cuda") * width
        at = (at + torch.randint(width, (T, K), device="cuda", generator=_gen(seed, 9))) % real
        have = torch.randint(K // 2, K + 1, (T, 1), device="cuda", generator=_gen(seed, 10))      # shorter lists end in -1
        have[torch.rand(T, 1, device="cuda", generator=_gen(seed, 11)) < 0.02] = 0                # a few tokens without any
        at[torch.arange(K, device="cuda") >= have] = -1
        s["top_index"] = at.to(torch.int32)
        top = torch.sort(_normal(seed, 12, (T, K), torch.float32, 2.0), dim=1, descending=True).values + 4.0
        s["top_logit"] = top.contiguous()
        s["teacher_lse"] = None
        if c["lse"]:
            kept = 0.7 + 0.3 * torch.rand(T, device="cuda", generator=_gen(seed, 13))
            s["teacher_lse"] = torch.logsumexp(torch.where(at >= 0, top / c["tau"], -1e30), 1) - torch.log(kept)
        s["weight"] = torch.full((T,), 1.0 / T, device="cuda")
        s["weight"][torch.rand(T, device="cuda", generator=_gen(seed, 14)) < 0.05] = 0.0          # padding
        s["loss"], s["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        if c["op"] != "distill_loss":
            s["dlogits"] = torch.empty(T, V, dtype=dt, device="cuda")
        if c["op"] == "distill_grad":
            s["dloss"] = 0.5 + torch.rand(T, device="cuda", generator=_gen(seed, 15))
            for i in range(0, T, 256):               # what the forward pass left
                s["lse"][i:i + 256] = torch.logsumexp(s["logits"][i:i + 256].float() / c["tau"], 1)
    else:
        T, E, N, K = c["T"], c["E"], c["N"], c["K"]
        s["displs"] = _shares(seed, T, E)
        s["cuts"] = s["displs"].tolist()             # a host copy: the plain form's slices need it, the library's calls do not
        s["w"] = _normal(seed, 16, (E, N, K), torch.bfloat16, 1.0 / math.sqrt(K))
        s["x"] = _normal(seed, 17, (T, K), torch.bfloat16)
        if c["op"] == "experts":
            s["y"] = torch.empty(T, N, dtype=DT[c["dst"]], device="cuda")
        else:
            s["dy"] = _normal(seed, 18, (T, N), torch.bfloat16, 1e-2)
            s["dx"] = torch.empty(T, K, dtype=torch.bfloat16, device="cuda")
            s["dw"] = torch.empty(E, N, K, dtype=DT[c["dst"]], device="cuda")
    return s


def _teacher(s):
    """Teacher's probabilities [T][K], 0 for absent entries, and which rows count."""
    a = s["top_logit"].float() / s["tau"]
    there = s["top_index"] >= 0
    rows = there.any(1) & (s["weight"] != 0)
    if s["teacher_lse"] is not None:
        p = torch.exp(a - s["teacher_lse"][:, None])
    else:
        a = torch.where(there, a, torch.full_like(a, -1e30))
        p = torch.exp(a - a.max(1, keepdim=True).values)
        p = p / torch.where(there, p, torch.zeros_like(p)).sum(1, keepdim=True).clamp_min(1e-30)
    return torch.where(there & rows[:, None], p, torch.zeros_like(p)), rows


def _plain(s):
    op = s["op"]
    if op == "lookup":
        there = (s["tokens"] >= 0) & (s["tokens"] < s["V"])
        rows = s["table"][s["tokens"].clamp(0, s["V"] - 1)].float() * s["scale"]
        return (rows * there[:, None]).to(s["out"].dtype)
    if op == "lookup_grad":
        there = (s["tokens"] >= 0) & (s["tokens"] < s["V"])
        grad = torch.zeros(s["V"], s["D"], device="cuda")
        grad.index_add_(0, s["tokens"].clamp(0, s["V"] - 1), s["dout"].float() * there[:, None])
        return (grad * s["scale"]).to(s["grad"].dtype)
    if op.startswith("distill"):
        p, rows = _teacher(s)
        at = s["top_index"].clamp_min(0).long()
        u = s["logits"].float() / s["tau"]
        if op == "distill_grad":
            lse = s["lse"]
        else:
            top = u.max(1).values
            lse = top + torch.log(torch.exp(u - top[:, None]).sum(1))
        if op != "distill_grad":
            logp = torch.log(torch.where(p > 0, p, torch.ones_like(p)))
            loss = s["weight"] * (p * (logp - u.gather(1, at) + lse[:, None])).sum(1)
            loss = torch.where(rows, loss, torch.zeros_like(loss))
            kept = torch.where(rows, lse, torch.full_like(lse, -math.inf))
            if op == "distill_loss":
                return loss, kept
        g = s["weight"] / s["tau"] * (s["dloss"] if op == "distill_grad" else 1.0)
        d = torch.exp(u - lse[:, None]) * p.sum(1)[:, None]
        d.scatter_add_(1, at, -p)
        d = torch.where(rows[:, None], d * g[:, None], torch.zeros_like(d)).to(s["logits"].dtype)
        return d if op == "distill_grad" else (loss, kept, d)
    cuts = s["cuts"]
    if op == "experts":
        y = [s["x"][a:b].float() @ s["w"][e].float().T for e, (a, b) in enumerate(zip(cuts, cuts[1:]))]
        return torch.cat(y).to(s["y"].dtype)
    dx = [s["dy"][a:b].float() @ s["w"][e].float() for e, (a, b) in enumerate(zip(cuts, cuts[1:]))]
    dw = [s["dy"][a:b].float().T @ s["x"][a:b].float() for a, b in zip(cuts, cuts[1:])]
    return torch.cat(dx).to(s["dx"].dtype), torch.stack(dw).to(s["dw"].dtype)


def run(s):
    if not own:
        return _plain(s)
    from paper_2203_17063_b200 import binding as ec

    op = s["op"]
    if op == "lookup":
        ec.embed_lookup(s["table"], s["tokens"], s["out"], s["scale"])
        return s["out"]
    if op == "lookup_grad":
        if "workspace" not in s:                     # kept from step to step, as a training loop does
            need = ec.embed_grad_workspace_bytes(s["T"], s["V"], s["D"])
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        ec.embed_grad(s["dout"], s["tokens"], s["grad"], s["workspace"], s["scale"])
        return s["grad"]
    if op == "distill_loss":
        ec.distill_loss(s["logits"], s["top_index"], s["top_logit"], s["loss"], s["lse"], s["tau"], s["weight"], s["teacher_lse"])
        return s["loss"], s["lse"]
    if op == "distill_grad":
        ec.distill_grad(s["logits"], s["top_index"], s["top_logit"], s["lse"], s["dlogits"], s["tau"], s["weight"],
                        s["teacher_lse"], s["dloss"])
        return s["dlogits"]
    if op == "distill_step":
        ec.distill_step(s["logits"], s["top_index"], s["top_logit"], s["loss"], s["lse"], s["dlogits"], s["tau"], s["weight"],
                        s["teacher_lse"])
        return s["loss"], s["lse"], s["dlogits"]
    if op == "experts":
        ec.expert_forward(s["x"], s["displs"], s["w"], s["y"])
        return s["y"]
    ec.expert_input_grad(s["dy"], s["displs"], s["w"], s["dx"])
    ec.expert_weight_grad(s["dy"], s["x"], s["displs"], s["dw"])
    return s["dx"], s["dw"]


def work(case):
    c = case
    if c["op"] in ("lookup", "lookup_grad"):
        T, V, D, ids = c["T"], c["V"], c["D"], c["T"] * (4 if c["idx"] == "i32" else 8)
        if c["op"] == "lookup":
            return {"bytes": ids + _distinct(T, V) * D * SIZE[c["src"]] + T * D * SIZE[c["dst"]], "flops": T * D}
        return {"bytes": ids + T * D * SIZE[c["src"]] + V * D * SIZE[c["dst"]], "flops": T * D + V * D}
    if c["op"].startswith("distill"):
        n, lists = c["T"] * c["V"], c["T"] * (c["K"] * 8 + 16)
        return {"bytes": n * SIZE[c["src"]] * (1 if c["op"] == "distill_loss" else 2) + lists, "flops": 4 * n}
    T, E, N, K = c["T"], c["E"], c["N"], c["K"]
    f = 2.0 * T * N * K
    if c["op"] == "experts":
        return {"bytes": 2.0 * (T * K + E * N * K) + T * N * SIZE[c["dst"]], "flops": f}
    return {"bytes": 2.0 * (2 * T * K + T * N + E * N * K) + E * N * K * SIZE[c["dst"]], "flops": 2 * f}


def exact(case, seed):
    s = prepare(case, seed)
    op, f64 = s["op"], torch.float64
    if op == "lookup":
        padded = torch.cat([s["table"], s["table"].new_zeros(1, s["D"])])
        return padded[torch.where(s["tokens"] < 0, s["V"], s["tokens"].long())].to(f64) * s["scale"]
    if op == "lookup_grad":
        order = torch.argsort(s["tokens"].long(), stable=True)
        ids, n = torch.unique_consecutive(s["tokens"].long()[order], return_counts=True)
        sums = torch.segment_reduce(s["dout"].to(f64)[order], "sum", lengths=n, axis=0)
        grad = torch.zeros(s["V"], s["D"], dtype=f64, device="cuda")
        grad[ids[ids >= 0]] = sums[ids >= 0] * s["scale"]
        return grad
    if op.startswith("distill"):
        T, V, tau = s["T"], s["V"], s["tau"]
        loss, kept = torch.zeros(T, dtype=f64, device="cuda"), torch.full((T,), -math.inf, dtype=f64, device="cuda")
        grad = torch.zeros(T, V, dtype=f64, device="cuda") if op != "distill_loss" else None
        use = torch.nonzero((s["weight"] != 0) & (s["top_index"] >= 0).any(1)).flatten()
        for at in use.split(512):
            z = s["logits"][at].to(f64) / tau
            lse = s["lse"][at].to(f64) if op == "distill_grad" else torch.logsumexp(z, 1)
            idx = s["top_index"][at].long()
            a = (s["top_logit"][at].to(f64) / tau).masked_fill(idx < 0, -math.inf)
            logp = a - (torch.logsumexp(a, 1) if s["teacher_lse"] is None else s["teacher_lse"][at].to(f64))[:, None]
            p = logp.exp()
            logq = z.gather(1, idx.clamp_min(0)) - lse[:, None]
            w = s["weight"][at].to(f64)
            loss[at] = w * torch.where(idx >= 0, p * (logp - logq), 0.0).sum(1)
            kept[at] = lse
            if grad is not None:
                q = (z - lse[:, None]).exp_().mul_(p.sum(1)[:, None])
                q.scatter_add_(1, idx.clamp_min(0), -p)
                if op == "distill_grad":
                    w = w * s["dloss"][at].to(f64)
                grad[at] = q.mul_((w / tau)[:, None])
        return {"distill_loss": (loss, kept), "distill_grad": grad, "distill_step": (loss, kept, grad)}[op]
    E, cuts = s["E"], s["cuts"]
    if op == "experts":
        y = torch.zeros(s["T"], s["N"], dtype=f64, device="cuda")
        for e in range(E):
            y[cuts[e]:cuts[e + 1]] = torch.mm(s["x"][cuts[e]:cuts[e + 1]].to(f64), s["w"][e].to(f64).t())
        return y
    dx = torch.zeros(s["T"], s["K"], dtype=f64, device="cuda")
    dw = torch.zeros(E, s["N"], s["K"], dtype=f64, device="cuda")
    for e in range(E):
        x, dy = s["x"][cuts[e]:cuts[e + 1]].to(f64), s["dy"][cuts[e]:cuts[e + 1]].to(f64)
        dx[cuts[e]:cuts[e + 1]] = torch.mm(dy, s["w"][e].to(f64))
        dw[e] = torch.mm(dy.t(), x)
    return dx, dw
