"""The operators at the vocabulary ends of a replay trainer, as cases that can be timed.

Kinds (``case["kind"]``):

* ``embed_fwd``  rows of the embedding table for a batch of tokens, scaled (``policy_embed_fwd``);
* ``embed_bwd``  the table's gradient from the gradient of those rows (``policy_embed_bwd``),
                 overwritten or added to the gradient that a tied head has already filled;
* ``verify``     drafted tokens accepted or replaced by the target's probabilities from given
                 random numbers, with the behaviour log-probs of what is emitted
                 (``policy_verify_drafts``); without drafts, one sampled token per sequence;
* ``distill``    the KL divergence from a teacher's top logits to the policy's logits, with its
                 gradient or alone (``policy_distill_fwd_bwd``).

``own`` false: the plain form, elementary torch operations; true: the package's entry points.
Sizes: heads from the tiny to the 7B one of ``paper_2604_08706_amd/workloads.py``, batches from
one token to the 16384 of the benchmark.
"""

import math

import torch

own = False


def listed():
    return [
        # the embedding of one decoding step of a few sequences, 0.5B table
        {"name": "embed_fwd_05b_step", "kind": "embed_fwd", "T": 5, "d": 896, "V": 151936,
         "scale": 1.0},
        # the embedding of a full micro-batch, 7B table
        {"name": "embed_fwd_7b", "kind": "embed_fwd", "T": 16384, "d": 3584, "V": 152064,
         "scale": 1.0},
        # the tiny model's gradient: a unit test, a tutorial; bound by launches
        {"name": "embed_bwd_tiny", "kind": "embed_bwd", "T": 256, "d": 64, "V": 1024,
         "scale": 8.0, "dx": "float32", "accumulate": False},
        # a 0.5B micro-batch whose head is not tied: the whole gradient is written
        {"name": "embed_bwd_05b_whole", "kind": "embed_bwd", "T": 10007, "d": 896, "V": 151936,
         "scale": 1.0, "dx": "bfloat16", "accumulate": False},
        # the 7B micro-batch, added to the gradient that the tied head filled
        {"name": "embed_bwd_7b_tied", "kind": "embed_bwd", "T": 16384, "d": 3584, "V": 152064,
         "scale": 1.0, "dx": "float32", "accumulate": True},
        # one decoding step without drafts: a token sampled per sequence
        {"name": "sample_05b", "kind": "verify", "B": 5, "K": 0, "V": 151936,
         "dtype": "bfloat16", "draft": "none", "temperature": 1.0},
        # a generation batch with a draft model's four tokens per sequence
        {"name": "verify_7b", "kind": "verify", "B": 64, "K": 4, "V": 152064,
         "dtype": "bfloat16", "draft": "model", "temperature": 1.0},
        # drafts copied from earlier rollouts (no draft distribution), ragged numbers of them
        {"name": "verify_lookup_15b", "kind": "verify", "B": 24, "K": 7, "V": 151936,
         "dtype": "float32", "draft": "lookup", "temperature": 0.75},
        # a short answer under the tiny vocabulary
        {"name": "distill_tiny", "kind": "distill", "T": 37, "V": 1024, "K": 8,
         "dtype": "float32", "temperature": 1.0, "grad": True, "mass": False},
        # the divergence alone, as an evaluation asks for it
        {"name": "distill_eval_15b", "kind": "distill", "T": 3003, "V": 151936, "K": 20,
         "dtype": "bfloat16", "temperature": 1.0, "grad": False, "mass": True},
        # one rollout's logits in 32 bits
        {"name": "distill_05b_f32", "kind": "distill", "T": 1301, "V": 151936, "K": 64,
         "dtype": "float32", "temperature": 2.0, "grad": True, "mass": False},
        # the full micro-batch under the 7B vocabulary
        {"name": "distill_7b", "kind": "distill", "T": 16384, "V": 152064, "K": 32,
         "dtype": "bfloat16", "temperature": 1.0, "grad": True, "mass": False},
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """A case of the same kinds: vocabularies from 1024 to 152064, widths from 64 to 3584, batches
    from one token to 16384, both types."""
    kind = rng.choice(["embed_fwd", "embed_bwd", "embed_bwd", "verify", "verify", "distill",
                       "distill"])
    V = _log_uniform(rng, 1024, 152064)
    if kind in ("embed_fwd", "embed_bwd"):
        case = {"kind": kind, "T": _log_uniform(rng, 1, 16384), "d": 8 * _log_uniform(rng, 8, 448),
                "V": V, "scale": rng.choice([1.0, 0.5, 8.0])}
        if kind == "embed_bwd":
            case["dx"] = rng.choice(["float32", "bfloat16"])
            case["accumulate"] = rng.random() < 0.6
        return case
    dtype = rng.choice(["bfloat16", "float32"])
    temperature = rng.choice([1.0, 1.0, 0.75, 1.5])
    if kind == "verify":
        draft = rng.choice(["none", "model", "model", "lookup"])
        return {"kind": kind, "B": _log_uniform(rng, 1, 64),
                "K": 0 if draft == "none" else rng.randint(1, 4 if draft == "model" else 8),
                "V": V, "dtype": dtype, "draft": draft, "temperature": temperature}
    return {"kind": kind, "T": _log_uniform(rng, 1, 8192), "V": V, "K": _log_uniform(rng, 1, 128),
            "dtype": dtype, "temperature": temperature, "grad": rng.random() < 0.8,
            "mass": rng.random() < 0.3}


# ---- inputs, from the seed alone ----------------------------------------------------------------


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + salt)
    return g


def _randn(shape, g, dtype=torch.float32, sd=1.0):
    """N(0, sd^2), made in pieces so that a large 16-bit tensor needs no 32-bit copy of itself."""
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - at)
        flat[at:at + n] = torch.randn(n, generator=g, device="cuda").mul_(sd)
    return x


def _tokens(T, V, g):
    """Token ids whose frequencies fall like 1 / rank, as a text's do; ranks are spread over the ids."""
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(V + 1)).floor().long() - 1
    return ((rank.clamp(0, V - 1) * 7919 + 13) % V).int()


def _sequences(T, g):
    """(seq_of_token, seq_len) of a packed batch of about 600-token sequences whose last thirtieth is
    padding."""
    B = 1 + T // 600
    valid = T - T // 30
    cuts = torch.rand(B - 1, generator=g, device="cuda").mul(valid).long().sort().values
    t = torch.arange(T, device="cuda")
    seq = torch.searchsorted(cuts, t, right=True).int()
    seq[valid:] = -1
    length = torch.bincount(seq[:valid].long(), minlength=B).clamp(min=1).int()
    return seq, length


def prepare(case, seed):
    kind, V = case["kind"], case["V"]
    g = _gen(seed, 1)
    st = {"case": case}
    if kind in ("embed_fwd", "embed_bwd"):
        T, d = case["T"], case["d"]
        st["tokens"] = _tokens(T, V, g)
        st["seq"], _ = _sequences(T, g)
        if kind == "embed_fwd":
            st["table"] = _randn((V, d), g, torch.bfloat16, 0.02)
            st["out"] = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
        else:
            st["dx"] = _randn((T, d), g, getattr(torch, case["dx"]), 1e-3)
            st["dW"] = _randn((V, d), g, torch.float32, 1e-3)
            if own:
                import paper_2604_08706_amd as rbp

                st["ws"] = rbp.workspace(rbp.RBP_OP_EMBED_BWD, T, d, V)
        return st
    dtype = getattr(torch, case["dtype"])
    if kind == "verify":
        B, K, draft = case["B"], case["K"], case["draft"]
        z = _randn((B, K + 1, V), g, torch.float32, 3.0)
        st["draft_logits"] = st["draft_tokens"] = st["n_draft"] = None
        if K:
            zd = z[:, :K] + _randn((B, K, V), g, torch.float32, 0.7)
            if draft == "lookup":  # mostly what the target finds likely
                zd = zd.mul_(1.5)
            pick = torch.rand((B, K, V), generator=g, device="cuda").log_().neg_().log_().neg_()
            st["draft_tokens"] = pick.add_(zd).argmax(-1).int()
            del pick
            if draft == "model":
                st["draft_logits"] = zd.to(dtype)
            st["n_draft"] = torch.randint(0, K + 1, (B,), generator=g, device="cuda",
                                          dtype=torch.int32)
            if draft == "model":
                st["n_draft"].fill_(K)
            del zd
        st["logits"] = z.to(dtype)
        st["u"] = torch.rand((B, K + 1), generator=g, device="cuda")
        st["out_tokens"] = torch.empty((B, K + 1), dtype=torch.int32, device="cuda")
        st["out_logp"] = torch.empty((B, K + 1), device="cuda")
        st["n_out"] = torch.empty(B, dtype=torch.int32, device="cuda")
        if own:
            import paper_2604_08706_amd as rbp

            st["ws"] = rbp.workspace(rbp.RBP_OP_VERIFY, B, K, V)
        return st
    T, K = case["T"], case["K"]
    st["logits"] = _randn((T, V), g, dtype, 2.0)
    # a teacher's top logits, in falling order, at ids anywhere in the vocabulary
    st["ids"] = torch.randint(0, V, (T, K), generator=g, device="cuda", dtype=torch.int32)
    st["teacher"] = torch.randn((T, K), generator=g, device="cuda").mul_(2.0).add_(8.0) \
        .sort(dim=1, descending=True).values.contiguous()
    st["mass"] = (torch.logsumexp(st["teacher"] / case["temperature"], 1)
                  + 0.3 * torch.rand(T, generator=g, device="cuda")) if case["mass"] else None
    st["seq"], st["len"] = _sequences(T, g)
    st["kl"] = torch.empty(T, device="cuda")
    st["loss"] = torch.zeros(1, device="cuda")
    st["stats"] = torch.zeros(2, device="cuda")
    st["dlogits"] = torch.empty_like(st["logits"]) if case["grad"] else None
    if own:
        import paper_2604_08706_amd as rbp

        st["ws"] = rbp.workspace(rbp.RBP_OP_DISTILL, T, K, V)
    return st


# ---- one pass -----------------------------------------------------------------------------------


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"embed_fwd": _embed_fwd_own, "embed_bwd": _embed_bwd_own, "verify": _verify_own,
                "distill": _distill_own}[kind](state)
    return {"embed_fwd": _embed_fwd, "embed_bwd": _embed_bwd, "verify": _verify,
            "distill": _distill}[kind](state)


def _embed_fwd_own(st):
    import paper_2604_08706_amd as rbp

    rbp.policy_embed_fwd(st["table"], st["tokens"], st["seq"], st["out"],
                         scale=st["case"]["scale"])
    return st["out"]


def _embed_bwd_own(st):
    import paper_2604_08706_amd as rbp

    c = st["case"]
    rbp.policy_embed_bwd(st["dx"], st["tokens"], st["seq"], st["dW"], st["ws"], scale=c["scale"],
                         accumulate_dW=c["accumulate"])
    return st["dW"]


def _verify_own(st):
    import paper_2604_08706_amd as rbp

    rbp.policy_verify_drafts(st["logits"], st["draft_logits"], st["draft_tokens"], st["n_draft"],
                             st["u"], st["out_tokens"], st["out_logp"], st["n_out"], st["ws"],
                             temperature=st["case"]["temperature"])
    return {"tokens": st["out_tokens"], "logp": st["out_logp"], "n": st["n_out"]}


def _distill_own(st):
    import paper_2604_08706_amd as rbp

    c = st["case"]
    rbp.policy_distill_fwd_bwd(st["logits"], st["ids"], st["teacher"], st["mass"], st["seq"],
                               st["len"], st["len"].numel(), st["kl"], st["loss"], st["stats"],
                               st["dlogits"], st["ws"], temperature=c["temperature"], scale=0.5)
    return {"kl": st["kl"], "loss": st["loss"], "stats": st["stats"], "dlogits": st["dlogits"]}


def _embed_fwd(st):
    rows = st["table"][st["tokens"].long()].float() * st["case"]["scale"]
    st["out"].copy_(rows.masked_fill_((st["seq"] < 0)[:, None], 0.0))
    return st["out"]


def _embed_bwd(st):
    c = st["case"]
    dx = st["dx"].double().mul_(c["scale"]).masked_fill_((st["seq"] < 0)[:, None], 0.0)
    start = st["dW"].double() if c["accumulate"] else torch.zeros_like(st["dW"], dtype=dx.dtype)
    st["dW"].copy_(start.index_add_(0, st["tokens"].long(), dx))
    return st["dW"]


def _softmax64(z, temperature):
    z = z.double() / temperature
    e = torch.exp(z - z.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _verify(st):
    c = st["case"]
    B, K, V = c["B"], c["K"], c["V"]
    # in 64 bits: the draws lie next to borders of a distribution over up to 152064 tokens
    p = _softmax64(st["logits"], c["temperature"])
    b = torch.arange(B, device="cuda")
    if K:
        x = st["draft_tokens"].long()
        px = p[:, :K].gather(2, x[..., None])[..., 0]
        if st["draft_logits"] is not None:
            q = _softmax64(st["draft_logits"], c["temperature"])
            qx = q.gather(2, x[..., None])[..., 0]
        else:
            q, qx = None, torch.ones_like(px)
        k = torch.arange(K, device="cuda")
        ok = (st["u"][:, :K].double() * qx < px) & (k < st["n_draft"][:, None])
        n = ok.long().cumprod(1).sum(1)
        rejected = n < st["n_draft"]
        at = n.clamp(max=K - 1)
        row = p[b, n]
        if q is not None:
            left = (row - q[b, at]).clamp_(min=0.0)
        else:
            left = row.scatter(1, x[b, at][:, None], 0.0)
        weight = torch.where((rejected & (left.sum(1) > 0))[:, None], left, row)
    else:
        x = torch.zeros((B, 0), dtype=torch.long, device="cuda")
        n = torch.zeros(B, dtype=torch.long, device="cuda")
        weight = p[:, 0]
    cdf = weight.cumsum(1)
    hit = (cdf > st["u"][:, K:].double() * cdf[:, -1:]) & (weight > 0)
    token = torch.where(hit, torch.arange(V, device="cuda"), V).amin(1)
    emitted = torch.cat([x, torch.zeros((B, 1), dtype=torch.long, device="cuda")], 1)
    emitted[b, n] = token
    place = torch.arange(K + 1, device="cuda")
    lp = p.gather(2, emitted[..., None])[..., 0].log()
    st["out_tokens"].copy_(torch.where(place <= n[:, None], emitted, -1))
    st["out_logp"].copy_(torch.where(place <= n[:, None], lp, 0.0))
    st["n_out"].copy_(n + 1)
    return {"tokens": st["out_tokens"], "logp": st["out_logp"], "n": st["n_out"]}


def _distill(st):
    c = st["case"]
    tau, scale, n_seq = c["temperature"], 0.5, st["len"].numel()
    valid = st["seq"] >= 0
    z = st["logits"].float()
    if tau != 1.0:
        z = z / tau
    m = z.amax(1, keepdim=True)
    zk = z.gather(1, st["ids"].long())
    e = torch.exp_(z.sub_(m) if z.data_ptr() != st["logits"].data_ptr() else z - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    lt = st["teacher"] / tau
    mass = st["mass"][:, None] if st["mass"] is not None else torch.logsumexp(lt, 1, keepdim=True)
    logp = lt - mass
    p = torch.exp(logp)
    kl = (p * (logp - zk + lse)).sum(1).masked_fill(~valid, 0.0)
    w = (scale / n_seq) / st["len"][st["seq"].clamp(min=0).long()].float()
    w = torch.where(valid, w, 0.0)
    st["kl"].copy_(kl)
    st["loss"] += (w * kl).double().sum()
    st["stats"] += torch.stack([valid.double().sum(), kl.double().sum()])
    if st["dlogits"] is not None:
        w = w[:, None] / tau
        dz = e.mul_(w * p.sum(1, keepdim=True) / total)
        st["dlogits"].copy_(dz.scatter_add_(1, st["ids"].long(), -w * p))
    return {"kl": st["kl"], "loss": st["loss"], "stats": st["stats"], "dlogits": st["dlogits"]}


# ---- what a pass cannot do without ----------------------------------------------------------------


def _distinct(T, V):
    """Expected number of distinct ids among T tokens of _tokens."""
    r = torch.arange(1, V + 1, dtype=torch.float64)
    p = torch.log1p(1.0 / r) / math.log(V + 1)
    return float((1.0 - torch.exp(T * torch.log1p(-p))).sum())


def work(case):
    kind, V = case["kind"], case["V"]
    if kind == "embed_fwd":
        T, d = case["T"], case["d"]
        return {"bytes": _distinct(T, V) * d * 2 + T * d * 2 + 8 * T}
    if kind == "embed_bwd":
        T, d = case["T"], case["d"]
        dw = _distinct(T, V) * d * 8 if case["accumulate"] else V * d * 4
        return {"bytes": T * d * (4 if case["dx"] == "float32" else 2) + dw + 8 * T,
                "flops": T * d}
    s = 4 if case["dtype"] == "float32" else 2
    if kind == "verify":
        rows = case["K"] + 1 + (case["K"] if case["draft"] == "model" else 0)
        return {"bytes": case["B"] * rows * V * s, "flops": 4 * case["B"] * rows * V}
    T, K = case["T"], case["K"]
    return {"bytes": T * V * s * (2 if case["grad"] else 1) + 8 * T * K, "flops": 6 * T * V}


# ---- the definitions in 64 bits -------------------------------------------------------------------


def exact(case, seed):
    st = prepare(case, seed)
    kind, V = case["kind"], case["V"]
    if kind == "embed_fwd":
        keep = (st["seq"] >= 0).double()
        picked = torch.index_select(st["table"], 0, st["tokens"])
        return picked.double() * (keep * case["scale"])[:, None]
    if kind == "embed_bwd":
        order = torch.argsort(st["tokens"].long() * case["T"] + torch.arange(case["T"], device="cuda"))
        order = order[(st["seq"] >= 0)[order]]
        ids, counts = torch.unique_consecutive(st["tokens"][order], return_counts=True)
        out = st["dW"].double() if case["accumulate"] else \
            torch.zeros((V, case["d"]), dtype=torch.float64, device="cuda")
        run_of = torch.repeat_interleave(torch.arange(ids.numel(), device="cuda"), counts)
        for rows in torch.arange(ids.numel(), device="cuda").split(4096):
            here = (run_of >= rows[0]) & (run_of <= rows[-1])
            grads = st["dx"][order[here]].double()
            ends = torch.cumsum(counts[rows], 0)
            sums = torch.cat([grads.new_zeros((1, case["d"])), torch.cumsum(grads, 0)])
            out[ids[rows].long()] += case["scale"] * (sums[ends] - sums[ends - counts[rows]])
        return out
    tau = case["temperature"]
    if kind == "verify":
        B, K = case["B"], case["K"]
        tokens = torch.full((B, K + 1), -1, dtype=torch.int32)
        logp = torch.zeros((B, K + 1), dtype=torch.float64)
        count = torch.zeros(B, dtype=torch.int32)
        u = st["u"].double().cpu()
        for i in range(B):
            drafts = int(st["n_draft"][i]) if K else 0
            n = 0
            while True:
                lp = torch.log_softmax(st["logits"][i, n].double() / tau, 0)
                weight = torch.exp(lp)
                if n == drafts:
                    break
                x = int(st["draft_tokens"][i, n])
                if st["draft_logits"] is not None:
                    lq = torch.log_softmax(st["draft_logits"][i, n].double() / tau, 0)
                else:
                    lq = torch.full_like(lp, -math.inf)
                    lq[x] = 0.0
                if float(u[i, n]) < math.exp(float(lp[x]) - float(lq[x])):
                    tokens[i, n], logp[i, n] = x, float(lp[x])
                    n += 1
                    continue
                rest = torch.relu(weight - torch.exp(lq))
                weight = rest if float(rest.sum()) > 0 else weight
                break
            cdf = torch.cumsum(weight, 0)
            v = int(torch.searchsorted(cdf, u[i, K].cuda() * cdf[-1], right=True))
            tokens[i, n], logp[i, n], count[i] = v, float(lp[v]), n + 1
        return {"tokens": tokens, "logp": logp, "n": count}
    T, n_seq = case["T"], st["len"].numel()
    kl = torch.zeros(T, dtype=torch.float64, device="cuda")
    weight = torch.zeros(T, dtype=torch.float64, device="cuda")
    grad = torch.empty((T, V), dtype=torch.float64, device="cuda") if case["grad"] else None
    for rows in torch.arange(T, device="cuda").split(max(1, (1 << 28) // V)):
        live = (st["seq"][rows] >= 0).double()
        weight[rows] = live * 0.5 / (n_seq * st["len"].double()[st["seq"][rows].clamp(min=0).long()])
        lq = torch.log_softmax(st["logits"][rows].double() / tau, 1)
        top = st["teacher"][rows].double() / tau
        lp = torch.log_softmax(top, 1) if st["mass"] is None else top - st["mass"][rows, None].double()
        ids = st["ids"][rows].long()
        kl[rows] = live * (lp.exp() * (lp - torch.gather(lq, 1, ids))).sum(1)
        if grad is not None:
            target = torch.zeros_like(lq).scatter_add_(1, ids, lp.exp())
            target = lp.exp().sum(1, keepdim=True) * lq.exp() - target
            grad[rows] = target * (weight[rows] / tau)[:, None]
    stats = torch.stack([(st["seq"] >= 0).double().sum(), kl.sum()])
    return {"kl": kl, "loss": (weight * kl).sum().reshape(1), "stats": stats, "dlogits": grad}
