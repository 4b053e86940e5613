"""The operators of a decode step in which every row picks weights of its own, each beside its plain form.

An operator is one of

  route     logits of a router to the ``top_k`` experts of every token and their softmax weights.
  moe       a whole mixture-of-experts layer on 4-bit experts, from the router's logits to the layer's output:
            out[m] = sum_j w[m, j] * (silu(x[m] G_e) * (x[m] U_e)) D_e  with e the token's j-th expert, where G_e, U_e (gate
            and up, one packed matrix) and D_e (down) are dequantised as everywhere in this library.
  experts   the same from given experts and weights (a router of another kind, or experts spread over several GPUs:
            those that live elsewhere have the id -1 and add nothing).
  lora      a shared 4-bit projection with the low-rank adapter of every row's own request beside it:
            out[m] = x[m] W + s_l (x[m] A_l^T) B_l^T  with l the row's adapter, or none.
  lora_add  the adapters alone, added to the output of a projection that has been made (here the first columns of a
            wider one: adapters on the queries of a fused projection of queries, keys and values).

Where ``own`` is false ``run`` computes them in elementary torch operations in 32 bits, rounded once at the end.
Codes, zero points and scales have the distributions of the library's workloads: codes and zero points uniform in
0..15, scales uniform in 0.001..0.01; inputs are drawn on the GPU from the seed.
"""
import math

import torch

own = False

HIDDEN, INTER = 4096, 11008  # of the 7B set of the library's workloads
QKV = 12288


def _route(name, m, experts, top_k, dtype="fp16", renormalize=True):
    return {"name": name, "op": "route", "m": m, "experts": experts, "top_k": top_k, "dtype": dtype,
            "renormalize": renormalize}


def _moe(name, op, m, hidden, inter, experts, top_k, group=128, dtype="fp16", absent=0.0):
    return {"name": name, "op": op, "m": m, "hidden": hidden, "inter": inter, "experts": experts, "top_k": top_k,
            "group": group, "dtype": dtype, "absent": absent, "renormalize": True}


def _lora(name, op, m, k, n, rank, adapters, group=128, packed=False, bare=0.0, row=0):
    return {"name": name, "op": op, "m": m, "k": k, "n": n, "rank": rank, "adapters": adapters, "group": group,
            "packed": packed, "bare": bare, "row": row or n}


def listed():
    return [
        # the smallest call: the experts of one token
        _route("route_m1", 1, 8, 2),
        # routing a prompt's tokens over many experts
        _route("route_m2048", 2048, 64, 6, dtype="fp32", renormalize=False),
        # single-stream decoding through a layer of few large experts
        _moe("moe_m1", "moe", 1, HIDDEN, INTER, 8, 2),
        # the largest: a decode step of 64 streams through the same layer; every expert is hit
        _moe("moe_m64", "moe", 64, HIDDEN, INTER, 8, 2),
        # single-stream decoding through many small experts, where latency counts
        _moe("moe_small_m1", "moe", 1, 2048, 1024, 64, 4, dtype="fp32"),
        # sixteen streams on one of two GPUs that hold half of the experts each
        _moe("experts_m16", "experts", 16, 2048, 1024, 64, 4, absent=0.5),
        # an odd batch on a layer with small groups whose sizes are no multiple of a tile
        _moe("experts_ragged_m33", "experts", 33, 2752, 1376, 12, 3, group=32),
        # one request with an adapter on an attention output projection
        _lora("lora_m1", "lora", 1, HIDDEN, HIDDEN, 16, 16),
        # a decode step of 32 requests, each with an adapter of its own choice; some have none
        _lora("lora_m32", "lora", 32, HIDDEN, QKV, 16, 32, bare=0.1),
        # prompts of several requests packed into one chunk of 512 tokens
        _lora("lora_m512", "lora", 512, HIDDEN, QKV, 32, 8, packed=True, bare=0.1),
        # adapters of a higher rank on the queries of a fused projection
        _lora("lora_add_m16", "lora_add", 16, HIDDEN, HIDDEN, 64, 16, row=QKV),
        # an odd batch and rank on an odd layer
        _lora("lora_add_m77", "lora_add", 77, 2752, 6888, 24, 5, bare=0.2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _multiple(rng, lo, hi, unit):
    return max(1, round(_log_int(rng, lo, hi) / unit)) * unit


def draw(rng):
    """One more case: routing of 1..4096 tokens over 4..256 experts; layers of 1..64 tokens with 2..64 experts of
    1024..8192 by 512..14336; projections of 1..512 rows, 1024..11008 by 1024..22016, with 1..64 adapters of rank 8..128."""
    op = rng.choice(["route", "moe", "moe", "experts", "experts", "lora", "lora", "lora_add"])
    if op == "route":
        experts = rng.choice([8, 16, 60, 64, 128, 256, _log_int(rng, 4, 256)])
        case = _route(None, _log_int(rng, 1, 4096), experts, min(experts, rng.choice([1, 2, 2, 4, 6, 8])),
                      rng.choice(["fp16", "fp32"]), rng.random() < 0.7)
    elif op in ("moe", "experts"):
        most = work(_moe("", "moe", 64, HIDDEN, INTER, 8, 2))
        while True:
            group = rng.choice([128, 128, 128, 64, 32])
            experts = rng.choice([4, 8, 16, 32, 64, _log_int(rng, 2, 64)])
            case = _moe(None, op, 1 if rng.random() < 0.25 else _log_int(rng, 1, 64), _multiple(rng, 1024, 8192, group),
                        _multiple(rng, 512, 14336, group), experts, min(experts, rng.choice([1, 2, 2, 4, 6, 8])), group,
                        rng.choice(["fp16", "fp32"]), rng.choice([0.0, 0.0, 0.5]) if op == "experts" else 0.0)
            need = work(case)
            held = experts * case["hidden"] * case["inter"]  # what the program has in memory: no more either
            if need["bytes"] <= most["bytes"] and need["flops"] <= most["flops"] and held <= 8 * HIDDEN * INTER:
                break
    else:
        group = rng.choice([128, 128, 128, 64, 32])
        m = _log_int(rng, 1, 512)
        k, n = _multiple(rng, 1024, 11008, group), _multiple(rng, 1024, 22016, rng.choice([8, 64, 128]))
        case = _lora(None, op, m, k, n, _multiple(rng, 8, 128, 8), _log_int(rng, 1, 64), group,
                     packed=m > 64 or rng.random() < 0.3, bare=rng.choice([0.0, 0.1, 0.5]),
                     row=n + rng.choice([0, 0, 8, 4096]) if op == "lora_add" else 0)
    del case["name"]
    return case


# ---- what a program has in hand before the call ----

def _words(gen, *shape):
    return torch.randint(-2 ** 31, 2 ** 31, shape, dtype=torch.int32, device="cuda", generator=gen)


def _packed(gen, k, n, group, *lead):
    return (_words(gen, *lead, k // 8, n), _words(gen, *lead, k // group, n // 8),
            torch.empty(*lead, k // group, n, device="cuda").uniform_(0.001, 0.01, generator=gen).half())


def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, m = case["op"], case["m"]
    state = dict(case)
    if op in ("route", "moe", "experts"):
        logits = _normal(gen, m, case["experts"])
        state["logits"] = logits.half() if case["dtype"] == "fp16" else logits
        state["ids"] = torch.empty(m, case["top_k"], dtype=torch.int32, device="cuda")
        state["weights"] = torch.empty(m, case["top_k"], device="cuda")
    if op in ("moe", "experts"):
        state["x"] = _normal(gen, m, case["hidden"]).half()
        state["gate_up"] = _packed(gen, case["hidden"], 2 * case["inter"], case["group"], case["experts"])
        state["down"] = _packed(gen, case["inter"], case["hidden"], case["group"], case["experts"])
        state["out"] = torch.empty(m, case["hidden"], dtype=torch.float16, device="cuda")
        if op == "experts":
            ids, weights = _route_plain(logits, case["top_k"], True)
            here = case["experts"] - round(case["absent"] * case["experts"])
            gone = torch.randperm(case["experts"], device="cuda", generator=gen) >= here
            state["ids"] = torch.where(gone[ids.long()], -1, ids)
            state["weights"] = weights
    if op in ("lora", "lora_add"):
        k, n, rank, adapters = case["k"], case["n"], case["rank"], case["adapters"]
        state["x"] = _normal(gen, m, k).half()
        state["a"] = (_normal(gen, adapters, rank, k) / math.sqrt(k)).half()
        state["b"] = (_normal(gen, adapters, n, rank) * 0.1).half()
        state["scaling"] = torch.empty(adapters, device="cuda").uniform_(0.5, 2.0, generator=gen)
        rows = torch.randint(0, adapters, (m,), device="cuda", generator=gen)
        bare = torch.rand(m, device="cuda", generator=gen) < case["bare"]
        if case["packed"]:  # rows of one request stand together: a request's rows have the adapter of its first one
            start = torch.rand(m, device="cuda", generator=gen) < 1.0 / 48
            first = torch.cummax(torch.where(start, torch.arange(m, device="cuda"), 0), 0).values
            rows, bare = rows[first], bare[first]
        state["adapter"] = torch.where(bare, -1, rows).int()
        state["out"] = torch.empty(m, case["row"], dtype=torch.float16, device="cuda")[:, :n]
        if op == "lora":
            state["packed_w"] = _packed(gen, k, n, case["group"])
        else:
            state["base"] = (_normal(gen, m, case["row"]) * 2).half()[:, :n]
    return state


# ---- the plain forms ----

def _dequant_plain(qweight, qzeros, scales):
    """fp32 [..., K, N] of packed matrices."""
    shift = torch.arange(0, 32, 4, dtype=torch.int32, device=qweight.device)
    q = (qweight[..., :, None, :] >> shift[:, None] & 15).flatten(-3, -2)
    z = (qzeros[..., None] >> shift & 15).flatten(-2)
    q = q.unflatten(-2, (z.shape[-2], -1))  # [..., groups, rows of a group, N]
    return ((q - z[..., None, :]).float() * scales.float()[..., None, :]).flatten(-3, -2)


def _route_plain(logits, top_k, renormalize):
    """The largest logits, the lower index first among equal ones; an expert masked by -inf is none."""
    logits = logits.float()
    value, index = torch.sort(logits, dim=1, descending=True, stable=True)
    e = torch.exp(logits - value[:, :1])
    chosen = torch.exp(value[:, :top_k] - value[:, :1])
    total = chosen.sum(1, keepdim=True) if renormalize else e.sum(1, keepdim=True)
    none = value[:, :top_k] == -math.inf
    return (torch.where(none, -1, index[:, :top_k]).int(),
            torch.where(none, 0.0, chosen / total))


def _experts_plain(state, ids, weights):
    x = state["x"].float()
    m, top_k = ids.shape
    experts, inter = state["experts"], state["inter"]
    few = m * top_k <= experts  # then only the experts that the tokens are sent to, looked up on the GPU; else all
    if few:
        chosen = ids.flatten().clamp(min=0).long()
        gate_up, down = [t[chosen] for t in state["gate_up"]], [t[chosen] for t in state["down"]]
        x = x.repeat_interleave(top_k, 0)[:, None, :]
    else:
        gate_up, down = state["gate_up"], state["down"]
    gu = x @ _dequant_plain(*gate_up)
    gate, up = gu[..., :inter], gu[..., inter:]
    y = (gate / (1 + torch.exp(-gate)) * up) @ _dequant_plain(*down)
    if few:
        share = torch.where(ids >= 0, weights, 0.0)
        out = (share[..., None] * y.view(m, top_k, -1)).sum(1)
    else:
        expert = torch.arange(experts, dtype=torch.int32, device=x.device)
        share = torch.where(ids[..., None] == expert, weights[..., None], 0.0).sum(1)  # [tokens, experts]
        out = (share.t()[..., None] * y).sum(0)
    return out.half()


def _lora_plain(state, base):
    x = state["x"].float()
    a, b = state["a"].float(), state["b"].float()
    adapters, rank, _ = a.shape
    own_one = state["adapter"][:, None] == torch.arange(adapters, dtype=torch.int32, device=x.device)
    t = (x @ a.flatten(0, 1).t()).view(-1, adapters, rank)
    t = t * torch.where(own_one, state["scaling"], 0.0)[..., None]  # nothing of the other adapters
    return (base + t.flatten(1) @ b.transpose(1, 2).reshape(adapters * rank, -1)).half()


# ---- one pass ----

def run(state):
    op = state["op"]
    if not own:
        if op == "route":
            return _route_plain(state["logits"], state["top_k"], state["renormalize"])
        if op == "moe":
            return _experts_plain(state, *_route_plain(state["logits"], state["top_k"], state["renormalize"]))
        if op == "experts":
            return _experts_plain(state, state["ids"], state["weights"])
        if op == "lora":
            return _lora_plain(state, state["x"].float() @ _dequant_plain(*state["packed_w"]))
        return _lora_plain(state, state["base"].float())

    from paper_2511_19438_amd import serving

    if op == "route":
        return serving.gptq_w4a16_moe_route(state["logits"], state["ids"], state["weights"], state["renormalize"])
    if op == "moe":
        return serving.gptq_w4a16_moe(state["x"], state["logits"], state["gate_up"], state["down"], state["out"],
                                      state["top_k"], state["group"], state["renormalize"])
    if op == "experts":
        return serving.gptq_w4a16_moe_experts(state["x"], state["ids"], state["weights"], state["gate_up"],
                                              state["down"], state["out"], state["group"])
    if op == "lora":
        return serving.gptq_w4a16_gemm_lora(state["x"], *state["packed_w"], state["a"], state["b"], state["scaling"],
                                            state["adapter"], state["out"], state["group"])
    return serving.gptq_w4a16_lora_add(state["x"], state["a"], state["b"], state["scaling"], state["adapter"],
                                       state["base"], state["out"])


# ---- what a pass cannot do without ----

def _expected_hit(buckets, picks, rows):
    """Buckets that `rows` draws of `picks` different ones are expected to hit, all alike."""
    return buckets * (1 - (1 - picks / buckets) ** rows)


def _matrix_bytes(k, n, group):
    return k * n // 2 + (k // group) * (2 * n + n // 2)


def work(case):
    """Each input read once - of experts and adapters those that the rows are expected to use - and each output written
    once; two operations per multiply-add."""
    op, m = case["op"], case["m"]
    logit = 2 if case.get("dtype") == "fp16" else 4
    if op == "route":
        size = m * case["experts"]
        return {"bytes": size * logit + m * case["top_k"] * 8, "flops": 4 * size}
    if op in ("moe", "experts"):
        h, i, e, k = case["hidden"], case["inter"], case["experts"], case["top_k"]
        here = e - round(case["absent"] * e)
        picks = k * here / e  # of a token's experts, those that live here
        hit = _expected_hit(here, picks, m)
        routing = m * e * logit if op == "moe" else m * k * 8
        one = _matrix_bytes(h, 2 * i, case["group"]) + _matrix_bytes(i, h, case["group"])
        return {"bytes": int(hit * one) + routing + 4 * m * h, "flops": int(m * picks * 6 * h * i)}
    k, n, rank = case["k"], case["n"], case["rank"]
    segments = m / 48 + 1 if case["packed"] else m
    hit = _expected_hit(case["adapters"], 1 - case["bare"], segments)
    nbytes = int(hit * (2 * rank * (k + n) + 4)) + 4 * m + 2 * m * k + 2 * m * n
    flops = int(2 * m * (1 - case["bare"]) * rank * (k + n))
    if op == "lora":
        return {"bytes": nbytes + _matrix_bytes(k, n, case["group"]), "flops": flops + 2 * m * k * n}
    return {"bytes": nbytes + 2 * m * n, "flops": flops}


# ---- the definitions in 64 bits ----

def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("route", "moe"):
        # an expert's place is the number of experts ahead of it: a larger logit, or an equal one and a lower index
        l = state["logits"].double()
        order = torch.arange(case["experts"], device="cuda")
        ids = torch.empty(case["m"], case["top_k"], dtype=torch.int32, device="cuda")
        weights = torch.empty(case["m"], case["top_k"], dtype=torch.float64, device="cuda")
        for lo in range(0, case["m"], 256):
            part = l[lo:lo + 256]
            ahead = (part[:, None, :] > part[:, :, None]) | ((part[:, None, :] == part[:, :, None])
                                                             & (order[None, None, :] < order[None, :, None]))
            place = ahead.sum(2)
            p = torch.softmax(part, 1)
            for j in range(case["top_k"]):
                pick = (place == j).int().argmax(1)
                ids[lo:lo + 256, j] = pick.int()
                weights[lo:lo + 256, j] = p.gather(1, pick[:, None])[:, 0]
        if case["renormalize"]:
            weights /= weights.sum(1, keepdim=True)
        if op == "route":
            return ids, weights
    if op == "experts":
        ids, weights = state["ids"], state["weights"].double()
    if op in ("moe", "experts"):
        out = torch.zeros(case["m"], case["hidden"], dtype=torch.float64, device="cuda")
        x = state["x"].double()
        for e in sorted(set(ids.flatten().tolist()) - {-1}):
            rows, slot = (ids == e).nonzero(as_tuple=True)
            gate = _product64(x[rows], state["gate_up"], e, 0, case["inter"])
            up = _product64(x[rows], state["gate_up"], e, case["inter"], 2 * case["inter"])
            y = _product64(gate * torch.sigmoid(gate) * up, state["down"], e, 0, case["hidden"])
            out.index_add_(0, rows, y * weights[rows, slot][:, None])
        return out
    x = state["x"].double()
    if op == "lora":
        out = _product64(x, [t[None] for t in state["packed_w"]], 0, 0, case["n"])
    else:
        out = state["base"].double()
    for l in sorted(set(state["adapter"].tolist()) - {-1}):
        rows = (state["adapter"] == l).nonzero()[:, 0]
        t = x[rows] @ state["a"][l].double().t().contiguous()
        out[rows] += state["scaling"][l].double() * (t @ state["b"][l].double().t().contiguous())
    return out


def _product64(x, packed, e, lo, hi):
    """x times columns lo..hi of matrix e in 64 bits, a block of columns at a time."""
    qweight, qzeros, scales = (t[e] for t in packed)
    rows = qweight.shape[0] * 8
    k = torch.arange(rows, device="cuda")
    group = k // (rows // scales.shape[0])
    parts = []
    for a in range(lo, hi, 4096):
        n = torch.arange(a, min(a + 4096, hi), device="cuda")
        q = qweight[k // 8][:, n] >> (4 * (k % 8))[:, None].int() & 15
        z = qzeros[:, n // 8] >> (4 * (n % 8))[None, :].int() & 15
        parts.append(x @ ((q - z[group]).double() * scales[:, n].double()[group]))
    return torch.cat(parts, 1)
