"""What the operators around the optimizer step are timed on that score a model's tokens, clip its gradients and run its experts
on a few tokens.

Kinds of call:
  score   log probabilities of given tokens with the entropy of the whole distribution and its top alternatives, from hidden states and
          the head's weight
  policy  the same without alternatives, and the gradients of hidden states and weight for given gradients of log probabilities and
          entropies, as a policy gradient with an entropy bonus takes them
  clip    the norm of all gradients together and the gradients scaled in place where it exceeds a limit
  adamw   the norm, and an AdamW step that takes the gradients times the scale that the limit asks for
  layer   the experts of a mixture on a few tokens: gated products, the way back, the weighted sum
Widths, experts and inner widths are those of this repository's workloads (1024 with 4096, 2048 with 1408; 66 experts) and generic ones;
vocabularies are generic, powers of two and odd sizes.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def score(name, tokens, vocab, width, top, *, tau=1.0, dtype="bf16"):
    return {"name": name, "kind": "score", "tokens": tokens, "vocab": vocab, "width": width, "top": top, "tau": tau, "dtype": dtype}


def policy(name, tokens, vocab, width, *, tau=1.0, entropy=0.01, dtype="bf16"):
    return {"name": name, "kind": "policy", "tokens": tokens, "vocab": vocab, "width": width, "top": 0, "tau": tau, "entropy": entropy,
            "dtype": dtype}


def gradients(name, kind, *, layers=0, width=0, inner=0, attention=4, experts=1, spread=0, least=1, most=1, dtype="bf16"):
    """`layers` of `attention` square matrices and `experts` of three, and `spread` tensors of sizes between two."""
    return {"name": name, "kind": kind, "layers": layers, "width": width, "inner": inner, "attention": attention, "experts": experts,
            "spread": spread, "least": least, "most": most, "dtype": dtype}


def layer(name, tokens, width, inner, experts, top, *, shared=0, gated=True, dtype="bf16", dropped=0.0):
    return {"name": name, "kind": "layer", "tokens": tokens, "width": width, "inner": inner, "experts": experts, "top": top,
            "shared": shared, "gated": gated, "dtype": dtype, "dropped": dropped}


def listed():
    return [
        # the next tokens of a few running requests, with five alternatives each: the weight is read once, latency counts
        score("score_few", 8, 32768, 1024, 5),
        # scoring a batch of text, alternatives kept as a teacher's entries, odd vocabulary
        score("score_text", 4096, 100003, 2048, 8),
        # a small fp32 model, ragged sizes, a sampler's temperature
        score("score_f32", 300, 8191, 512, 20, tau=0.7, dtype="f32"),
        # one micro batch of policy training of a width-1024 model
        policy("policy_w1024", 2048, 32768, 1024),
        # the same with a large odd vocabulary at width 2048: the largest call
        policy("policy_w2048", 8192, 100003, 2048),
        # gains, biases and small matrices of a small model, both types, odd sizes: launches count
        gradients("clip_small", "clip", spread=48, least=1, most=20000, dtype="mixed"),
        # all matrices of the 12-layer model of width 1024
        gradients("clip_w1024", "clip", layers=12, width=1024, inner=4096),
        # the expert bank of a mixture's layer, 198 matrices
        gradients("clip_bank", "clip", layers=1, width=2048, inner=1408, attention=0, experts=66),
        # embedding, head and gains, which stay with AdamW
        gradients("adamw_w2048", "adamw", spread=24, least=2048, most=67108864),
        # one running request through a layer's experts
        layer("layer_one", 1, 2048, 1408, 64, 6),
        # a batch of them, with two experts that every token goes to
        layer("layer_batch", 32, 2048, 1408, 66, 8, shared=2),
        # a small fp32 mixture without gates, odd sizes, a share of the pairs dropped (experts that live on another device)
        layer("layer_f32", 5, 777, 333, 16, 2, gated=False, dtype="f32", dropped=0.3),
    ]


MAX_FLOPS = 8e12                  # of a drawn head call in bf16: below the largest listed one
MAX_BANK = 5e8                    # elements of a drawn layer's matrices


def draw(rng):
    """One more case of the same ranges: 1 to 8192 tokens for the head, vocabularies of 1000 to 131072, widths of 64 to 4096, up to 32
    alternatives; 1 to 400 gradients of 1 to 30 million elements; layers of 1 to 64 tokens, 4 to 66 experts, 1 to 8 of them per token;
    odd sizes among all of them."""
    def between(low, high, grain=16):
        v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
        return v if v < 2 * grain else rng.choice([v | 1, grain * (v // grain | 1)])

    def width():
        return rng.choice([512, 1024, 1408, 2048, 4096, between(64, 4096, 8)])

    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kind = rng.choice(["score", "score", "policy", "policy", "clip", "adamw", "layer", "layer"])
    if kind in ("score", "policy"):
        while True:
            tokens, vocab, d = between(1, 8192), between(1000, 131072, 64), width()
            if 8 * tokens * vocab * d <= (MAX_FLOPS if dtype == "bf16" else MAX_FLOPS / 8):
                break
        tau = rng.choice([1.0, 1.0, 0.7, 1.3])
        if kind == "score":
            case = score("", tokens, vocab, d, rng.choice([0, 1, 5, 8, 20, 32]), tau=tau, dtype=dtype)
        else:
            case = policy("", tokens, vocab, d, tau=tau, entropy=rng.choice([0.0, 0.01, 0.1]), dtype=dtype)
    elif kind in ("clip", "adamw"):
        if rng.random() < 0.4:
            d = rng.choice([512, 1024, 2048])
            case = gradients("", kind, layers=rng.randint(1, 6), width=d, inner=between(d // 2, 4 * d), dtype=rng.choice(["bf16", "f32"]))
        else:
            least = between(1, 1000)
            while True:
                count, most = between(1, 400), between(2000, 30000000)
                if count * most <= 1e9:
                    break
            case = gradients("", kind, spread=count, least=least, most=most, dtype=rng.choice(["bf16", "f32", "mixed"]) if kind == "clip" else dtype)
    else:
        while True:
            d, inner, experts = width(), between(64, 4096, 8), rng.choice([4, 8, 16, 64, 66])
            if 3 * experts * d * inner <= MAX_BANK:
                break
        top = rng.randint(1, min(8, experts))
        case = layer("", between(1, 64), d, inner, experts, top, shared=rng.choice([0, 0, min(2, top - 1)]), gated=rng.random() < 0.7,
                     dtype=dtype, dropped=rng.choice([0.0, 0.0, 0.3]))
    del case["name"]
    return case


def generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 29)
    return gen


def head_inputs(case, seed):
    """Hidden states as a last norm leaves them, pulled towards the rows of the given tokens by an amount that differs from token to
    token, so that some are nearly certain and some open; a few places have no token (a prompt's, padding)."""
    gen = generator(seed)
    t, v, d, dt = case["tokens"], case["vocab"], case["width"], DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, 1.0, generator=gen)

    weight = normal(v, d).mul_(0.02)
    unit = 0.02 * math.sqrt(d)                                         # norm of a weight's row
    targets = torch.randint(v, (t,), device=DEV, generator=gen)
    pull = torch.empty(t, 1, device=DEV).uniform_(0.0, 9.0, generator=gen)
    hidden = normal(t, d) + pull / unit ** 2 * weight[targets]
    gone = torch.empty(t, device=DEV).uniform_(0.0, 1.0, generator=gen) < 0.05
    gone[:1] = False
    state = {"weight": weight.to(dt), "hidden": hidden.to(dt), "targets": torch.where(gone, -1, targets)}
    if case["kind"] == "policy":
        share = torch.where(gone, 0.0, 1.0 / (~gone).sum()).float()    # the mean over the tokens that count
        state["d_log_prob"] = -normal(t) * share                       # advantages
        state["d_entropy"] = -case["entropy"] * share
    return state


def sizes_of(case):
    """Sizes of the gradients, in their order."""
    d, inner = case["width"], case["inner"]
    one = [d * d] * case["attention"] + [d * inner] * 3 * case["experts"]
    pick = random.Random(case["spread"])
    ratio = math.log(case["most"] / case["least"])
    return one * case["layers"] + [max(case["least"], int(case["least"] * math.exp(ratio * pick.random() ** 2))) for _ in range(case["spread"])]


def gradient_inputs(case, seed):
    """Gradients as they lie in buckets, one behind the other in a buffer for each type; a hundredth of them are outliers."""
    gen = generator(seed)
    sizes = sizes_of(case)
    dtypes = [("bf16", "f32")[i % 3 == 2] if case["dtype"] == "mixed" else case["dtype"] for i in range(len(sizes))]
    state = {"flat": {}, "grads": []}
    for name in sorted(set(dtypes)):
        n = sum(s for s, x in zip(sizes, dtypes) if x == name)
        flat = torch.empty(n, dtype=torch.float32, device=DEV).normal_(0.0, 1e-3, generator=gen)
        flat[::97] *= 30.0
        state["flat"][name] = flat.to(DTYPES[name])
    at = dict.fromkeys(state["flat"], 0)
    for s, x in zip(sizes, dtypes):
        state["grads"].append(state["flat"][x][at[x]:at[x] + s])
        at[x] += s
    state["max_norm"] = 0.5 * math.sqrt(sum(sizes) * 1e-6 * (1.0 + 899.0 / 97.0))      # about half of the norm
    if case["kind"] == "adamw":
        g = state["flat"][case["dtype"]]
        state["p"] = torch.empty_like(g).normal_(0.0, 0.02, generator=gen)
        state["m"] = torch.empty(g.shape, device=DEV).normal_(0.0, 1e-3, generator=gen)
        state["v"] = torch.empty(g.shape, device=DEV).uniform_(1e-7, 1e-5, generator=gen)
        at, state["tensors"] = 0, []
        for s in sizes:
            state["tensors"].append((state["p"][at:at + s], g[at:at + s], state["m"][at:at + s], state["v"][at:at + s]))
            at += s
    return state


ADAMW = {"lr": 4e-4, "weight_decay": 0.1, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "step": 100}


def layer_inputs(case, seed):
    """Normalised hidden states and the top experts of a router that likes some more than others, `shared` of them everybody's."""
    gen = generator(seed)
    t, d, n, e, dt = case["tokens"], case["width"], case["inner"], case["experts"], DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device=DEV).normal_(0.0, std, generator=gen)

    routed, shared = e - case["shared"], case["shared"]
    best, expert = (normal(t, routed) + 0.7 * normal(routed)).topk(case["top"] - shared, dim=1)
    gates = best.exp()
    weights = torch.cat([gates / gates.sum(1, keepdim=True), torch.ones(t, shared, device=DEV)], dim=1)
    expert = torch.cat([expert, torch.arange(routed, e, device=DEV).expand(t, shared)], dim=1)
    away = torch.empty(t, case["top"], device=DEV).uniform_(0.0, 1.0, generator=gen) < case["dropped"]
    state = {"x": normal(t, d).to(dt), "expert": torch.where(away, -1, expert), "weights": weights.contiguous(),
             "up": normal(e, d, n, std=d ** -0.5, dtype=dt), "down": normal(e, n, d, std=n ** -0.5, dtype=dt), "gate": None}
    if case["gated"]:
        state["gate"] = normal(e, d, n, std=d ** -0.5, dtype=dt)
    return state


INPUTS = {"score": head_inputs, "policy": head_inputs, "clip": gradient_inputs, "adamw": gradient_inputs, "layer": layer_inputs}


def prepare(case, seed):
    state = INPUTS[case["kind"]](case, seed)
    state["case"] = case
    if own and case["kind"] in ("score", "policy"):
        from paper_2502_16982_amd import losses
        state["head"] = losses.LossHead(case["tokens"], case["vocab"], case["width"], dtype=DTYPES[case["dtype"]],
                                        gradients=case["kind"] == "policy")
    if own and case["kind"] in ("clip", "adamw"):
        from paper_2502_16982_amd import clipping
        state["clipper"] = clipping.GradClipper(state["grads"])
    return state


def head_plain(state):
    case = state["case"]
    h, w, tau = state["hidden"].float(), state["weight"].float(), case["tau"]
    z = h @ w.T
    if tau != 1.0:
        z = z / tau
    peak = z.amax(1, keepdim=True)
    lse = peak + (z - peak).exp().sum(1, keepdim=True).log()
    p = (z - lse).exp()
    entropy = -(p * (z - lse)).sum(1, keepdim=True)
    there = state["targets"] >= 0
    at = state["targets"].clamp(min=0)
    given = (state["hidden"].double() * state["weight"][at].double()).sum(1) / tau     # 64 bits: z - lse cancels where a token is certain
    out = {"log_prob": torch.where(there, given - lse[:, 0].double(), 0.0).float(), "entropy": entropy[:, 0], "lse": lse[:, 0]}
    if case["kind"] == "score":
        if case["top"]:
            out["top_index"], out["top_log_prob"] = top_plain(state, z, lse)
        return out
    g, e = torch.where(there, state["d_log_prob"], 0.0)[:, None], state["d_entropy"][:, None]
    dz = p.mul_(-(g + e * (z - lse + entropy)))
    dz.scatter_add_(1, at[:, None], g)
    dz /= tau
    dt = state["hidden"].dtype
    out["d_hidden"], out["d_weight"] = (dz @ w).to(dt), (dz.T @ h).to(dt)
    return out


def top_plain(state, z, lse):
    """The largest logits, of a few more than are asked for by their values in 64 bits; ties go to the lowest index."""
    case = state["case"]
    near = z.topk(min(case["vocab"], case["top"] + 16), dim=1).indices.sort(dim=1).values
    values = torch.bmm(state["weight"][near].double(), state["hidden"].double()[:, :, None])[:, :, 0]
    values, order = (values / case["tau"]).sort(dim=1, descending=True, stable=True)
    index = near.gather(1, order)[:, :case["top"]]
    return index, (values[:, :case["top"]] - lse.double()).float()


def scale_plain(state):
    """(norm, scale) of all gradients, in 64 bits."""
    norm = sum(flat.double().square().sum() for flat in state["flat"].values()).sqrt()
    return norm, torch.where(norm > state["max_norm"], state["max_norm"] / norm, 1.0).float()


def clip_plain(state):
    norm, scale = scale_plain(state)
    for flat in state["flat"].values():
        flat.copy_(flat.float() * scale)
    return {"norm": norm, "grads": state["flat"]}


def adamw_plain(state):
    norm, scale = scale_plain(state)
    h, p, m, v = ADAMW, state["p"], state["m"], state["v"]
    g = state["flat"][state["case"]["dtype"]].float() * scale
    m.copy_(h["beta1"] * m + (1.0 - h["beta1"]) * g)
    v.copy_(h["beta2"] * v + (1.0 - h["beta2"]) * g * g)
    update = (m / (1.0 - h["beta1"] ** h["step"])) / ((v / (1.0 - h["beta2"] ** h["step"])).sqrt() + h["eps"])
    p.copy_(p.float() - h["lr"] * (update + h["weight_decay"] * p.float()))
    return {"norm": norm, "p": p, "m": m, "v": v}


def layer_plain(state):
    """The matrices of each pair's expert, or, where there are more pairs than experts, all experts' on all tokens."""
    x, weights, expert = state["x"].float(), state["weights"], state["expert"]
    tokens, top = expert.shape
    experts = state["up"].shape[0]
    weights, by_pair = torch.where(expert >= 0, weights, 0.0), tokens * top < experts
    at = expert.clamp(min=0)
    if by_pair:
        pick, x = at.reshape(-1), x.repeat_interleave(top, 0)[:, None, :]
    else:
        pick, x = slice(None), x.expand(experts, *x.shape)
    lead = inner = torch.bmm(x, state["up"][pick].float())
    if state["gate"] is not None:
        lead = torch.bmm(x, state["gate"][pick].float())
        inner = inner * (lead / (1.0 + (-lead).exp()))
    else:
        inner = lead / (1.0 + (-lead).exp())
    rows = torch.bmm(inner, state["down"][pick].float())
    if by_pair:
        out = (rows.reshape(tokens, top, -1) * weights[:, :, None]).sum(1)
    else:
        share = torch.zeros(tokens, experts, device=x.device).scatter_add_(1, at, weights)
        out = (rows * share.T[:, :, None]).sum(0)
    return {"out": out.to(state["x"].dtype)}


PLAIN = {"score": head_plain, "policy": head_plain, "clip": clip_plain, "adamw": adamw_plain, "layer": layer_plain}


def run(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "clip":
        state["max_norm"] *= 0.999            # the limit falls a little from pass to pass, so that every pass has to clip
    if not own:
        return PLAIN[kind](state)
    if kind in ("score", "policy"):
        head, args = state["head"], (state["hidden"], state["weight"], state["targets"])
        r = head.log_probs(*args, top=case["top"], temperature=case["tau"])
        out = {"log_prob": r.log_prob, "entropy": r.entropy, "lse": r.lse}
        if case["top"]:
            out["top_index"], out["top_log_prob"] = r.top_index, r.top_log_prob
        if kind == "policy":
            out["d_hidden"], out["d_weight"] = head.log_probs_backward(*args, r, state["d_log_prob"], state["d_entropy"],
                                                                       temperature=case["tau"])
        return out
    if kind == "clip":
        return {"norm": state["clipper"].clip_(state["max_norm"]).norm, "grads": state["flat"]}
    if kind == "adamw":
        from paper_2502_16982_amd import binding
        r = state["clipper"].scale(state["max_norm"])
        binding.muon_adamw_step(state["tensors"], **ADAMW, grad_scale=r.scale, stream_ptr=torch.cuda.current_stream().cuda_stream)
        return {"norm": r.norm, "p": state["p"], "m": state["m"], "v": state["v"]}
    from paper_2502_16982_amd import experts
    return {"out": experts.layer(state["x"], state["up"], state["down"], state["expert"], state["weights"], gate=state["gate"])}


def work(case):
    """Each input read once and each output written once; the multiply-adds of the products."""
    kind, e = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind in ("score", "policy"):
        t, v, d = case["tokens"], case["vocab"], case["width"]
        if kind == "score":
            return {"bytes": (t + v) * d * e + t * (8 + 12 + 12 * case["top"]), "flops": 2 * t * v * d}
        return {"bytes": 2 * (t + v) * d * e + t * (8 + 12 + 8), "flops": 6 * t * v * d}
    if kind in ("clip", "adamw"):
        sizes = sizes_of(case)
        n = sum(sizes)
        if kind == "adamw":
            return {"bytes": n * (3 * e + 16), "flops": 16 * n}
        if case["dtype"] == "mixed":
            e = sum(s * (4 if i % 3 == 2 else 2) for i, s in enumerate(sizes)) / n
        return {"bytes": 2 * n * e, "flops": 3 * n}
    t, d, n, x, k, shared = (case[key] for key in ("tokens", "width", "inner", "experts", "top", "shared"))
    per, there = (3 if case["gated"] else 2) * d * n, 1.0 - case["dropped"]
    hit = (x - shared) * (1.0 - (1.0 - there * (k - shared) / max(1, x - shared)) ** t) + shared * (1.0 - case["dropped"] ** t)
    return {"bytes": hit * per * e + 2 * t * d * e + t * k * 12, "flops": 2 * t * k * there * per}


def head_exact(case, state):
    """Row by row of the definition: a softmax over the vocabulary, its logarithm at the token, its expected logarithm, the chain rule."""
    w = state["weight"].double()
    wt = w.T.contiguous()
    policy_case, top, tau = case["kind"] == "policy", case["top"], case["tau"]
    parts, d_weight = [], torch.zeros_like(w) if policy_case else None
    for a in range(0, case["tokens"], 1024):
        b = min(case["tokens"], a + 1024)
        h = state["hidden"][a:b].double()
        logp = torch.log_softmax(torch.mm(h, wt) / tau, 1)
        p = logp.exp()
        y = state["targets"][a:b]
        row = (y >= 0).nonzero()[:, 0]
        given = torch.zeros(b - a, dtype=torch.float64, device=DEV)
        given[row] = logp[row, y[row]]
        entropy = torch.special.entr(p).sum(1)
        part = {"log_prob": given, "entropy": entropy, "lse": torch.logsumexp(torch.mm(h, wt) / tau, 1)}
        if top:
            best = torch.topk(logp, min(case["vocab"], top + 8), dim=1)
            order = sorted_rows(best.values, best.indices)
            part["top_index"], part["top_log_prob"] = best.indices.gather(1, order)[:, :top], best.values.gather(1, order)[:, :top]
        if policy_case:
            # d entropy / d z_v = -p_v (log p_v + entropy); d log p_y / d z_v = [v = y] - p_v
            g, e = torch.zeros_like(given), state["d_entropy"][a:b].double()
            g[row] = state["d_log_prob"][a:b].double()[row]
            dz = -e[:, None] * p * (logp + entropy[:, None]) - g[:, None] * p
            dz[row, y[row]] += g[row]
            dz /= tau
            part["d_hidden"] = torch.mm(dz, w)
            d_weight += torch.mm(dz.T.contiguous(), h)
        parts.append(part)
    out = {key: torch.cat([part[key] for part in parts]) for key in parts[0]}
    if policy_case:
        out["d_weight"] = d_weight
    return out


def sorted_rows(values, indices):
    """Order of each row by falling value, then by index."""
    by_index = indices.sort(dim=1).indices
    by_value = values.gather(1, by_index).sort(dim=1, descending=True, stable=True).indices
    return by_index.gather(1, by_value)


def gradients_exact(case, state):
    parts = [g.double() for g in state["grads"]]
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(g) for g in parts]))
    limit = state["max_norm"] * (0.999 if case["kind"] == "clip" else 1.0)
    scale = min(1.0, limit / float(norm))
    if case["kind"] == "clip":
        kept = {name: torch.cat([g for g, raw in zip(parts, state["grads"]) if raw.dtype == flat.dtype]) for name, flat in state["flat"].items()}
        return {"norm": norm, "grads": {name: flat * scale for name, flat in kept.items()}}
    h = ADAMW
    out = {"norm": norm, "p": [], "m": [], "v": []}
    for g, (p, _, m, v) in zip(parts, state["tensors"]):
        m = torch.lerp(m.double(), g * scale, 1.0 - h["beta1"])
        v = torch.lerp(v.double(), (g * scale).square(), 1.0 - h["beta2"])
        way = m / (1.0 - h["beta1"] ** h["step"]) / (torch.sqrt(v / (1.0 - h["beta2"] ** h["step"])) + h["eps"])
        out["p"].append(p.double() * (1.0 - h["lr"] * h["weight_decay"]) - h["lr"] * way)
        out["m"].append(m)
        out["v"].append(v)
    return {key: torch.cat(x) if isinstance(x, list) else x for key, x in out.items()}


def layer_exact(case, state):
    """Pair by pair."""
    out = torch.zeros(case["tokens"], case["width"], dtype=torch.float64, device=DEV)
    expert = state["expert"].tolist()
    for t, row in enumerate(expert):
        for j, e in enumerate(row):
            if e < 0:
                continue
            x = state["x"][t].double()
            inner = torch.mv(state["up"][e].double().T.contiguous(), x)
            lead = inner if state["gate"] is None else torch.mv(state["gate"][e].double().T.contiguous(), x)
            inner = lead * torch.sigmoid(lead) * (1.0 if state["gate"] is None else inner)
            out[t] += state["weights"][t, j].double() * torch.mv(state["down"][e].double().T.contiguous(), inner)
    return {"out": out}


def exact(case, seed):
    state = INPUTS[case["kind"]](case, seed)
    how = {"score": head_exact, "policy": head_exact, "clip": gradients_exact, "adamw": gradients_exact, "layer": layer_exact}
    return how[case["kind"]](case, state)
