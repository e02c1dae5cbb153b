"""Routing to experts and expert layers with 8-bit floating point weights as timing cases.

Labels are held as the library holds them: for every CRT prime p a uint8 tensor [chunks][elements][16], the lambda_p digits of an
element's label in [0, p) cut into chunks of 16, zeros past lambda_p.  Elements are ordered [batch element][feature].

  kind "choose"    the experts of every row and their gates from a router's logits l (float32, bfloat16 or float16): scores s = softmax(l)
                   or sigmoid(l); choice values c = s + bias, without a bias the order of l; of `groups` equal groups of experts the
                   top_groups with the largest c (or the largest sum of two); among these the top_k largest c, in descending order, ties
                   to the lower number.  w = scale * s (renormalise: / sum of the chosen s); gate = w 2^gate_bits to the nearest integer, ties to
                   the even.  Logits of -infinity are never chosen; what is missing of top_k, and rows that are not valid: expert -1,
                   w = 0, gate 0.  Outputs: experts, gates, w in float32
  kind "quantise"  weights (float32, bfloat16 or float16) to e4m3 floats with an integer scale S for each block of 128 x 128:
                   S = clamp(ceil(amax / (448 * 2^base)), 1, max_scale), the nearest e4m3 value of w / (S 2^base), ties to the even code,
                   saturated at 448.  Output: the values that the weights stand for, e4m3 S 2^base
  kind "experts"   out[r][j] = sum_i W_e(r)[j][i] in[r / top_k][i] on every digit, mod p, W = 512 e4m3 S; e(r): the public expert of row r,
                   -1: none (zeros).  experts = 1: a dense layer
"""
import math

import numpy as np
import torch

own = False

PRIMES = [2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37]
# mixed-radix digits of the sign gadget by number of primes
DIGITS = {7: (10,) + (13,) * 5, 8: (26,) + (12,) * 6, 9: (22,) + (10,) * 8, 12: (46,) + (17,) * 10}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _lambda(p):
    """smallest label length with p^lambda >= 2^128"""
    n = 1
    while p ** n < 2 ** 128:
        n += 1
    return n


LAMBDA = {p: _lambda(p) for p in PRIMES}


def _chunks(p):
    return (LAMBDA[p] + 15) // 16


def _choose(name, rows, experts, top_k, dtype, score, bias=False, groups=1, top_groups=1, pairs=False, renormalise=True, scale=1.0,
            gate_bits=8, pad=0, masked=0.0, invalid=0.0):
    return dict(name=name, kind="choose", rows=rows, experts=experts, top_k=top_k, dtype=dtype, score=score, bias=bias, groups=groups,
                top_groups=top_groups, pairs=pairs, renormalise=renormalise, scale=scale, gate_bits=gate_bits, pad=pad, masked=masked, invalid=invalid)


def listed():
    return [
        # one token, two of eight experts: latency
        _choose("choose_1_of_8", 1, 8, 2, "f32", "softmax"),
        # a prompt, odd sizes: the logits a slice of a wider matrix, padding at the end of batch elements, experts taken out of service
        _choose("choose_odd_strided", 1000, 160, 6, "f16", "softmax", groups=8, top_groups=3, renormalise=False, scale=16.0, pad=5,
                masked=0.02, invalid=0.1),
        # a batch of prompts, balanced by a bias: the best four of eight groups of 32, eight experts of these
        _choose("choose_groups_256", 4096, 256, 8, "f32", "sigmoid", bias=True, groups=8, top_groups=4, pairs=True, scale=2.5, gate_bits=12),
        # a large batch of prompts, the largest of its kind
        _choose("choose_64k_of_256", 65536, 256, 8, "bf16", "softmax", bias=True),
        # the last layer of the small dense network (128 -> 10): less than a block
        dict(name="quantise_128_10", kind="quantise", dtype="f32", experts=1, out_c=10, K=128, pad=0, base=-12, max_scale=255),
        # odd sizes, rows that lie further apart than they are long
        dict(name="quantise_odd_strided", kind="quantise", dtype="f16", experts=3, out_c=257, K=1030, pad=26, base=-16, max_scale=4095),
        # a 4096 x 4096 layer as it leaves training
        dict(name="quantise_4096", kind="quantise", dtype="bf16", experts=1, out_c=4096, K=4096, pad=0, base=-14, max_scale=255),
        # one image through the first layer of the small dense network: latency
        dict(name="f8_784_128_b1", kind="experts", k=8, experts=1, top_k=1, rows=1, K=784, out_c=128, skew=0, none=0.0),
        # one token through a large dense layer on the 12-prime base
        dict(name="f8_4096_b1", kind="experts", k=12, experts=1, top_k=1, rows=1, K=4096, out_c=4096, skew=0, none=0.0),
        # the dense benchmark layer, batch 128: the largest
        dict(name="f8_4096_b128", kind="experts", k=12, experts=1, top_k=1, rows=128, K=4096, out_c=4096, skew=0, none=0.0),
        # 64 images of the CIFAR-sized network, 12 clients of very different shares, some images of no client
        dict(name="f8_clients_4096_256", kind="experts", k=12, experts=12, top_k=1, rows=64, K=4096, out_c=256, skew=2, none=0.1),
        # a mixture of 32 experts, two for each of 128 tokens, ragged
        dict(name="f8_mixture_32", kind="experts", k=12, experts=32, top_k=2, rows=256, K=1024, out_c=2048, skew=1, none=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["choose", "choose", "quantise", "experts", "experts"])
        if kind == "choose":
            groups = rng.choice([1, 1, 2, 4, 8, 16])
            experts = groups * _log(rng, 8 if groups == 1 else 2, 512 // groups)
            top_groups = rng.randint(1, groups)
            bias = rng.random() < 0.5
            c = _choose(None, _log(rng, 1, 65536), experts, min(_log(rng, 1, 16), top_groups * (experts // groups)), rng.choice(["f32", "bf16", "f16"]),
                        rng.choice(["softmax", "sigmoid"]), bias, groups, top_groups, groups > 1 and rng.random() < 0.5, rng.random() < 0.7,
                        rng.choice([1.0, 1.0, 2.5, 16.0]), rng.randint(4, 16), rng.choice([0, 0, rng.randint(1, 40)]),
                        rng.choice([0.0, 0.0, 0.02]), rng.choice([0.0, 0.0, 0.1]))
            del c["name"]
            if c["rows"] * experts > 65536 * 256:
                continue
        elif kind == "quantise":
            c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16"]), experts=rng.randint(1, 8), out_c=_log(rng, 8, 4096), K=_log(rng, 32, 4096),
                     pad=rng.choice([0, 0, rng.randint(1, 40)]), base=rng.randint(-18, -8), max_scale=rng.choice([1, 255, 255, 4095, 32767]))
        else:
            top_k = rng.choice([1, 1, 2, 4])
            c = dict(kind=kind, k=rng.choice([7, 8, 9, 12]), experts=_log(rng, 1, 64), top_k=top_k, rows=top_k * _log(rng, 1, 256),
                     K=_log(rng, 60, 4096), out_c=_log(rng, 8, 4096), skew=rng.randint(0, 2), none=rng.choice([0.0, 0.0, 0.1]))
        w, top = work(c), work(listed()[9])
        if w["flops"] <= top["flops"] and w["bytes"] <= 2 ** 31:
            return c


def work(case):
    if case["kind"] == "choose":
        n = case["rows"] * case["experts"]
        # an exponential, a sum and two comparisons for every logit
        return {"bytes": n * SIZE[case["dtype"]] + 12 * case["rows"] * case["top_k"], "flops": 4 * n}
    if case["kind"] == "quantise":
        E, M, K = case["experts"], case["out_c"], case["K"]
        blocks = E * ((M + 127) // 128) * ((K + 127) // 128)
        return {"bytes": 2 * E * M * K * SIZE[case["dtype"]] + E * M * K + 4 * blocks, "flops": 4 * E * M * K}
    primes = PRIMES[:case["k"]]
    stored, digits = sum(16 * _chunks(p) for p in primes), sum(LAMBDA[p] for p in primes)
    rows, top_k, K, M = case["rows"], case["top_k"], case["K"], case["out_c"]
    numbers = [e for e in _expert_numbers(case, 0) if e >= 0]
    weights = len(set(numbers)) * (M * K + 4 * ((M + 127) // 128) * ((K + 127) // 128))
    return {"bytes": (rows // top_k * K + rows * M) * stored + weights, "flops": 2 * len(numbers) * M * K * digits}


def _expert_numbers(case, seed):
    """public expert of every row: shares of 1 / (e + 1)^skew, a batch element's rows on different experts where there are enough"""
    g = np.random.Generator(np.random.Philox(key=[seed, 77]))
    E, top_k = case["experts"], case["top_k"]
    share = 1.0 / np.arange(1, E + 1) ** case["skew"]
    share /= share.sum()
    out = []
    for _ in range(case["rows"] // top_k):
        out += g.choice(E, top_k, replace=top_k > E, p=share).tolist()
    none = g.random(len(out)) < case["none"]
    return [-1 if z else int(e) for e, z in zip(out, none)]


def _labels(g, primes, n):
    out = []
    for p in primes:
        t = torch.randint(0, p, (_chunks(p), n, 16), dtype=torch.uint8, device="cuda", generator=g)
        t[-1, :, LAMBDA[p] - 16 * (_chunks(p) - 1):] = 0
        out.append(t)
    return out


def _context(k):
    from paper_2302_06361_amd import Context
    return Context(PRIMES[:k], bytes(range(64, 80)), DIGITS[k])


def _bundle(ctx, n, tensors=None):
    from paper_2302_06361_amd import Labels
    b = Labels(ctx, n) if tensors is None else Labels(ctx, 0)
    if tensors is not None:
        b.n_elem, b.tensors = n, list(tensors)
    return b


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=case, own=own)
    if case["kind"] == "choose":
        # logits as a trained router gives them: some experts liked more than others, a few strong opinions; a bias that works against that
        T, E = case["rows"], case["experts"]
        liked = 0.5 * torch.randn(E, device="cuda", generator=g)
        l = 1.5 * torch.randn(T, E + case["pad"], device="cuda", generator=g)
        l[:, :E] += liked
        if case["masked"]:
            l = torch.where(torch.rand(l.shape, device="cuda", generator=g) < case["masked"], torch.full_like(l, -math.inf), l)
            l[T // 2] = -math.inf                              # no expert at all
        s["logits"] = l.to(DTYPES[case["dtype"]])[:, :E]
        s["bias"] = -0.1 * liked + 0.01 * torch.randn(E, device="cuda", generator=g) if case["bias"] else None
        s["valid"] = (torch.rand(T, device="cuda", generator=g) >= case["invalid"]).to(torch.uint8) if case["invalid"] else None
        if own:
            from paper_2302_06361_amd import GROUP_MAX, GROUP_PAIR, SIGMOID, SOFTMAX, Choice, Router
            s["ctx"] = _context(8)
            s["router"] = Router(E, case["top_k"], score=SIGMOID if case["score"] == "sigmoid" else SOFTMAX, bias=s["bias"], groups=case["groups"],
                                 top_groups=case["top_groups"], group_score=GROUP_PAIR if case["pairs"] else GROUP_MAX,
                                 renormalise=case["renormalise"], scale=case["scale"], gate_bits=case["gate_bits"])
            s["choice"] = Choice(s["ctx"], T, case["top_k"])
        return s
    if case["kind"] == "quantise":
        # weights as they leave training: normal, of a different size for every row, a few much larger, some exactly zero
        E, M, K = case["experts"], case["out_c"], case["K"]
        w = torch.randn(E, M, K + case["pad"], device="cuda", generator=g)
        w *= torch.exp2(torch.randn(E, M, 1, device="cuda", generator=g) - 5)
        u = torch.rand(w.shape, device="cuda", generator=g)
        w = torch.where(u < 0.01, w * 8, torch.where(u > 0.97, torch.zeros_like(w), w))
        s["w"] = w.to(DTYPES[case["dtype"]])[:, :, :K]
        if own:
            from paper_2302_06361_amd import F8, ExpertWeights
            s["ctx"] = _context(8)
            s["weights"] = ExpertWeights(s["ctx"], F8, E, M, K)
            s["values"] = torch.empty((E, M, K), dtype=s["w"].dtype, device="cuda")
        return s
    primes, rows, top_k = PRIMES[:case["k"]], case["rows"], case["top_k"]
    E, K, M = case["experts"], case["K"], case["out_c"]
    s["in"] = _labels(g, primes, rows // top_k * K)
    s["experts"] = _expert_numbers(case, seed)
    # codes as a quantised checkpoint holds them: normal weights, the largest of a block close to 448; scales that differ by some powers of two
    w = torch.randn(E, M, K, device="cuda", generator=g)
    s["codes"] = (w * 100).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    del w
    blocks = (E, (M + 127) // 128, (K + 127) // 128)
    s["scales"] = torch.exp2(4 + 1.5 * torch.randn(blocks, device="cuda", generator=g)).round().clamp(1, 255).to(torch.int32)
    if own:
        from paper_2302_06361_amd import EXPERTS, Layer
        s["ctx"] = ctx = _context(case["k"])
        s["weights"] = ctx.f8_prepare(s["codes"], s["scales"])
        s["src"], s["dst"] = _bundle(ctx, rows // top_k * K, s["in"]), _bundle(ctx, rows * M)
        routing = None
        if E > 1 or -1 in s["experts"]:
            routing = ctx.route(torch.tensor(s["experts"], dtype=torch.int32, device="cuda"), E)
        s["layer"] = Layer(EXPERTS, 1, rows, top_k=top_k, weights=s["weights"], routing=routing)
    return s


# ---- plain forms ----
def _plain_choose(s):
    # doubles: the choice and the rounding of the gates compare values that float32 does not tell apart
    case, T, E, top_k = s["case"], s["case"]["rows"], s["case"]["experts"], s["case"]["top_k"]
    l = s["logits"].double()
    if case["score"] == "softmax":
        m = l.amax(-1, keepdim=True)
        x = torch.exp(l - torch.where(m > -math.inf, m, torch.zeros_like(m)))
        total = x.sum(-1, keepdim=True)
        score = x / torch.where(total > 0, total, torch.ones_like(total))
    else:
        score = 1 / (1 + torch.exp(-l))
    none = l == -math.inf
    c = l if s["bias"] is None else score + s["bias"].double()
    c = torch.where(none, torch.full_like(c, -math.inf), c)
    if s["valid"] is not None:
        c = torch.where(s["valid"][:, None] != 0, c, torch.full_like(c, -math.inf))

    def best(v, n):
        """the numbers of the n largest, first among equals; -1 where nothing is left"""
        v, at = v.clone(), torch.arange(v.shape[1], device=v.device)[None]
        out = torch.full((v.shape[0], n), -1, dtype=torch.int64, device=v.device)
        for j in range(n):
            m = v.amax(-1, keepdim=True)
            i = torch.where(v == m, at, v.shape[1]).amin(-1, keepdim=True)
            out[:, j:j + 1] = torch.where(m > -math.inf, i, torch.full_like(i, -1))
            v.scatter_(1, i, -math.inf)
        return out
    G = case["groups"]
    if case["top_groups"] < G:
        of = c.view(T, G, E // G)
        first = of.amax(-1)
        if case["pairs"]:
            value = (c if s["bias"] is not None else torch.where(c > -math.inf, score, c)).view(T, G, E // G)
            at = torch.arange(E // G, device=c.device)
            i = torch.where(of == first[..., None], at, E // G).amin(-1, keepdim=True).clamp(max=E // G - 1)
            rest = torch.where(at == i, torch.full_like(of, -math.inf), of)
            j = torch.where(rest == rest.amax(-1, keepdim=True), at, E // G).amin(-1, keepdim=True).clamp(max=E // G - 1)
            two = torch.where(rest.amax(-1) > -math.inf, value.gather(-1, j)[..., 0], torch.zeros_like(first))
            first = torch.where(first > -math.inf, value.gather(-1, i)[..., 0] + two, first)
        kept = torch.zeros(T, G + 1, dtype=torch.bool, device=c.device)
        chosen = best(first, case["top_groups"])
        kept.scatter_(1, torch.where(chosen < 0, G, chosen), True)
        c = torch.where(kept[:, :G].repeat_interleave(E // G, 1), c, torch.full_like(c, -math.inf))
    experts = best(c, top_k)
    w = torch.where(experts >= 0, score.gather(1, experts.clamp(min=0)), torch.zeros((), dtype=torch.float64, device=c.device))
    if case["renormalise"]:
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
    w = w * case["scale"]
    return [experts.to(torch.int32), torch.round(w * 2.0 ** case["gate_bits"]).to(torch.int32), w.float()]


def _plain_quantise(s):
    case, w = s["case"], s["w"].double()                       # (quotients next to the middle of two e4m3 values)
    E, M, K = w.shape
    mb, kb = (M + 127) // 128, (K + 127) // 128
    wp = torch.zeros(E, mb * 128, kb * 128, dtype=torch.float64, device=w.device)
    wp[:, :M, :K] = w * 2.0 ** -case["base"]
    wp = wp.view(E, mb, 128, kb, 128)
    S = torch.ceil(wp.abs().amax((2, 4), keepdim=True) / 448).clamp(1, case["max_scale"])
    a = (wp.abs() / S).clamp(max=448.0)
    step = torch.exp2(torch.frexp(a)[1].clamp(min=-5).double() - 4)      # a = f 2^e, f in [1/2, 1): four significant bits, down to 2^-9
    q = torch.sign(wp) * torch.round(a / step) * step * S * 2.0 ** case["base"]
    return q.view(E, mb * 128, kb * 128)[:, :M, :K].to(s["w"].dtype)


def _by_expert(experts):
    rows = {}
    for r, e in enumerate(experts):
        rows.setdefault(e, []).append(r)
    rows.pop(-1, None)
    return rows


def _integer_weights(s, e):
    """the integers of expert e's matrix: 512 e4m3 S, below 2^26"""
    c = s["codes"][e].to(torch.int32)
    mant, exp = c & 7, (c >> 3) & 15
    mag = torch.where(exp > 0, (8 + mant) << (exp - 1).clamp(min=0), mant)
    S = s["scales"][e].repeat_interleave(128, 0)[:c.shape[0]].repeat_interleave(128, 1)[:, :c.shape[1]]
    return torch.where(c >> 7 > 0, -mag, mag) * S


def _plain_experts(s):
    case = s["case"]
    K, M, rows, top_k = case["K"], case["out_c"], case["rows"], case["top_k"]
    groups = {e: torch.tensor(r, device="cuda") for e, r in _by_expert(s["experts"]).items()}
    weights = {e: _integer_weights(s, e) for e in groups}
    out = []
    for p, x in zip(PRIMES, s["in"]):
        nch = x.shape[0]
        x = x.view(nch, rows // top_k, K, 16)
        o = torch.zeros(nch, rows, M, 16, dtype=torch.uint8, device="cuda")
        for e, r in groups.items():
            # residues below 37: sums of up to 12 945 products are exact in 32 bits
            w = torch.remainder(weights[e], p).float()
            for at in range(0, len(r), 64):
                rr = r[at:at + 64]
                a = x[:, torch.div(rr, top_k, rounding_mode="floor")].permute(2, 1, 0, 3).reshape(K, -1).float()
                y = torch.remainder(torch.mm(w, a), p).to(torch.uint8)
                o[:, rr] = y.view(M, len(rr), nch, 16).permute(2, 1, 0, 3)
        out.append(o.view(nch, rows * M, 16))
    return out


def run(state):
    case = state["case"]
    if not state["own"]:
        return {"choose": _plain_choose, "quantise": _plain_quantise, "experts": _plain_experts}[case["kind"]](state)
    ctx = state["ctx"]
    if case["kind"] == "choose":
        choice = ctx.choose(state["router"], state["logits"], valid=state["valid"], out=state["choice"])
        return [choice.experts, choice.gates, choice.weights]
    if case["kind"] == "quantise":
        ctx.f8_quantise(state["w"], base=case["base"], max_scale=case["max_scale"], out=state["weights"], values=state["values"])
        return state["values"]
    ctx.eval_layer(state["layer"], state["src"], None, state["dst"])
    return state["dst"].tensors


# ---- the definitions in 64 bits ----
def _exact_choose(s):
    """by whole-row sorts: numbers in a stable descending order"""
    case, T, E, k = s["case"], s["case"]["rows"], s["case"]["experts"], s["case"]["top_k"]
    l = s["logits"].double()
    able = ~torch.isneginf(l)
    if s["valid"] is not None:
        able &= s["valid"].bool()[:, None]
    if case["score"] == "softmax":
        score = torch.exp(l - torch.logsumexp(l, -1, keepdim=True).nan_to_num(neginf=0.0))
    else:
        score = torch.where(l > 0, 1 / (1 + torch.exp(-l.abs())), torch.exp(-l.abs()) / (1 + torch.exp(-l.abs())))
    key = l if s["bias"] is None else score + s["bias"].double()
    order = torch.sort(key.masked_fill(~able, -math.inf), dim=1, descending=True, stable=True)[1]
    G, n = case["groups"], E // case["groups"]
    if case["top_groups"] < G:
        ranked = torch.zeros(T, G, dtype=torch.float64, device="cuda")
        value = key if s["bias"] is not None else score if case["pairs"] else l
        for gi in range(G):
            part, ok = key[:, gi * n:(gi + 1) * n], able[:, gi * n:(gi + 1) * n]
            inside = torch.sort(part.masked_fill(~ok, -math.inf), dim=1, descending=True, stable=True)[1][:, :2 if case["pairs"] else 1]
            v = torch.where(ok.gather(1, inside), value[:, gi * n:(gi + 1) * n].gather(1, inside), torch.zeros((), dtype=torch.float64, device="cuda"))
            ranked[:, gi] = v.sum(1).masked_fill(~ok.any(1), -math.inf)
        rank = torch.argsort(torch.sort(ranked, dim=1, descending=True, stable=True)[1], dim=1)
        able &= (rank < case["top_groups"]).repeat_interleave(n, 1)
        order = torch.sort(key.masked_fill(~able, -math.inf), dim=1, descending=True, stable=True)[1]
    first = order[:, :k]
    there = able.gather(1, first)
    w = score.gather(1, first) * there
    if case["renormalise"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-300)
    w = w * case["scale"]
    return [first.masked_fill(~there, -1).int(), torch.round(torch.ldexp(w, torch.tensor(case["gate_bits"], device="cuda"))).int(), w]


def _exact_quantise(s):
    case, w = s["case"], s["w"].double()
    E, M, K = w.shape
    # the 127 magnitudes of e4m3, in the order of their codes
    grid = torch.tensor([m / 512 if e == 0 else (8 + m) / 8 * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64, device="cuda")
    out = torch.zeros_like(w)
    for i in range(0, M, 128):
        for j in range(0, K, 128):
            b = w[:, i:i + 128, j:j + 128]
            unit = 2.0 ** case["base"]
            S = torch.ceil(b.abs().flatten(1).amax(1) / (448 * unit)).clamp(1, case["max_scale"])[:, None, None] * unit
            a = (b.abs() / S).clamp(max=448.0)
            hi = torch.bucketize(a, grid).clamp(1, 126)
            up, down = grid[hi] - a, a - grid[hi - 1]
            q = grid[torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)]
            out[:, i:i + 128, j:j + 128] = torch.sign(b) * q * S
    return out


def _exact_experts(s):
    case = s["case"]
    K, M, rows, top_k = case["K"], case["out_c"], case["rows"], case["top_k"]
    # doubles hold every sum: weights below 2^26, labels below 37, up to 4096 terms
    values = torch.tensor([(-1) ** (c >> 7) * ((c & 7) if c >> 3 & 15 == 0 else (8 + (c & 7)) * 2 ** ((c >> 3 & 15) - 1)) for c in range(256)],
                          dtype=torch.float64, device="cuda")
    weights = {}
    for e in sorted(set(s["experts"]) - {-1}):
        w = values[s["codes"][e].long()]
        for i in range(0, M, 128):
            for j in range(0, K, 128):
                w[i:i + 128, j:j + 128] *= s["scales"][e, i // 128, j // 128]
        weights[e] = w
    out = []
    for p, x in zip(PRIMES, s["in"]):
        nch = x.shape[0]
        o = torch.zeros(nch, rows, M, 16, dtype=torch.uint8, device="cuda")
        x = x.view(nch, rows // top_k, K, 16)
        for r, e in enumerate(s["experts"]):
            if e >= 0:
                a = x[:, r // top_k].double().permute(1, 0, 2).reshape(K, nch * 16)
                o[:, r] = torch.remainder(weights[e] @ a, float(p)).to(torch.uint8).view(M, nch, 16).permute(1, 0, 2)
        out.append(o.view(nch, rows * M, 16))
    return out


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return {"choose": _exact_choose, "quantise": _exact_quantise, "experts": _exact_experts}[case["kind"]](s)
