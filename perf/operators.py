"""Expert layers of a garbled network as timing cases: 4-bit weights, products grouped by expert, the weighted sum of a
batch element's experts.

Labels are held as the library holds them: for every CRT prime p a uint8 tensor [chunks][elements][16], the lambda_p digits of an
element's label in [0, p) cut into chunks of 16, zeros past lambda_p.  Elements are ordered [batch element][feature].

  kind "quantise"  weights (float32, bfloat16 or float16) to blocks of 32 four-bit floats (e2m1) with a shared power of two:
                   E = clamp(floor(log2 amax) - 2, base, base + max_shift), the nearest e2m1 value of w / 2^E, ties to the even
                   code, saturated at 6.  Output: the values that the 4-bit weights stand for
  kind "experts"   out[r][j] = sum_i W_e(r)[j][i] in[r / top_k][i] on every digit, mod p; e(r): the public expert of row r, -1: none
                   (zeros).  fmt "w8": weights in int8; "mx4": 4-bit floats, integers 2 q 2^shift.  experts = 1: a dense layer
  kind "combine"   out[t][v] = sum_j gate[t][j] in[t top_k + j][v] on every digit, mod p
"""
import math

import numpy as np
import torch

own = False

PRIMES = [2, 3, 5, 7, 11, 13, 17, 19, 23, 29, 31, 37]
# mixed-radix digits of the sign gadget by number of primes
DIGITS = {7: (10,) + (13,) * 5, 8: (26,) + (12,) * 6, 9: (22,) + (10,) * 8, 12: (46,) + (17,) * 10}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
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


def listed():
    return [
        # the last layer of the small dense network (128 -> 10): the smallest matrix
        dict(name="quantise_128_10", kind="quantise", dtype="f32", experts=1, out_c=10, K=128, pad=0, base=-6, max_shift=8),
        # odd sizes, rows that lie further apart than they are long (a slice of a wider matrix)
        dict(name="quantise_odd_strided", kind="quantise", dtype="f16", experts=3, out_c=257, K=1030, pad=26, base=-9, max_shift=255),
        # a 4096 x 4096 layer as it leaves training
        dict(name="quantise_4096", kind="quantise", dtype="bf16", experts=1, out_c=4096, K=4096, pad=0, base=-10, max_shift=20),
        # one image through the first layer of the small dense network with 4-bit weights: latency
        dict(name="mx4_784_128_b1", kind="experts", fmt="mx4", k=8, experts=1, top_k=1, rows=1, K=784, out_c=128, skew=0, none=0.0),
        # one token through a large dense layer on the 12-prime base
        dict(name="mx4_4096_b1", kind="experts", fmt="mx4", k=12, experts=1, top_k=1, rows=1, K=4096, out_c=4096, skew=0, none=0.0),
        # the dense benchmark layer, batch 128: the largest
        dict(name="mx4_4096_b128", kind="experts", fmt="mx4", k=12, experts=1, top_k=1, rows=128, K=4096, out_c=4096, skew=0, none=0.0),
        # 16 images of 8 clients, each client with a layer of its own in place of the first dense layer of LeNet-5
        dict(name="w8_clients_400_120", kind="experts", fmt="w8", k=8, experts=8, top_k=1, rows=16, K=400, out_c=120, skew=0, none=0.0),
        # 64 images of the CIFAR-sized network, 12 clients of very different shares, some images of no client
        dict(name="w8_clients_4096_256", kind="experts", fmt="w8", k=12, experts=12, top_k=1, rows=64, K=4096, out_c=256, skew=2, none=0.1),
        # a mixture of 32 experts, two for each of 128 tokens, ragged
        dict(name="mx4_mixture_32", kind="experts", fmt="mx4", k=12, experts=32, top_k=2, rows=256, K=1024, out_c=2048, skew=1, none=0.0),
        # the two experts of each of 16 images joined, 84 values each
        dict(name="combine_84_b16", kind="combine", k=8, top_k=2, rows=32, V=84),
        # the four experts of each of 128 tokens joined
        dict(name="combine_4096_b128", kind="combine", k=12, top_k=4, rows=512, V=4096),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["quantise", "experts", "experts", "combine"])
        if kind == "quantise":
            c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16"]), experts=rng.randint(1, 8), out_c=_log(rng, 8, 4096), K=_log(rng, 32, 4096),
                     pad=rng.choice([0, 0, rng.randint(1, 40)]), base=rng.randint(-12, -4), max_shift=rng.choice([4, 8, 20, 255]))
        elif kind == "experts":
            top_k = rng.choice([1, 1, 2, 4])
            c = dict(kind=kind, fmt=rng.choice(["w8", "mx4"]), k=rng.choice([7, 8, 9, 12]), experts=_log(rng, 1, 64), top_k=top_k,
                     rows=top_k * _log(rng, 1, 256), K=_log(rng, 60, 4096), out_c=_log(rng, 8, 4096), skew=rng.randint(0, 2),
                     none=rng.choice([0.0, 0.0, 0.1]))
        else:
            top_k = rng.randint(1, 8)
            c = dict(kind=kind, k=rng.choice([7, 8, 9, 12]), top_k=top_k, rows=top_k * _log(rng, 1, 256), V=_log(rng, 8, 4096))
        w, top = work(c), work(listed()[5])
        # the plain form's passes are dominated by operations of products and by bytes of the others
        if w["flops"] <= top["flops"] and w["bytes"] <= 2 ** 31:
            return c


def work(case):
    if case["kind"] == "quantise":
        n = case["experts"] * case["out_c"] * case["K"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + n * 17 / 32, "flops": 4 * n}
    primes = PRIMES[:case["k"]]
    stored, digits = sum(16 * _chunks(p) for p in primes), sum(LAMBDA[p] for p in primes)
    rows, top_k = case["rows"], case["top_k"]
    if case["kind"] == "combine":
        return {"bytes": (rows + rows // top_k) * case["V"] * stored + 4 * rows, "flops": 2 * rows * case["V"] * digits}
    K, M = case["K"], case["out_c"]
    busy = sum(1 for r in _expert_numbers(case, 0) if r >= 0)
    used = len({r for r in _expert_numbers(case, 0) if r >= 0})
    weights = used * M * K * (1 if case["fmt"] == "w8" else 17 / 32)
    return {"bytes": (rows // top_k * K + rows * M) * stored + weights, "flops": 2 * busy * M * K * digits}


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
    if case["kind"] == "quantise":
        # weights as they leave training: normal, of a different size for every row, a few much larger, some exactly zero
        E, M, K = case["experts"], case["out_c"], case["K"]
        w = torch.randn(E, M, K + case["pad"], device="cuda", generator=g)
        w *= torch.exp2(2 * torch.randn(E, M, 1, device="cuda", generator=g) - 5)
        u = torch.rand(w.shape, device="cuda", generator=g)
        w = torch.where(u < 0.01, w * 16, torch.where(u > 0.97, torch.zeros_like(w), w))
        s["w"] = w.to(DTYPES[case["dtype"]])[:, :, :K]
        if own:
            from paper_2302_06361_amd import MX4, ExpertWeights
            s["ctx"] = _context(8)
            s["weights"] = ExpertWeights(s["ctx"], MX4, E, M, K)
            s["values"] = torch.empty((E, M, K), dtype=s["w"].dtype, device="cuda")
        return s
    primes, rows, top_k = PRIMES[:case["k"]], case["rows"], case["top_k"]
    if own:
        s["ctx"] = _context(case["k"])
    if case["kind"] == "combine":
        V = case["V"]
        s["in"] = _labels(g, primes, rows * V)
        s["gates"] = torch.randint(-64, 64, (rows // top_k, top_k), dtype=torch.int32, device="cuda", generator=g)
        if own:
            from paper_2302_06361_amd import COMBINE, Layer
            s["src"], s["dst"] = _bundle(s["ctx"], rows * V, s["in"]), _bundle(s["ctx"], rows // top_k * V)
            s["layer"] = Layer(COMBINE, 1, rows // top_k, in_c=V, top_k=top_k, gates=s["gates"])
        return s
    E, K, M = case["experts"], case["K"], case["out_c"]
    s["in"] = _labels(g, primes, rows // top_k * K)
    s["experts"] = _expert_numbers(case, seed)
    if case["fmt"] == "w8":
        s["w"] = torch.randint(-64, 64, (E, M, K), dtype=torch.int8, device="cuda", generator=g)
    else:
        # codes (bit 3: sign) and a power of two for every 32 weights of a row
        s["codes"] = torch.randint(0, 16, (E, M, K), dtype=torch.uint8, device="cuda", generator=g)
        s["shifts"] = torch.randint(0, 12, (E, M, (K + 31) // 32), dtype=torch.uint8, device="cuda", generator=g)
    if own:
        from paper_2302_06361_amd import EXPERTS, Layer
        ctx = s["ctx"]
        if case["fmt"] == "w8":
            s["weights"] = ctx.weights8_prepare(s["w"])
        else:
            w = torch.zeros(E, M, K, device="cuda")
            for e in range(E):                                 # on the grid of the 4-bit floats: quantised without a loss
                v = torch.tensor(E2M1, device="cuda")[(s["codes"][e] & 7).long()] * (1 - 2 * (s["codes"][e] >> 3).float())
                w[e] = v * torch.exp2(s["shifts"][e].float()).repeat_interleave(32, 1)[:, :K]
            s["weights"] = ctx.mx4_quantise(w, base=0, max_shift=255)
        s["src"], s["dst"] = _bundle(ctx, rows // top_k * K, s["in"]), _bundle(ctx, rows * M)
        routing = None
        if E > 1 or -1 in s["experts"]:
            routing = ctx.route(torch.tensor(s["experts"], dtype=torch.int32, device="cuda"), E)
        s["layer"] = Layer(EXPERTS, 1, rows, top_k=top_k, weights=s["weights"], routing=routing)
    return s


def _power(e):
    """2^e, -127 < e < 128, from its bits"""
    return ((e + 127) << 23).view(torch.float32)


def _scale_e2m1(w):
    """nearest e2m1 magnitude, ties to the even code"""
    a = w.abs()
    n = ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float()) * 0.5
    return n + (a > 2.5).float() + (a >= 3.5).float() + 2 * (a > 5).float()


def _plain_quantise(s):
    case, w = s["case"], s["w"].float()
    E, M, K = w.shape
    n = (K + 31) // 32
    wp = torch.zeros(E, M, n * 32, device=w.device)
    wp[:, :, :K] = w
    wp = wp.view(E, M, n, 32)
    amax = wp.abs().amax(-1, keepdim=True)
    e = torch.frexp(amax)[1] - 3                               # amax = m 2^e', m in [1/2, 1): floor(log2 amax) = e' - 1
    e = torch.where(amax > 0, e, torch.full_like(e, case["base"])).clamp(case["base"], min(case["base"] + case["max_shift"], 126))
    q = torch.sign(wp) * _scale_e2m1(wp * _power(-e)) * _power(e)
    return q.view(E, M, n * 32)[:, :, :K].to(s["w"].dtype)


def _by_expert(experts):
    rows = {}
    for r, e in enumerate(experts):
        rows.setdefault(e, []).append(r)
    rows.pop(-1, None)
    return rows


def _integer_weights(s, e, dtype):
    """the integers of expert e's matrix"""
    if s["case"]["fmt"] == "w8":
        return s["w"][e].to(dtype)
    c = s["codes"][e]
    mag = torch.tensor([int(2 * v) for v in E2M1], dtype=dtype, device=c.device)[(c & 7).long()]
    two = torch.ones((), dtype=dtype, device=c.device) << s["shifts"][e].to(dtype)
    return mag * (1 - 2 * (c >> 3).to(dtype)) * two.repeat_interleave(32, 1)[:, :c.shape[1]]


def _plain_experts(s):
    case = s["case"]
    K, M, rows, top_k = case["K"], case["out_c"], case["rows"], case["top_k"]
    groups = {e: torch.tensor(r, device="cuda") for e, r in _by_expert(s["experts"]).items()}
    weights = {e: _integer_weights(s, e, torch.int32) for e in groups}
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


def _plain_combine(s):
    case = s["case"]
    V, rows, top_k = case["V"], case["rows"], case["top_k"]
    out = []
    for p, x in zip(PRIMES, s["in"]):
        x = x.view(x.shape[0], rows // top_k, top_k, V, 16)
        gate = torch.remainder(s["gates"], p).float()
        acc = torch.zeros(x.shape[0], rows // top_k, V, 16, device="cuda")
        for j in range(top_k):
            acc += x[:, :, j].float() * gate[None, :, j, None, None]
        out.append(torch.remainder(acc, p).to(torch.uint8).view(x.shape[0], -1, 16))
    return out


def run(state):
    case = state["case"]
    if not state["own"]:
        return {"quantise": _plain_quantise, "experts": _plain_experts, "combine": _plain_combine}[case["kind"]](state)
    ctx = state["ctx"]
    if case["kind"] == "quantise":
        ctx.mx4_quantise(state["w"], base=case["base"], max_shift=case["max_shift"], out=state["weights"], values=state["values"])
        return state["values"]
    ctx.eval_layer(state["layer"], state["src"], None, state["dst"])
    return state["dst"].tensors


def exact(case, seed):
    """the definitions in 64 bits"""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "quantise":
        w = s["w"].double()
        grid = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
        out = torch.zeros_like(w)
        for at in range(0, case["K"], 32):
            b = w[:, :, at:at + 32]
            amax = b.abs().amax(-1, keepdim=True)
            e = (amax.view(torch.int64) >> 52) - 1025          # the exponent's bits: floor(log2 amax) - 2 (zero: below every base)
            e = e.clamp(case["base"], case["base"] + case["max_shift"])
            two = ((e + 1023) << 52).view(torch.float64)
            a = (b.abs() / two).clamp(max=6.0)
            hi = torch.bucketize(a, grid).clamp(1, 7)          # grid[hi - 1] < a <= grid[hi] (hi = 1 for zero)
            up, down = grid[hi] - a, a - grid[hi - 1]
            out[:, :, at:at + 32] = torch.sign(b) * grid[torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)] * two
        return out
    if case["kind"] == "combine":
        V, rows, top_k = case["V"], case["rows"], case["top_k"]
        out = []
        for p, x in zip(PRIMES, s["in"]):
            res = torch.empty(x.shape[0], rows // top_k, V, 16, dtype=torch.int64, device="cuda")
            x = x.view(x.shape[0], rows // top_k, top_k, V, 16)
            for t in range(rows // top_k):
                res[:, t] = (x[:, t].long() * s["gates"][t].long()[None, :, None, None]).sum(1) % p
            out.append(res.to(torch.uint8).view(x.shape[0], -1, 16))
        return out
    K, M, rows, top_k = case["K"], case["out_c"], case["rows"], case["top_k"]
    used = sorted(set(s["experts"]) - {-1})
    # doubles hold every sum: integers below 12 * 2^11 (4-bit) or 128 (int8), labels below 37, up to 4096 terms
    weights = {e: _integer_weights(s, e, torch.int64).double() for e in used}
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
