"""Performance cases of the 8-bit operators around a linear layer and a mixture-of-experts
block: rows in 8-bit integers with a scale each, RMS norm with the residual's addition (and
its backward pass, and its output in 8 bits), products of 8-bit matrices with scales for each
token and channel, and the same by experts.

Kinds of call:
  quantize     fo.quantize_rows, the values that its codes stand for returned;
  norm_train   fo.norm_add_forward with 16-bit outputs, then fo.norm_add_backward;
  norm_linear  fo.norm_add_forward with 8-bit outputs, then fo.int8_product of them: the way
               into an attention or MLP projection when a model is served;
  product      fo.int8_product of activations and weights that are there in 8 bits;
  experts      fo.int8_experts over the rows that fo.route_sort has put in order, the rows
               taken from the tokens (gather) or standing in that order.

M, N: rows and columns, of the result where there is a product; H: its inner size;
T, K, E: tokens, choices per token, experts.
"""
import math

import torch

own = False

EPS = 1e-6
MOST_FLOPS, MOST_BYTES, MOST_WEIGHTS = 9.0e11, 1.2e9, 3.7e9      # of a drawn case
_DTYPE = {"fp16": torch.float16, "bf16": torch.bfloat16}


def listed():
    def case(name, op, **more):
        return dict({"name": name, "op": op}, **more)

    return [
        # a small activation of odd sizes
        case("quantize_517x1001", "quantize", M=517, N=1001, dtype="fp16"),
        # the input of an MLP's second projection (FFN 14336) over 8192 tokens
        case("quantize_8192x14336", "quantize", M=8192, N=14336, dtype="bf16"),
        # training on a ragged batch, hidden size 2880
        case("norm_train_1217x2880", "norm_train", M=1217, N=2880, dtype="fp16"),
        # a training micro-batch of 16384 tokens
        case("norm_train_16384x4096", "norm_train", M=16384, N=4096, dtype="bf16"),
        # one token of one sequence into a square projection
        case("norm_linear_1x4096x4096", "norm_linear", M=1, N=4096, H=4096, dtype="bf16", bias=False),
        # a long prompt into an MLP's first projection
        case("norm_linear_8192x14336x4096", "norm_linear", M=8192, N=14336, H=4096, dtype="bf16", bias=False),
        # a decode step of 16 sequences through an output projection
        case("product_16x7168x2048", "product", M=16, N=7168, H=2048, dtype="bf16", bias=False),
        # a short ragged prompt, sizes that no tile divides, with a bias
        case("product_333x2881x1985", "product", M=333, N=2881, H=1985, dtype="fp16", bias=True),
        # an MLP's down projection shard (hidden 8192, FFN 28672 / 8) over 8192 tokens
        case("product_8192x8192x3584", "product", M=8192, N=8192, H=3584, dtype="fp16", bias=False),
        # a decode step of 16 sequences into 8 of 256 experts each
        case("experts_16x2048x7168", "experts", T=16, K=8, E=256, N=2048, H=7168, dtype="bf16", gather=True, align=1, drop=0.0, bias=False),
        # a ragged batch back out of 4 of 60 experts each, some choices dropped, odd widths, with biases
        case("experts_1217x2881x1409", "experts", T=1217, K=4, E=60, N=2881, H=1409, dtype="fp16", gather=False, align=64, drop=0.02, bias=True),
        # a prompt of 4096 tokens into 8 of 64 experts each
        case("experts_4096x2048x7168", "experts", T=4096, K=8, E=64, N=2048, H=7168, dtype="bf16", gather=True, align=64, drop=0.0, bias=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A hidden size: mostly whole multiples of 64, and now and then odd."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.7 else n


def draw(rng):
    op = rng.choice(["quantize", "norm_train", "norm_linear", "product", "product", "experts", "experts"])
    while True:
        case = {"op": op, "dtype": rng.choice(["fp16", "bf16"])}
        if op in ("quantize", "norm_train"):
            case.update(M=_log(rng, 1, 32768), N=_width(rng, 64, 16384))
            if case["M"] * case["N"] > 16384 * 4096:
                continue
        elif op in ("norm_linear", "product"):
            case.update(M=_log(rng, 1, 16384), N=_width(rng, 64, 16384), H=_width(rng, 64, 16384), bias=rng.random() < 0.3)
        else:
            case.update(T=_log(rng, 1, 8192), K=rng.choice([1, 2, 4, 6, 8]), E=rng.choice([8, 16, 60, 64, 128, 160, 256]),
                        N=_width(rng, 64, 8192), H=_width(rng, 64, 8192), gather=rng.random() < 0.5, align=rng.choice([1, 64, 256]),
                        drop=rng.choice([0.0, 0.0, 0.03]), bias=rng.random() < 0.3)
            while case["align"] > 1 and min(case["E"], case["T"] * case["K"]) * case["align"] > 2 * case["T"] * case["K"]:
                case["align"] = {256: 64, 64: 1}[case["align"]]      # padding stays the smaller part
            if case["E"] * case["N"] * case["H"] > MOST_WEIGHTS:
                continue
        w = work(case)
        if w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES:
            return case


# ---- inputs ---------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def padded(n):
    """Bytes of a row of n codes: whole chunks of 16."""
    return -(-n // 16) * 16


def capacity_of(case):
    """Rows that hold every choice, each expert's padded to a multiple of `align`."""
    P = case["T"] * case["K"]
    return P + min(case["E"], P) * (case["align"] - 1)


def _codes(v):
    """(codes, scales) of rows of 32-bit values, codes behind a row's end 0."""
    top = v.abs().amax(dim=1)
    codes = torch.zeros(v.shape[0], padded(v.shape[1]), dtype=torch.int8, device="cuda")
    codes[:, :v.shape[1]] = (v * 127.0 / top[:, None]).round().to(torch.int8)
    return codes, top / 127.0


def _weights(case, gen, count):
    """A weight's rows in 8 bits: normal values, the largest of a row 3.5 to 4.5 deviations out."""
    N, H = case["N"], case["H"]
    codes = torch.randn(count * N, H, generator=gen, device="cuda").mul_(32.0).round_().clamp_(-127, 127).to(torch.int8)
    if padded(H) != H:
        codes = torch.nn.functional.pad(codes, (0, padded(H) - H))
    return codes, (0.75 + 0.5 * torch.rand(count * N, generator=gen, device="cuda")) / (32.0 * math.sqrt(H))


def prepare(case, seed):
    gen, dtype = _generator(seed), _DTYPE[case["dtype"]]

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(dtype)

    def empty(*shape, dtype=dtype):
        return torch.empty(*shape, dtype=dtype, device="cuda")

    def stream(M, N):
        """A residual stream: columns of uneven size."""
        size = 0.5 + torch.rand(N, generator=gen, device="cuda") * 2
        return torch.randn(M, N, generator=gen, device="cuda") * size

    s = {"case": case}
    op = case["op"]
    if op == "quantize":
        M, N = case["M"], case["N"]
        s["x"], s["values"] = stream(M, N).to(dtype), empty(M, N)
        s["codes"], s["scales"] = empty(M, padded(N), dtype=torch.int8), empty(M, dtype=torch.float32)
        return s
    if op in ("norm_train", "norm_linear"):
        M, H = case["M"], case["N"] if op == "norm_train" else case["H"]
        s["x"], s["residual"], s["h"] = normal(M, H), stream(M, H).to(dtype), empty(M, H)
        s["gamma"] = (0.5 + torch.rand(H, generator=gen, device="cuda")).to(dtype)
        if op == "norm_train":
            s["dy"], s["dh"], s["dx"], s["y"] = normal(M, H), normal(M, H), empty(M, H), empty(M, H)
            s["rstd"], s["dgamma"] = empty(M, dtype=torch.float32), empty(H, dtype=torch.float32)
            return s
        s["a"], s["a_scales"] = empty(M, padded(H), dtype=torch.int8), empty(M, dtype=torch.float32)
    if op in ("norm_linear", "product"):
        if op == "product":
            s["a"], s["a_scales"] = _codes(stream(case["M"], case["H"]))
        s["b"], s["b_scales"] = _weights(case, gen, 1)
        s["bias"] = normal(case["N"], scale=0.1) if case["bias"] else None
        s["c"] = empty(case["M"], case["N"])
        return s
    # the router's choices, distinct within a token, experts unevenly popular; -1: dropped
    T, K, E, N, rows = case["T"], case["K"], case["E"], case["N"], capacity_of(case)
    logits = torch.randn(T, E, generator=gen, device="cuda") + 0.7 * torch.randn(E, generator=gen, device="cuda")
    ids = torch.topk(logits, K, dim=1)[1]
    ids = torch.where(torch.rand(T, K, generator=gen, device="cuda") < case["drop"], -1, ids)
    s["offsets"], s["counts"], s["pair_of"] = _sorted(case, ids)
    s["most"] = max(1, int(s["counts"].max()))          # rows of the busiest expert
    s["a"], s["a_scales"] = _codes(stream(T if case["gather"] else rows, case["H"]))
    b, b_scales = _weights(case, gen, E)
    s["b"], s["b_scales"] = b.reshape(E, N, -1), b_scales.reshape(E, N)
    s["bias"] = normal(E, N, scale=0.1) if case["bias"] else None
    s["c"] = torch.zeros(rows, N, dtype=dtype, device="cuda")
    return s


def _sorted(case, ids):
    """(offsets, counts, pair_of) of the choices, experts in order, a choice's order within its expert kept."""
    T, K, E, align = case["T"], case["K"], case["E"], case["align"]
    flat = ids.reshape(-1)
    kept = flat >= 0
    key = torch.where(kept, flat, E)
    order = torch.argsort(key, stable=True)
    counts = torch.bincount(key, minlength=E + 1)[:E]
    zero = counts.new_zeros(1)
    offsets = torch.cat([zero, torch.cumsum((counts + align - 1) // align * align, 0)])
    first = torch.cat([zero, torch.cumsum(counts, 0)])
    slot = torch.arange(T * K, device=ids.device) - first[key[order]] + offsets[key[order]]
    pair_of = torch.full((capacity_of(case) + 1,), -1, dtype=torch.int32, device=ids.device)
    pair_of[torch.where(kept[order], slot, capacity_of(case))] = order.to(torch.int32)
    return offsets.to(torch.int32), counts.to(torch.int32), pair_of[:-1].contiguous()


# ---- one pass -------------------------------------------------------------

def run(s):
    return _calls(s) if own else _plain(s)


def _calls(s):
    import paper_2504_19519_amd as fo
    case = s["case"]
    op, dtype = case["op"], case["dtype"]
    if op == "quantize":
        fo.quantize_rows(s["x"], s["codes"], s["scales"], case["M"], case["N"], dtype)
        return {"values": torch.mul(s["codes"][:, :case["N"]], s["scales"][:, None], out=s["values"]), "scales": s["scales"]}
    if op == "norm_train":
        M, N = case["M"], case["N"]
        if "work" not in s:        # a program's one workspace
            s["work"] = torch.empty(fo.norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        fo.norm_add_forward(s["x"], s["residual"], s["gamma"], s["h"], s["y"], M, N, dtype, EPS, rstd=s["rstd"])
        fo.norm_add_backward(s["dy"], s["dh"], s["h"], s["gamma"], s["rstd"], s["dx"], s["dgamma"], M, N, dtype, s["work"])
        return {k: s[k] for k in ("h", "y", "rstd", "dx", "dgamma")}
    if op in ("norm_linear", "product"):
        M, N, H = case["M"], case["N"], case["H"]
        if "work" not in s:
            s["work"] = torch.empty(fo.int8_workspace_bytes(M, N, H), dtype=torch.uint8, device="cuda")
        if op == "norm_linear":
            fo.norm_add_forward(s["x"], s["residual"], s["gamma"], s["h"], None, M, H, dtype, EPS, codes=s["a"], scales=s["a_scales"])
        fo.int8_product(s["a"], s["a_scales"], s["b"], s["b_scales"], s["c"], M, N, H, dtype, bias=s["bias"], workspace=s["work"])
        return {"h": s["h"], "c": s["c"]} if op == "norm_linear" else {"c": s["c"]}
    fo.int8_experts(s["a"], s["a_scales"], s["b"], s["b_scales"], s["c"], case["N"], case["H"], case["E"], dtype, len(s["c"]),
                    s["offsets"], s["counts"], len(s["a"]), pair_of=s["pair_of"] if case["gather"] else None, choices=case["K"],
                    bias=s["bias"])
    return {"c": s["c"]}


def _plain(s):
    case = s["case"]
    op, dtype = case["op"], _DTYPE[case["dtype"]]
    if op == "quantize":
        x = s["x"].float()
        top = x.abs().amax(dim=1, keepdim=True)
        scales = top / 127.0
        codes = torch.where(top > 0, x * 127.0 / top, 0.0).round()
        return {"values": (codes * scales).to(dtype), "scales": scales.reshape(-1)}
    if op in ("norm_train", "norm_linear"):
        h = (s["x"].float() + s["residual"].float()).to(dtype)
        hf, gamma = h.float(), s["gamma"].float()
        rstd = 1.0 / torch.sqrt((hf * hf).mean(dim=1, keepdim=True) + EPS)
        y = hf * rstd * gamma
        if op == "norm_train":
            dy = s["dy"].float()
            hh, g = hf * rstd, dy * gamma
            dx = s["dh"].float() + rstd * (g - hh * (g * hh).mean(dim=1, keepdim=True))
            return {"h": h, "y": y.to(dtype), "rstd": rstd.reshape(-1), "dx": dx.to(dtype), "dgamma": (dy * hh).sum(dim=0)}
        top = y.abs().amax(dim=1, keepdim=True)
        a = torch.where(top > 0, y * 127.0 / top, 0.0).round()
        a_scales = top / 127.0
    if op in ("norm_linear", "product"):
        H = case["H"]
        if op == "product":
            a, a_scales = s["a"][:, :H].float(), s["a_scales"][:, None]
        c = torch.matmul(a, s["b"][:, :H].float().t()) * a_scales * s["b_scales"]
        c = (c if s["bias"] is None else c + s["bias"].float()).to(dtype)
        return {"h": h, "c": c} if op == "norm_linear" else {"c": c}
    E, N, H, rows, most = case["E"], case["N"], case["H"], len(s["c"]), s["most"]
    place = torch.arange(most, device="cuda")
    there = place < s["counts"][:, None]                                         # [E, most]
    at = torch.where(there, s["offsets"][:E, None] + place, rows).long()
    src = torch.where(there, s["pair_of"][at.clamp(max=rows - 1)].long() // case["K"] if case["gather"] else at, 0)
    right = s["a"][src][:, :, :H].transpose(1, 2).float().contiguous()           # [E, H, most]
    out = torch.bmm(s["b"][:, :, :H].float(), right).transpose(1, 2)
    out = out * s["a_scales"][src][:, :, None] * s["b_scales"][:, None, :]
    if s["bias"] is not None:
        out = out + s["bias"].float()[:, None, :]
    c = torch.zeros(rows + 1, N, dtype=dtype, device="cuda")
    c[at.reshape(-1)] = out.to(dtype).reshape(-1, N)
    return {"c": c[:-1]}


def work(case):
    op = case["op"]
    if op == "quantize":       # values in, codes and scales out; those in, values out
        MN = float(case["M"] * case["N"])
        return {"bytes": 6.0 * MN + 8.0 * case["M"], "flops": 4.0 * MN}
    if op == "norm_train":     # x, residual in, h, y out; dy, dh, h in, dx out
        MN = float(case["M"] * case["N"])
        return {"bytes": 16.0 * MN + 8.0 * case["M"] + 8.0 * case["N"], "flops": 16.0 * MN}
    N, H = case["N"], case["H"]
    if op == "experts":
        T, E = case["T"], case["E"]
        P = T * case["K"] * (1.0 - case["drop"])
        active = E * (1.0 - (1.0 - 1.0 / E) ** P)
        return {"bytes": active * (N * H + 4.0 * N) + (T if case["gather"] else P) * (H + 4.0) + 2.0 * P * N, "flops": 2.0 * P * N * H}
    M = case["M"]
    # (the norm: x, residual in, h, codes out, which the product reads)
    head = M * (8.0 * H + 4.0) + 2.0 * H if op == "norm_linear" else M * (H + 4.0)
    return {"bytes": head + float(N) * H + 4.0 * N + 2.0 * M * N, "flops": 2.0 * M * N * H}


# ---- the same in 64 bits ---------------------------------------------------

def _whole(v):
    """(codes, scales) of rows in 64 bits."""
    top = v.abs().max(dim=1, keepdim=True).values
    return torch.round(127 * v / torch.where(top > 0, top, 1.0)), top / 127


def exact(case, seed):
    s = prepare(case, seed)
    op, dtype = case["op"], _DTYPE[case["dtype"]]
    if op == "quantize":
        codes, scales = _whole(s["x"].double())
        return {"values": codes * scales, "scales": scales[:, 0]}
    if op in ("norm_train", "norm_linear"):
        h = s["x"].double() + s["residual"].double()
        h16 = h.float().to(dtype).double()       # (as it is kept)
        width = h.shape[1]
        rstd = (h16.square().sum(1) / width + EPS) ** -0.5
        if op == "norm_train":
            dy, gamma = s["dy"].double(), s["gamma"].double()
            dot = torch.einsum("mn,mn,n->m", dy, h16, gamma) / width
            dx = s["dh"].double() + rstd[:, None] * dy * gamma - h16 * (dot * rstd ** 3)[:, None]
            return {"h": h, "y": gamma * (h16 * rstd[:, None]), "rstd": rstd, "dx": dx, "dgamma": torch.einsum("mn,mn,m->n", dy, h16, rstd)}
        a, a_scales = _whole(s["gamma"].double() * (h16 * rstd[:, None]))
    if op in ("norm_linear", "product"):
        if op == "product":
            a, a_scales = s["a"][:, :case["H"]].double(), s["a_scales"].double()[:, None]
        c = (a * a_scales) @ (s["b"][:, :case["H"]].double() * s["b_scales"].double()[:, None]).t()
        if s["bias"] is not None:
            c += s["bias"].double()
        return {"h": h, "c": c} if op == "norm_linear" else {"c": c}
    H = case["H"]
    c = torch.zeros(s["c"].shape, dtype=torch.float64, device="cuda")
    offsets, counts = s["offsets"].tolist(), s["counts"].tolist()
    for e in range(case["E"]):
        if counts[e]:
            lo, hi = offsets[e], offsets[e] + counts[e]
            src = s["pair_of"][lo:hi].long() // case["K"] if case["gather"] else torch.arange(lo, hi, device="cuda")
            a = s["a"][src, :H].double() * s["a_scales"][src].double()[:, None]
            c[lo:hi] = a @ (s["b"][e, :, :H].double() * s["b_scales"][e].double()[:, None]).t()
            if s["bias"] is not None:
                c[lo:hi] += s["bias"][e].double()
    return {"c": c}
