"""The products of expert layers and the orthogonalised update of their weights, as cases that can be timed.

A layer of experts sends each token to some of its experts.  With the tokens sorted by expert the layer is a product grouped
by ragged sizes, and training it takes three of them:

  forward      y[t] = w[g] x[t]                     for the tokens t of expert g   (oz_gemm_grouped, transA = 1)
  input_grad   dx[t] = w[g]^T dy[t]                                                (oz_gemm_grouped, transA = 0)
  weight_grad  dw[g] = sum over its tokens of dy[t] x[t]^T                         (oz_gemm_grouped_wgrad)

  orthogonalise  the update of a matrix parameter by Newton-Schulz products (oz_orthogonalise):
               x = g / (|g|_F + 1e-7), then `steps` times  x <- a x + (b s + c s s) x  with s = x x^T

Fields of a case
  kind    one of the four;  type: type of the inputs (bf16, f16; orthogonalise also f32);  out: type of the result
  grouped: groups experts, tokens rows in all, m outputs and k inputs of an expert, skew: spread of the group sizes (standard deviation
          of their logarithm; sizes of zero are among them where tokens are few), behind: rows behind the last group, which stay as they are
  orthogonalise: count matrices of rows x cols, steps
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def _grouped(kind, groups, tokens, m, k, type="bf16", out=None, skew=0.5, behind=0):
    return {"kind": kind, "groups": groups, "tokens": tokens, "m": m, "k": k, "type": type, "out": out or type, "skew": skew, "behind": behind}


def _square(count, rows, cols, type="bf16", out=None, steps=5):
    return {"kind": "orthogonalise", "count": count, "rows": rows, "cols": cols, "type": type, "out": out or type, "steps": steps}


def listed():
    return [
        # one generated token through two of eight experts: reads two weight matrices, latency counts
        {"name": "forward_one_token", **_grouped("forward", 8, 2, 4096, 2048, skew=0.0)},
        # a batch of generated tokens over many experts: every weight is read for a handful of tokens
        {"name": "forward_decode", **_grouped("forward", 32, 128, 2048, 4096, skew=0.7)},
        # a prompt, or a training batch, in a layer of few large experts
        {"name": "forward_prompt", **_grouped("forward", 8, 8192, 4096, 4096)},
        # many small experts, uneven sizes, a padded batch, widths that no tile divides
        {"name": "forward_ragged_f16", **_grouped("forward", 64, 4099, 1000, 520, type="f16", skew=1.0, behind=101)},
        # gradient of the inputs of a training batch
        {"name": "input_grad", **_grouped("input_grad", 16, 16384, 2048, 4096)},
        # gradient of the weights of the same batch, kept in 32 bits for the optimiser
        {"name": "weight_grad_f32", **_grouped("weight_grad", 16, 16384, 2048, 4096, out="f32")},
        # gradient of the weights of a small uneven batch
        {"name": "weight_grad_small", **_grouped("weight_grad", 32, 1021, 1024, 1536, skew=1.0, behind=3)},
        # update of one narrow parameter: launches count
        {"name": "orthogonalise_narrow", **_square(1, 128, 512, type="f32")},
        # update of an ordinary square projection
        {"name": "orthogonalise_1024", **_square(1, 1024, 1024)},
        # update of all experts of a layer at once
        {"name": "orthogonalise_experts", **_square(16, 512, 2048)},
        # odd sizes, taller than wide, from a 16-bit gradient into 32 bits
        {"name": "orthogonalise_tall_f16", **_square(3, 1009, 517, type="f16", out="f32")},
        # update of a large projection held in 32 bits
        {"name": "orthogonalise_4096", **_square(1, 4096, 4096, type="f32")},
    ]


def _log_int(rng, low, high, multiple=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(low, min(high, round(v / multiple) * multiple))


def draw(rng):
    if rng.random() < 0.6:
        while True:
            type = rng.choice(["bf16", "f16"])
            c = _grouped(rng.choice(["forward", "input_grad", "weight_grad"]), _log_int(rng, 1, 64), _log_int(rng, 1, 16384),
                         _log_int(rng, 128, 4096, 8), _log_int(rng, 128, 4096, 8), type=type, out=rng.choice([type, type, "f32"]),
                         skew=rng.choice([0.0, 0.5, 1.0]), behind=rng.choice([0, 0, 1, 77]))
            # no dearer than the largest listed one, in operations and in weights
            if c["tokens"] * c["m"] * c["k"] <= 16384 * 2048 * 4096 and c["groups"] * c["m"] * c["k"] <= 32 * 2048 * 4096:
                return c
    while True:
        type = rng.choice(["bf16", "f16", "f32"])
        c = _square(_log_int(rng, 1, 16), _log_int(rng, 32, 4096), _log_int(rng, 32, 4096), type=type, out=rng.choice([type, "f32"]))
        if work(c)["flops"] <= work(_square(1, 4096, 4096))["flops"]:
            return c


def _sizes(case):
    """Group sizes: shares exp(skew N(0,1)) of the tokens, cut at whole tokens; the same for every seed, which only shuffles them."""
    rng = random.Random(case["groups"] * 1000003 + case["tokens"])
    share = [math.exp(case["skew"] * rng.gauss(0.0, 1.0)) for _ in range(case["groups"])]
    total, at, cuts = sum(share), 0.0, [0]
    for s in share:
        at += s
        cuts.append(round(case["tokens"] * at / total))
    cuts[-1] = case["tokens"]
    return [b - a for a, b in zip(cuts, cuts[1:])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    type = TYPES[case["type"]]
    out = TYPES[case["out"]]
    if case["kind"] == "orthogonalise":
        count, rows, cols = case["count"], case["rows"], case["cols"]
        # a gradient: a part of low rank that many samples share, and noise
        rank = max(1, min(rows, cols) // 8)
        g = torch.randn(count, rows, rank, device="cuda", generator=gen) @ torch.randn(count, rank, cols, device="cuda", generator=gen) / rank ** 0.5
        g = 1e-3 * (g + torch.randn(count, rows, cols, device="cuda", generator=gen))
        return {"kind": case["kind"], "g": g.to(type), "steps": case["steps"], "out": out}
    groups, tokens, m, k = case["groups"], case["tokens"], case["m"], case["k"]
    sizes = _sizes(case)
    random.Random(seed).shuffle(sizes)
    offsets = torch.tensor([0] + sizes).cumsum(0)
    longest = max(sizes)
    # the padded batch of the plain form: where row i of group g lies, and where token t went
    at = offsets[:-1, None] + torch.arange(longest)[None, :]
    inside = at < offsets[1:, None]
    place = torch.arange(groups * longest).reshape(groups, longest)[inside]
    all_rows = tokens + case["behind"]
    s = {"kind": case["kind"], "groups": groups, "tokens": tokens, "m": m, "k": k, "out": out, "offsets": offsets.cuda(),
         "rows": torch.where(inside, at, 0).cuda(), "inside": inside.cuda(), "place": place.cuda()}
    if case["kind"] != "input_grad":
        s["x"] = torch.randn(all_rows, k, device="cuda", generator=gen).to(type)
    if case["kind"] != "forward":
        s["dy"] = torch.randn(all_rows, m, device="cuda", generator=gen).to(type)
    if case["kind"] != "weight_grad":
        s["w"] = (torch.randn(groups, m, k, device="cuda", generator=gen) / k ** 0.5).to(type)
    if case["kind"] == "weight_grad":
        s["result"] = torch.zeros(groups, m, k, dtype=out, device="cuda")
    else:
        s["result"] = torch.zeros(all_rows, m if case["kind"] == "forward" else k, dtype=out, device="cuda")
    return s


def run(state):
    if own:
        return _run_own(state)
    if state["kind"] == "orthogonalise":
        return _plain_orthogonalise(state["g"], state["steps"]).to(state["out"])
    if state["kind"] == "weight_grad":
        return torch.bmm(_padded(state, "dy").transpose(1, 2), _padded(state, "x")).to(state["out"])
    w = state["w"].float()
    y = torch.bmm(_padded(state, "x"), w.transpose(1, 2)) if state["kind"] == "forward" else torch.bmm(_padded(state, "dy"), w)
    result = torch.zeros_like(state["result"])
    result[:state["tokens"]] = y.flatten(0, 1)[state["place"]].to(state["out"])
    return result


def _padded(state, name):
    """The rows of each group, filled up with zeros to the longest group."""
    return torch.where(state["inside"][:, :, None], state[name].float()[state["rows"]], 0.0)


def _plain_orthogonalise(g, steps):
    a, b, c = COEFFICIENTS
    x = g.float()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(steps):
        s = x @ x.transpose(1, 2)
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.transpose(1, 2) if tall else x


_names = {torch.bfloat16: "OZ_BF16", torch.float16: "OZ_F16", torch.float32: "OZ_F32"}


def _run_own(state):
    import paper_2609_09095_b200 as oz

    if state["kind"] == "orthogonalise":
        g = state["g"]
        count, rows, cols = g.shape
        x = torch.empty(count, rows, cols, dtype=state["out"], device=g.device)
        workspace = torch.empty(oz.oz_orthogonalise_workspace_bytes(cols, rows, count), dtype=torch.uint8, device=g.device)
        # a row-major matrix is the column-major transpose, and the update of the transpose is the transpose of the update
        oz.check(oz.oz_orthogonalise(cols, rows, count, getattr(oz, _names[g.dtype]), g, cols, rows * cols, state["steps"], COEFFICIENTS, EPS,
                                     getattr(oz, _names[state["out"]]), x, cols, rows * cols, workspace), "oz_orthogonalise")
        return x
    groups, m, k, offsets, result = state["groups"], state["m"], state["k"], state["offsets"], state["result"]
    out = getattr(oz, _names[state["out"]])
    if state["kind"] == "weight_grad":
        x, dy = state["x"], state["dy"]
        oz.check(oz.oz_gemm_grouped_wgrad(k, m, x.shape[0], groups, offsets, getattr(oz, _names[x.dtype]), x, k, dy, m, out, 0.0, result, k, m * k),
                 "oz_gemm_grouped_wgrad")
    elif state["kind"] == "forward":
        x, w = state["x"], state["w"]
        oz.check(oz.oz_gemm_grouped(1, m, x.shape[0], k, groups, offsets, getattr(oz, _names[x.dtype]), w, k, m * k, x, k, out, 0.0, result, m),
                 "oz_gemm_grouped")
    else:
        dy, w = state["dy"], state["w"]
        oz.check(oz.oz_gemm_grouped(0, k, dy.shape[0], m, groups, offsets, getattr(oz, _names[dy.dtype]), w, k, m * k, dy, m, out, 0.0, result, k),
                 "oz_gemm_grouped")
    return result


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}
    i, o = size[case["type"]], size[case["out"]]
    if case["kind"] == "orthogonalise":
        r, c = sorted((case["rows"], case["cols"]))
        # a step: half of the symmetric x x^T, half of the symmetric s s, and the product with x
        return {"bytes": case["count"] * r * c * (i + o), "flops": case["count"] * case["steps"] * (r * r * c + r * r * r + 2 * r * r * c)}
    m, k, tokens = case["m"], case["k"], case["tokens"]
    used = sum(1 for s in _sizes(case) if s)
    flops = 2 * tokens * m * k
    if case["kind"] == "weight_grad":
        return {"bytes": i * tokens * (m + k) + o * case["groups"] * m * k, "flops": flops}
    return {"bytes": i * used * m * k + tokens * (i * (k if case["kind"] == "forward" else m) + o * (m if case["kind"] == "forward" else k)), "flops": flops}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "orthogonalise":
        return torch.stack([_exact_update(g, case["steps"]) for g in s["g"].double()])
    result = s["result"].double()
    cuts = s["offsets"].tolist()
    for g, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
        if case["kind"] == "forward":
            result[lo:hi] = torch.einsum("tk,mk->tm", s["x"][lo:hi].double(), s["w"][g].double())
        elif case["kind"] == "input_grad":
            result[lo:hi] = torch.einsum("tm,mk->tk", s["dy"][lo:hi].double(), s["w"][g].double())
        else:
            result[g] = torch.einsum("tm,tk->mk", s["dy"][lo:hi].double(), s["x"][lo:hi].double())
    return result


def _exact_update(g, steps):
    """In terms of the singular values: g = u diag(d) v^T, and a step takes d to a d + b d^3 + c d^5, so that the update is
    u diag(p(d) / d) u^T g; from the eigenvectors of g g^T, whose rounding (2^-53 of the largest d^2) falls on directions that matter least."""
    a, b, c = COEFFICIENTS
    if g.shape[0] > g.shape[1]:
        return _exact_update(g.T, steps).T
    g = g / (torch.linalg.norm(g) + EPS)
    squares, u = torch.linalg.eigh(g @ g.T)
    factor, square = torch.ones_like(squares), squares.clamp_min(0.0)
    for _ in range(steps):
        f = a + square * (b + square * c)
        factor, square = factor * f, square * f * f
    return u @ (factor[:, None] * (u.T @ g))
