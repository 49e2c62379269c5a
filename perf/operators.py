"""Cases for the operators around the classifier: what a network answers with, what it is scored on, what updates it.

  logprobs  log probabilities of given classes, log-sum-exp, entropy and the top alternatives of rows of logits
            (vgg19_logprobs), and with "train" their gradient as well (vgg19_logprobs_backward)
  q4        a dense layer over 4-bit weights with group scales, for a few rows at a time (vgg19_q4_linear)
  muon      momentum, Newton-Schulz orthogonalisation and the update of weight matrices (vgg19_muon_update)

Each has its plain form here, in elementary torch operations, beside the call a program makes of the library.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
PAD = -1  # an id that asks for nothing
NS = (3.4445, -4.7750, 2.0315)  # the quintic step of the Newton-Schulz iteration


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # one image's answer: 1000 classes, the five best
        {"name": "answer one image", "op": "logprobs", "rows": 1, "classes": 1000, "dtype": "fp32", "ids": 1, "top": 5,
         "masked": False, "train": False},
        # one step of sampling over a long list of classes, some of them excluded
        {"name": "answer one long row", "op": "logprobs", "rows": 1, "classes": 131072, "dtype": "bf16", "ids": 1, "top": 20,
         "masked": True, "train": False},
        # scoring a batch of texts: an odd number of classes, so that no row but the first starts on 16 bytes
        {"name": "score many rows", "op": "logprobs", "rows": 2048, "classes": 50021, "dtype": "fp32", "ids": 3, "top": 8,
         "masked": True, "train": False},
        # a training step's loss: forward and gradient, an entropy term, padded rows
        {"name": "train many rows", "op": "logprobs", "rows": 4096, "classes": 32003, "dtype": "bf16", "ids": 1, "top": 0,
         "masked": False, "train": True},
        # the three dense layers of a 224 x 224 network answering for one image or a few
        {"name": "dense 3, one image", "op": "q4", "batch": 1, "in": 4096, "out": 1000, "group": 128, "dtype": "bf16", "relu": False},
        {"name": "dense 1, one image", "op": "q4", "batch": 1, "in": 25088, "out": 4096, "group": 128, "dtype": "bf16", "relu": True},
        {"name": "dense 2, sixteen images", "op": "q4", "batch": 16, "in": 4096, "out": 4096, "group": 32, "dtype": "bf16", "relu": True},
        # sizes that divide nothing, fp32 activations
        {"name": "odd sizes, five rows", "op": "q4", "batch": 5, "in": 5003, "out": 4099, "group": 64, "dtype": "fp32", "relu": False},
        # the update of one small filter, of all convolution filters, of the classifier, of its largest matrix
        {"name": "one filter", "op": "muon", "shapes": "128x576", "nesterov": True, "decay": 0.0},
        {"name": "sixteen filters", "op": "muon", "nesterov": True, "decay": 0.01,
         "shapes": "64x27 64x576 128x576 128x1152 256x1152 256x2304 256x2304 256x2304 512x2304 512x4608 512x4608 512x4608 "
                   "512x4608 512x4608 512x4608 512x4608"},
        {"name": "odd and tall matrices", "op": "muon", "shapes": "1001x333 77x2049 1x513", "nesterov": False, "decay": 0.01},
        {"name": "dense layers", "op": "muon", "shapes": "4096x25088 4096x4096 1000x4096", "nesterov": True, "decay": 0.01},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    op = rng.choice(["logprobs", "q4", "muon"])
    if op == "logprobs":
        rows = log(1, 4096)
        classes = log(2, min(131072, 100_000_000 // rows))
        return {"op": op, "rows": rows, "classes": classes, "dtype": rng.choice(["fp32", "bf16"]), "ids": rng.randint(1, 8),
                "top": rng.randint(0, min(32, classes)), "masked": rng.random() < 0.5, "train": rng.random() < 0.5}
    if op == "q4":
        inner = log(64, 25088)
        return {"op": op, "batch": rng.randint(1, 16), "in": inner, "out": log(16, min(16384, 100_000_000 // inner)),
                "group": rng.choice([32, 64, 128]), "dtype": rng.choice(["fp32", "bf16"]), "relu": rng.random() < 0.5}
    shapes = []
    for _ in range(rng.randint(1, 4)):
        small = log(1, 1500)
        big = log(small, 8192)
        shapes.append((small, big) if rng.random() < 0.75 else (big, small))
    return {"op": op, "shapes": " ".join("%dx%d" % s for s in shapes), "nesterov": rng.random() < 0.7,
            "decay": rng.choice([0.0, 0.01, 0.1])}


def shapes_of(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split()]


def work(case):
    if case["op"] == "logprobs":
        r, n, elt = case["rows"], case["classes"], 4 if case["dtype"] == "fp32" else 2
        small = r * (8 + 8 * case["ids"] + 8 * case["top"])
        if case["train"]:  # the logits twice: the gradient needs the sums over the whole row
            return {"bytes": 3 * r * n * elt + small + r * 4 * (case["ids"] + 1), "flops": 10 * r * n}
        return {"bytes": r * n * elt + small, "flops": 5 * r * n}
    if case["op"] == "q4":
        b, i, o, elt = case["batch"], case["in"], case["out"], 4 if case["dtype"] == "fp32" else 2
        return {"bytes": o * (i / 2 + 2 * -(-i // case["group"]) + 4) + elt * b * (i + o), "flops": 2 * b * i * o}
    shapes = shapes_of(case)
    # gradient read; momentum and weights read and written; bf16 weights written.  Products: two Gram matrices (each
    # symmetric), three steps and two steps on m x m symmetric matrices, two products back to m x n
    return {"bytes": sum(22 * r * c for r, c in shapes),
            "flops": sum(6 * min(s) ** 2 * max(s) + 14 * min(s) ** 3 for s in shapes)}


# ---- inputs ------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=g, device=DEV) * std

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device=DEV)

    s = {"case": case}
    if case["op"] == "logprobs":
        r, n, k = case["rows"], case["classes"], case["ids"]
        x = normal(r, n, std=2.5)
        if case["masked"]:  # excluded classes; the first of every 64 rows but row 0 has nothing left
            x = torch.where(uniform(r, n) < 0.05, torch.full_like(x, -math.inf), x)
            x[64::64] = -math.inf
        s["logits"] = x.to(TYPES[case["dtype"]])
        del x
        s["ids"] = torch.randint(0, n, (r, k), generator=g, device=DEV, dtype=torch.int32)
        if r > 1:
            s["ids"][uniform(r, k) < 0.1] = PAD
        f32 = {"dtype": torch.float32, "device": DEV}
        s["logprob"], s["lse"], s["entropy"] = torch.empty(r, k, **f32), torch.empty(r, **f32), torch.empty(r, **f32)
        s["top_id"] = torch.empty(r, case["top"], dtype=torch.int32, device=DEV)
        s["top_logprob"] = torch.empty(r, case["top"], **f32)
        if case["train"]:
            s["d_logprob"] = normal(r, k, std=1.0 / r) - 1.0 / r
            s["d_entropy"] = normal(r, std=0.01 / r)
            s["d_logits"] = torch.empty(r, n, dtype=TYPES[case["dtype"]], device=DEV)
    elif case["op"] == "q4":
        b, i, o, group = case["batch"], case["in"], case["out"], case["group"]
        s["x"] = normal(b, i).abs().to(TYPES[case["dtype"]])
        s["bias"] = normal(o, std=0.1)
        tiles, blocks = -(-o // 16), -(-i // 128)
        w = normal(tiles * 16, blocks * 128, std=math.sqrt(2.0 / i))
        w[o:] = 0
        w[:, i:] = 0
        w = w.view(tiles * 16, -1, group)
        scale = (w.abs().amax(2, keepdim=True) / 7).to(torch.bfloat16)
        q = torch.where(scale > 0, (w / scale.float()).round().clamp(-8, 7), torch.zeros_like(w)) + 8
        q = q.to(torch.uint8).view(tiles, 16, blocks, 4, 4, 8)                  # tile, row, block, u, t, j: k = 32 u + 8 t + j
        q = q.permute(0, 2, 1, 4, 3, 5).reshape(tiles, blocks, 16, 64, 2)       # tile, block, row, (t, u, j / 2), low and high
        s["codes"] = (q[..., 0] | (q[..., 1] << 4)).contiguous()
        s["scales"] = scale.view(tiles, 16, blocks, 128 // group).permute(0, 2, 1, 3).contiguous()
        s["y"] = torch.empty(b, o, dtype=TYPES[case["dtype"]], device=DEV)
    else:
        s["tensors"] = []
        for rows, cols in shapes_of(case):
            # a gradient of a batch of 100: a hundred strong directions over a weaker rest
            k = min(100, rows, cols)
            grad = normal(rows, k, std=1e-2) @ normal(k, cols, std=1e-2) + normal(rows, cols, std=1e-4)
            w = normal(rows, cols, std=math.sqrt(2.0 / cols))
            s["tensors"].append({"w": w, "w16": w.to(torch.bfloat16), "grad": grad, "momentum": normal(rows, cols, std=1e-3)})
        s["lr"], s["mu"], s["steps"] = 0.02, 0.95, 5
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    import paper_1810_09868_b200 as p
    case, stream = s["case"], torch.cuda.current_stream()
    if case["op"] == "logprobs":
        p.vgg19_logprobs(s["logits"], s["ids"], s["logprob"], s["lse"], s["entropy"], s["top_id"], s["top_logprob"], stream=stream)
        if not case["train"]:
            return {n: s[n] for n in ("logprob", "lse", "entropy", "top_id", "top_logprob")}
        p.vgg19_logprobs_backward(s["logits"], s["ids"], s["lse"], s["entropy"], s["d_logprob"], s["d_entropy"], s["d_logits"],
                                  stream=stream)
        return {n: s[n] for n in ("logprob", "lse", "entropy", "d_logits")}
    if case["op"] == "q4":
        p.vgg19_q4_linear(s["x"], s["codes"], s["scales"], case["out"], case["group"], s["bias"], case["relu"], s["y"],
                          stream=stream)
        return s["y"]
    if "table" not in s:  # what a program keeps: the list of its tensors and the workspace
        s["table"] = p.vgg19_muon_tensors([(t["w"], t["w16"], t["grad"], t["momentum"]) for t in s["tensors"]])
        s["workspace"] = torch.empty(p.vgg19_muon_workspace_bytes(s["table"]), dtype=torch.uint8, device=DEV)
    p.vgg19_muon_update(s["table"], s["lr"], s["mu"], case["decay"], s["steps"], case["nesterov"], s["workspace"], stream=stream)
    return [{n: t[n] for n in ("w", "w16", "momentum")} for t in s["tensors"]]


def run_plain(s):
    case = s["case"]
    if case["op"] == "logprobs":
        return plain_logprobs(s)
    if case["op"] == "q4":
        q = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).float() - 8
        tiles, blocks = q.shape[:2]
        w = q.view(tiles, blocks, 16, 4, 4, 8).permute(0, 2, 1, 4, 3, 5).reshape(tiles * 16, -1, case["group"])
        w = w * s["scales"].float().permute(0, 2, 1, 3).reshape(tiles * 16, -1, 1)
        y = s["x"].float() @ w.view(tiles * 16, -1)[: case["out"], : case["in"]].T + s["bias"]
        return (y.clamp_min(0) if case["relu"] else y).to(s["y"].dtype)
    for t in s["tensors"]:
        w, grad, m = t["w"], t["grad"], t["momentum"]
        m.mul_(s["mu"]).add_(grad)
        x = grad + s["mu"] * m if case["nesterov"] else m.clone()
        norm = x.double().square().sum().sqrt()
        x = torch.where(norm > 0, x / norm.float(), torch.zeros_like(x))
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        for _ in range(s["steps"]):
            a = x @ x.T
            x = NS[0] * x + (NS[1] * a + NS[2] * (a @ a)) @ x
        x = x.T if tall else x
        w.mul_(1 - s["lr"] * case["decay"]).sub_(s["lr"] * math.sqrt(max(1.0, w.shape[0] / w.shape[1])) * x)
        t["w16"].copy_(w)
    return [{n: t[n] for n in ("w", "w16", "momentum")} for t in s["tensors"]]


def plain_logprobs(s):
    case = s["case"]
    x = s["logits"].float()
    n, ids = case["classes"], s["ids"].long()
    top = x.amax(1, keepdim=True)
    alive = top > -math.inf  # whether the row has a class left
    e = torch.exp(torch.where(alive, x - top, torch.zeros_like(x)))
    lse = torch.where(alive, top + torch.log(e.sum(1, keepdim=True)), top)
    logp = torch.where(alive, x - lse, x)  # a row with nothing left keeps -inf
    p = torch.exp(logp)
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    entropy = -plogp.sum(1, keepdim=True)
    given = torch.where(ids == PAD, torch.zeros_like(s["logprob"]), torch.gather(logp, 1, ids.clamp_min(0)))
    out = {"logprob": given, "lse": lse[:, 0], "entropy": entropy[:, 0]}
    if case["train"]:
        d = torch.where(ids == PAD, torch.zeros_like(given), s["d_logprob"])
        grad = -p * d.sum(1, keepdim=True) - s["d_entropy"][:, None] * (plogp + p * entropy)
        grad.scatter_add_(1, ids.clamp_min(0), torch.where(alive, d, torch.zeros_like(d)))
        out["d_logits"] = grad.to(s["logits"].dtype)
        return out
    # the largest first, the lower index first among equals: one whole number per class that orders them so
    bits = (x + 0.0).view(torch.int32).long()
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) | (n - 1 - torch.arange(n, device=x.device))
    key = torch.topk(key, case["top"], 1).values
    top_id = n - 1 - (key & 0xFFFFFFFF)
    top_logprob = torch.gather(logp, 1, top_id)
    out["top_id"] = torch.where(top_logprob > -math.inf, top_id, torch.full_like(top_id, -1)).int()
    out["top_logprob"] = top_logprob
    return out


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "logprobs":
        out = {n: [] for n in ("logprob", "lse", "entropy", "top_logprob", "d_logits")}
        step = max(1, 20_000_000 // case["classes"])
        for a in range(0, case["rows"], step):
            z = s["logits"][a:a + step].double()
            ids = s["ids"][a:a + step].long()
            lse = torch.logsumexp(z, 1)
            empty = torch.isinf(lse)
            logp = torch.log_softmax(z, 1)
            logp[empty] = -math.inf
            h = -torch.special.xlogy(logp.exp(), logp.exp()).sum(1)
            pad = ids < 0
            out["logprob"].append(logp.gather(1, ids.masked_fill(pad, 0)).masked_fill(pad, 0.0))
            out["lse"].append(lse)
            out["entropy"].append(h)
            if case["train"]:
                # d/dz of sum_i g_i log p[id_i] + w H: p is softmax(z)
                p = logp.exp()
                g = torch.zeros_like(z).scatter_add_(1, ids.masked_fill(pad, 0), s["d_logprob"][a:a + step].double().masked_fill(pad, 0.0))
                g[empty] = 0
                dh = -p * (logp.masked_fill(torch.isinf(logp), 0.0) + h[:, None])
                out["d_logits"].append(g - p * g.sum(1, keepdim=True) + s["d_entropy"][a:a + step].double()[:, None] * dh)
            else:
                out["top_logprob"].append(logp.topk(case["top"], 1).values)
        got = {n: torch.cat(v) for n, v in out.items() if v}
        if not case["train"]:
            got["top_id"] = None
        return got
    if case["op"] == "q4":
        # element k of a row: block k / 128; within it word 4 t + u, nibble j, with k % 128 = 32 u + 8 t + j
        k = torch.arange(case["in"], device=DEV)
        row = torch.arange(case["out"], device=DEV)[:, None]
        inside = k % 128
        byte = (inside // 8 % 4 * 4 + inside // 32) * 4 + inside % 8 // 2
        code = s["codes"][row // 16, k // 128, row % 16, byte].to(torch.int64) >> (4 * (inside % 2))
        w = ((code & 15) - 8).double() * s["scales"][row // 16, k // 128, row % 16, inside // case["group"]].double()
        y = torch.einsum("bk,ok->bo", s["x"].double(), w) + s["bias"].double()
        return torch.relu(y) if case["relu"] else y
    out = []
    for t in s["tensors"]:
        grad = t["grad"].double()
        m = s["mu"] * t["momentum"].double() + grad
        u = grad + s["mu"] * m if case["nesterov"] else m
        x = u / torch.linalg.matrix_norm(u)
        for _ in range(s["steps"]):
            gram = x @ x.mT if x.shape[0] <= x.shape[1] else x.mT @ x
            poly = NS[1] * gram + NS[2] * gram @ gram
            x = NS[0] * x + (poly @ x if x.shape[0] <= x.shape[1] else x @ poly)
        w = t["w"].double() * (1 - s["lr"] * case["decay"]) - s["lr"] * max(1.0, x.shape[0] / x.shape[1]) ** 0.5 * x
        out.append({"w": w, "w16": w, "momentum": m})
    return out
