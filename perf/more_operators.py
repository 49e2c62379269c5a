"""Cases for the operators that train a classifier's head: dropout in front of its layers, and its last layer with the loss.

  dropout  dropout from a counter-based generator, whose mask is computed and never stored (vgg19_dropout), and with
           "train" the gradient, which computes the same mask again (vgg19_dropout_backward)
  loss     the last dense layer and the softmax cross entropy of its rows in one, over pieces of the classes, without
           keeping the logits (vgg19_linear_cross_entropy), and with "train" the gradients at the layer's input, weights and
           bias (vgg19_linear_cross_entropy_backward)

Each has its plain form here, in elementary torch operations, beside the calls a program makes of the library.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
NO_CLASS = -1  # the label of a row that only fills the batch
# Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011)
MULTIPLY, WEYL = (0xD2511F53, 0xCD9E8D57), (0x9E3779B9, 0xBB67AE85)


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # between the dense layers of a network in training: one batch of 100 images
        {"name": "dropout, one batch", "op": "dropout", "rows": 100, "cols": 4096, "pad": 0, "rate": 0.5, "dtype": "bf16", "train": True},
        # the features in front of the first dense layer, for many images
        {"name": "dropout, many features", "op": "dropout", "rows": 4096, "cols": 25088, "pad": 0, "rate": 0.5, "dtype": "bf16",
         "train": True},
        # rows of a wider buffer, sizes that divide nothing
        {"name": "dropout, odd rows", "op": "dropout", "rows": 1001, "cols": 4099, "pad": 13, "rate": 0.1, "dtype": "fp32", "train": True},
        # the score of one image's known class
        {"name": "loss of one image", "op": "loss", "rows": 1, "in": 4096, "classes": 1000, "pad": 0, "dtype": "bf16", "masked": False,
         "train": False},
        # a training step's last layer at 224 x 224, for a batch of 100, of a bf16 network and of an fp32 one
        {"name": "last layer, one batch", "op": "loss", "rows": 100, "in": 4096, "classes": 1000, "pad": 0, "dtype": "bf16",
         "masked": False, "train": True},
        {"name": "last layer, fp32", "op": "loss", "rows": 100, "in": 4096, "classes": 1000, "pad": 0, "dtype": "fp32",
         "masked": False, "train": True},
        # the same batch against a long list of classes: the weights are all there is to read
        {"name": "one batch, many classes", "op": "loss", "rows": 100, "in": 4096, "classes": 50021, "pad": 0, "dtype": "bf16",
         "masked": True, "train": True},
        # scoring many rows, no gradient
        {"name": "score many rows", "op": "loss", "rows": 2048, "in": 4096, "classes": 50021, "pad": 0, "dtype": "bf16", "masked": True,
         "train": False},
        # training on short rows, where the exponentials count against the products
        {"name": "train many rows", "op": "loss", "rows": 4096, "in": 1024, "classes": 32003, "pad": 0, "dtype": "bf16", "masked": False,
         "train": True},
        # fp32 rows and weights over a long list
        {"name": "train fp32 rows", "op": "loss", "rows": 512, "in": 1024, "classes": 32003, "pad": 0, "dtype": "fp32", "masked": True,
         "train": True},
        # sizes that divide nothing; rows of a wider buffer
        {"name": "odd sizes", "op": "loss", "rows": 1001, "in": 333, "classes": 2049, "pad": 5, "dtype": "bf16", "masked": True, "train": True},
        # the largest
        {"name": "train long rows", "op": "loss", "rows": 4096, "in": 4096, "classes": 131072, "pad": 0, "dtype": "bf16", "masked": False,
         "train": True},
    ]


def draw(rng):
    def log(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))

    dtype, pad, train = rng.choice(["fp32", "bf16", "bf16"]), rng.choice([0, 0, 0, 1, 8]), rng.random() < 0.7
    if rng.random() < 0.3:
        return {"op": "dropout", "rows": log(1, 4096), "cols": log(64, 25088 if dtype == "bf16" else 12544), "pad": pad,
                "rate": rng.choice([0.1, 0.5, round(rng.random(), 3)]), "dtype": dtype, "train": train}
    rows, inner = log(1, 4096), log(16, 4096)
    # fp32 products cost several times bf16's
    most = 131072 if dtype == "bf16" else max(1000, min(131072, 20_000_000_000 // (rows * inner)))
    return {"op": "loss", "rows": rows, "in": inner, "classes": log(32, most), "pad": pad, "dtype": dtype,
            "masked": rng.random() < 0.5, "train": train}


def work(case):
    elt = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"] * (2 if case["train"] else 1)
        # a block of ten rounds, of two products and four exclusive ors each, makes eight values
        return {"bytes": 2 * n * elt, "flops": n * (10 * 6 / 8 + 2)}
    r, i, n = case["rows"], case["in"], case["classes"]
    small = 4 * n + 12 * r  # bias; labels, loss and log-sum-exp
    if not case["train"]:
        return {"bytes": elt * (r * i + n * i) + small, "flops": 2 * r * n * i}
    return {"bytes": 2 * elt * (r * i + n * i) + small + 4 * n + 4 * r, "flops": 6 * r * n * i}


# ---- inputs ------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dtype = TYPES[case["dtype"]]

    def normal(rows, cols, std, pad=0):
        """Rows that lie `pad` values apart."""
        buffer = torch.empty(rows, cols + pad, dtype=dtype, device=DEV)
        return buffer.normal_(0.0, std, generator=g)[:, :cols]

    s = {"case": case}
    if case["op"] == "dropout":
        s["x"] = normal(case["rows"], case["cols"], 1.0, case["pad"])
        s["y"] = normal(case["rows"], case["cols"], 1.0, case["pad"])
        s["seed"], s["step"] = (seed * 0x9E3779B97F4A7C15 + 12345) % (1 << 64), 7
        if case["train"]:
            s["dy"] = normal(case["rows"], case["cols"], 1.0 / case["rows"], case["pad"])
            s["dx"] = normal(case["rows"], case["cols"], 1.0, case["pad"])
        return s
    r, i, n = case["rows"], case["in"], case["classes"]
    s["x"] = normal(r, i, 1.0, case["pad"])
    s["w"] = normal(n, i, 2.0 / math.sqrt(i), case["pad"])
    s["bias"] = torch.randn(n, generator=g, device=DEV) * 0.1
    s["labels"] = torch.randint(0, n, (r,), generator=g, device=DEV, dtype=torch.int32)
    if case["masked"]:  # classes that are left out: nothing is labelled with them
        out = torch.rand(n, generator=g, device=DEV) < 0.05
        out[s["labels"].long()] = False
        s["bias"][out] = -math.inf
    if r > 1:  # rows that only fill the batch
        s["labels"][torch.rand(r, generator=g, device=DEV) < 0.05] = NO_CLASS
    f32 = {"dtype": torch.float32, "device": DEV}
    s["loss"], s["lse"] = torch.empty(r, **f32), torch.empty(r, **f32)
    if case["train"]:
        s["d_loss"] = (0.5 + torch.rand(r, generator=g, device=DEV)) / r
        s["dx"] = torch.empty(r, i, dtype=dtype, device=DEV)
        s["dw"] = torch.empty(n, i, dtype=dtype, device=DEV)
        s["db"] = torch.empty(n, **f32)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def run(s):
    return (run_own if own else run_plain)(s)


def run_own(s):
    import paper_1810_09868_b200 as p
    case, stream = s["case"], torch.cuda.current_stream()
    if case["op"] == "dropout":
        p.vgg19_dropout(s["x"], s["y"], case["rate"], s["seed"], s["step"], stream=stream)
        if not case["train"]:
            return s["y"]
        p.vgg19_dropout_backward(s["dy"], s["dx"], case["rate"], s["seed"], s["step"], stream=stream)
        return {n: s[n] for n in ("y", "dx")}
    if "workspace" not in s:  # what a program keeps
        s["workspace"] = torch.empty(p.vgg19_linear_cross_entropy_bytes(s["x"], s["w"], case["train"]), dtype=torch.uint8, device=DEV)
    p.vgg19_linear_cross_entropy(s["x"], s["w"], s["bias"], s["labels"], s["loss"], s["lse"], s["workspace"], stream=stream)
    if not case["train"]:
        return {n: s[n] for n in ("loss", "lse")}
    p.vgg19_linear_cross_entropy_backward(s["x"], s["w"], s["bias"], s["labels"], s["lse"], s["d_loss"], s["dx"], s["dw"], s["db"],
                                          s["workspace"], stream=stream)
    return {n: s[n] for n in ("loss", "lse", "dx", "dw", "db")}


def run_plain(s):
    case = s["case"]
    if case["op"] == "dropout":
        keep, scale = plain_keep(case["rows"], case["cols"], case["rate"], s["seed"], s["step"])
        y = torch.where(keep, s["x"].float() * scale, 0.0).to(s["x"].dtype)
        if not case["train"]:
            return y
        keep, scale = plain_keep(case["rows"], case["cols"], case["rate"], s["seed"], s["step"])
        return {"y": y, "dx": torch.where(keep, s["dy"].float() * scale, 0.0).to(s["x"].dtype)}
    x, w = s["x"].float(), s["w"].float()
    labels = s["labels"].long()
    real = labels != NO_CLASS
    at = labels.clamp_min(0)[:, None]
    z = x @ w.T + s["bias"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    lse = top + torch.log(e.sum(1, keepdim=True))
    loss = torch.where(real, (lse - torch.gather(z, 1, at))[:, 0], 0.0)
    if not case["train"]:
        return {"loss": loss, "lse": lse[:, 0]}
    del e
    d = torch.exp(z - lse)  # the softmax, then the gradient at the logits
    del z
    d.scatter_add_(1, at, torch.full_like(lse, -1.0))
    d *= torch.where(real, s["d_loss"], 0.0)[:, None]
    return {"loss": loss, "lse": lse[:, 0], "dx": (d @ w).to(s["x"].dtype), "dw": (d.T @ x).to(s["x"].dtype), "db": d.sum(0)}


def plain_keep(rows, cols, rate, seed, step):
    """Which values stay, and what they are multiplied by.  Value e (row by row) takes 16 bits of block e / 8, a 64-bit
    counter beside the step's: bits of word (e % 8) / 2, the low half first."""
    low = 0xFFFFFFFF
    n = rows * cols
    block = torch.arange((n + 7) // 8, device=DEV)
    c = [block & low, block >> 32, torch.full_like(block, step & low), torch.full_like(block, step >> 32)]
    k = [seed & low, seed >> 32]
    for _ in range(10):
        a, b = c[0] * MULTIPLY[0], c[2] * MULTIPLY[1]  # (64-bit products, as bits)
        c = [(b >> 32 & low) ^ c[1] ^ k[0], b & low, (a >> 32 & low) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + WEYL[0]) & low, (k[1] + WEYL[1]) & low]
    words = torch.stack(c, 1)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:n].view(rows, cols)
    dropped = math.floor(rate * 65536 + 0.5)
    return halves >= dropped, 65536 / (65536 - dropped) if dropped < 65536 else 0.0


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        # the generator in numpy's unsigned arithmetic, on the host
        n = case["rows"] * case["cols"]
        index = np.arange(-(-n // 8), dtype=np.uint64)
        mask, half = np.uint64(0xFFFFFFFF), np.uint64(32)
        x0, x1 = index & mask, index >> half
        x2, x3 = np.uint64(s["step"] & 0xFFFFFFFF), np.uint64(s["step"] >> 32)
        for r in range(10):
            k0 = np.uint64(((s["seed"] & 0xFFFFFFFF) + r * WEYL[0]) & 0xFFFFFFFF)
            k1 = np.uint64(((s["seed"] >> 32) + r * WEYL[1]) & 0xFFFFFFFF)
            p, q = np.uint64(MULTIPLY[0]) * x0, np.uint64(MULTIPLY[1]) * x2
            x0, x1, x2, x3 = (q >> half) ^ x1 ^ k0, q & mask, (p >> half) ^ x3 ^ k1, p & mask
        bits = np.empty((index.size, 8), dtype=np.uint16)
        for j, v in enumerate(np.broadcast_arrays(x0, x1, x2, x3)):
            bits[:, 2 * j], bits[:, 2 * j + 1] = v & np.uint64(0xFFFF), v >> np.uint64(16)
        limit = int(case["rate"] * 65536 + 0.5)
        factor = torch.from_numpy(bits.reshape(-1)[:n].astype(np.int32)).to(DEV).view(case["rows"], case["cols"])
        factor = (factor >= limit).double() * (65536 / max(1, 65536 - limit))
        y = s["x"].double() * factor
        return {"y": y, "dx": s["dy"].double() * factor} if case["train"] else y
    w, bias = s["w"].double().requires_grad_(case["train"]), s["bias"].double().requires_grad_(case["train"])
    out = {"loss": [], "lse": [], "dx": []}
    step = max(1, 200_000_000 // case["classes"])
    for a in range(0, case["rows"], step):
        x = s["x"][a:a + step].double().requires_grad_(case["train"])
        z = torch.nn.functional.linear(x, w, bias)
        loss = torch.nn.functional.cross_entropy(z, s["labels"][a:a + step].long(), ignore_index=NO_CLASS, reduction="none")
        out["lse"].append(torch.logsumexp(z.detach(), 1))
        out["loss"].append(loss.detach())
        if case["train"]:
            loss.backward(s["d_loss"][a:a + step].double())
            out["dx"].append(x.grad)
        del x, z, loss
    got = {n: torch.cat(v) for n, v in out.items() if v}
    return {**got, "dw": w.grad, "db": bias.grad} if case["train"] else got
