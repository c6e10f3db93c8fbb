"""Attention in one call, as measurable cases: m queries to k states, over all positions or those of a
sparse matrix, with a learned relative position bias by buckets, and the gradients of both.

  forward   O and the logarithm of each row's sum: a decoder's queries to an encoder's states of another
            length, or sparse self-attention with a position bias
  token     the same for one query or a few of each sequence (a decoding step), where reading K and V is the cost
  train     forward, then backward: gradients of Q, K, V and, with a bias, of the bias table

Every head of query i of sequence b sees state j where j < lengths[b] and, with a mask, where the sparse matrix stores (i, j):

  s_ij = scale Q_i . K_j + table[head, bucket_of[span + clamp(j - i - positions[b], -span, span)]]
  P_ij = exp(s_ij - lse_i),  lse_i = log sum_j exp(s_ij),  O_i = sum_j P_ij V_j     (rows that see nothing: O = 0, lse = -inf)

Consecutive groups of heads / kv_heads query heads share a head of K and V.  The sequence of 4096 with a band of 256 and scattered entries at
10 % and its eight heads of 64 are those of workloads.py; the sequence of 12288 with heads of 128, a band of 256 and 95 % sparsity
beside it are the sparse Transformer's of the paper.  The other sizes are generic.
"""
import math

import torch

own = False


def _case(op, dtype, batch, heads, kv_heads, m, k, d, ragged=False, mask="none", density=1.0, buckets=0, distance=0, both=True):
    """ragged: sequences of unequal length.  buckets, distance: the bias table's and how far its buckets tell positions apart;
    both: whether they tell states before a query from those behind it."""
    return {"op": op, "dtype": dtype, "batch": batch, "heads": heads, "kv_heads": kv_heads, "m": m, "k": k, "d": d, "ragged": ragged,
            "mask": mask, "density": density, "buckets": buckets, "distance": distance, "both": both}


def listed():
    return [
        # one token of one sequence: launches and latency are the cost
        dict(_case("token", "f16", 1, 8, 8, 1, 512, 64), name="token_small"),
        # one token of each of 32 sequences over a long cache of unequal lengths, four query heads to a head of the cache
        dict(_case("token", "f16", 32, 32, 8, 1, 8192, 128, ragged=True), name="token_long"),
        # one token of a self-attention with a position bias, in single precision
        dict(_case("token", "f32", 16, 8, 8, 1, 2048, 64, ragged=True, buckets=32, distance=128, both=False), name="token_bias_f32"),
        # a short target and a short source, sizes that are multiples of nothing
        dict(_case("forward", "f32", 2, 8, 8, 37, 203, 64, ragged=True), name="cross_small_f32"),
        # targets of 512 to sources of up to 2048: an encoder-decoder's forward
        dict(_case("forward", "f16", 8, 16, 16, 512, 2048, 64, ragged=True), name="cross_forward"),
        # long target, longer source, heads of 128, four query heads to one of the source
        dict(_case("forward", "f16", 1, 16, 4, 4096, 8192, 128), name="cross_long"),
        # sparse self-attention: sequence 4096, eight heads of 64, band and scatter at 10 %, with a position bias
        dict(_case("forward", "f32", 1, 8, 8, 4096, 4096, 64, mask="banded", density=0.10, buckets=32, distance=128), name="sparse_forward_f32"),
        # the sparse Transformer's layer: sequence 12288, eight heads of 128
        dict(_case("forward", "f16", 1, 8, 8, 12288, 12288, 128, mask="banded", density=0.07, buckets=32, distance=128), name="sparse_long"),
        # training steps: of the cross attention above, of an encoder's self-attention with a position bias, of the sparse layer, and of
        # a small layer whose sizes are multiples of nothing
        dict(_case("train", "f16", 8, 16, 16, 512, 2048, 64, ragged=True), name="cross_train"),
        dict(_case("train", "f16", 4, 8, 8, 2048, 2048, 64, buckets=32, distance=128), name="bias_train"),
        dict(_case("train", "f32", 1, 8, 8, 4096, 4096, 64, mask="banded", density=0.10, buckets=32, distance=128), name="sparse_train_f32"),
        dict(_case("train", "f32", 3, 6, 2, 77, 203, 40, ragged=True, buckets=32, distance=128), name="small_train_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng, most):
    """(heads, kv_heads, d): heads of their own or shared by two, four or eight."""
    group = rng.choice([1, 1, 2, 4, 8])
    kv = max(1, _log(rng, 1, most) // group)
    return kv * group, kv, rng.choice([32, 40, 64, 64, 64, 80, 96, 128, 128])


def _bias(rng):
    return dict(buckets=rng.choice([16, 32, 32, 64]), distance=rng.choice([64, 128, 128, 256]), both=rng.random() < 0.7) if rng.random() < 0.5 else {}


def draw(rng):
    kind = rng.choice(["token", "token", "token", "forward", "forward", "forward", "train", "train", "train"])
    dtype = rng.choice(["f16", "f16", "f32"])
    more = _bias(rng)
    if kind == "token":
        heads, kv, d = _heads(rng, 32)
        k = _log(rng, 100, 8192)
        room = 2 ** 28 // (kv * k * d * (2 if dtype == "f32" else 1))        # values of K: the largest listed token's
        return _case("token", dtype, min(64, _log(rng, 1, max(1, min(64, room)))), heads, kv, rng.choice([1, 1, 1, 2, 4, 7]), k, d, ragged=rng.random() < 0.6, **more)
    heads, kv, d = _heads(rng, 16)
    if rng.random() < 0.4:                               # sparse self-attention
        m = _log(rng, 300, 4096)
        density = round(min(0.9, math.exp(rng.uniform(math.log(0.05), math.log(0.2))) + 257.0 / m), 4)
        return _case(kind, dtype, 1, min(heads, 8), min(heads, 8), m, m, d, mask="banded", density=density, **more)
    m, k = _log(rng, 16, 2048), _log(rng, 50, 2048)
    room = 2 ** 27 // (m * k * heads)                    # positions of the largest listed training step
    return _case(kind, dtype, max(1, min(8, _log(rng, 1, max(1, room)))), heads, kv, m, k, d, ragged=rng.random() < 0.6, **more)


def _bucket_of(buckets, distance, both):
    """Bucket of each relative position -distance .. distance (state minus query): a bucket to each of the nearest, the others' widths
    growing in proportion.  In whole numbers: position n is in bucket exact + e, e the most with n / exact >= (distance / exact)^(e / steps)."""
    half = buckets // 2 if both else buckets
    exact = half // 2
    steps = half - exact

    def bucket(n):
        if n < exact:
            return n
        e = 0
        while e + 1 < steps and n ** steps * exact ** (e + 1) >= distance ** (e + 1) * exact ** steps:
            e += 1
        return exact + e
    return [(half if both and r > 0 else 0) + bucket(abs(r) if both else max(0, -r)) for r in range(-distance, distance + 1)]


def _topology(case, gen):
    """CSR offsets and ascending column indices of a band of 257 and entries beside it, more of them near it, int(density m k) in all."""
    m, k = case["m"], case["k"]
    i, j = torch.arange(m, device="cuda")[:, None], torch.arange(k, device="cuda")[None, :]
    far = (i - j).abs()
    keep = far <= 128
    free = max(0, int(case["density"] * m * k) - int(keep.sum()))
    weight = torch.where(keep, 0.0, 1.0 / far.clamp(min=1).float())
    p = weight * (free / max(1e-30, float(weight.sum())))
    for _ in range(6):
        p = (p * (free / max(1e-30, float(p.sum())))).clamp(max=1.0)
    keep |= torch.rand((m, k), generator=gen, device="cuda") < p
    ro = torch.zeros(m + 1, dtype=torch.int32, device="cuda")
    ro[1:] = torch.cumsum(keep.sum(dim=1, dtype=torch.int32), 0)
    return ro, torch.nonzero(keep)[:, 1].to(torch.int32)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    b, h, kv, m, k, d = (case[x] for x in ("batch", "heads", "kv_heads", "m", "k", "d"))
    dt = torch.float16 if case["dtype"] == "f16" else torch.float32

    def heads_of(n, rows):
        """As a projection leaves them, [batch, rows, heads, d]; a cache keeps a head's rows together."""
        if case["op"] == "token" and rows == k:
            return torch.randn((b, n, rows, d), generator=gen, device="cuda").to(dt)
        return torch.randn((b, rows, n, d), generator=gen, device="cuda").to(dt).transpose(1, 2)

    s = {"op": case["op"], "scale": 1.0 / math.sqrt(d), "Q": heads_of(h, m), "K": heads_of(kv, k), "V": heads_of(kv, k),
         "lengths": None, "positions": None, "rows": None, "bucket_of": None, "table": None}
    if case["ragged"]:
        lengths = torch.randint(max(1, k // 4), k + 1, (b,), generator=gen, device="cuda", dtype=torch.int32)
        lengths[0] = k
        s["lengths"] = lengths
    if case["buckets"]:
        s["bucket_of"] = torch.tensor(_bucket_of(case["buckets"], case["distance"], case["both"]), dtype=torch.int32, device="cuda")
        s["table"] = torch.randn((h, case["buckets"]), generator=gen, device="cuda").to(dt)
        s["span"] = case["distance"]
        if case["op"] == "token":                        # the newest m positions of each sequence
            s["positions"] = (s["lengths"] if case["ragged"] else torch.full((b,), k, dtype=torch.int32, device="cuda")) - m
    if case["mask"] != "none":
        s["rows"] = _topology(case, gen)
    if case["op"] == "train":
        s["dO"] = heads_of(h, m)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2006_10901_amd as spdl
        m, k = case["m"], case["k"]
        s["f16"] = case["dtype"] == "f16"
        s["mask"] = None
        if s["rows"] is not None:
            s["mask"] = torch.empty(spdl.spdl_attention_mask_bytes(m, k), dtype=torch.uint8, device="cuda")
            spdl.spdl_build_attention_mask(m, k, s["rows"][1].numel(), *s["rows"], s["mask"])
        s["O"] = torch.empty_like(s["Q"])
        s["lse"] = torch.empty(s["Q"].shape[:3], dtype=torch.float32, device="cuda")
        for name in ("Q", "K", "V") if s["op"] == "train" else ():
            s["d" + name] = torch.empty_like(s[name])
        s["dtable"] = torch.empty_like(s["table"]) if s["op"] == "train" and s["table"] is not None else None
        s["problem"] = spdl.attention_problem(s["Q"], s["K"], s["V"], s["O"], s["scale"], bucket_of=s["bucket_of"], table=s["table"],
                                              dO=s.get("dO"), dQ=s.get("dQ"), dK=s.get("dK"), dV=s.get("dV"))
        s["workspace"] = torch.empty(spdl.spdl_attention_workspace(s["problem"], 2 if s["f16"] else 4, s["op"] == "train"), dtype=torch.uint8, device="cuda")
    return s


def _run_own(s):
    import paper_2006_10901_amd as spdl
    forward, backward = ((spdl.spdl_attention_f16, spdl.spdl_attention_backward_f16) if s["f16"] else
                         (spdl.spdl_attention, spdl.spdl_attention_backward))
    forward(s["problem"], s["Q"], s["K"], s["V"], s["lengths"], s["positions"], s["mask"], s["bucket_of"], s["table"], s["O"], s["lse"],
            s["workspace"])
    if s["op"] != "train":
        return {"O": s["O"], "lse": s["lse"]}
    backward(s["problem"], s["Q"], s["K"], s["V"], s["lengths"], s["positions"], s["mask"], s["bucket_of"], s["table"], s["O"], s["lse"],
             s["dO"], s["dQ"], s["dK"], s["dV"], s["dtable"], s["workspace"])
    out = {"O": s["O"], "lse": s["lse"], "dQ": s["dQ"], "dK": s["dK"], "dV": s["dV"]}
    if s["dtable"] is not None:
        out["dtable"] = s["dtable"]
    return out


def run(s):
    if own:
        return _run_own(s)
    Q, K, V, scale = s["Q"], s["K"], s["V"], s["scale"]
    (b, h, m, d), (_, kv, k, _) = Q.shape, K.shape
    dt, dev = Q.dtype, Q.device
    q = Q.float().reshape(b, kv, h // kv * m, d)          # the query heads that share a head of K and V, one below the other
    kt = K.float().transpose(-1, -2).contiguous()
    v = V.float().contiguous()
    x = torch.matmul(q, kt).reshape(b, h, m, k).mul_(scale)
    if s["table"] is not None:
        rel = torch.arange(k, device=dev)[None, None, :] - torch.arange(m, device=dev)[None, :, None]
        if s["positions"] is not None:
            rel = rel - s["positions"].long()[:, None, None]
        bucket = s["bucket_of"].long()[rel.clamp(-s["span"], s["span"]) + s["span"]]     # [1 or b, m, k]
        x += s["table"].float()[:, bucket].transpose(0, 1)
    if s["lengths"] is not None:
        x.masked_fill_(torch.arange(k, device=dev) >= s["lengths"].long()[:, None, None, None], -math.inf)
    if s["rows"] is not None:
        ro, ci = s["rows"]
        seen = torch.zeros((m, k), dtype=torch.bool, device=dev)
        seen[torch.repeat_interleave(torch.arange(m, device=dev), (ro[1:] - ro[:-1]).long()), ci.long()] = True
        x.masked_fill_(~seen, -math.inf)
    most = x.amax(dim=-1, keepdim=True)
    most = torch.where(most == -math.inf, 0.0, most)      # rows that see nothing
    x = x.sub_(most).exp_()
    total = x.sum(dim=-1, keepdim=True)
    lse = (most + total.log())[..., 0]
    P = x.div_(torch.where(total == 0, 1.0, total))
    O = torch.matmul(P.reshape(b, kv, -1, k), v).reshape(b, h, m, d)
    if s["op"] != "train":
        return {"O": O.to(dt), "lse": lse}
    dO = s["dO"].float()
    delta = (dO * O).sum(dim=-1, keepdim=True)
    do = dO.reshape(b, kv, -1, d)
    dV = torch.matmul(P.reshape(b, kv, -1, k).transpose(-1, -2).contiguous(), do)
    dS = torch.matmul(do, v.transpose(-1, -2).contiguous()).reshape(b, h, m, k).sub_(delta).mul_(P)
    ds = dS.reshape(b, kv, -1, k)
    dQ = torch.matmul(ds, K.float().contiguous()).reshape(b, h, m, d) * scale
    dK = torch.matmul(ds.transpose(-1, -2).contiguous(), q) * scale
    out = {"O": O.to(dt), "lse": lse, "dQ": dQ.to(dt), "dK": dK.to(dt), "dV": dV.to(dt)}
    if s["table"] is not None:
        # sums of up to millions of terms of either sign, in 64 bits: first over the positions of one distance, which a row that
        # is one element longer than the next puts into one column, then over a bucket's
        skewed = torch.nn.functional.pad(dS.sum(dim=0).flip(1), (0, m)).reshape(h, -1)[:, :m * (m + k - 1)].reshape(h, m, m + k - 1)
        sums = skewed.sum(dim=1, dtype=torch.float64)
        at = (torch.arange(m + k - 1, device=dev) - (m - 1)).clamp(-s["span"], s["span"]) + s["span"]
        dtable = torch.zeros(s["table"].shape, dtype=torch.float64, device=dev).index_add_(1, s["bucket_of"].long()[at], sums)
        out["dtable"] = dtable.to(dt)
    return out


def _pairs(case):
    """Positions that a head of every sequence sees, in the mean."""
    seen = case["density"] if case["mask"] != "none" else 1.0
    share = (1 + (case["batch"] - 1) * 0.625) / case["batch"] if case["ragged"] else 1.0     # lengths from a quarter of k to all of it
    return case["batch"] * case["m"] * case["k"] * seen * share, share


def work(case):
    pairs, share = _pairs(case)
    size = 2 if case["dtype"] == "f16" else 4
    q = case["batch"] * case["heads"] * case["m"] * case["d"] * size
    kv = 2 * case["batch"] * case["kv_heads"] * case["k"] * case["d"] * size * share
    lse = case["batch"] * case["heads"] * case["m"] * 4
    extra = (case["m"] * case["k"] / 8 if case["mask"] != "none" else 0) + case["heads"] * case["buckets"] * size
    products = 2.0 * pairs * case["heads"] * case["d"]    # operations of one of the products of Q, K, P, V and their gradients
    if case["op"] != "train":
        return {"bytes": 2 * q + kv + lse + extra, "flops": 2 * products}
    # two products forward; backward the scores again and four gradients.  Q, K, V, dO read, O, lse and the three gradients written
    return {"bytes": 4 * q + 2 * kv + lse + 2 * extra, "flops": 7 * products}


def exact(case, seed):
    s = _inputs(case, seed)
    Q, K, V = s["Q"], s["K"], s["V"]
    (b, h, m, d), (_, kv, k, _) = Q.shape, K.shape
    if 14.0 * b * h * m * k * d > 2e13:                  # some 20 seconds
        return None
    dev, f64 = Q.device, torch.float64
    train = s["op"] == "train"
    out = {"O": torch.zeros((b, h, m, d), dtype=f64, device=dev), "lse": torch.zeros((b, h, m), dtype=f64, device=dev)}
    if train:
        out.update(dQ=torch.zeros((b, h, m, d), dtype=f64, device=dev), dK=torch.zeros((b, kv, k, d), dtype=f64, device=dev),
                   dV=torch.zeros((b, kv, k, d), dtype=f64, device=dev))
        if s["table"] is not None:
            out["dtable"] = torch.zeros(s["table"].shape, dtype=f64, device=dev)
    stored = None
    if s["rows"] is not None:
        offsets, columns = (t.cpu().tolist() for t in s["rows"])
        stored = torch.zeros((m, k), dtype=torch.bool)
        for i in range(m):
            stored[i, columns[offsets[i]:offsets[i + 1]]] = True
        stored = stored.to(dev)
    for c in range(b):
        n = k if s["lengths"] is None else int(s["lengths"][c])
        if s["table"] is not None:
            first = 0 if s["positions"] is None else int(s["positions"][c])
            far = torch.arange(n, device=dev).view(1, n) - (torch.arange(m, device=dev).view(m, 1) + first)
            where = s["bucket_of"].long()[torch.clamp(far, min=-s["span"], max=s["span"]) + s["span"]]
        for e in range(h):
            g = e * kv // h
            q, kk, v = Q[c, e].to(f64), K[c, g, :n].to(f64), V[c, g, :n].to(f64)
            logits = s["scale"] * (q @ kk.T)
            if s["table"] is not None:
                logits = logits + s["table"][e].to(f64)[where]
            if stored is not None:
                logits = torch.where(stored[:, :n], logits, -math.inf)
            lse = torch.logsumexp(logits, dim=1)
            weights = torch.where(logits == -math.inf, 0.0, torch.exp(logits - lse[:, None]))
            out["lse"][c, e] = lse
            out["O"][c, e] = weights @ v
            if train:
                do = s["dO"][c, e].to(f64)
                slope = do @ v.T
                slope = weights * (slope - (weights * slope).sum(dim=1, keepdim=True))
                out["dV"][c, g, :n] += weights.T @ do
                out["dQ"][c, e] = s["scale"] * (slope @ kk)
                out["dK"][c, g, :n] += s["scale"] * (slope.T @ q)
                if s["table"] is not None:
                    out["dtable"][e] += torch.bincount(where.reshape(-1), weights=slope.reshape(-1), minlength=case["buckets"])
    return out
