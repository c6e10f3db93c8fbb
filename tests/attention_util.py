"""Attention and its gradients in 64 bits, from the definition, with the scale of each result's error; and calls of the library
on the same inputs.

Tolerances (tol * S, those of gpu_util): S is the sum of the absolute values of what a result adds up.  Single precision: a score is a
sum of at most 128 products, off by (d + 2) 2^-24 sum |q k| scale, which for the inputs here is at most 5e-5 where P is not negligible;
P is then off by 1e-4 of itself.  Half precision adds roundings of at most 2^-11: of P and of the result (O, dV), of D = dO . O
through O, of dS and of the result (dQ, dK, dtable): at most 3 * 2^-11 + 1e-4 = 1.6e-3."""
import math

import numpy as np
import torch

import paper_2006_10901_amd as spdl
from tests.gpu_util import TOL_F16, TOL_F32, assert_close


def reference(Q, K, V, scale, lengths=None, positions=None, seen=None, bucket_of=None, table=None, dO=None):
    """Everything in float64 on the CPU: {name: (result, S)}."""
    f = lambda t: t.detach().cpu().double()
    Q, K, V = f(Q), f(K), f(V)
    (B, H, m, d), (_, G, k, _) = Q.shape, K.shape
    group = H // G
    zero = lambda *s: torch.zeros(s, dtype=torch.float64)
    out = {n: [zero(B, H, m, d), zero(B, H, m, d)] for n in ("O", "dQ")}
    out.update({n: [zero(B, G, k, d), zero(B, G, k, d)] for n in ("dK", "dV")})
    out["lse"] = [torch.full((B, H, m), -math.inf, dtype=torch.float64), torch.ones((B, H, m), dtype=torch.float64)]
    if table is not None:
        table, bucket_of = f(table), bucket_of.cpu().long()
        span = (bucket_of.numel() - 1) // 2
        out["dtable"] = [torch.zeros_like(table), torch.zeros_like(table)]
    for b in range(B):
        n = k if lengths is None else min(max(int(lengths[b]), 0), k)
        can = torch.ones((m, n), dtype=torch.bool) if seen is None else seen[:, :n].clone()
        if table is not None:
            rel = torch.arange(n)[None, :] - torch.arange(m)[:, None] - (0 if positions is None else int(positions[b]))
            bucket = bucket_of[rel.clamp(-span, span) + span]
        for h in range(H):
            g = h // group
            q, kk, v = Q[b, h], K[b, g, :n], V[b, g, :n]
            s = scale * (q @ kk.T)
            if table is not None:
                s = s + table[h][bucket]
            s = torch.where(can, s, -math.inf)
            lse = torch.logsumexp(s, dim=1) if n else torch.full((m,), -math.inf, dtype=torch.float64)
            P = torch.where(can, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            O = P @ v
            out["O"][0][b, h], out["O"][1][b, h] = O, P @ v.abs()
            out["lse"][0][b, h] = lse
            if dO is None:
                continue
            do = f(dO)[b, h]
            dP = do @ v.T
            D = (do * O).sum(1, keepdim=True)
            dS = torch.where(can, P * (dP - D), 0.0)
            S = P * (do.abs() @ v.abs().T + (do.abs() * O.abs()).sum(1, keepdim=True))
            out["dV"][0][b, g, :n] += P.T @ do
            out["dV"][1][b, g, :n] += P.T @ do.abs()
            out["dQ"][0][b, h], out["dQ"][1][b, h] = scale * (dS @ kk), abs(scale) * (S @ kk.abs())
            out["dK"][0][b, g, :n] += scale * (dS.T @ q)
            out["dK"][1][b, g, :n] += abs(scale) * (S.T @ q.abs())
            if table is not None and n:
                for to, x in ((0, dS), (1, S)):
                    out["dtable"][to][h].index_add_(0, bucket.reshape(-1), x.reshape(-1))
    return out


class Case:
    """Inputs of one attention, on the GPU."""

    def __init__(self, dtype="f32", batch=1, heads=2, kv_heads=None, m=8, k=8, d=64, scale=None, lengths=None, positions=None, mask=None,
                 buckets=0, span=16, both=True, layout="heads", seed=0, device="cuda"):
        self.f16 = dtype == "f16"
        self.dt = torch.float16 if self.f16 else torch.float32
        self.device = device
        kv = kv_heads or heads
        gen = torch.Generator().manual_seed(1000 + seed)
        self.scale = 1.0 / math.sqrt(d) if scale is None else scale

        def heads_of(n, rows):
            x = torch.randn((batch, n, rows, d), generator=gen)
            return self.place(x.to(self.dt), layout)

        self.Q, self.K, self.V, self.dO = heads_of(heads, m), heads_of(kv, k), heads_of(kv, k), heads_of(heads, m)
        self.layout = layout
        ints = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=device)
        self.lengths, self.positions = ints(lengths), ints(positions)
        self.bucket_of = self.table = None
        if buckets:
            # spans too short for the library's buckets: any bucket at each relative position
            of = (spdl.spdl_build_relative_buckets_host(buckets, span, both) if span > buckets // 2 else
                  np.random.default_rng(seed).integers(0, buckets, 2 * span + 1).astype(np.int32))
            self.bucket_of = torch.from_numpy(of).to(device)
            self.table = torch.randn((heads, buckets), generator=gen).to(self.dt).to(device)
        self.seen = self.mask = None
        if mask is not None:
            rng = np.random.default_rng(seed)
            self.seen = torch.from_numpy(mask(m, k, rng))
            self.mask = self.build_mask()
        if lengths is not None:                          # what lies behind a sequence's states is not read
            for b, n in enumerate(lengths):
                self.K[b, :, max(0, n):], self.V[b, :, max(0, n):] = float("nan"), float("nan")

    def place(self, x, layout):
        """x as the library may meet it: heads of their own, as a projection leaves them, or an element past a border of 16 bytes."""
        b, n, rows, d = x.shape
        if layout == "rows":
            return x.transpose(1, 2).contiguous().to(self.device).transpose(1, 2)
        if layout == "odd":
            room = torch.full((b * n * rows * (d + 3) + 1,), float("nan"), dtype=x.dtype, device=self.device)
            view = room[1:].view(b, n, rows, d + 3)[..., :d]
            view.copy_(x)
            return view
        return x.contiguous().to(self.device)

    def build_mask(self):
        m, k = self.seen.shape
        ro = torch.zeros(m + 1, dtype=torch.int32)
        ro[1:] = torch.cumsum(self.seen.sum(1), 0)
        ci = self.seen.nonzero()[:, 1].to(torch.int32)
        mask = torch.full((spdl.spdl_attention_mask_bytes(m, k),), 255, dtype=torch.uint8, device=self.device)
        spdl.spdl_build_attention_mask(m, k, ci.numel(), ro.to(self.device), ci.to(self.device), mask)
        return mask

    def output(self, like):
        return self.place(torch.full(like.shape, float("nan"), dtype=like.dtype), self.layout)

    def prepare(self, backward=True):
        self.O = self.output(self.Q)
        self.lse = torch.full(self.Q.shape[:3], float("nan"), device=self.device)
        self.dQ, self.dK, self.dV = (self.output(t) for t in (self.Q, self.K, self.V))
        self.dtable = None if self.table is None else torch.full_like(self.table, float("nan"))
        self.problem = spdl.attention_problem(self.Q, self.K, self.V, self.O, self.scale, bucket_of=self.bucket_of, table=self.table,
                                              dO=self.dO, dQ=self.dQ, dK=self.dK, dV=self.dV)
        n = spdl.spdl_attention_workspace(self.problem, 2 if self.f16 else 4, backward)
        self.workspace = torch.full((n,), 255, dtype=torch.uint8, device=self.device) if n else None
        return self

    def forward(self, stream=None):
        fn = spdl.spdl_attention_f16 if self.f16 else spdl.spdl_attention
        fn(self.problem, self.Q, self.K, self.V, self.lengths, self.positions, self.mask, self.bucket_of, self.table, self.O, self.lse,
           self.workspace, stream)

    def backward(self, stream=None):
        fn = spdl.spdl_attention_backward_f16 if self.f16 else spdl.spdl_attention_backward
        fn(self.problem, self.Q, self.K, self.V, self.lengths, self.positions, self.mask, self.bucket_of, self.table, self.O, self.lse,
           self.dO, self.dQ, self.dK, self.dV, self.dtable, self.workspace, stream)

    def results(self, backward=True):
        r = {"O": self.O, "lse": self.lse}
        if backward:
            r.update(dQ=self.dQ, dK=self.dK, dV=self.dV)
            if self.dtable is not None:
                r["dtable"] = self.dtable
        return r

    def check(self, backward=True, what=""):
        self.prepare(backward)
        self.forward()
        if backward:
            self.backward()
        torch.cuda.synchronize()
        ref = reference(self.Q, self.K, self.V, self.scale, self.lengths, self.positions, self.seen, self.bucket_of, self.table,
                        self.dO if backward else None)
        tol = TOL_F16 if self.f16 else TOL_F32
        for name, got in self.results(backward).items():
            want, S = ref[name]
            got, want, S = got.cpu().numpy(), want.numpy(), S.numpy()
            if name == "lse":
                none = np.isneginf(want)
                assert np.array_equal(none, np.isneginf(got)), f"{what} lse: which rows see nothing"
                err = np.abs(np.where(none, 0.0, got.astype(np.float64)) - np.where(none, 0.0, want))
                assert np.all(err <= 1e-4), f"{what} lse off by {np.nanmax(err) if err.size else 0}"
                continue
            assert_close(got, want, S, tol, f"{what} {name}")


def banded(m, k, rng):
    """A band beside the diagonal and scattered entries."""
    i, j = np.arange(m)[:, None], np.arange(k)[None, :]
    return (np.abs(i - j) <= 9) | (rng.random((m, k)) < 0.05)


def causal(m, k, rng):
    return np.arange(k)[None, :] <= np.arange(m)[:, None] + (k - m)


def blocks(m, k, rng):
    """Whole tiles empty, others full, and rows and columns that nothing sees."""
    s = np.repeat(np.repeat(rng.random((m // 64 + 1, k // 64 + 1)) < 0.4, 64, 0), 64, 1)[:m, :k].copy()
    s[m // 2] = False
    s[:, k // 2] = False
    return s


def nothing(m, k, rng):
    return np.zeros((m, k), dtype=bool)


def sparse_rows(m, k, rng):
    s = rng.random((m, k)) < 0.03
    s[::3] = False
    return s
