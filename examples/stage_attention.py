"""One pipeline stage's attention sublayer, as it answers and as it trains.

    python examples/stage_attention.py [--tokens 16] [--fp4]

Serving: coordinates arrive, are decompressed, give queries, keys and values;
``kv_append`` norms and rotates them and files keys and values in a paged cache,
``paged_attention`` reads it, the reparameterized output projection adds to the
residual stream, and the coordinates of the result leave.  Prompts go through in
chunks, then every sequence advances a token at a time.  With --fp4 the cache holds
4 bits an element (``kv_append_fp4``, ``paged_attention_fp4``); ``move`` takes a
sequence of it to another cache (``kv_read_fp4``).

Training: ``qk_norm_rope`` and its backward as a torch autograd function.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_13332_amd import ssn  # noqa: E402

DEV = "cuda:0"


class Stage:
    """Random weights of one layer's attention: d wide, rank k, Hq query heads
    over Hk key heads of D."""

    def __init__(self, d=1024, k=64, Hq=10, Hk=2, D=128, V=1000, max_len=2048, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rand = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.Hq, self.Hk, self.D, self.max_len = Hq, Hk, D, max_len
        self.U = torch.linalg.qr(rand(d, k).cpu())[0].to(DEV).bfloat16().contiguous()
        self.E = (0.02 * rand(V, d)).bfloat16()
        self.wqkv = (rand(d, (Hq + 2 * Hk) * D) / d ** 0.5).bfloat16()
        self.wq, self.wk = ((1 + 0.1 * rand(D)).bfloat16() for _ in range(2))
        self.Zp = (rand(Hq * D, k) / (Hq * D) ** 0.5).bfloat16()
        self.table = ssn.rope_table(max_len, D, 5e5, device=DEV)

    def heads(self, X):
        qkv = torch.nn.functional.rms_norm(X, X.shape[-1:]) @ self.wqkv
        return qkv.view(X.shape[0], self.Hq + 2 * self.Hk, self.D).split([self.Hq, self.Hk, self.Hk], 1)

    def serve(self, Z, ids, cache, batch):
        """Coordinates of a batch's new tokens in, coordinates out."""
        X = ssn.decompress(Z, ids, self.E, self.U)
        q, k, v = self.heads(X)
        pages, starts, lens, max_q, max_len = batch
        append, attention, workspace = ssn.kv_append, ssn.paged_attention, ssn.paged_attention_workspace
        if len(cache) == 4:            # codes and scales of keys and of values
            append, attention, workspace = ssn.kv_append_fp4, ssn.paged_attention_fp4, ssn.paged_attention_fp4_workspace
        q = append(k, v, *cache, pages, starts, lens, Q=q, table=self.table, wq=self.wq, wk=self.wk)
        ws = workspace(X.shape[0], pages.shape[0], self.Hq, self.Hk, self.D, max_q, max_len, DEV)
        O = attention(q, *cache, pages, starts, lens, max_q, max_len, workspace=ws)
        _, Y = ssn.reparam_forward(O.view(X.shape[0], -1), self.Zp, self.U)
        return ssn.compress(X + Y, ids, self.E, self.U)


class Pages:
    """Pages of one layer's cache, handed out as sequences grow."""

    def __init__(self, stage, npages, size, B, fp4=False):
        shape = (npages, stage.Hk, size, stage.D)
        if fp4:
            self.cache = [*ssn.fp4_cache(*shape, DEV), *ssn.fp4_cache(*shape, DEV)]
        else:
            self.cache = [torch.empty(shape, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        self.size, self.free = size, list(range(npages))
        self.lens = [0] * B
        self.table = [[] for _ in range(B)]
        self.width = -(-stage.max_len // size)

    def batch(self, new):
        """The device arrays for `new[b]` tokens more of every sequence."""
        for b, n in enumerate(new):
            self.lens[b] += n
            while len(self.table[b]) * self.size < self.lens[b]:
                self.table[b].append(self.free.pop())
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        pages = [row + [-1] * (self.width - len(row)) for row in self.table]
        return i32(pages), i32(starts), i32(self.lens), max(new), max(self.lens)


class QKNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, pos, table):
        ctx.save_for_backward(q, k, wq, wk, pos, table)
        return ssn.qk_norm_rope(q, k, pos, table, wq, wk)

    @staticmethod
    def backward(ctx, gq, gk):
        q, k, wq, wk, pos, table = ctx.saved_tensors
        gq, gk, gwq, gwk = ssn.qk_norm_rope_backward(q, k, gq.contiguous(), gk.contiguous(), pos, table, wq, wk)
        return gq, gk, gwq.to(wq.dtype), gwk.to(wk.dtype), None, None


def move(cache, pages, length, size):
    """A sequence of a 4-bit cache, its page numbers [1, width], into a cache of
    its own with pages of another size: read back, appended as it is.  Returns
    that cache and its page numbers."""
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    rows = (i32([0, length]), i32([length]))
    K, V = ssn.kv_read_fp4(*cache, pages, *rows, length)
    need = -(-length // size)
    shape = (need, K.shape[1], size, K.shape[2])
    other = [*ssn.fp4_cache(*shape, DEV), *ssn.fp4_cache(*shape, DEV)]
    numbers = i32([list(range(need))])
    ssn.kv_append_fp4(K, V, *other, numbers, *rows, eps=None)
    return other, numbers


def serve(tokens=16, prompts=(300, 41, 700), chunk=256, fp4=False):
    """Coordinates of each sequence's last token: fed in chunks and then token
    by token, and fed whole."""
    stage = Stage()
    g = torch.Generator(device=DEV).manual_seed(1)
    ids = [torch.randint(0, 1000, (n + tokens,), generator=g, device=DEV, dtype=torch.int32) for n in prompts]
    Z = [torch.randn((len(i), 64), generator=g, device=DEV) for i in ids]
    pages = Pages(stage, 200, 16, len(prompts), fp4)
    done = [0] * len(prompts)
    total = [len(i) for i in ids]
    out = [None] * len(prompts)
    while done != total:
        new = [min(chunk, n - d) if d < n else min(1, t - d) for d, n, t in zip(done, prompts, total)]
        rows = [slice(d, d + n) for d, n in zip(done, new)]
        batch = pages.batch(new)
        z = stage.serve(torch.cat([a[r] for a, r in zip(Z, rows)]), torch.cat([a[r] for a, r in zip(ids, rows)]),
                        pages.cache, batch)
        for b, part in enumerate(z.split(new)):
            if new[b]:
                out[b] = part[-1]
        done = [d + n for d, n in zip(done, new)]
    whole = Pages(stage, 200, 16, len(prompts), fp4)
    z = stage.serve(torch.cat(Z), torch.cat(ids), whole.cache, whole.batch(total))
    return torch.stack(out), torch.stack([part[-1] for part in z.split(total)])


def train():
    """A loss of the rotated queries and keys, and its gradients."""
    stage = Stage()
    X = torch.randn((64, 1024), device=DEV).bfloat16()
    pos = torch.arange(64, dtype=torch.int32, device=DEV)
    params = [t.clone().requires_grad_() for t in (stage.wqkv, stage.wq, stage.wk)]
    stage.wqkv = params[0]
    q, k, _ = stage.heads(X)
    q, k = QKNormRope.apply(q, k, params[1], params[2], pos, stage.table)
    # scores of each query head with its key head
    s = torch.einsum("ihd,jhd->hij", q.float(), k.float().repeat_interleave(stage.Hq // stage.Hk, 1))
    loss = torch.logsumexp(s / stage.D ** 0.5, -1).mean()
    loss.backward()
    return loss.item(), [p.grad.float().norm().item() for p in params]


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=16)
    ap.add_argument("--fp4", action="store_true", help="a cache of 4 bits an element")
    a = ap.parse_args()
    steps, whole = serve(a.tokens, fp4=a.fp4)
    print(f"serving: chunks and {a.tokens} single tokens against whole prompts: "
          f"rel {((steps - whole).norm() / whole.norm()).item():.2e}")
    if a.fp4:
        stored = serve(a.tokens)[1]
        print(f"serving: the 4-bit cache against the bf16 one: rel {((whole - stored).norm() / stored.norm()).item():.2e}")
    loss, norms = train()
    print(f"training: loss {loss:.4f}, gradient norms " + ", ".join(f"{n:.3e}" for n in norms))


if __name__ == "__main__":
    main()
