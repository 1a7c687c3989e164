"""Several samples of one prompt from a small random decoder on the 4-bit paged cache: python examples/kv4_samples.py [--samples 4] [--tokens 48]

The prompt runs once.  Its pages are then shared by the samples (thi_kv4_fork), each sample's tokens go where the page table says
(thi_qk_norm_rope_kv4), attention reads all of it (thi_kv4_attention), and the pool is compacted now and then (thi_kv4_compact).  Tables, lengths and
counts of references stay on the device."""
from __future__ import annotations

import argparse
import os
import sys

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

EPS = 1e-5


class Decoder:
    """Random weights of a few layers, and the pool of pages they share the numbering of."""

    def __init__(self, seed=0, layers=2, hidden=512, inter=1024, Hq=8, Hkv=4, D=64, vocab=1000, pages=64):
        import torch
        import paper_2605_25655_amd as thi
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(n, k):
            return (torch.randn(n, k, device="cuda", generator=g) * k ** -0.5).half()

        self.thi, self.torch, self.hidden, self.inter, self.Hq, self.Hkv, self.D, self.vocab = thi, torch, hidden, inter, Hq, Hkv, D, vocab
        ones = torch.ones(max(hidden, D), device="cuda").half()
        self.gamma, self.head_gamma = ones[:hidden], ones[:D]
        self.layers = [dict(qkv=w((Hq + 2 * Hkv) * D, hidden), o=w(hidden, Hq * D), gate=w(inter, hidden), up=w(inter, hidden), down=w(hidden, inter)) for _ in range(layers)]
        self.embedding, self.head = torch.randn(vocab, hidden, device="cuda", generator=g).half(), w(vocab, hidden)
        self.theta = torch.tensor([10000.0 ** (-2 * i / D) for i in range(D // 2)], device="cuda")
        self.pool = torch.zeros(layers, pages, Hkv, 68 * D, dtype=torch.uint8, device="cuda")
        self._ws = {}

    def empty(self, *shape):
        return self.torch.empty(*shape, dtype=self.torch.float16, device="cuda")

    def ints(self, x):
        return self.torch.as_tensor(x, dtype=self.torch.int32).cuda()

    def workspace(self, name, nbytes, init):
        if name not in self._ws or self._ws[name].nbytes < nbytes:
            self._ws[name] = self.thi.Workspace(nbytes, init=init)
        return self._ws[name]

    def step(self, tokens, table, lens, new):
        """Logits of each row's last token: `new` tokens of every row of the table, which end at its length `lens`."""
        torch, thi = self.torch, self.thi
        B, MP = table.shape
        T, N = B * new, (self.Hq + 2 * self.Hkv) * self.D
        positions = lens[:, None] - new + torch.arange(new, dtype=torch.int32, device="cuda")
        page = table.gather(1, positions.long() // thi.THI_KV4_PAGE)
        slots = torch.where(page >= 0, page * thi.THI_KV4_PAGE + positions % thi.THI_KV4_PAGE, -1).int().flatten()
        positions, offsets = positions.flatten(), None if new == 1 else torch.arange(0, T + 1, new, dtype=torch.int32, device="cuda")
        sizes = [thi.thi_workspace_bytes(0, T, N, self.hidden), thi.thi_workspace_bytes(1, T, max(self.hidden, self.vocab), max(self.hidden, self.Hq * self.D)),
                 thi.thi_workspace_bytes(2, T, self.hidden, self.inter)]
        ws = self.workspace("layers", max(sizes), True)
        wa = self.workspace("attention", thi.thi_kv4_attention_workspace_bytes(B, T, self.Hq, self.Hkv, self.D, new, MP), False)
        x, qkv, q, a, y = self.embedding[tokens.flatten()], self.empty(T, N), self.empty(T, self.Hq, self.D), self.empty(T, self.Hq, self.D), self.empty(T, self.hidden)
        for w, pages in zip(self.layers, self.pool):
            thi.thi_rmsnorm_qkv(x, self.gamma, EPS, w["qkv"], qkv, ws)
            thi.thi_qk_norm_rope_kv4(qkv, self.head_gamma, self.head_gamma, EPS, positions, self.theta, slots, q, pages)
            thi.thi_kv4_attention(q, pages, table, lens, offsets, self.D ** -0.5, a, new, wa)
            thi.thi_linear_residual(a.view(T, -1), w["o"], x, y, ws)
            thi.thi_rmsnorm_swiglu_mlp(y, self.gamma, EPS, w["gate"], w["up"], w["down"], y, x, ws)
        logits = self.empty(B, self.vocab)
        thi.thi_linear(x.view(B, new, -1)[:, -1].contiguous(), self.head, logits, ws)
        return logits


class Rows:
    """Who has which page: the table, the lengths, the counts of references, as they are now."""

    def __init__(self, decoder, max_pages):
        self.m = decoder
        self.table, self.lens = decoder.ints([[-1] * max_pages]), decoder.ints([0])
        self.refs = decoder.ints([0] * decoder.pool.shape[1])

    def _workspace(self, rows):
        thi = self.m.thi
        return self.m.workspace("pages", thi.thi_kv4_pages_workspace_bytes(rows, self.table.shape[0], self.table.shape[1], len(self.refs)), False)

    def fork(self, parents, room):
        """Row i continues parents[i] (-1: starts empty), with `room` positions of new tokens, by which its length grows."""
        torch = self.m.torch
        n = len(parents)
        table, lens, info = (torch.empty(*s, dtype=torch.int32, device="cuda") for s in ((n, self.table.shape[1]), (n,), (2,)))
        refs = torch.empty_like(self.refs)
        self.m.thi.thi_kv4_fork(self.refs, self.table, self.lens, self.m.ints(parents), self.m.ints([room] * n), refs, table, lens, info, self.m.pool, self._workspace(n))
        self.refs, self.table, self.lens = refs, table, lens + room
        return info

    def compact(self):
        torch = self.m.torch
        table, refs, info = torch.empty_like(self.table), torch.empty_like(self.refs), torch.empty(2, dtype=torch.int32, device="cuda")
        self.m.thi.thi_kv4_compact(self.refs, self.table, refs, table, info, self.m.pool, self._workspace(len(table)))
        self.refs, self.table = refs, table
        return info


def generate(decoder, prompt, noise, share=True, compact_every=16, drop_at=None):
    """Tokens [steps, samples], logits of the last step, and the rows as they end.  prompt [n] token numbers; noise [steps, samples, vocab] is added to the logits.
    share=False: every sample runs the prompt itself.  drop_at: the step behind which the first sample ends and the last goes on in its place too."""
    torch = decoder.torch
    steps, samples = noise.shape[:2]
    n = len(prompt)
    rows = Rows(decoder, -(-(n + steps) // decoder.thi.THI_KV4_PAGE))
    if share:
        rows.fork([-1], n)
        logits = decoder.step(prompt, rows.table, rows.lens, n).expand(samples, -1)
        rows.fork([0] * samples, 1)
    else:
        rows.fork([-1] * samples, n)
        logits = torch.cat([decoder.step(prompt, rows.table[i:i + 1], rows.lens[i:i + 1], n) for i in range(samples)])
        rows.fork(list(range(samples)), 1)
    out = []
    for i in range(steps):
        out.append((logits.float() + noise[i]).argmax(-1))
        if i + 1 == steps:
            break
        logits = decoder.step(out[-1], rows.table, rows.lens, 1)
        order = list(range(samples))
        if drop_at == i:
            order[0] = samples - 1
            logits = logits[order]
        rows.fork(order, 1)
        if i % compact_every == compact_every - 1:
            rows.compact()
    return torch.stack(out), logits, rows


def main():
    p = argparse.ArgumentParser()
    p.add_argument("--samples", type=int, default=4)
    p.add_argument("--tokens", type=int, default=48)
    p.add_argument("--prompt", type=int, default=150)
    a = p.parse_args()
    import torch
    pages = a.samples * (-(-(a.prompt + a.tokens) // 64) + 1) + 1
    decoder = Decoder(pages=pages)
    g = torch.Generator(device="cuda").manual_seed(1)
    prompt = torch.randint(0, decoder.vocab, (a.prompt,), device="cuda", generator=g)
    noise = -torch.log(-torch.log(torch.rand(a.tokens, a.samples, decoder.vocab, device="cuda", generator=g).clamp(1e-6, 1 - 1e-6)))
    tokens, _, rows = generate(decoder, prompt, noise)
    held = int((rows.refs > 0).sum())
    for i, row in enumerate(tokens.T.tolist()):
        print(f"sample {i}: {row[:12]} ...")
    print(f"{held} of {pages} pages held for {a.samples} samples of {a.prompt} + {a.tokens} positions, {decoder.thi.thi_kv4_page_bytes(decoder.Hkv, decoder.D)} bytes a page and layer")


if __name__ == "__main__":
    main()
