"""A serving loop over paged caches, layers with random keys, values and queries: prompts in chunks, steps of one token, three
continuations of a prompt, ends, compaction, and the span decode step for the sequences that have grown long.  The layers share
the table, the lengths and the counts: room, forks, ends and compaction go once, copies and the rest for every layer.

    python examples/paged_serving.py [--prompts 8] [--chunk 1024] [--steps 32] [--span-from 4096] [--layers 2]

Prints the tokens that went through and checks the last step against attention over a contiguous copy.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2601_18401_b200 as sla  # noqa: E402
from paper_2601_18401_b200.paged import PagedCache  # noqa: E402


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def run(prompts=8, chunk=1024, steps=32, span_from=4096, q_heads=32, kv_heads=8, head_dim=128, layers=2, seed=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def rand(*shape):
        return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)

    lengths = [200 + 777 * i for i in range(prompts)]        # tokens of the prompts: a program knows what it was sent
    slots = prompts + 3
    most = max(lengths) + steps + 64
    pages = sum(-(-(n + steps) // 64) + 1 for n in lengths) + 3 * (-(-(lengths[0] + steps) // 64) + 2)
    params = sla.make_params(8, 0, head_dim=head_dim)
    shape = dict(n_q_heads=q_heads, n_kv_heads=kv_heads, head_dim=head_dim, max_new=prompts * chunk)
    c = PagedCache(pages, slots, most, params=params, **shape)
    caches = [c] + [PagedCache(pages, slots, most, share=c, **shape) for _ in range(layers - 1)]
    done, tokens = [0] * prompts, 0
    began = time.perf_counter()

    # the prompts, a chunk of each that has some left at a time
    while any(d < n for d, n in zip(done, lengths)):
        seq = [s for s in range(prompts) if done[s] < lengths[s]]
        new = [min(chunk, lengths[s] - done[s]) for s in seq]
        cu = ints([0] + torch.tensor(new).cumsum(0).tolist())
        first = c.extend(cu, seq=ints(seq))
        for layer in caches:
            layer.append(cu, first, rand(sum(new), kv_heads, head_dim), rand(sum(new), kv_heads, head_dim), seq=ints(seq))
            layer.attend(rand(sum(new), q_heads, head_dim), cu, seq=ints(seq), max_new=max(new), first=first)
        for s, n in zip(seq, new):
            done[s] += n
        tokens += sum(new)

    # three continuations of the first prompt, in the slots behind the others
    pairs = c.fork(ints([0, 0, 0]), ints([prompts, prompts + 1, prompts + 2]))
    for layer in caches[1:]:
        layer.copy(pairs)
    live = lengths + [lengths[0]] * 3
    out = q = None
    for step in range(steps):
        if step == steps // 2:                                # the second prompt is answered; what it held goes to the others
            c.release(ints([1]))
            pairs = c.compact()
            for layer in caches[1:]:
                layer.copy(pairs)
            live[1] = 0
        short = [s for s in range(slots) if live[s] and live[s] < span_from]
        long_ = [s for s in range(slots) if live[s] >= span_from]
        for group, spans in ((short, False), (long_, True)):
            if not group:
                continue
            seq = ints(group)
            first = c.extend(seq=seq)
            for layer in caches:
                layer.append(None, first, rand(len(group), kv_heads, head_dim), rand(len(group), kv_heads, head_dim), seq=seq)
                q = rand(len(group), q_heads, head_dim)
                if spans:
                    layer.step(rand(len(group), q_heads, head_dim), q, seq=seq, max_tokens=most, first=first)
                else:
                    out, _ = layer.attend(q, seq=seq, first=first)
                    last = (group, q, out)
            for s in group:
                live[s] += 1
            tokens += len(group)
    status = c.poll()
    seconds = time.perf_counter() - began

    # the last layer's last dense step again, each sequence by itself
    worst = 0.0
    for x, s in enumerate(last[0]):
        n = live[s]
        rows = c.table[s, : -(-n // 64)].long()
        k, v = (p[rows].transpose(1, 2).reshape(-1, kv_heads, head_dim)[:n].float().repeat_interleave(q_heads // kv_heads, 1)
                for p in (caches[-1].k, caches[-1].v))
        w = torch.softmax(torch.einsum("hd,jhd->hj", last[1][x].float(), k) * head_dim ** -0.5, -1)
        worst = max(worst, (torch.einsum("hj,jhd->hd", w, v) - last[2][x].float()).abs().max().item())
    assert c.n_tokens.tolist() == live
    return dict(tokens=tokens, seconds=seconds, status=status, worst=worst)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, default=8)
    ap.add_argument("--chunk", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--span-from", type=int, default=4096)
    ap.add_argument("--layers", type=int, default=2)
    a = ap.parse_args()
    r = run(a.prompts, a.chunk, a.steps, a.span_from, layers=a.layers)
    assert r["status"] == sla.SLA_OK and r["worst"] < 2e-2, r
    print(f"{r['tokens']} tokens of {a.layers} layer(s) in {r['seconds'] * 1e3:.1f} ms; last step off by at most {r['worst']:.1e}")
