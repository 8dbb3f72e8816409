"""One attention layer served from KV pages behind the keys of a KeyTable.

Two workers' worth of steps on one GPU, with random weights:
  1. keys of the prompts' chunks, and each prompt's longest cached prefix (KeyTable);
  2. the prefix's K and V read back from its pages, the rest projected, and attention over the whole (a hit skips the
     prefix's part);
  3. the missed chunks written to the pages of the slots that the table gave them, so that a second batch hits them;
  4. decode steps: the new token's K and V appended, attention over the pages, each page's attention weight accumulated;
  5. each request cut to a budget of pages by that weight, and decoding goes on over what is left.

    python examples/serve_from_pages.py
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_38706_gb300.service import KeyTable, KVPages  # noqa: E402

CHUNK, VOCAB, WIDTH, Q_HEADS, KV_HEADS, D = 16, 1000, 256, 8, 2, 64


class Layer:
    """Embedding and projections of one attention layer (random, no positions: a page's state is its tokens')."""

    def __init__(self, seed: int):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: (torch.randn(s, generator=g, device="cuda") / s[0] ** 0.5).to(torch.bfloat16)
        self.embed, self.wq = r(VOCAB, WIDTH) * VOCAB ** 0.5, r(WIDTH, Q_HEADS * D)
        self.wkv, self.wo = r(WIDTH, 2 * KV_HEADS * D), r(Q_HEADS * D, VOCAB)

    def project(self, tokens):
        x = self.embed[tokens.long()]
        kv = (x @ self.wkv).view(-1, 2, KV_HEADS, D)
        return (x @ self.wq).view(-1, Q_HEADS, D), kv[:, 0], kv[:, 1]

    def logits(self, attended):
        return attended.reshape(-1, Q_HEADS * D) @ self.wo


class Server:
    def __init__(self, layer: Layer, slots: int = 512):
        self.layer, self.free = layer, list(range(slots))
        self.private = set()  # slots that one request has to itself: no key of the table leads to them
        self.kt = KeyTable(CHUNK, 12)
        self.kv = KVPages(slots, CHUNK, KV_HEADS, D)
        self.descriptors = [{"model_id": "example/one-layer", "weight_precision": "bf16", "weight_version": "1",
                             "kv_format": self.kv.kv_format}]

    def prefill(self, prompts, room: int):
        """Prompts (lists of token ids) to (logits of their last tokens, page table, lengths, hit chunks)."""
        lens = [len(p) for p in prompts]
        R = len(prompts)
        tok_off = np.concatenate(([0], np.cumsum(lens))).astype(np.int64)
        tokens = torch.tensor([t for p in prompts for t in p], dtype=torch.int32, device="cuda")
        n = sum(x // CHUNK for x in lens)
        fresh = [self.free.pop() for _ in range(n)]
        _, key_off, _, hit, slots, result, slot_out = self.kt.derive_lookup_store(
            tokens, tok_off, np.zeros(R, np.uint32), self.descriptors, np.array(fresh, np.uint32))
        self.kt.check("prefill")
        key_off, hit = key_off.tolist(), hit.tolist()
        used = torch.where(slots >= 0, slots, slot_out).tolist()       # a hit's slot, or the one a miss was given
        taken = set(used)
        self.free += [s for s in fresh if s not in taken]

        # page tables: the chunks' slots, then private pages for the rest of the prompt and what is decoded
        stride = max(-(-(x + room) // CHUNK) for x in lens)
        table = torch.full((R, stride), -1, dtype=torch.int32)
        for r in range(R):
            row = used[key_off[r]: key_off[r + 1]]
            own = [self.free.pop() for _ in range(-(-(lens[r] + room) // CHUNK) - len(row))]
            self.private.update(own)
            row += own
            table[r, : len(row)] = torch.tensor(row, dtype=torch.int32)
        table = table.cuda()

        # a hit may cover the whole prompt: its last token is still needed as a query
        start = [min(h * CHUNK, x - 1) for h, x in zip(hit, lens)]
        off = lambda v: torch.tensor(np.concatenate(([0], np.cumsum(v))), dtype=torch.int64, device="cuda")
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        new = [x - s for x, s in zip(lens, start)]
        mine = torch.cat([tokens[a + s: a + x] for a, s, x in zip(tok_off, start, lens)])
        q, k_new, v_new = self.layer.project(mine)
        k_old, v_old = self.kv.read(off(start), i32([0] * R), table, sum(start))
        olds, news = np.cumsum([0] + start), np.cumsum([0] + new)
        k, v = (torch.cat([p for r in range(R) for p in (old[olds[r]: olds[r + 1]], fresh_[news[r]: news[r + 1]])])
                for old, fresh_ in ((k_old, k_new), (v_old, v_new)))
        out, _ = self.kv.attend_prompt(q, k, v, off(new), off(lens))

        # only what no page holds yet: the missed chunks and the tail (a fully hit prompt's last token is there)
        first = [max(s, min(h * CHUNK, x)) for s, h, x in zip(start, hit, lens)]
        keep = torch.cat([torch.arange(news[r] + first[r] - start[r], news[r + 1]) for r in range(R)]).cuda()
        self.kv.write(k_new[keep], v_new[keep], off([x - f for x, f in zip(lens, first)]), i32(first), table)
        self.kv.check("prefill")
        last = torch.tensor(news[1:] - 1, device="cuda")
        return self.layer.logits(out[last]), table, i32(lens), hit

    def decode(self, tokens, table, kv_len, weight):
        """One step: tokens [R] appended, attention over the pages, weights accumulated; logits and the new lengths."""
        R = tokens.numel()
        q, k, v = self.layer.project(tokens)
        self.kv.write(k, v, torch.arange(R + 1, device="cuda"), kv_len, table)
        kv_len = kv_len + 1
        out, _ = self.kv.attend(q.unsqueeze(1), kv_len, table, weight=weight)
        return self.layer.logits(out), kv_len


    def evict(self, table, weight, kv_len, budget: int):
        """Cuts each request to the pages that attention has weighed most; the rest of its room follows them."""
        stride = table.shape[1]
        held = (kv_len + CHUNK - 1) // CHUNK
        kept, kept_weight, kv_len, gone = self.kv.evict(table, weight, kv_len, budget, sinks=1, recent=2)
        left = (kv_len + CHUNK - 1) // CHUNK
        at = torch.arange(stride, device="cuda").view(1, -1)
        room = at + (held - left).view(-1, 1)  # where a place behind the kept pages was before
        moved = torch.where(room < stride, table.gather(1, room.clamp(max=stride - 1)), -1)
        kept, kept_weight = (torch.nn.functional.pad(x, (0, max(0, stride - budget)))[:, :stride] for x in (kept, kept_weight))
        table = torch.where(at < left.view(-1, 1), kept, moved).to(torch.int32).contiguous()
        self.release(gone)
        return table, kept_weight.contiguous(), kv_len

    def release(self, slots):
        """Gives back what of `slots` no key leads to: a chunk's page may be another request's, now or later."""
        mine = self.private.intersection(slots.flatten().tolist())
        self.private -= mine
        self.free += sorted(mine)

    def serve(self, batch, steps: int, budget: int):
        """Answers of 2 * steps tokens a request, cut to `budget` pages after the first half; a report."""
        logits, table, kv_len, hit = self.prefill(batch, room=2 * steps)
        weight = torch.zeros(table.shape, dtype=torch.float32, device="cuda")
        answers = []
        for step in range(2 * steps):
            if step == steps:
                table, weight, kv_len = self.evict(table, weight, kv_len, budget)
            token = logits.argmax(-1).to(torch.int32)
            answers.append(token)
            logits, kv_len = self.decode(token, table, kv_len, weight)
        self.kv.check("decode")
        self.release(table)
        return dict(hit=hit, kv_len=kv_len.tolist(), answers=torch.stack(answers).T.tolist(), weight=weight.sum(1).tolist())


def main(steps: int = 24, budget: int = 8, quiet: bool = False):
    rng = np.random.default_rng(0)
    server = Server(Layer(0))
    document = rng.integers(0, VOCAB, 100).tolist()
    first = [document + rng.integers(0, VOCAB, n).tolist() for n in (40, 7)]
    second = [document + rng.integers(0, VOCAB, 60).tolist(), first[0], rng.integers(0, VOCAB, 5).tolist()]
    report = {}
    for name, batch in (("first", first), ("second", second)):
        report[name] = server.serve(batch, steps, budget)
        if not quiet:
            print(f"{name} batch: hit chunks {report[name]['hit']}, positions held {report[name]['kv_len']}, "
                  f"first answers {[a[:6] for a in report[name]['answers']]}")
    server.kt.close()
    return report


if __name__ == "__main__":
    main()
