"""A request from its context to its answer's tokens, with every operator of the library at its place (paper Section 3.3; random weights stand in for a model):

  1. the context is streamed in chunks through the layer below the retrieval layer: queries and keys turned to their positions, keys and values stored in a
     paged cache (ilre_rope_append), attention over the sink part and a sliding window (ilre_paged_attention);
  2. at the retrieval layer only keys are made, turned straight into the recall's key cache (ilre_rope);
  3. the question's queries recall the tokens to keep (ilre_recall, ilre_gather_ids);
  4. the compressed prompts of several requests are attended to whole, packed (ilre_prompt_attention), and stored in a paged cache;
  5. the answers' tokens come one at a time (ilre_rope_append, ilre_paged_attention).

    python examples/stream_recall_answer.py [context tokens]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2508_17892_amd as il  # noqa: E402

HQ, HKV, D, PAGE = 32, 8, 128, 64
HIDDEN, VOCAB = 512, 4096
SINK, WINDOW, CHUNK = 4, 512, 1024
STEPS = 4


class Layer:
    def __init__(self, g):
        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") / rows ** 0.5).bfloat16()
        self.qkv, self.out = weight(HIDDEN, (HQ + 2 * HKV) * D), weight(HQ * D, HIDDEN)

    def project(self, x):
        """Queries, keys and values of tokens x [T, hidden], side by side in one row as a fused projection leaves them."""
        y = (x @ self.qkv).reshape(x.shape[0], HQ + 2 * HKV, D)
        return y[:, :HQ], y[:, HQ:HQ + HKV], y[:, HQ + HKV:]

    def leave(self, x, attended):
        return x + attended.reshape(x.shape[0], HQ * D) @ self.out


class Cache:
    """Pages for sequences of up to `lens` tokens, handed out in no particular order."""

    def __init__(self, lens, g):
        pages = [-(-n // PAGE) for n in lens]
        order = torch.randperm(sum(pages), generator=g, device="cuda").int()
        self.table = torch.full((len(lens), max(pages)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for s, n in enumerate(pages):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.k = torch.empty(at, HKV, PAGE, D, dtype=torch.bfloat16, device="cuda")
        self.v = torch.empty_like(self.k)
        self.kv_len = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
        self.cu_q = torch.zeros(len(lens) + 1, dtype=torch.int32, device="cuda")
        self.view = il.PagedKV(self.k, self.v, self.table, self.kv_len, self.cu_q)

    def extend(self, new):
        """`new` tokens of every sequence are about to come."""
        new = torch.tensor(new, dtype=torch.int32, device="cuda")
        self.kv_len += new
        self.cu_q[1:] = new.cumsum(0)


def main(L=20000, budget=2048, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    embed = torch.randn(VOCAB, HIDDEN, generator=g, device="cuda").bfloat16()
    below, answering = Layer(g), Layer(g)
    at_recall = Layer(g)
    freqs = il.ilre_rope_frequencies(D, 500000.0, scaling=il.ILRE_ROPE_BANDS, factor=8.0, low=1.0, high=4.0, original_len=8192)

    # 1, 2: the context, chunk by chunk (the first one brings the sink part along)
    ids = torch.randint(0, VOCAB, (L,), generator=g, device="cuda", dtype=torch.int32)
    question = torch.randint(0, VOCAB, (24,), generator=g, device="cuda", dtype=torch.int32)
    cache = Cache([L + len(question)], g)
    key_cache = torch.empty(HKV, L, D, dtype=torch.bfloat16, device="cuda")

    def stream(tokens, at):
        x = embed[tokens.long()]
        q, k, v = below.project(x)
        cache.extend([len(tokens)])
        q = il.ilre_rope_append(q, k, v, cache.view, freqs)
        attended, _ = il.ilre_paged_attention(q, cache.view, max_q=len(tokens), max_kv=at + len(tokens), sink=SINK, window=WINDOW)
        return below.leave(x, attended)

    at = 0
    while at < L:
        n = min(CHUNK + (SINK if at == 0 else 0), L - at)
        _, k, _ = at_recall.project(stream(ids[at:at + n], at))
        il.ilre_rope(k, freqs, first_position=at, out=key_cache[:, at:at + n].transpose(0, 1))
        at += n

    # 3: the question recalls
    q, _, _ = at_recall.project(stream(question, L))
    q = il.ilre_rope(q, freqs, first_position=L)
    idx, _ = il.ilre_recall(q.transpose(0, 1), key_cache, budget, (1, 3, 7, 15, 31), sink=SINK)
    kept = il.ilre_gather_ids(ids, idx)

    # 4: its compressed prompt, packed with a shorter request's, through a layer of the answering model
    prompts = [torch.cat((kept, question)), question]
    lens = [len(p) for p in prompts]
    answers = Cache([n + STEPS for n in lens], g)
    answers.extend(lens)
    x = embed[torch.cat(prompts).long()]
    q, k, v = answering.project(x)
    q = il.ilre_rope_append(q, k, v, answers.view, freqs)
    positions = torch.cat([torch.arange(n, device="cuda", dtype=torch.int32) for n in lens])
    k = il.ilre_rope(k, freqs, positions)
    whole, whole_lse = il.ilre_prompt_attention(q, k, v, answers.cu_q, max_q=max(lens))
    last = answering.leave(x, whole)[answers.cu_q[1:].long() - 1]

    # 5: one token each, again and again
    steps = []
    for step in range(STEPS):
        token = (last @ embed.T).argmax(-1)
        steps.append(token)
        x = embed[token]
        q, k, v = answering.project(x)
        answers.extend([1, 1])
        q = il.ilre_rope_append(q, k, v, answers.view, freqs)
        attended, lse = il.ilre_paged_attention(q, answers.view, max_q=1, max_kv=max(lens) + step + 1, total_kv=sum(lens) + 2 * (step + 1))
        last = answering.leave(x, attended)
    return {"kept": kept, "idx": idx, "answer": torch.stack(steps, 1), "lens": lens, "prompts": prompts, "embed": embed, "layer": answering, "freqs": freqs,
            "attended": attended, "lse": lse, "whole": whole, "whole_lse": whole_lse}


if __name__ == "__main__":
    r = main(int(sys.argv[1]) if len(sys.argv) > 1 else 20000)
    torch.cuda.synchronize()
    print(f"kept {len(r['idx'])} tokens, prompts of {r['lens']} tokens, answers {r['answer'].tolist()}")
