"""A small transformer decoded with PLD+ over paged caches: every call of a step where it belongs.

    python examples/cached_decode.py [--cache e4m3] [--no-draft]

The model is a few attention layers with random weights (no MLP, no training), enough to produce queries,
keys, values and logits; what is shown is the step around it:

  prompts     pldp_pages_reserve, then per layer pldp_cache_append_prompt and pldp_attend_prompt, all
              sequences' tokens packed
  a step      pldp_pages_reserve   pages for the tokens that it appends
  per layer   pldp_cache_append    norms and rotates the step's queries and keys, writes keys and values
              pldp_attend_cache    attends over the cache with all of the step's tokens at once
  then        pldp_verify_greedy   accepts the draft's prefix and appends it with the bonus token
              pldp_token_logprobs  scores the tokens that the step emitted
  next draft  pldp_find_candidates, pldp_rank_cache (Eq. 2 from the last layers' caches, a layer at a time),
              pldp_extract_draft

Greedy decoding emits the same tokens with and without drafts; drafts only save steps.
"""
import argparse
import dataclasses
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2412_01447_gb300 as pk  # noqa: E402


@dataclasses.dataclass
class Shape:
    layers: int = 3
    q_heads: int = 8
    heads: int = 2
    head_dim: int = 64
    vocab: int = 512
    K: int = 6                  # draft length at most
    page: int = 16
    cache: str = "bf16"         # or "e4m3"
    rank_layers: int = 2        # the last layers rank the candidates


def context_of(prompt, new, shape):
    """Positions to hold: the slowest sequence may take a step a token, in which another appends K+1."""
    return prompt + (new + 1) * (shape.K + 1)


class Decoder:
    def __init__(self, shape, B, context, seed=0, device="cuda"):
        s, g = shape, torch.Generator(device).manual_seed(seed)
        self.s, self.B, self.dev = s, B, device
        d = self.d = s.q_heads * s.head_dim

        def w(*size):
            return torch.randn(size, generator=g, device=device) * size[0] ** -0.5

        self.embed, self.unembed = torch.randn((s.vocab, d), generator=g, device=device), w(d, s.vocab) * 4
        self.qkv = [w(d, (s.q_heads + 2 * s.heads) * s.head_dim) for _ in range(s.layers)]
        self.proj = [w(d, d) for _ in range(s.layers)]
        self.norms = [(torch.full((s.head_dim,), 1.5, device=device, dtype=torch.bfloat16),) * 2 for _ in range(s.layers)]
        angle = torch.arange(context, device=device, dtype=torch.float64)[:, None] * (
            10000.0 ** (-torch.arange(0, s.head_dim, 2, device=device, dtype=torch.float64) / s.head_dim))
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

        # one pool of pages a layer; every sequence has its pages anywhere in it, the same in all layers, as it needs them
        per = -(-context // s.page)
        n_pages = B * per
        self.pages = torch.full((B, per), -1, dtype=torch.int32, device=device)
        self.table = pk.pldp_page_table(self.pages, torch.zeros(n_pages, dtype=torch.int32, device=device), s.page)
        kind = torch.bfloat16 if s.cache == "bf16" else torch.float8_e4m3fn
        pool = lambda: torch.zeros((n_pages, s.page, s.heads, s.head_dim), device=device, dtype=torch.bfloat16).to(kind)  # noqa: E731
        scale = lambda: torch.ones((n_pages, s.heads, s.page), device=device) if s.cache == "e4m3" else None  # noqa: E731
        self.caches = [pk.pldp_cache(pool(), pool(), self.pages, scale(), scale()) for _ in range(s.layers)]

        n, i32 = s.K + 1, dict(dtype=torch.int32, device=device)
        self.workspace = torch.zeros(pk.pldp_attend_workspace_size(B, n, s.q_heads, s.heads, s.head_dim), dtype=torch.uint8, device=device)
        self.prompt_ws = torch.empty(pk.pldp_attend_prompt_workspace_size(s.q_heads, s.heads, s.head_dim), dtype=torch.uint8, device=device)
        self.pages_ws = torch.empty(pk.pldp_pages_workspace_size(self.table), dtype=torch.uint8, device=device)
        self.copies = torch.empty((B, 2), **i32)
        self.verify_ws = torch.zeros(pk.pldp_verify_workspace_size(B, s.K, s.vocab), dtype=torch.uint8, device=device)
        self.score_ws = torch.empty(pk.pldp_token_logprobs_workspace_size(B * n, s.vocab), dtype=torch.uint8, device=device)
        self.draft, self.draft_len = torch.zeros((B, s.K), **i32), torch.zeros(B, **i32)
        self.accepted, self.next_token, self.kv_keep = (torch.zeros(B, **i32) for _ in range(3))
        self.cand, self.count, self.match = torch.full((B, 1024), -1, **i32), torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.scores, self.best = torch.zeros((B, 1024), device=device), torch.zeros(B, **i32)
        self.status = torch.zeros(B, **i32)

    def reserve(self, start, n, count=None):
        # (no page here is held by two sequences, so that none has to be copied)
        pk.pldp_pages_reserve(self.table, start, self.copies, self.pages_ws, n, count=count, status=self.status)

    def prompts(self, tokens, rows, n):
        """Takes the prompts into the caches: sequence b's tokens are tokens[rows[b]:rows[b + 1]], n of one at most."""
        s, R = self.s, tokens.shape[0]
        x, start = self.embed[tokens.long()], torch.zeros_like(rows[:-1])
        self.reserve(start, n, rows[1:] - rows[:-1])
        for layer in range(s.layers):
            h = torch.nn.functional.layer_norm(x, (self.d,))
            qkv = (h @ self.qkv[layer]).to(torch.bfloat16).view(R, s.q_heads + 2 * s.heads, s.head_dim)
            q, k, v = qkv.split((s.q_heads, s.heads, s.heads), 1)
            out = torch.empty((R, s.q_heads, s.head_dim), device=self.dev, dtype=torch.bfloat16)
            pk.pldp_cache_append_prompt(self.caches[layer], q, k, v, rows, q, start=start, q_norm=self.norms[layer][0],
                                        k_norm=self.norms[layer][1], cos=self.cos, sin=self.sin, status=self.status)
            if layer + 1 < s.layers:                              # (nothing reads what the last layer would give)
                pk.pldp_attend_prompt(self.caches[layer], q, rows, out, self.prompt_ws, start=start, status=self.status)
                x = x + out.float().view(R, self.d) @ self.proj[layer]

    def forward(self, tokens, seq_len, draft_len):
        """Logits [B, n, vocab] of x_t and its draft (tokens [B, n], x_t first); what ranking needs of
        each layer stays in self.rows."""
        s, B, n = self.s, self.B, tokens.shape[1]
        x = self.embed[tokens.long()]
        self.rows = []
        ws = self.workspace
        self.reserve(seq_len - 1, n, draft_len + 1)
        for layer in range(s.layers):
            h = torch.nn.functional.layer_norm(x, (self.d,))
            qkv = (h @ self.qkv[layer]).to(torch.bfloat16).view(B, n, s.q_heads + 2 * s.heads, s.head_dim)
            q, k, v = qkv.split((s.q_heads, s.heads, s.heads), 2)  # slices of one tensor, as they are
            out = torch.empty((B, n, s.q_heads, s.head_dim), device=self.dev, dtype=torch.bfloat16)
            lse = torch.empty((B, n, s.q_heads), device=self.dev)
            pk.pldp_cache_append(self.caches[layer], q, k, v, seq_len, q, draft_len=draft_len, q_norm=self.norms[layer][0],
                                 k_norm=self.norms[layer][1], cos=self.cos, sin=self.sin, status=self.status)
            pk.pldp_attend_cache(self.caches[layer], q, seq_len, out, ws, draft_len=draft_len, lse=lse, status=self.status)
            self.rows.append((q, lse))
            x = x + out.float().view(B, n, self.d) @ self.proj[layer]
        return torch.nn.functional.layer_norm(x, (self.d,)) @ self.unembed

    def next_draft(self, ids, seq_len):
        """Candidates of the new x_t, ranked by the attention of the query before it, and the draft behind
        the best of them."""
        pk.pldp_find_candidates(ids, seq_len, 1, 3, self.cand, self.count, self.match, self.status)
        layers = range(self.s.layers - self.s.rank_layers, self.s.layers)
        for i, layer in enumerate(layers):
            q, lse = self.rows[layer]
            pk.pldp_rank_cache(self.caches[layer], q, self.accepted, self.kv_keep, lse, self.cand, self.count, self.best,
                               scores=self.scores, accumulate=i > 0, status=self.status)
        pk.pldp_extract_draft(ids, seq_len, self.best, self.draft, self.draft_len)

    def decode(self, prompt, new, draft=True):
        """Greedy decoding of `new` tokens a sequence.  Returns (contexts, steps, accepted tokens, the emitted tokens'
        log probabilities and leads over the runner-up, by sequence)."""
        s, B = self.s, self.B
        ids = torch.zeros((B, context_of(prompt.shape[1], new, s)), dtype=torch.int32, device=self.dev)
        ids[:, : prompt.shape[1]] = prompt
        seq_len = torch.full((B,), prompt.shape[1], dtype=torch.int32, device=self.dev)
        start = seq_len.clone()
        # the prompts but their last tokens
        n = prompt.shape[1] - 1
        self.prompts(prompt[:, :-1].reshape(-1), torch.arange(B + 1, dtype=torch.int32, device=self.dev) * n, n)
        self.draft_len.zero_()
        self.draft.zero_()
        rows = torch.arange(s.K + 1, device=self.dev)
        steps, taken = 0, 0
        logprobs, leads = ([[] for _ in range(B)] for _ in range(2))
        while int((seq_len - start).min()) < new:
            x_t = torch.gather(ids, 1, seq_len.long()[:, None] - 1)
            logits = self.forward(torch.cat((x_t, self.draft.clamp(min=0)), 1), seq_len, self.draft_len)
            pk.pldp_verify_greedy(logits, self.draft, self.draft_len, self.accepted, self.next_token, self.verify_ws, ids=ids,
                                  seq_len=seq_len, kv_keep_len=self.kv_keep, status=self.status)
            emitted = torch.cat((self.draft, self.next_token[:, None]), 1)
            emitted.scatter_(1, self.accepted.long()[:, None], self.next_token[:, None])
            lp, ids2 = torch.empty((B, s.K + 1), device=self.dev), torch.empty((B, s.K + 1, 2), dtype=torch.int32, device=self.dev)
            top = torch.empty((B, s.K + 1, 2), device=self.dev)
            pk.pldp_token_logprobs(logits, emitted, lp, self.score_ws, top_id=ids2, top_logprob=top)
            live = rows <= self.accepted[:, None]
            for b in range(B):
                logprobs[b] += lp[b][live[b]].tolist()
                leads[b] += (top[b, :, 0] - top[b, :, 1])[live[b]].tolist()
            steps, taken = steps + 1, taken + int(self.accepted.sum())
            if draft:
                self.next_draft(ids, seq_len)
        assert int(self.status.abs().sum()) == 0, self.status
        return [ids[b, : int(seq_len[b])].tolist() for b in range(B)], steps, taken, logprobs, leads


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--no-draft", action="store_true")
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--new", type=int, default=64)
    a = ap.parse_args()
    pk.build()
    shape = Shape(cache=a.cache)
    g = torch.Generator("cuda").manual_seed(1)
    prompt = torch.randint(0, shape.vocab, (a.batch, 40), generator=g, device="cuda", dtype=torch.int32)
    prompt = torch.cat((prompt, prompt[:, :20]), 1)               # a text that repeats itself
    model = Decoder(shape, a.batch, context_of(prompt.shape[1], a.new, shape))
    texts, steps, taken, logprobs, _ = model.decode(prompt, a.new, draft=not a.no_draft)
    for b, t in enumerate(texts):
        print(f"sequence {b}: {t[prompt.shape[1]:][:24]} ... mean log probability {sum(logprobs[b]) / len(logprobs[b]):.3f}")
    print(f"{a.new} tokens in {steps} steps, {taken / a.batch:.1f} draft tokens accepted a sequence")


if __name__ == "__main__":
    main()
