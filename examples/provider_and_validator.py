"""A provider serves a small decoder and proves what it generated; a validator recomputes it.

    python examples/provider_and_validator.py

The model is a Llama-shaped decoder with random weights and norms of queries and keys, small enough to run in seconds.  The
provider reads ragged prompts, forks every one into samples (the j-th begins with the j-th likeliest token) and decodes 32
tokens a sequence over a paged cache: every step plans its pages on the GPU, norms and turns queries and keys, writes keys
and values, attends over the cache, commits to the final norm's rows and takes the likeliest token with its log probability.
At the end the sequences give their pages back.  The validator has the tokens and the weights, recomputes all sequences in
one packed pass of whole prompts, checks the proofs and compares the log probabilities.  The products in between are torch's.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_16007_b200 as tl  # noqa: E402

HIDDEN, LAYERS, Q_HEADS, KV_HEADS, HEAD_DIM, MLP, VOCAB = 1024, 2, 16, 4, 64, 2048, 1000
EPS, PAGE, GENERATED, K, SAMPLES = 1e-5, 16, 32, 128, 2


class Model:
    """Weights, and one pass over packed rows; how a layer attends is the caller's."""

    def __init__(self, seed, device):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(*shape):
            return (torch.randn(shape, generator=g, device=device) * shape[0] ** -0.5).to(torch.bfloat16)

        self.embedding = torch.randn((VOCAB, HIDDEN), generator=g, device=device).to(torch.bfloat16)
        self.layers = [dict(qkv=weight(HIDDEN, (Q_HEADS + 2 * KV_HEADS) * HEAD_DIM),
                            out=weight(Q_HEADS * HEAD_DIM, HIDDEN), up=weight(HIDDEN, 2 * MLP),
                            down=weight(MLP, HIDDEN), norm1=self._norm(g, device), norm2=self._norm(g, device))
                       for _ in range(LAYERS)]
        self.final = self._norm(g, device)
        self.head = weight(HIDDEN, VOCAB)
        for w in self.layers:
            w["q_norm"], w["k_norm"] = self._norm(g, device, HEAD_DIM), self._norm(g, device, HEAD_DIM)
        self.inv_freq = 10000.0 ** (-torch.arange(HEAD_DIM // 2, device=device) / (HEAD_DIM // 2))

    @staticmethod
    def _norm(g, device, size=HIDDEN):
        return (1.0 + 0.1 * torch.randn(size, generator=g, device=device)).to(torch.bfloat16)

    def forward(self, tokens, attend):
        """Last hidden states of packed rows.  attend(layer, q, k, v) -> [rows, Q_HEADS, HEAD_DIM], from queries and keys
        that are neither normed nor turned yet."""
        residual, x = self.embedding[tokens], None
        for i, w in enumerate(self.layers):
            # the residual stream takes the layer before; its norm feeds this one
            if x is None:
                h, _, _ = tl.toploc_rmsnorm_residual(residual, None, w["norm1"], EPS)
            else:
                h, residual, _ = tl.toploc_rmsnorm_residual(x, residual, w["norm1"], EPS, residual_out=residual)
            qkv = (h @ w["qkv"]).view(-1, Q_HEADS + 2 * KV_HEADS, HEAD_DIM)
            q, k, v = qkv.split((Q_HEADS, KV_HEADS, KV_HEADS), dim=1)
            x = attend(i, q, k, v).reshape(-1, HIDDEN) @ w["out"]
            # the second norm stores 8 bits with a scale per 128 channels, as an 8-bit product would take them
            h8, residual, scales = tl.toploc_rmsnorm_residual(x, residual, w["norm2"], EPS, residual_out=residual,
                                                              quantize=True, group=128)
            h = (h8.float().view(-1, HIDDEN // 128, 128) * scales[:, :, None]).view(-1, HIDDEN).to(torch.bfloat16)
            gate, up = (h @ w["up"]).chunk(2, dim=1)
            x = (torch.nn.functional.silu(gate) * up) @ w["down"]
        return tl.toploc_rmsnorm_residual(x, residual, self.final, EPS, residual_out=residual)[0]


def check_status(status):
    """Raises where a call has flagged a sequence.  Waits for the GPU: once behind many steps is enough."""
    for i, code in enumerate(status.tolist()):
        if code != tl.TOPLOC_SEQ_OK:
            raise tl.ToplocError("sequence %d: %s" % (i, tl.toploc_sequence_status_string(code)))


class Provider:
    """Ragged prompts in, GENERATED tokens a sequence and their proofs out."""

    def __init__(self, model, num_prompts, longest, device, samples=1):
        self.model, self.n, self.samples, self.device = model, num_prompts * samples, samples, device
        self.width = -(-(longest + GENERATED) // PAGE)
        pages = self.n * self.width
        self.caches = [torch.empty((2, pages, PAGE, KV_HEADS, HEAD_DIM), dtype=torch.bfloat16, device=device)
                       for _ in range(LAYERS)]
        self.table = torch.full((self.n, self.width), -1, dtype=torch.int32, device=device)
        self.free = torch.randperm(pages, device=device).to(torch.int32)
        self.heads = [torch.zeros(1, dtype=torch.int32, device=device) for _ in range(2)]   # of the free list, in turn
        self.shares = [torch.zeros(pages, dtype=torch.int32, device=device) for _ in range(2)]   # of the pages, in turn
        self.planned, self.status = (torch.zeros(self.n, dtype=torch.uint8, device=device) for _ in range(2))

    def _flag(self):
        torch.maximum(self.status, self.planned, out=self.status)      # what any step flags stays

    def step(self, tokens, cached, new, longest):
        """One step: packed new tokens behind `cached` ones of every sequence; the last hidden states of all rows."""
        i32, dev, rows = torch.int32, self.device, tokens.shape[0]
        offsets = torch.empty(self.n + 1, dtype=i32, device=dev)
        kv_lens = torch.empty(self.n, dtype=i32, device=dev)
        slots = torch.empty(rows, dtype=torch.int64, device=dev)
        positions = torch.empty(rows, dtype=i32, device=dev)
        tl.toploc_plan_pages(cached, new, self.free, self.heads[0], self.table, PAGE, offsets, kv_lens, slots, positions,
                             self.heads[1], self.planned)
        self._flag()
        self.heads.reverse()

        def attend(layer, q, k, v):
            (k_cache, v_cache), w = self.caches[layer], self.model.layers[layer]
            q = tl.toploc_norm_rotary_paged(q, k, v, positions, slots, self.model.inv_freq, k_cache, v_cache, w["q_norm"],
                                            w["k_norm"], EPS)
            return tl.toploc_attention_paged(q, k_cache, v_cache, self.table, offsets, kv_lens, longest,
                                             status=self.status)[0]

        return self.model.forward(tokens, attend), offsets, kv_lens

    def fork(self, lens):
        """Every prompt's other samples begin as copies of its first sequence; their lengths."""
        i32, dev = torch.int32, self.device
        i = torch.arange(self.n, dtype=i32, device=dev)
        parents = torch.where(i % self.samples == 0, -1, i - i % self.samples).to(i32)
        forked, source, target = (torch.empty(self.n, dtype=i32, device=dev) for _ in range(3))
        copies = torch.empty(1, dtype=i32, device=dev)
        tl.toploc_fork_pages(parents, lens, self.shares[0], self.free, self.heads[0], self.table, PAGE, forked,
                             self.shares[1], source, target, copies, self.heads[1], self.planned)
        tl.toploc_copy_pages([half for cache in self.caches for half in cache], source, target, copies)
        self._flag()
        self.heads.reverse()
        self.shares.reverse()
        return forked

    def release(self, lens):
        """All sequences give their pages back."""
        everyone, none = torch.ones(self.n, dtype=torch.uint8, device=self.device), torch.empty_like(lens)
        tl.toploc_release_pages(everyone, lens, self.table, self.shares[0], PAGE, self.free, self.heads[0], none,
                                self.shares[1], self.heads[1], self.planned)
        self._flag()
        self.heads.reverse()
        self.shares.reverse()

    def generate(self, prompts):
        """prompts: list of token lists.  Returns (tokens [n, GENERATED], proofs, log probabilities [n, GENERATED]), a
        prompt's samples one after the other."""
        i32, dev = torch.int32, self.device
        lens = torch.tensor([len(p) if j == 0 else 0 for p in prompts for j in range(self.samples)], dtype=i32, device=dev)
        packed = torch.tensor([t for p in prompts for t in p], device=dev)
        hidden, offsets, cached = self.step(packed, torch.zeros_like(lens), lens, max(len(p) for p in prompts))
        last = hidden[offsets[1:].long() - 1]          # (of a prompt's other samples, which have no rows yet: the prompt's)
        if self.samples > 1:
            cached = self.fork(cached)
        one = torch.ones_like(lens)
        layout, _ = tl.make_layout(last, GENERATED, K, self.n, 1)
        state = torch.empty(tl.toploc_stream_state_bytes(layout), dtype=torch.uint8, device=dev)
        tl.toploc_stream_begin(state, layout)
        generated, logprobs = [], []
        for t in range(GENERATED):
            top = self.samples if t == 0 else 1        # sample j begins with the j-th likeliest token
            _, _, ids, likely = tl.toploc_token_logprobs(last @ self.model.head, top=top)
            pick = torch.arange(self.n, device=dev)[:, None] % top
            generated.append(ids.gather(1, pick)[:, 0])
            logprobs.append(likely.gather(1, pick)[:, 0])
            last, _, cached = self.step(generated[-1], cached, one, 1)
            tl.toploc_stream_append(last, layout, t, state)
        proofs, _, _ = tl.toploc_stream_finish(state, layout)
        self.release(cached)
        check_status(self.status)
        return torch.stack(generated, dim=1), proofs, torch.stack(logprobs, dim=1)


def validate(model, prompts, generated, proofs, logprobs):
    """Recomputes all sequences in one packed pass; one verdict a sequence, and how far any generated token's log probability
    is from the provider's."""
    dev = generated.device
    whole = [p + g for p, g in zip(prompts, generated.tolist())]
    ends = torch.tensor([0] + [len(w) for w in whole]).cumsum(0)
    offsets = ends.to(torch.int32).to(dev)
    tokens = torch.tensor([t for w in whole for t in w], device=dev)
    positions = torch.cat([torch.arange(len(w)) for w in whole]).to(torch.int32).to(dev)

    status = torch.zeros(len(whole), dtype=torch.uint8, device=dev)

    def attend(layer, q, k, v):
        w = model.layers[layer]
        q, k = tl.toploc_norm_rotary_prompt(q, k, positions, model.inv_freq, w["q_norm"], w["k_norm"], EPS)
        return tl.toploc_attention_prompt(q, k, v, offsets, max(len(w) for w in whole), status=status)[0]

    hidden = model.forward(tokens, attend)
    check_status(status)
    rows = torch.cat([torch.arange(int(e) - GENERATED, int(e)) for e in ends[1:]]).to(dev)
    recomputed = hidden[rows]
    layout, _ = tl.make_layout(recomputed, GENERATED, K, len(prompts), GENERATED)
    results = tl.toploc_verify_proofs(recomputed, layout, proofs, tl.default_thresholds(K))
    again = tl.toploc_token_logprobs(hidden[rows - 1] @ model.head, generated.reshape(-1))[0]
    return results.cpu().numpy().view(tl.RESULT_DTYPE).reshape(-1), (again - logprobs.reshape(-1)).abs().max().item()


def main(device="cuda:0"):
    torch.manual_seed(0)
    lens = [5, 33, 200, 1, 64, 129]
    prompts = [torch.randint(0, VOCAB, (n,)).tolist() for n in lens]
    model = Model(1, device)
    provider = Provider(model, len(prompts), max(lens), torch.device(device), SAMPLES)
    generated, proofs, logprobs = provider.generate(prompts)
    prompts = [p for p in prompts for _ in range(SAMPLES)]
    honest, near = validate(model, prompts, generated, proofs, logprobs)
    other, far = validate(Model(2, device), prompts, generated, proofs, logprobs)
    for name, results, off in (("honest", honest, near), ("other", other, far)):
        print("%s weights: %d of %d proofs accepted (exponent mismatches %s), log probabilities off by up to %.3f"
              % (name, results["accept"].sum(), results.size, results["exp_mismatch"].tolist(), off))
    return honest, other


if __name__ == "__main__":
    main()
