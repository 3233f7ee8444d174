"""Generation over a long context: a small decoder whose layers share KV heads (MLKV), with a sliding
window and sinks, its cache held in 4 bits.

    python examples/long_context.py --batch 8 --prompt 6000 --new 64

Every layer's attention is three calls of the library:

  prompt   mlkv_qk_norm_rope       the projection's rows -> normed, rotated queries and keys, values
           MLKVQ4Cache.prefill     windowed attention over the prompt; an owner layer's K and V stored
  token    mlkv_qk_norm_rope
           MLKVQ4Cache.append      owner layers only
           MLKVQ4Cache.decode_attention   over the layer's owner's codes, window and sinks

The weights are random (sizes of Pythia-160M by default): this shows the calls, not a model's answers.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2406_09297_gb300 as mlkv  # noqa: E402


class Decoder:
    """Pre-norm layers of attention and an MLP on a bf16 residual stream."""

    def __init__(self, n_layers=12, hidden=768, n_q_heads=12, head_dim=64, n_owners=2, kv_heads=4,
                 rot_dim=16, vocab=50304, window=4096, sinks=4, batch=8, max_seq=8192, seed=0):
        self.l, self.h, self.d, self.g, self.b = n_layers, n_q_heads, head_dim, kv_heads, batch
        self.window, self.sinks, self.max_seq = window, sinks, max_seq
        self.owner = [int(o) for o in mlkv.mlkv_block_owner_map(n_layers, n_owners)]
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n_out, n_in):
            w = torch.empty((n_out, n_in), dtype=torch.bfloat16, device="cuda")
            return w.normal_(0.0, 1.0 / math.sqrt(n_in), generator=gen)

        self.embed = weight(vocab, hidden) * math.sqrt(hidden)
        # an owner layer projects to queries, keys and values, a reader to queries alone
        heads = [n_q_heads + (2 * kv_heads if o == n else 0) for n, o in enumerate(self.owner)]
        self.w_in = [weight(k * head_dim, hidden) for k in heads]
        self.w_out = [weight(hidden, n_q_heads * head_dim) for _ in heads]
        self.w_up = [weight(4 * hidden, hidden) for _ in heads]
        self.w_down = [weight(hidden, 4 * hidden) for _ in heads]
        gains = 1.0 + 0.1 * torch.randn((2, n_layers, head_dim), generator=gen, device="cuda")
        self.q_gain, self.k_gain = gains.bfloat16()
        half = rot_dim // 2
        rate = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
        angle = torch.arange(max_seq, dtype=torch.float64, device="cuda")[:, None] * rate
        self.cos, self.sin = angle.cos().float(), angle.sin().float()
        self.cache = mlkv.MLKVQ4Cache(n_layers, n_q_heads, head_dim, self.owner, kv_heads, batch,
                                      max_seq)

    @staticmethod
    def _norm(x):
        return torch.nn.functional.rms_norm(x, x.shape[-1:], eps=1e-6)

    def _qkv(self, layer, x, positions):
        """x [b][s][hidden] -> Q [b][s][h][d] and, for an owner layer, K and V [b][g][s][d]."""
        b, s, _ = x.shape
        rows = (self._norm(x) @ self.w_in[layer].T).view(b, s, -1, self.d)
        Q, K, V = rows[:, :, :self.h], None, None
        Q_out, K_out, V_out = torch.empty(Q.shape, dtype=Q.dtype, device="cuda"), None, None
        if self.owner[layer] == layer:
            K, V = rows[:, :, self.h:self.h + self.g], rows[:, :, self.h + self.g:]
            K_out, V_out = torch.empty((2, b, self.g, s, self.d), dtype=Q.dtype, device="cuda")
        mlkv.mlkv_qk_norm_rope(Q, K, V, self.q_gain[layer], self.k_gain[layer], self.cos, self.sin,
                               positions, Q_out, K_out, V_out)
        return Q_out, K_out, V_out

    def _rest(self, layer, x, attention):
        x = x + attention.flatten(-2) @ self.w_out[layer].T
        up = torch.nn.functional.gelu(self._norm(x) @ self.w_up[layer].T)
        return x + up @ self.w_down[layer].T

    def prefill(self, tokens, lens):
        """tokens [b][s], the first lens[i] of each row a prompt: the logits after each prompt."""
        s = tokens.shape[1]
        x = self.embed[tokens]
        positions = torch.arange(s, dtype=torch.int32, device="cuda").expand(self.b, s).contiguous()
        kv = {}
        for n in range(self.l):
            Q, K, V = self._qkv(n, x, positions)
            if K is not None:
                kv = {self.owner[n]: (K, V)}   # its readers follow it
            out = torch.zeros_like(Q)          # rows past a prompt's end are not written
            self.cache.prefill(n, Q, *kv[self.owner[n]], out, lens, self.window, self.sinks)
            x = self._rest(n, x, out)
        last = torch.as_tensor(lens, device="cuda").long() - 1
        x = x[torch.arange(self.b, device="cuda"), last]
        return self._norm(x) @ self.embed.T

    def step(self, tokens, lens):
        """One token a sequence, the lens[i]-th: the logits after it."""
        x = self.embed[tokens][:, None]
        positions = torch.as_tensor(lens, dtype=torch.int32).sub(1).cuda()[:, None]
        lens = mlkv.as_seq_lens(lens)
        for n in range(self.l):
            Q, K, V = self._qkv(n, x, positions)
            if K is not None:
                self.cache.append(n, K, V, lens)
            out = torch.empty_like(Q)
            self.cache.decode_attention(n, Q, out, lens, self.window, self.sinks)
            x = self._rest(n, x, out)
        return self._norm(x[:, 0]) @ self.embed.T


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--batch", type=int, default=8)
    p.add_argument("--prompt", type=int, default=6000)
    p.add_argument("--new", type=int, default=64)
    p.add_argument("--window", type=int, default=4096)
    p.add_argument("--sinks", type=int, default=4)
    a = p.parse_args()
    max_seq = a.prompt + a.new
    model = Decoder(batch=a.batch, max_seq=max_seq, window=a.window, sinks=a.sinks)
    gen = torch.Generator(device="cuda").manual_seed(1)
    prompts = torch.randint(0, 50304, (a.batch, a.prompt), generator=gen, device="cuda")
    # uneven prompts: the i-th is shorter by i tokens
    lens = [max(1, a.prompt - i) for i in range(a.batch)]
    times = []
    token = model.prefill(prompts, lens).argmax(-1)
    answers = [token]
    for _ in range(a.new - 1):
        torch.cuda.synchronize()
        t0 = time.perf_counter()
        lens = [n + 1 for n in lens]
        token = model.step(token, lens).argmax(-1)
        answers.append(token)
        torch.cuda.synchronize()
        times.append(time.perf_counter() - t0)
    model.cache.sync_status()
    bf16 = 4 * a.batch * max_seq * model.g * model.d * len(set(model.owner))
    print(f"first answer's tokens: {torch.stack(answers, 1)[0, :8].tolist()} ...")
    print(f"cache {model.cache.cache_bytes() / 2**20:.1f} MiB ({bf16 / 2**20:.1f} in bf16)")
    if times:
        print(f"{1e3 * sorted(times)[len(times) // 2]:.2f} ms a step of {a.batch} tokens")


if __name__ == "__main__":
    main()
