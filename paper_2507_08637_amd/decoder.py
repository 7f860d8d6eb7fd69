"""A small decoder of linear-time layers: what the causal operators are for, together.

    python -m paper_2507_08637_amd.decoder [--steps 200] [--eight-bit]

trains it on sequences of two tokens that take turns, takes a batch of packed prompts of unequal lengths into a cache of states
and goes on token by token, for a prompt's length no more than for any other.  A layer is
    h, r = norm(x + r);  q, k, v = h Wqkv;  x = norm_per_head(decay attention(q, k, v)) Wo
    h, r = norm(x + r);  x = silu(h Wup) Wdown
with the residual stream r added where it is normed next.  The decays are fixed: memories from 8 tokens to 1024.
Products with weights are torch's; with eight_bit, serving has the norms leave 8 bits with a scale for each row, and the
weights in 8 bits with a scale for each column.
"""
import argparse

import torch

from . import autograd, binding


class Decoder(torch.nn.Module):
    def __init__(self, vocabulary=64, hidden=256, heads=4, layers=2, dtype=torch.bfloat16, device="cuda"):
        super().__init__()
        self.heads, self.width, self.hidden, self.dtype = heads, hidden // heads, hidden, dtype
        param = lambda *shape, scale=1.0: torch.nn.Parameter(scale * torch.randn(*shape, device=device))
        ones = lambda: torch.nn.Parameter(torch.ones(hidden, device=device))
        self.embedding = param(vocabulary, hidden)
        self.layers = torch.nn.ModuleList()
        for _ in range(layers):
            layer = torch.nn.Module()
            layer.norm_mix, layer.norm_mlp = ones(), ones()
            layer.qkv, layer.out = param(hidden, 3 * hidden, scale=hidden ** -0.5), param(hidden, hidden, scale=hidden ** -0.5)
            layer.up, layer.down = param(hidden, 2 * hidden, scale=hidden ** -0.5), param(2 * hidden, hidden, scale=(2 * hidden) ** -0.5)
            self.layers.append(layer)
        self.norm_last, self.head = ones(), param(hidden, vocabulary, scale=hidden ** -0.5)
        memory = torch.exp2(3 + 7 * torch.arange(heads, device=device) / max(1, heads - 1))
        self.register_buffer("log_decay", torch.log1p(-1 / memory))

    def cache(self, slots):
        """States of `slots` sequences, for each layer."""
        return [torch.zeros(slots, self.heads, self.width, self.width, device=self.log_decay.device) for _ in self.layers]

    def _heads(self, qkv):
        """(B, n, 3 hidden) as q, k, v (B, heads, n, width), by stride."""
        return qkv.unflatten(-1, (3, self.heads, self.width)).permute(2, 0, 3, 1, 4).unbind(0)

    # ---- training: whole sequences, all of them at once
    def forward(self, tokens):
        """(B, n) -> logits (B, n, vocabulary)."""
        x, r = self.embedding[tokens].to(self.dtype), None
        for layer in self.layers:
            h, r = (autograd.wersa_rms_norm(x, layer.norm_mix), x) if r is None else autograd.wersa_rms_norm(x, layer.norm_mix, residual=r)
            o, _ = autograd.wersa_decay_attention(*self._heads(h @ layer.qkv.to(self.dtype)), self.log_decay)
            o = autograd.wersa_rms_norm(o.transpose(1, 2)).flatten(2)
            h, r = autograd.wersa_rms_norm(o @ layer.out.to(self.dtype), layer.norm_mlp, residual=r)
            x = torch.nn.functional.silu(h @ layer.up.to(self.dtype)) @ layer.down.to(self.dtype)
        h, r = autograd.wersa_rms_norm(x, self.norm_last, residual=r)
        return (h @ self.head.to(self.dtype)).float()

    # ---- serving: the weights laid out once, a cache of states, prompts and then tokens
    @torch.no_grad()
    def serving(self, eight_bit=False):
        """The weights as prefill() and step() take them: in the model's type, and those that follow a norm of the stream with eight_bit in 8 bits, a scale for each column."""
        def after_norm(w):
            if not eight_bit:
                return w.to(self.dtype), None
            most = w.abs().amax(0)
            scale = torch.where(most > 0, most / 448, 1.0)   # (a column of zeros)
            return (w / scale).to(torch.float8_e4m3fn).t().contiguous().t(), scale[None]
        return ([dict(qkv=after_norm(x.qkv), out=x.out.to(self.dtype), up=after_norm(x.up), down=x.down.to(self.dtype)) for x in self.layers],
                after_norm(self.head))

    def _normed(self, x, weight, r, w):
        """norm(x + r) times w, and the stream."""
        w, scale = w
        if scale is None:
            y, r, _ = binding.wersa_rms_norm_forward(x, weight, residual=r)
            return y @ w, r
        y, r, rows = binding.wersa_rms_norm_eight_bit(x, weight, residual=r)
        return torch._scaled_mm(y, w, scale_a=rows[:, None], scale_b=scale, out_dtype=self.dtype), r

    def _serve(self, tokens, weights, attend):
        """Logits (rows, vocabulary) of rows of tokens; attend(layer's number, q, k, v (1, heads, rows, width)) gives (1, heads, rows, width)."""
        layers, head = weights
        x, r = self.embedding[tokens].to(self.dtype), None
        for i, (layer, w) in enumerate(zip(self.layers, layers)):
            qkv, r = self._normed(x, layer.norm_mix, r, w["qkv"])
            o = attend(i, *self._heads(qkv[None]))
            o, _, _ = binding.wersa_rms_norm_forward(o.transpose(1, 2).reshape(-1, self.width))
            h, r = self._normed(o.view(-1, self.hidden) @ w["out"], layer.norm_mlp, r, w["up"])
            x = torch.nn.functional.silu(h) @ w["down"]
        return self._normed(x, self.norm_last, r, head)[0].float()

    @torch.no_grad()
    def prefill(self, tokens, offsets, cache, slots, weights):
        """Prompts one behind the other: tokens (all), offsets (prompts + 1) and slots (prompts) int32.  Leaves their states in the cache; logits of every token."""
        def attend(i, q, k, v):
            return binding.wersa_decay_forward(q, k, v, self.log_decay, offsets=offsets, final_state=cache[i], slots=slots)[0]
        return self._serve(tokens, weights, attend)

    @torch.no_grad()
    def step(self, tokens, cache, slots, weights):
        """The next token of each of B sequences (tokens, slots (B)): logits (B, vocabulary), states updated in place."""
        def attend(i, q, k, v):
            q, k, v = (x[0].transpose(0, 1) for x in (q, k, v))
            return binding.wersa_decay_step(q, k, v, self.log_decay, cache[i], slots=slots).transpose(0, 1)[None]
        return self._serve(tokens, weights, attend)


def batch(sequences, n, vocabulary, period, generator):
    """Sequences that repeat themselves: (sequences, n + 1)."""
    once = torch.randint(vocabulary, (sequences, period), generator=generator, device=generator.device)
    return once.repeat(1, n // period + 2)[:, :n + 1]


def train(model, steps, sequences=16, n=128, period=2, seed=0, report=None):
    """Losses of the steps."""
    generator = torch.Generator(device=model.log_decay.device).manual_seed(seed)
    optimizer = torch.optim.AdamW(model.parameters(), lr=3e-3)
    losses = []
    for i in range(steps):
        tokens = batch(sequences, n, model.embedding.shape[0], period, generator)
        loss = torch.nn.functional.cross_entropy(model(tokens[:, :-1]).flatten(0, 1), tokens[:, 1:].flatten())
        optimizer.zero_grad(set_to_none=True)
        loss.backward()
        optimizer.step()
        losses.append(loss.item())
        if report and (i % report == 0 or i == steps - 1):
            print(f"step {i}: loss {losses[-1]:.3f}", flush=True)
    return losses


def generate(model, prompts, tokens, eight_bit=False):
    """The most likely continuation, `tokens` long, of each prompt (a list of 1-D tensors): (prompts, tokens)."""
    assert prompts and all(len(p) > 0 for p in prompts), "a prompt has at least one token to go on from"
    device, B = model.log_decay.device, len(prompts)
    lengths = torch.tensor([len(p) for p in prompts])
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), lengths.cumsum(0)]).to(torch.int32).to(device)
    slots = torch.arange(B, dtype=torch.int32, device=device)
    weights, cache = model.serving(eight_bit), model.cache(B)
    logits = model.prefill(torch.cat(prompts), offsets, cache, slots, weights)[offsets[1:].long() - 1]
    out = [logits.argmax(1)]
    for _ in range(tokens - 1):
        out.append(model.step(out[-1], cache, slots, weights).argmax(1))
    return torch.stack(out, 1)


def main():
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--steps", type=int, default=200)
    parser.add_argument("--eight-bit", action="store_true", help="serve with activations and weights in 8 bits")
    args = parser.parse_args()
    torch.manual_seed(0)
    model = Decoder()
    train(model, args.steps, report=50)
    generator = torch.Generator(device="cuda").manual_seed(1)
    rows = batch(4, 64, model.embedding.shape[0], 2, generator)
    prompts = [row[:length] for row, length in zip(rows, (17, 40, 23, 31))]
    out = generate(model, prompts, 16, args.eight_bit)
    for row, prompt, got in zip(rows, prompts, out):
        want = row[len(prompt):len(prompt) + 16]
        print(f"prompt of {len(prompt)}: {int((got == want).sum())} of 16 tokens as they repeat")


if __name__ == "__main__":
    main()
