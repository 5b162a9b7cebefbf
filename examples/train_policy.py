"""A whole training program around one MoE layer: python -m examples.train_policy

A small policy learns, from rewards alone, which token answers which.  Everything but the plain matrix products goes through
the library:

    tokens -> symi_embed_fwd -> gate network, route, dispatch, experts, combine -> + residual -> product with the same table
           -> symi_token_logp of the sampled answers
    update:   symi_policy_loss (loss and gradient of the logits, in their place) -> product's gradients -> the layer's backward
           -> symi_embed_bwd (added to the table's gradient from the product)
           -> symi_adamw_step (table with 8-bit states, gate network with 32-bit ones) and symi_adam_to_replicas (experts)
"""
import argparse
import math

import torch

import harness as Hn
import paper_2504_19925_amd as symi
import workloads as wl


class Policy:
    """Table [V, d], gate network and one MoE layer with all its optimizer partitions; weights and activations in fp32."""

    def __init__(self, c, V, seed=0):
        self.c, self.V = c, V
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
        self.layer = Hn.State(c, all_shards=True)
        self.layer.place_current()
        self.ctx = self.layer.ctx
        self.scale = 1.0
        self.table, self.dtable = rand(V, c.d) / math.sqrt(c.d), torch.empty(V, c.d, device="cuda")
        self.Wr, self.dWr = rand(c.E, c.d) * 0.02, torch.empty(c.E, c.d, device="cuda")
        self.b, self.db = torch.zeros(c.E, device="cuda"), torch.empty(c.E, device="cuda")
        self.X, self.dX = torch.empty(c.T, c.d, device="cuda"), torch.empty(c.T, c.d, device="cuda")
        self.scores = torch.empty(c.T, c.E, device="cuda")
        self.ws = torch.empty(symi.symi_embed_workspace_bytes(self.ctx, V), dtype=torch.uint8, device="cuda")
        blocks = -(-self.table.numel() // 256)
        zeros = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")   # noqa: E731
        self.opt = symi.symi_adamw_create([
            dict(param=self.table, grad=self.dtable, m=zeros(V, c.d, dtype=torch.int8), v=zeros(V, c.d, dtype=torch.uint8),
                 m_scale=zeros(blocks), v_scale=zeros(blocks)),
            dict(param=self.Wr, grad=self.dWr, m=zeros(c.E, c.d), v=zeros(c.E, c.d)),
            dict(param=self.b, grad=self.db, m=zeros(c.E), v=zeros(c.E), decay=0.0)])
        self.step = 0

    def forward(self, tokens):
        """Logits [T, V]."""
        symi.symi_embed_fwd(self.ctx, tokens, self.table, self.V, self.scale, self.X)
        symi.symi_router_fwd(self.ctx, self.X, self.Wr, self.b, self.scores)
        self.layer.forward(self.X, self.scores)
        self.H = self.X + self.layer.Y
        return self.H @ self.table.t()

    def backward(self, tokens, dlogits):
        layer = self.layer
        torch.mm(dlogits.t(), self.H, out=self.dtable)
        dH = dlogits @ self.table
        layer.backward(dH, self.scores)
        symi.symi_router_bwd(self.ctx, self.X, self.Wr, layer.dlogits, self.dWr, self.db, layer.dX, layer.ws)
        torch.add(dH, layer.dX, out=self.dX)
        symi.symi_embed_bwd(self.ctx, tokens, self.dX, self.V, self.scale, 1, self.dtable, self.ws)

    def update(self, lr, clip=1.0):
        """One optimizer step of everything, the dense part's gradient clipped at norm `clip` without leaving the device."""
        self.step += 1
        norm = torch.stack([g.square().sum() for g in (self.dtable, self.dWr, self.db)]).sum().sqrt()
        factor = (clip / (norm + 1e-6)).clamp(max=1.0).reshape(1)
        hp, _ = Hn.make_adam(lr=lr, step=self.step)
        symi.symi_adamw_step(self.ctx, self.opt, hp, factor, 1)
        self.layer.optimizer(hp)
        self.layer.advance()


def train(iterations=60, epochs=4, V=61, seed=0, lr=3e-3, say=print):
    """Mean reward of every iteration's samples."""
    c = wl.scaled(wl.get_config("c1"), T=1024)
    policy = Policy(c, V, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    hp = symi.SymiPolicy.make(clip_low=0.2, clip_high=0.3, kl_coef=0.01, dtype="f32")
    ctx, rewards = policy.ctx, []
    logp_old, logp, stats = torch.empty(c.T, device="cuda"), torch.empty(c.T, device="cuda"), torch.empty(4, device="cuda")
    ws = torch.empty(symi.symi_policy_workspace_bytes(ctx), dtype=torch.uint8, device="cuda")
    for it in range(iterations):
        tokens = torch.randint(0, V, (c.T,), generator=g, device="cuda", dtype=torch.int32)
        real = torch.rand(c.T, generator=g, device="cuda") > 0.05
        tokens = torch.where(real, tokens, -1)                       # padding: no embedding, no loss
        logits = policy.forward(tokens)
        answer = torch.multinomial(torch.softmax(logits, 1), 1, generator=g)[:, 0].to(torch.int32)
        weight = real / real.sum()
        symi.symi_token_logp(ctx, hp, logits, V, V, answer, weight, logp_old)
        reward = (answer == (tokens * 7 + 3) % V).float()
        mean = (reward * weight).sum()
        advantage = (reward - mean) / (mean * (1 - mean)).sqrt().clamp(min=0.05)
        for _ in range(epochs):
            logits = policy.forward(tokens)
            symi.symi_policy_loss(ctx, hp, logits, V, V, answer, logp_old, logp_old, advantage, weight, logp, stats, logits, ws)
            policy.backward(tokens, logits)
            policy.update(lr)
        rewards.append(mean.item())
        if say and (it % 10 == 0 or it == iterations - 1):
            loss, _, kl, clipped = stats.tolist()
            say(f"iteration {it:3d}: reward {rewards[-1]:.3f}  loss {loss:+.4f}  kl {kl:.4f}  clipped {clipped:.2f}", flush=True)
    return rewards


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--iterations", type=int, default=60)
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args()
    train(a.iterations, seed=a.seed)
