"""One policy-training step of a small token model, as a sequence of calls into the C-ABI library.

The model: an embedding; blocks of two products (D -> F with ReLU -> D), each with a norm before it, a norm, a gate
vector and a scaled residual sum after it; an output product over the vocabulary.  The step: log-probabilities of
the tokens that were drawn, clipped policy loss with a KL term, backward pass with the loss scale folded in,
AdamW on the FP32 master (moments in 32 or in 8 bits), loss-scale state machine.  Like the stack of linear layers this
module only owns device buffers and orders the calls; nothing returns to the host inside a step, and a step can
be recorded into a CUDA graph.

    python -m paper_1805_10387_b200.token_model [--steps 50] [--state-bits 8]

trains a model on a toy task (a token is rewarded when it continues a fixed cycle) and prints how the reward moves.
"""
from __future__ import annotations

import math

import torch

from . import mp


def _align(n: int, a: int = 8) -> int:
    return (n + a - 1) // a * a


class TokenModel:
    def __init__(self, vocab, width, inner, blocks, tokens, kind=mp.MP_NORM_RMS, eps=1e-6, res_scale=1.0, pad_id=-1,
                 lr=1e-3, beta1=0.9, beta2=0.95, adam_eps=1e-8, weight_decay=0.1, state_bits=32, clip_lo=0.2, clip_hi=0.2,
                 kl_coef=0.0, init_scale=65536.0, growth_interval=1000, seed=0, device="cuda"):
        """tokens: rows of a step (fixed, as the buffers are).  state_bits: 32, or 8 for E4M3 moments."""
        self.V, self.D, self.F, self.L, self.n = vocab, width, inner, blocks, tokens
        self.kind, self.eps, self.res, self.pad_id = kind, eps, res_scale, pad_id
        self.loss_args = dict(clip_lo=clip_lo, clip_hi=clip_hi, kl_coef=kl_coef)
        self.device = torch.device(device)
        self.state = mp.State(init_scale, growth_interval)
        self.opt = mp.AdamWConfig(lr, beta1, beta2, adam_eps, weight_decay)
        g = torch.Generator().manual_seed(seed)
        V, D, F = vocab, width, inner
        # name -> (rows, columns, standard deviation, mean); a vector has one row.  Vectors do not decay.
        spec = {"embed": (V, D, D ** -0.5, 0.0), "out": (D, V, D ** -0.5, 0.0), "gain0": (1, D, 0.0, 1.0)}
        for l in range(blocks):
            spec.update({f"w1.{l}": (D, F, D ** -0.5, 0.0), f"w2.{l}": (F, D, F ** -0.5, 0.0),
                         f"post{l}": (1, D, 0.0, 1.0), f"gate{l}": (1, D, 0.0, 0.5), f"gain{l + 1}": (1, D, 0.0, 1.0)})
        f16 = dict(dtype=torch.float16, device=self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.w32, self.w16, self.dw = {}, {}, {}
        flat = {k: [] for k in ("g", "w", "m", "v", "w16", "ms", "vs")}
        for name, (r, c, std, mean) in spec.items():
            full = torch.zeros(r, _align(c))             # rows start on 16-byte boundaries; the padding stays 0
            full[:, :c] = torch.randn(r, c, generator=g) * std + mean
            w32, size = full.to(self.device), full.numel()
            w16, dw = w32.half(), torch.zeros(r, _align(c), **f16)
            view = (lambda t: t[0, :c]) if r == 1 else (lambda t: t[:, :c])
            self.w32[name], self.w16[name], self.dw[name] = view(w32), view(w16), view(dw)
            if state_bits == 32:
                m, v = torch.zeros(size, **f32), torch.zeros(size, **f32)
            else:
                m, v = (torch.zeros(size, dtype=torch.uint8, device=self.device).view(torch.float8_e4m3fn) for _ in "mv")
                n_scales = -(-size // mp.MP_ADAMW_BLOCK)
                flat["ms"].append(torch.zeros(n_scales, **f32))
                flat["vs"].append(torch.zeros(n_scales, **f32))
            for k, t in (("g", dw), ("w", w32), ("m", m), ("v", v), ("w16", w16)):
                flat[k].append(t.view(-1))
        self.flat = flat
        self.plan = mp.AdamWPlan(flat["g"], flat["w"], flat["m"], flat["v"], flat["w16"],
                                 flat["ms"] or None, flat["vs"] or None,
                                 decay=[0.0 if r == 1 else 1.0 for r, _, _, _ in spec.values()])
        n = tokens
        buf = lambda c: torch.zeros(n, _align(c), **f16)[:, :c]  # noqa: E731
        self.x = [buf(D) for _ in range(blocks + 1)]             # the residual stream before each block and after the last
        self.nx = [buf(D) for _ in range(blocks + 1)]            # its norms: the blocks' inputs, the output product's
        self.stats = [torch.zeros(n, 4, **f32) for _ in range(blocks + 1)]
        self.act, self.y = [buf(F) for _ in range(blocks)], [buf(D) for _ in range(blocks)]
        self.logits = buf(V)
        self.dx, self.dn, self.dact = buf(D), buf(D), buf(F)
        self.logp, self.token_loss = torch.zeros(n, **f32), torch.zeros(n, **f32)
        self.loss = torch.zeros(1, **f32)
        need = max([mp.mp_embedding_bwd_workspace_bytes(n, V, D), mp.mp_block_norm_bwd_workspace_bytes(n, D)] +
                   [mp.mp_gemm_workspace_bytes(n, k, c, op) for k, c in ((D, F), (F, D), (D, V))
                    for op in (mp.MP_OP_FWD, mp.MP_OP_DGRAD, mp.MP_OP_WGRAD)])
        self.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=self.device)

    # ---- the calls of a step ----
    def forward(self, ids):
        """ids [tokens] -> self.logits."""
        w, ws = self.w16, self.workspace
        mp.mp_embedding_fwd(ids, w["embed"], self.x[0], self.pad_id, math.sqrt(self.D), self.state)
        mp.mp_block_norm_fwd(self.x[0], w["gain0"], self.nx[0], self.stats[0], kind=self.kind, eps=self.eps)
        for l in range(self.L):
            mp.mp_linear_fwd_act(self.nx[l], w[f"w1.{l}"], None, self.act[l], mp.MP_ACT_RELU, workspace=ws)
            mp.mp_linear_fwd(self.act[l], w[f"w2.{l}"], self.y[l], ws)
            mp.mp_block_norm_fwd(self.x[l], w[f"gain{l + 1}"], self.nx[l + 1], self.stats[l + 1], self.y[l], w[f"post{l}"],
                                 w[f"gate{l}"], self.x[l + 1], self.kind, self.eps, self.res)
        mp.mp_linear_fwd(self.nx[self.L], w["out"], self.logits, ws)

    def log_probs(self, ids, targets, out):
        """out[i] = log-probability of targets[i] after ids[i], under the present weights."""
        self.forward(ids)
        mp.mp_token_logp(self.logits, targets, out, state=self.state)

    def backward(self, ids):
        """From the gradient that the loss left in the logits' place to the gradients of all weights."""
        w, dw, ws, st = self.w16, self.dw, self.workspace, self.state
        mp.mp_linear_bwd_wgrad(self.nx[self.L], self.logits, dw["out"], st, ws)
        mp.mp_linear_bwd_dgrad(self.logits, w["out"], self.dn, ws)
        above = None                                             # gradient that reaches x[l + 1] past its norm
        for l in reversed(range(self.L)):
            mp.mp_block_norm_bwd(self.dn, self.x[l + 1], w[f"gain{l + 1}"], self.stats[l + 1], self.dx, dw[f"gain{l + 1}"],
                                 above, self.y[l], w[f"post{l}"], w[f"gate{l}"], self.dn, dw[f"post{l}"], dw[f"gate{l}"],
                                 self.kind, self.res, st, ws)    # the gradient at y takes the place of that at n
            above = self.dx
            mp.mp_linear_bwd_wgrad(self.act[l], self.dn, dw[f"w2.{l}"], st, ws)
            mp.mp_linear_bwd_dgrad_act(self.dn, w[f"w2.{l}"], self.act[l], self.dact, mp.MP_ACT_RELU, workspace=ws)
            mp.mp_linear_bwd_wgrad(self.nx[l], self.dact, dw[f"w1.{l}"], st, ws)
            mp.mp_linear_bwd_dgrad(self.dact, w[f"w1.{l}"], self.dn, ws)
        mp.mp_block_norm_bwd(self.dn, self.x[0], w["gain0"], self.stats[0], self.dx, dw["gain0"], above, kind=self.kind,
                             state=st, workspace=ws)
        mp.mp_embedding_bwd(ids, self.dx, dw["embed"], self.pad_id, math.sqrt(self.D), st, ws)

    def gradients(self, ids, targets, old_logp, advantage, weight, ref_logp=None):
        self.forward(ids)
        mp.mp_policy_loss(self.logits, targets, old_logp, advantage, weight, self.logp, self.token_loss, self.loss,
                          self.logits, ref_logp, state=self.state, **self.loss_args)
        self.backward(ids)

    def step(self, ids, targets, old_logp, advantage, weight, ref_logp=None):
        """ids, targets [tokens] int32 or int64; the others [tokens] FP32.  weight: 0 for masked tokens, most often
        1 / (number of the others).  Padding tokens are masked too: their rows are zero throughout, and a
        gradient through the norms of zero rows grows by 1 / sqrt(eps) each, past what FP16 holds."""
        self.gradients(ids, targets, old_logp, advantage, weight, ref_logp)
        mp.mp_adamw_update(self.plan, self.state, self.opt)
        mp.mp_loss_scale_update(self.state)

    def capture(self, *args):
        """Records step(*args) into a CUDA graph that runs it with whatever the tensors hold then.  One real step
        comes first (the library's one-time set-up must not fall inside the capture)."""
        side = torch.cuda.Stream(device=self.device)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.step(*args)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self.step(*args)
        return graph

    def close(self):
        self.plan.close()
        self.state.close()


def demo(steps=50, state_bits=8, vocab=101, width=64, inner=256, blocks=2, tokens=2048, seed=0):
    """Policy gradient on a toy task: token t is rewarded when it is followed by (7 t + 3) mod vocab.  Returns the mean
    probability of the rewarded token before and after."""
    model = TokenModel(vocab, width, inner, blocks, tokens, lr=1e-2, weight_decay=0.0, kl_coef=0.0, state_bits=state_bits,
                       init_scale=1024.0, seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    ids = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    right = (7 * ids + 3) % vocab
    weight = torch.full((tokens,), 1.0 / tokens, device="cuda")
    old, best = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")

    def reward():
        model.log_probs(ids, right, best)
        return best.exp().mean().item()
    before = reward()
    for i in range(steps):
        # half of the tokens try the rewarded continuation, the others a random one
        tried = torch.where(torch.rand(tokens, generator=g, device="cuda") < 0.5, right,
                            torch.randint(0, vocab, (tokens,), generator=g, device="cuda"))
        model.log_probs(ids, tried, old)
        advantage = torch.where(tried == right, 1.0, -0.1)
        model.step(ids, tried, old, advantage, weight)
        if i % 10 == 9:
            print(f"step {i + 1}: probability of the rewarded token {reward():.3f}, S {model.state.read().scale:.0f}")
    after = reward()
    model.close()
    return before, after


if __name__ == "__main__":
    import argparse
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    b, e = demo(a.steps, a.state_bits)
    print(f"mean probability of the rewarded token: {b:.4f} -> {e:.4f}")
