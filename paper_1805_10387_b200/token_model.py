"""One training step of a small token model, as a sequence of calls into the C-ABI library.

The model: an embedding; blocks of two products (D -> F with ReLU -> D), each with a norm before it, a norm, a gate
vector and a scaled residual sum after it; an output product over the vocabulary.  With `heads` every block begins with
attention in the same manner: a product for queries, keys and values, norms of queries and keys for each head with the position
rotation, attention over the packed sequences, a product back.  The step: log-probabilities of
the tokens that were drawn, clipped policy loss with a KL term (or distillation from a teacher's top entries), backward
pass with the loss scale folded in, AdamW on the FP32 master (moments in 32 or in 8 bits), loss-scale state
machine.  Like the stack of linear layers this module only owns device buffers and orders the calls; nothing
returns to the host inside a step, and a step can be recorded into a CUDA graph.

    python -m paper_1805_10387_b200.token_model [--steps 50] [--state-bits 8] [--distill]

trains a model on a toy task (a token is rewarded when it continues a fixed cycle) and prints how the reward moves;
with --distill a model with attention then learns from that one's top alternatives.
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
                 kl_coef=0.0, init_scale=65536.0, growth_interval=1000, seed=0, device="cuda", heads=0, kv_heads=None,
                 head_dim=64, window=0, rope_base=10000.0, sequences=1):
        """tokens: rows of a step (fixed, as the buffers are).  state_bits: 32, or 8 for E4M3 moments.  heads: query heads of
        head_dim elements (a multiple of 8, at most mp.MP_ATTENTION_MAX_D), kv_heads of keys and values (None: as many; 0 heads: no
        attention), of which a query sees the last `window` (0: all) of its sequence; sequences: how many a step's rows are packed
        from at most (set_sequences)."""
        if heads:
            kv = heads if kv_heads is None else kv_heads
            if heads < 0 or kv <= 0 or heads % kv or window < 0 or sequences < 1:
                raise ValueError(f"expected key heads that divide the query heads, a window of at least 0 and at least one sequence, got "
                                 f"{heads} and {kv} heads, a window of {window}, {sequences} sequences")
            if head_dim <= 0 or head_dim % 8 or head_dim > mp.MP_ATTENTION_MAX_D:
                raise ValueError(f"expected heads of a multiple of 8 elements, at most {mp.MP_ATTENTION_MAX_D}, got {head_dim}")
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
        self.hq, self.hk = heads, (heads if kv_heads is None else kv_heads)
        self.hd, self.window = head_dim, window
        q_cols, kv_cols = self.hq * head_dim, self.hk * head_dim
        # what the residual stream passes through: (attention or not, block, norm after it, gate, norm before the next)
        self.subs = []
        for l in range(blocks):
            if heads:
                spec.update({f"qkv.{l}": (D, q_cols + 2 * kv_cols, D ** -0.5, 0.0), f"attn_out.{l}": (q_cols, D, q_cols ** -0.5, 0.0),
                             f"gq{l}": (1, head_dim, 0.0, 1.0), f"gk{l}": (1, head_dim, 0.0, 1.0), f"apost{l}": (1, D, 0.0, 1.0),
                             f"agate{l}": (1, D, 0.0, 0.5), f"again{l}": (1, D, 0.0, 1.0)})
                self.subs.append((True, l, f"apost{l}", f"agate{l}", f"again{l}"))
            self.subs.append((False, l, f"post{l}", f"gate{l}", f"gain{l + 1}"))
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
        subs = len(self.subs)
        self.x = [buf(D) for _ in range(subs + 1)]               # the residual stream before each of them and after the last
        self.nx = [buf(D) for _ in range(subs + 1)]              # its norms: their inputs, the output product's
        self.stats = [torch.zeros(n, 4, **f32) for _ in range(subs + 1)]
        self.act, self.y = [buf(F) for _ in range(blocks)], [buf(D) for _ in range(subs)]
        if heads:
            self.qk_cols, self.q_cols = q_cols + kv_cols, q_cols
            self.qkv, self.qk = [buf(q_cols + 2 * kv_cols) for _ in range(blocks)], [buf(q_cols + kv_cols) for _ in range(blocks)]
            self.o, self.lse = [buf(q_cols) for _ in range(blocks)], [torch.zeros(heads, n, **f32) for _ in range(blocks)]
            self.do, self.dqk, self.dqkv = buf(q_cols), buf(q_cols + kv_cols), buf(q_cols + 2 * kv_cols)
            rot = head_dim // 16 * 16
            self.freqs = rope_base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=self.device) / max(rot, 1)) if rot else None
            self.positions = torch.zeros(n, dtype=torch.int32, device=self.device)
            self.offsets = torch.zeros(sequences + 1, dtype=torch.int32, device=self.device)
            self.set_sequences([n])
        self.logits = buf(V)
        self.dx, self.dn, self.dact = buf(D), buf(D), buf(F)
        self.logp, self.token_loss = torch.zeros(n, **f32), torch.zeros(n, **f32)
        self.loss = torch.zeros(1, **f32)
        need = max([mp.mp_embedding_bwd_workspace_bytes(n, V, D), mp.mp_block_norm_bwd_workspace_bytes(n, D)] +
                   [mp.mp_gemm_workspace_bytes(n, k, c, op) for k, c in ((D, F), (F, D), (D, V))
                    for op in (mp.MP_OP_FWD, mp.MP_OP_DGRAD, mp.MP_OP_WGRAD)])
        if heads:
            need = max([need, mp.mp_head_norm_rope_bwd_workspace_bytes(n, self.hq, self.hk, head_dim),
                        mp.mp_attention_bwd_workspace_bytes(n, self.hq, self.hk, head_dim)] +
                       [mp.mp_gemm_workspace_bytes(n, k, c, op) for k, c in ((D, q_cols + 2 * kv_cols), (q_cols, D))
                        for op in (mp.MP_OP_FWD, mp.MP_OP_DGRAD, mp.MP_OP_WGRAD)])
        self.workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=self.device)

    def set_sequences(self, lengths):
        """How the rows of the next steps are packed: lengths of sequences that follow one another (padding rows as a sequence
        of their own).  Kept on the device, so a recorded step follows."""
        if sum(lengths) != self.n or min(lengths) < 0 or len(lengths) > self.offsets.shape[0] - 1:
            raise ValueError(f"expected at most {self.offsets.shape[0] - 1} lengths with the sum {self.n}, got {lengths}")
        at, where = [0], []
        for k in lengths:
            at.append(at[-1] + k)
            where += range(k)
        at += [self.n] * (self.offsets.shape[0] - len(at))
        self.offsets.copy_(torch.tensor(at, dtype=torch.int32))
        self.positions.copy_(torch.tensor(where, dtype=torch.int32))

    # ---- the calls of a step ----
    def _attend(self, i, l):
        """nx[i] -> y[i] through block l's attention."""
        w, ws, qkv, qk, c = self.w16, self.workspace, self.qkv[l], self.qk[l], self.q_cols
        mp.mp_linear_fwd(self.nx[i], w[f"qkv.{l}"], qkv, ws)
        mp.mp_head_norm_rope_fwd(qkv[:, :self.qk_cols], w[f"gq{l}"], w[f"gk{l}"], self.positions, self.freqs, qk, self.hq, self.hk,
                                 self.eps)
        mp.mp_attention_fwd(qk[:, :c], qk[:, c:], qkv[:, self.qk_cols:], self.o[l], self.lse[l], self.offsets, self.hq, self.hk,
                            window=self.window, state=self.state)
        mp.mp_linear_fwd(self.o[l], w[f"attn_out.{l}"], self.y[i], ws)

    def _attend_backward(self, i, l):
        """The gradient at y[i], in dn, to the one at nx[i], in its place."""
        w, dw, ws, st = self.w16, self.dw, self.workspace, self.state
        qkv, qk, c, k = self.qkv[l], self.qk[l], self.q_cols, self.qk_cols
        mp.mp_linear_bwd_wgrad(self.o[l], self.dn, dw[f"attn_out.{l}"], st, ws)
        mp.mp_linear_bwd_dgrad(self.dn, w[f"attn_out.{l}"], self.do, ws)
        mp.mp_attention_bwd(self.do, qk[:, :c], qk[:, c:], qkv[:, k:], self.o[l], self.lse[l], self.dqk[:, :c], self.dqk[:, c:],
                            self.dqkv[:, k:], self.offsets, self.hq, self.hk, window=self.window, state=st, workspace=ws)
        mp.mp_head_norm_rope_bwd(self.dqk, qkv[:, :k], w[f"gq{l}"], w[f"gk{l}"], self.positions, self.freqs, self.dqkv[:, :k],
                                 dw[f"gq{l}"], dw[f"gk{l}"], self.hq, self.hk, self.eps, state=st, workspace=ws)
        mp.mp_linear_bwd_wgrad(self.nx[i], self.dqkv, dw[f"qkv.{l}"], st, ws)
        mp.mp_linear_bwd_dgrad(self.dqkv, w[f"qkv.{l}"], self.dn, ws)

    def forward(self, ids):
        """ids [tokens] -> self.logits."""
        w, ws = self.w16, self.workspace
        mp.mp_embedding_fwd(ids, w["embed"], self.x[0], self.pad_id, math.sqrt(self.D), self.state)
        mp.mp_block_norm_fwd(self.x[0], w["gain0"], self.nx[0], self.stats[0], kind=self.kind, eps=self.eps)
        for i, (attends, l, post, gate, gain) in enumerate(self.subs):
            if attends:
                self._attend(i, l)
            else:
                mp.mp_linear_fwd_act(self.nx[i], w[f"w1.{l}"], None, self.act[l], mp.MP_ACT_RELU, workspace=ws)
                mp.mp_linear_fwd(self.act[l], w[f"w2.{l}"], self.y[i], ws)
            mp.mp_block_norm_fwd(self.x[i], w[gain], self.nx[i + 1], self.stats[i + 1], self.y[i], w[post], w[gate],
                                 self.x[i + 1], self.kind, self.eps, self.res)
        mp.mp_linear_fwd(self.nx[-1], w["out"], self.logits, ws)

    def log_probs(self, ids, targets, out):
        """out[i] = log-probability of targets[i] after ids[i], under the present weights."""
        self.forward(ids)
        mp.mp_token_logp(self.logits, targets, out, state=self.state)

    def top(self, ids, top_ids, top_logp, targets=None, logp=None, entropy=None, weight=None, temperature=1.0):
        """The likeliest next tokens after each of ids and their log-probabilities [tokens, k], the entropies, and the
        log-probabilities of targets: what a student's step takes, and what a policy run keeps an eye on."""
        self.forward(ids)
        mp.mp_token_top(self.logits, top_ids, top_logp, targets, logp, entropy, weight, temperature, self.state)

    def backward(self, ids):
        """From the gradient that the loss left in the logits' place to the gradients of all weights."""
        w, dw, ws, st = self.w16, self.dw, self.workspace, self.state
        mp.mp_linear_bwd_wgrad(self.nx[-1], self.logits, dw["out"], st, ws)
        mp.mp_linear_bwd_dgrad(self.logits, w["out"], self.dn, ws)
        above = None                                             # gradient that reaches x[i + 1] past its norm
        for i, (attends, l, post, gate, gain) in reversed(list(enumerate(self.subs))):
            mp.mp_block_norm_bwd(self.dn, self.x[i + 1], w[gain], self.stats[i + 1], self.dx, dw[gain],
                                 above, self.y[i], w[post], w[gate], self.dn, dw[post], dw[gate],
                                 self.kind, self.res, st, ws)    # the gradient at y takes the place of that at n
            above = self.dx
            if attends:
                self._attend_backward(i, l)
                continue
            mp.mp_linear_bwd_wgrad(self.act[l], self.dn, dw[f"w2.{l}"], st, ws)
            mp.mp_linear_bwd_dgrad_act(self.dn, w[f"w2.{l}"], self.act[l], self.dact, mp.MP_ACT_RELU, workspace=ws)
            mp.mp_linear_bwd_wgrad(self.nx[i], self.dact, dw[f"w1.{l}"], st, ws)
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

    def distill_gradients(self, ids, teacher_ids, teacher_logp, weight, temperature=1.0, tail=True):
        self.forward(ids)
        mp.mp_distill_loss(self.logits, teacher_ids, teacher_logp, weight, self.token_loss, self.loss, self.logits, temperature,
                           tail, state=self.state)
        self.backward(ids)

    def distill_step(self, ids, teacher_ids, teacher_logp, weight, temperature=1.0, tail=True):
        """A step towards a teacher's top entries [tokens, K] (its `top` at the same temperature); weight as in step."""
        self.distill_gradients(ids, teacher_ids, teacher_logp, weight, temperature, tail)
        mp.mp_adamw_update(self.plan, self.state, self.opt)
        mp.mp_loss_scale_update(self.state)

    def capture(self, *args, step=None):
        """Records step(*args) (or another step of this model) into a CUDA graph that runs it with whatever the tensors
        hold then.  One real step comes first (the library's one-time set-up must not fall inside the capture)."""
        step = self.step if step is None else step
        side = torch.cuda.Stream(device=self.device)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*args)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*args)
        return graph

    def close(self):
        self.plan.close()
        self.state.close()


def demo(steps=50, state_bits=8, vocab=101, width=64, inner=256, blocks=2, tokens=2048, seed=0, keep=False):
    """Policy gradient on a toy task: token t is rewarded when it is followed by (7 t + 3) mod vocab.  Returns the mean
    probability of the rewarded token before and after (and the model, if it is to be kept)."""
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
    if keep:
        return before, after, model
    model.close()
    return before, after


def demo_distill(teacher, steps=50, state_bits=8, k=8, length=256, seed=1):
    """A smaller model with attention learns from the teacher's top k alternatives, with the rest as one more outcome, over
    packed sequences of random tokens.  Returns the mean divergence of the first and of the last step."""
    n, V = teacher.n, teacher.V
    student = TokenModel(V, 32, 64, 1, n, lr=1e-2, weight_decay=0.0, state_bits=state_bits, init_scale=1024.0, seed=seed,
                         heads=2, kv_heads=1, head_dim=32, sequences=-(-n // length))
    student.set_sequences([length] * (n // length) + ([n % length] if n % length else []))
    g = torch.Generator(device="cuda").manual_seed(seed)
    weight = torch.full((n,), 1.0 / n, device="cuda")
    top_ids = torch.empty(n, k, dtype=torch.int32, device="cuda")
    top_logp, entropy = torch.empty(n, k, device="cuda"), torch.empty(n, device="cuda")
    losses = []
    for i in range(steps):
        ids = torch.randint(0, V, (n,), generator=g, device="cuda")
        teacher.top(ids, top_ids, top_logp, entropy=entropy)
        student.distill_step(ids, top_ids, top_logp, weight)
        if i in (0, steps - 1) or i % 10 == 9:
            losses.append(student.loss.item())
            print(f"step {i + 1}: divergence from the teacher {losses[-1]:.4f} (its entropy {entropy.mean().item():.3f})")
    student.close()
    return losses[0], losses[-1]


if __name__ == "__main__":
    import argparse
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--state-bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--distill", action="store_true", help="then train a smaller model with attention from that one's top alternatives")
    a = ap.parse_args()
    b, e, teacher = demo(a.steps, a.state_bits, keep=True)
    print(f"mean probability of the rewarded token: {b:.4f} -> {e:.4f}")
    if a.distill:
        b, e = demo_distill(teacher, a.steps, a.state_bits)
        print(f"mean divergence from the teacher: {b:.4f} -> {e:.4f}")
    teacher.close()
