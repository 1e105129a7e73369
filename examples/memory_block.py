"""A memory block as a policy's core would use it: trained over trajectories, then stepped on a table of states.

    python examples/memory_block.py [--steps 150] [--mixer linear|delta] [--max-norm 4.0]

The block is  x -> norm -> q, k, v, gate -> linear attention -> norm per head, gated -> projection
                -> norm, scale, residual stream, norm -> gated feed-forward -> norm, scale, residual stream,
with the operators of paper_2006_11751_amd/memory.py and two matrix products of its own.  With --mixer delta the gated delta rule stands
in the place of linear attention: queries and keys are brought to unit length by a norm over the heads, and a small product in fp32
gives each step its decay and writing strength.  The gradients' global norm is clipped as the paper's learner does.  The task needs a memory: the first
observation of an episode shows a cue, all others are noise, and the cue is asked for at every step.  Episodes end inside
the trajectories.  After training the same block is stepped one observation at a time, its states in the rows of a table
that environment ids name, and has to give what the pass over the trajectory gave.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2006_11751_amd import memory  # noqa: E402

CUES = 8


class MemoryBlock:
    """Parameters in fp32 (`p`), computed with in bf16; norm weights and residual scales stay fp32."""

    def __init__(self, D=128, H=4, d=32, F=256, seed=0, device="cuda", mixer="linear"):
        g = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=device) / s[-1] ** 0.5
        one = lambda n, v=1.0: torch.full((n,), v, device=device)
        self.H, self.d, self.D = H, d, D
        self.p = dict(w_in=r(4 * H * d, D), w_out=r(D, H * d), w_gate=r(F, D), w_up=r(F, D), w_down=r(D, F), head=r(CUES, D),
                      norm_in=one(D), norm_o=one(H * d), norm_b=one(D), scale_b=one(D, 0.5), norm_f_in=one(D), norm_f=one(D),
                      scale_f=one(D, 0.5))
        self.mixer = mixer
        if mixer == "delta":  # of each step and head: what is added to the decay's and the strength's argument
            self.p.update(w_step=r(2 * H, D))
        # memories of 4 .. 256 steps
        self.log_decay = -1.0 / (4.0 * 64.0 ** (torch.arange(H, device=device) / max(1, H - 1)))

    def weights(self):
        return {k: (v.bfloat16() if v.dim() == 2 else v) for k, v in self.p.items()}

    def _project(self, w, x):
        """The norm, and q, k, v and the gate as views of one product."""
        n = memory.residual_norm(x, post="none", pre="rms", pre_w=w["norm_in"])["n"]
        z = (n.flatten(0, -2) @ w["w_in"].T).unflatten(0, x.shape[:-1])
        parts = z.split(self.H * self.d, -1)
        heads = lambda a: a.unflatten(-1, (self.H, self.d))
        if self.mixer == "linear":
            return n, [heads(a) for a in parts[:3]], parts[3]
        qk = z[..., :2 * self.H * self.d]
        q, k = self._unit(qk).split(self.H * self.d, -1)
        step = (n.flatten(0, -2).float() @ w["w_step"].float().T).unflatten(0, x.shape[:-1])
        a, b = step.split(self.H, -1)
        # decays of exp(log_decay 2 sigmoid(a)), strengths of sigmoid(b)
        return n, (heads(q), heads(k), heads(parts[2]), (2.0 * self.log_decay * torch.sigmoid(a)).contiguous(), torch.sigmoid(b).contiguous(), qk), parts[3]

    def _unit(self, qk):
        """Every head's query and key at unit length."""
        return memory.residual_norm(qk, post="rms", scale=self._size(), groups=2 * self.H, pre="none")["y"]

    def _size(self):
        return torch.full((2 * self.H * self.d,), self.d ** -0.5, device=self.log_decay.device)

    def _behind(self, w, x, o, gate):
        """What follows the attention: the arrays that the backward pass wants, the block's result last."""
        o = o.flatten(-2)
        a = memory.residual_norm(o, gate=gate, gate_act="silu", post="rms", post_w=w["norm_o"], groups=self.H, pre="none")["y"]
        b = (a.flatten(0, -2) @ w["w_out"].T).view(x.shape)
        r = memory.residual_norm(b, x=x, post="rms", post_w=w["norm_b"], scale=w["scale_b"], pre="rms", pre_w=w["norm_f_in"])
        f = memory.gated_ffn(r["n"], w["w_gate"], w["w_up"], w["w_down"])["y"]
        y = memory.residual_norm(f, x=r["y"], post="rms", post_w=w["norm_f"], scale=w["scale_f"], pre="none")["y"]
        return o, a, b, r["y"], r["n"], f, y

    def unroll(self, w, x, done, state0):
        """x [T,N,D] -> y [T,N,D], the state behind the last step, and what the backward pass wants."""
        n, mix, gate = self._project(w, x)
        if self.mixer == "linear":
            r = memory.linear_attention(*mix, self.log_decay, done=done, state0=state0)
        else:
            r = memory.delta_rule(*mix[:5], done=done, state0=state0)
        rest = self._behind(w, x, r["o"], gate)
        return rest[-1], r["state"], (x, done, state0, n, mix, gate) + rest

    def backward(self, w, kept, dy):
        """Gradients of the parameters, given that of y."""
        x, done, state0, n, mix, gate, o, a, b, y1, n1, f, _ = kept
        flat = lambda t: t.flatten(0, -2)
        last = memory.residual_norm_backward(f, dy, x=y1, post="rms", post_w=w["norm_f"], scale=w["scale_f"], pre="none")
        ffn = memory.gated_ffn_backward(n1, w["w_gate"], w["w_up"], w["w_down"], last["db"])
        mid = memory.residual_norm_backward(b, last["dx"], ffn["dx"], x=x, post="rms", post_w=w["norm_b"], scale=w["scale_b"], pre="rms",
                                            pre_w=w["norm_f_in"])
        db = flat(mid["db"])
        head = memory.residual_norm_backward(o, (db @ w["w_out"]).view(a.shape), gate=gate, gate_act="silu", post="rms", post_w=w["norm_o"],
                                             groups=self.H, pre="none")
        do, more = head["db"].unflatten(-1, (self.H, self.d)), {}
        if self.mixer == "linear":
            att = memory.linear_attention_backward(*mix, self.log_decay, do, done=done, state0=state0)
            dqk, dn = [att["dq"].flatten(-2), att["dk"].flatten(-2)], 0.0
        else:
            q, k, v, log_decay, beta, qk = mix
            att = memory.delta_rule_backward(q, k, v, log_decay, beta, do, done=done, state0=state0)
            dunit = torch.cat([att["dq"].flatten(-2), att["dk"].flatten(-2)], -1)
            dqk = [memory.residual_norm_backward(qk, dunit, post="rms", scale=self._size(), groups=2 * self.H, pre="none")["db"]]
            half = log_decay / (2.0 * self.log_decay)  # sigmoid(a)
            dstep = flat(torch.cat([att["dlog_decay"] * log_decay * (1.0 - half), att["dbeta"] * beta * (1.0 - beta)], -1))
            more, dn = dict(w_step=dstep.T @ flat(n).float()), dstep @ w["w_step"].float()
        dz = flat(torch.cat(dqk + [att["dv"].flatten(-2), head["dgate"]], -1))
        first = memory.residual_norm_backward(x, None, (dz @ w["w_in"] + dn).to(x.dtype).view(x.shape), post="none", pre="rms", pre_w=w["norm_in"])
        return dict(more, w_in=dz.T @ flat(n), w_out=db.T @ flat(a), w_gate=ffn["dw_gate"], w_up=ffn["dw_up"], w_down=ffn["dw_down"],
                    norm_in=first["dpre_w"], norm_o=head["dpost_w"], norm_b=mid["dpost_w"], scale_b=mid["dscale"], norm_f_in=mid["dpre_w"],
                    norm_f=last["dpost_w"], scale_f=last["dscale"])

    def step(self, w, x, table, env_ids, done):
        """One observation of B environments, x [B,D]; their states are rows env_ids of the table."""
        _, mix, gate = self._project(w, x)
        if self.mixer == "linear":
            o = memory.linear_attention_step(*mix, self.log_decay, table, env_ids=env_ids, done=done)["o"]
        else:
            o = memory.delta_rule_step(*mix[:5], table, env_ids=env_ids, done=done)["o"]
        return self._behind(w, x, o, gate)[-1]


def trajectories(T, N, D, p_done, g, device="cuda"):
    """Observations bf16 [T,N,D], marks of first steps u8 [T,N], and the cue that each step's episode began with [T,N]."""
    done = torch.rand(T, N, generator=g, device=device) < p_done
    done[0] = True
    drawn = torch.randint(0, CUES, (T, N), generator=g, device=device)
    begin = torch.where(done, torch.arange(T, device=device)[:, None], 0).cummax(0).values
    cue = drawn.gather(0, begin)
    x = 0.3 * torch.randn(T, N, D, generator=g, device=device)
    x += 3.0 * done[..., None] * torch.nn.functional.one_hot(cue, D)
    return x.bfloat16(), done.byte(), cue


def train(steps, T=48, N=64, D=128, p_done=0.04, lr=3e-3, report=print, mixer="linear", max_norm=None):
    """The losses of `steps` updates, and the block.  max_norm: of all gradients together."""
    block, g = MemoryBlock(D=D, mixer=mixer), torch.Generator(device="cuda").manual_seed(1)
    opt = torch.optim.Adam(block.p.values(), lr=lr)
    losses = []
    for i in range(steps):
        x, done, cue = trajectories(T, N, D, p_done, g)
        w = block.weights()
        y, _, kept = block.unroll(w, x, done, None)
        logits = y.flatten(0, 1).float() @ block.p["head"].T
        prob = torch.softmax(logits, -1)
        losses.append(-torch.log(prob.gather(1, cue.view(-1, 1)) + 1e-9).mean().item())
        dlogits = (prob - torch.nn.functional.one_hot(cue.view(-1), CUES)) / prob.shape[0]
        grads = block.backward(w, kept, (dlogits @ block.p["head"]).bfloat16().view(y.shape))
        grads["head"] = dlogits.T @ y.flatten(0, 1).float()
        if max_norm is not None:
            memory.clip_gradients(list(grads.values()), max_norm)
        for name, p in block.p.items():
            p.grad = grads[name].float()
        opt.step()
        if report and (i % 25 == 0 or i == steps - 1):
            report("update %3d  loss %.3f" % (i, losses[-1]))
    return losses, block


def compare_steps(block, T=40, N=16, D=128):
    """How far steps on a table are from the pass over the trajectory (largest difference over largest value)."""
    g = torch.Generator(device="cuda").manual_seed(2)
    x, done, _ = trajectories(T, N, D, 0.05, g)
    w = block.weights()
    y, state, _ = block.unroll(w, x, done, None)
    table = torch.zeros(3 * N, block.H, block.d, block.d, device="cuda")
    ids = torch.randperm(3 * N, generator=g, device="cuda")[:N].int()
    ys = torch.stack([block.step(w, x[t], table, ids, done[t]) for t in range(T)])
    off = lambda a, b: ((a.float() - b.float()).abs().max() / b.float().abs().max()).item()
    return off(ys, y), off(table[ids.long()], state)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--mixer", choices=("linear", "delta"), default="linear")
    ap.add_argument("--max-norm", type=float, default=4.0)
    args = ap.parse_args()
    losses, block = train(args.steps, mixer=args.mixer, max_norm=args.max_norm)
    print("loss %.3f -> %.3f (chance %.3f)" % (losses[0], losses[-1], torch.log(torch.tensor(float(CUES)))))
    print("stepped against unrolled: outputs %.2g, states %.2g" % compare_steps(block))


if __name__ == "__main__":
    main()
