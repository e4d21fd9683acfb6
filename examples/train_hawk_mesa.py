"""A Hawk layer and a Mesa layer trained together, with 8-bit activation checkpoints.

    python examples/train_hawk_mesa.py [steps]

One block of the paper's Hawk-Mesa hybrid in its smallest form, on one GPU: tokens go through a
gated linear recurrence and then through a Mesa layer, each with its projections (torch matmuls)
and a residual connection, over rows that pack several documents (`reset` marks their starts
for the recurrence).  The task is to name the token seen a few places before.  What the
backward pass needs of the forward is kept in 8 bits (checkpoint_pack, and the recurrence's own
checkpoints); the Mesa layer's inputs are formed again from its projections' checkpoints.  At
the end the trained block decodes tokens one at a time from the states that a prefill leaves,
and the outputs are compared with those of the whole sequence at once.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2506_05233_amd import libmesa as L  # noqa: E402

VOCAB, DIM, WIDTH, HEADS, HEAD = 32, 128, 256, 2, 64
BACK = 3            # the answer at token t is the token at t - BACK
N_CG = 8


class Block:
    """Weights of the block, its forward, its backward from checkpoints, and one decoded token."""

    def __init__(self, device, seed=0):
        gen = torch.Generator().manual_seed(seed)

        def w(*shape, scale):
            return (torch.randn(shape, generator=gen) * scale).to(device)

        d = HEADS * HEAD
        self.p = {"embed": w(VOCAB, DIM, scale=1.0), "hawk_in": w(DIM, 3 * WIDTH, scale=DIM ** -0.5),
                  "theta": w(WIDTH, scale=0.5) - 4.0, "hawk_out": w(WIDTH, DIM, scale=WIDTH ** -0.5),
                  "mesa_in": w(DIM, 3 * d + 2 * HEADS, scale=DIM ** -0.5), "conv_q": w(d, 4, scale=0.5),
                  "conv_k": w(d, 4, scale=0.5), "conv_v": w(d, 4, scale=0.5), "lam": w(HEADS, HEAD, scale=0.5),
                  "norm": torch.ones((HEADS, HEAD), device=device), "mesa_out": w(d, DIM, scale=d ** -0.5),
                  "logits": w(DIM, VOCAB, scale=DIM ** -0.5)}

    def _mesa_inputs(self, proj):
        """The front end's arguments from the projection [B, T, 3 d + 2 H] of a token's features."""
        B, T = proj.shape[:2]
        d = HEADS * HEAD
        qp, kp, vp, gates = proj.split([d, d, d, 2 * HEADS], dim=-1)
        heads = [t.contiguous().view(B, T, HEADS, HEAD) for t in (qp, kp, vp)]
        return heads, (gates[..., :HEADS] + 3.0).contiguous(), gates[..., HEADS:].contiguous()

    def _front(self, heads, a_gamma, a_beta):
        p = self.p
        return L.frontend(*heads, p["conv_q"], p["conv_k"], p["conv_v"], a_gamma, a_beta, p["lam"])

    def forward(self, tokens, reset, keep=True):
        """Logits [B, T, VOCAB] and, with keep, what the backward pass needs."""
        p, B, T = self.p, *tokens.shape
        e = p["embed"][tokens]
        x, r, i = (e @ p["hawk_in"]).split(WIDTH, dim=-1)
        rec = L.recurrence(x, r, i, p["theta"], reset=reset, want_final=True, want_states=keep, want_checkpoints=keep)
        z = e + rec["y"] @ p["hawk_out"]
        heads, a_gamma, a_beta = self._mesa_inputs(z @ p["mesa_in"])
        f = self._front(heads, a_gamma, a_beta)
        fw = L.forward(f["q"], f["k"], f["v"], f["gamma"], f["beta"], f["lam"], N_CG, want_qstar=True, want_states=True)
        y = L.output_norm(fw["out"], p["norm"], out_dtype=torch.float32).view(B, T, HEADS * HEAD)
        out = z + y @ p["mesa_out"]
        logits = out @ p["logits"]
        if not keep:
            return logits, {"h": rec["h"], "H": fw["H"], "G": fw["G"], "heads": heads}
        # the projections as the front end's gradients take them: a token's heads in one row
        qp, kp, vp = (t.view(B, T, HEADS * HEAD) for t in heads)
        kept = {n: L.checkpoint_pack(t) for n, t in (("z", z), ("y", y), ("out", out), ("rec_y", rec["y"]), ("o", fw["out"]),
                                                    ("qstar", fw["qstar"]), ("qp", qp), ("kp", kp), ("vp", vp))}
        kept.update(tokens=tokens, reset=reset, states=rec["states"], x=rec["x"], r=rec["r"], i=rec["i"], a_gamma=a_gamma, a_beta=a_beta)
        return logits, kept

    def backward(self, kept, dlogits):
        """Gradients of every weight, from the checkpoints."""
        p, g = self.p, {}
        B, T = kept["tokens"].shape

        def value(n):
            return L.checkpoint_unpack(kept[n], torch.float32)

        def weight(a, da):
            return a.reshape(-1, a.shape[-1]).T @ da.reshape(-1, da.shape[-1])

        g["logits"] = weight(value("out"), dlogits)
        dz = dlogits @ p["logits"].T                                   # through the residual
        g["mesa_out"] = weight(value("y"), dz)
        dy = (dz @ p["mesa_out"].T).view(B, T, HEADS, HEAD)
        norm = L.output_norm_backward(kept["o"], p["norm"], dy)
        g["norm"] = norm["dweight"]
        heads = [value(n).view(B, T, HEADS, HEAD) for n in ("qp", "kp", "vp")]
        f = self._front(heads, kept["a_gamma"], kept["a_beta"])
        m = L.backward(f["k"], f["v"], f["gamma"], f["beta"], f["lam"], value("qstar"), norm["do"], N_CG)
        held = [L.Checkpoint(kept[n].buffer, (B, T, HEADS, HEAD)) for n in ("qp", "kp", "vp")]
        fg = L.frontend_backward(*held, p["conv_q"], p["conv_k"], p["conv_v"], kept["a_gamma"], kept["a_beta"], p["lam"],
                                 m["dq"], m["dk"], m["dv"], m["dgamma"], m["dbeta"], m["dlam"], grad_dtype=torch.float32)
        for n in ("conv_q", "conv_k", "conv_v"):
            g[n] = fg["d" + n]
        g["lam"] = fg["dtheta"]
        dproj = torch.cat([fg["dqp"].view(B, T, -1), fg["dkp"].view(B, T, -1), fg["dvp"].view(B, T, -1), fg["da_gamma"],
                           fg["da_beta"]], dim=-1)
        g["mesa_in"] = weight(value("z"), dproj)
        dz = dz + dproj @ p["mesa_in"].T
        g["hawk_out"] = weight(value("rec_y"), dz)
        dfused = torch.empty((B, T, 3 * WIDTH), device=dz.device)
        rg = L.recurrence_backward(kept["x"], kept["r"], kept["i"], p["theta"], kept["states"], dz @ p["hawk_out"].T,
                                   reset=kept["reset"], out=dfused.split(WIDTH, dim=-1))
        g["theta"] = rg["dtheta"]
        e = p["embed"][kept["tokens"]]
        g["hawk_in"] = weight(e, dfused)
        de = dz + dfused @ p["hawk_in"].T
        g["embed"] = torch.zeros_like(p["embed"]).index_add_(0, kept["tokens"].reshape(-1), de.reshape(-1, DIM))
        return g

    def decode(self, token, state):
        """Logits [B, VOCAB] of the next token [B], and `state` moved on by it."""
        p, B = self.p, token.shape[0]
        e = p["embed"][token]
        x, r, i = (e @ p["hawk_in"]).split(WIDTH, dim=-1)
        z = e + L.recurrence_step(state["h"], x, r, i, p["theta"]) @ p["hawk_out"]
        heads, a_gamma, a_beta = self._mesa_inputs((z @ p["mesa_in"])[:, None])
        # the front end's window: the last three tokens' projections and this one's
        state["heads"] = [torch.cat([old[:, -3:], new], dim=1).contiguous() for old, new in zip(state["heads"], heads)]
        n = state["heads"][0].shape[1]
        f = self._front(state["heads"], a_gamma.expand(B, n, HEADS).contiguous(), a_beta.expand(B, n, HEADS).contiguous())
        q, k, v = (f[n][:, :, -1].contiguous() for n in ("q", "k", "v"))
        o = L.decode_step(state["H"], state["G"], q, k, v, f["gamma"][..., -1].contiguous(), f["beta"][..., -1].contiguous(),
                          f["lam"], N_CG)
        y = L.output_norm(o[:, :, None].contiguous(), p["norm"], out_dtype=torch.float32).view(B, HEADS * HEAD)
        return (z + y @ p["mesa_out"]) @ p["logits"]


def batch(gen, device, rows=8, length=200):
    """Random tokens with document starts, and the answers (-1 where the document is too young)."""
    tokens = torch.randint(VOCAB, (rows, length), generator=gen)
    reset = (torch.rand((rows, length), generator=gen) < 0.01).to(torch.uint8)
    reset[:, 0] = 1
    answers = torch.full_like(tokens, -1)
    answers[:, BACK:] = tokens[:, :-BACK]
    for k in range(BACK):
        answers[:, BACK - 1 - k:][reset[:, :length - (BACK - 1 - k)] != 0] = -1
    return tokens.to(device), reset.to(device), answers.to(device)


def train(steps=60, device="cuda", say=print):
    """Trains a block; returns it and the losses."""
    block, gen, losses = Block(device), torch.Generator().manual_seed(1), []
    moments = {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in block.p.items()}
    for step in range(1, steps + 1):
        tokens, reset, answers = batch(gen, device)
        logits, kept = block.forward(tokens, reset)
        there = answers >= 0
        logp = torch.log_softmax(logits, dim=-1)
        losses.append(float(-logp[there, answers[there]].mean()))
        dlogits = logp.exp()
        dlogits[there, answers[there]] -= 1.0
        dlogits = torch.where(there[..., None], dlogits, 0.0) / there.sum()
        for n, grad in block.backward(kept, dlogits).items():
            m, v = moments[n]
            m.mul_(0.9).add_(grad, alpha=0.1)
            v.mul_(0.98).addcmul_(grad, grad, value=0.02)
            block.p[n] -= 1e-2 * (m / (1 - 0.9 ** step)) / ((v / (1 - 0.98 ** step)).sqrt() + 1e-8)
        if step == 1 or step % 20 == 0:
            held = sum(c.buffer.numel() for c in kept.values() if isinstance(c, L.Checkpoint))
            wide = sum(4 * c.rows * c.width for c in kept.values() if isinstance(c, L.Checkpoint))
            say("step %3d  loss %.4f  activations kept %.2f MB (fp32: %.2f MB)" % (step, losses[-1], held / 1e6, wide / 1e6))
    return block, losses


def check_decode(block, device="cuda", say=print):
    """Largest difference of the logits of tokens decoded one at a time from those of the whole
    sequence, relative to the largest logit."""
    tokens, reset, _ = batch(torch.Generator().manual_seed(2), device, rows=4, length=80)
    reset.zero_()
    want, _ = block.forward(tokens, reset, keep=False)
    _, state = block.forward(tokens[:, :70].contiguous(), reset[:, :70].contiguous(), keep=False)
    worst = max(float((block.decode(tokens[:, t], state) - want[:, t]).abs().max()) for t in range(70, 80))
    say("decoding a token at a time: largest difference %.1e of %.1f" % (worst, float(want.abs().max())))
    return worst / float(want.abs().max())


if __name__ == "__main__":
    trained, _ = train(int(sys.argv[1]) if len(sys.argv) > 1 else 60)
    check_decode(trained)
