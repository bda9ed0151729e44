"""A plain LLaMA forward in 64 bits over given visibility: every token (context and draft nodes) in one pass, each with its
position and the tokens that it sees.  On the GPU where there is one (elementary torch operations)."""
import numpy as np
import torch

import synth


class Model:
    def __init__(self, shape, seed=synth.BASE_SEED, random_gains=True):
        self.shape = shape
        self.dev = "cuda:0" if torch.cuda.is_available() else "cpu"
        self.w = {}
        for _, l, name in synth.tensor_names(shape.n_layers):
            t = synth.weight_tensor(shape, name, l, seed=seed, random_gains=random_gains)
            self.w[name, l] = torch.from_numpy(np.asarray(t, dtype=np.float64)).to(self.dev)

    def logits(self, tokens, pos, see, skip=(), skip_from=0):
        """[T][vocab] float64 of tokens at positions pos, see [T][T] (row sees column); rows from skip_from on skip the
        blocks of skip."""
        s, w = self.shape, self.w
        H, hd, half = s.n_heads, s.head_dim, s.head_dim // 2
        pos = torch.as_tensor(np.asarray(pos), device=self.dev).double()
        see = torch.as_tensor(np.asarray(see), device=self.dev)
        a = pos[:, None] * s.rope_base ** (-2.0 * torch.arange(half, device=self.dev).double() / hd)
        c, z = a.cos()[None], a.sin()[None]

        def norm(x, g):
            return x / torch.sqrt((x * x).mean(-1, keepdim=True) + s.rms_eps) * g

        def heads(y):
            return y.reshape(-1, H, hd).transpose(0, 1).contiguous()

        def turn(x):
            p, q = x[..., :half], x[..., half:]
            return torch.cat([p * c - q * z, q * c + p * z], -1)
        x = w["embed", -1][torch.as_tensor(np.asarray(tokens), device=self.dev).long()]
        for l in range(s.n_layers):
            if l in skip and skip_from == 0:
                continue
            kept = x[skip_from:] if l in skip else None
            y = norm(x, w["attn_norm", l])
            q, k = turn(heads(y @ w["wq", l].T)), turn(heads(y @ w["wk", l].T))
            v = heads(y @ w["wv", l].T)
            sc = torch.matmul(q, k.transpose(1, 2).contiguous()) / hd ** 0.5
            p = torch.softmax(sc.masked_fill(~see[None], -torch.inf), -1)
            o = torch.matmul(p, v).transpose(0, 1).reshape(-1, H * hd)
            x = x + o @ w["wo", l].T
            y = norm(x, w["mlp_norm", l])
            g = y @ w["w_gate", l].T
            x = x + (g * torch.sigmoid(g) * (y @ w["w_up", l].T)) @ w["w_down", l].T
            if kept is not None:
                x = torch.cat([x[:skip_from], kept])
        return (norm(x, w["final_norm", -1]) @ w["lm_head", -1].T).cpu().numpy()


def context_see(n, sinks, window):
    p, t = np.arange(n)[:, None], np.arange(n)[None]
    see = t <= p
    return see & ((t < sinks) | (t > p - window)) if window else see


def step_logits(model, ctx, draft, parent, sinks, window, skip=(), dense_context=False):
    """Logits of a draft's nodes behind a context whose tokens see sinks and window (0: all), as a prefill under the same
    window and mask (with dense_context: under no mask) leaves it."""
    n, m = len(ctx), len(draft)
    parent = np.arange(-1, m - 1) if parent is None else np.asarray(parent)
    depth, anc = np.zeros(m, np.int64), np.eye(m, dtype=bool)
    for i in range(1, m):
        depth[i] = depth[parent[i]] + 1
        anc[i] |= anc[parent[i]]
    see = np.zeros((n + m, n + m), bool)
    see[:n, :n] = context_see(n, sinks, window)
    p, t = n + depth[:, None], np.arange(n)[None]
    see[n:, :n] = (t < sinks) | (t > p - window) if window else True
    see[n:, n:] = anc
    return model.logits(np.concatenate([ctx, draft]), np.concatenate([np.arange(n), n + depth]), see, skip,
                        n if dense_context else 0)[n:]
