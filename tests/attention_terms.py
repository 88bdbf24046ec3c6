"""Float64 terms of the attention gradients, head by head, for tests whose
bounds are finer than those of attention_forms."""
import torch


def heads64(q, k, v, g, tau, causal=False, g_lse=None):
    """For every (problem, query head): a dict of the float64 rows, the
    probabilities p, dp = g v^T, delta, ds and the visible pairs, with

      eS  2^-21 (tau max_n |q|.|k_n| + 1) per row: error of a score, in units of p

    All of q's and k's rows count (no lengths)."""
    B, M, H, _ = q.shape
    N, Hk = k.shape[1:3]
    seen = torch.ones(M, N, dtype=torch.bool, device=q.device)
    if causal:
        seen = torch.arange(N, device=q.device)[None, :] <= \
            torch.arange(M, device=q.device)[:, None] + (N - M)
    for b in range(B):
        for h in range(H):
            j = h // (H // Hk)
            x = {"b": b, "h": h, "j": j, "seen": seen, "Q": q[b, :, h].double(),
                 "K": k[b, :, j].double(), "V": v[b, :, j].double(), "G": g[b, :, h].double()}
            s = (tau * x["Q"] @ x["K"].T).masked_fill(~seen, -float("inf"))
            some = seen.any(-1, keepdim=True)
            z = torch.where(some, torch.logsumexp(s, -1, keepdim=True), 0.0)
            x["lse"] = torch.where(some, z, -float("inf"))[:, 0]
            x["p"] = torch.where(some & seen, torch.exp(s - z), 0.0)
            x["out"] = x["p"] @ x["V"]
            x["dp"] = x["G"] @ x["V"].T
            x["delta"] = (x["G"] * x["out"]).sum(-1, keepdim=True)
            if g_lse is not None:
                x["delta"] = x["delta"] - g_lse[b, h, :, None].double()
            x["ds"] = x["p"] * (x["dp"] - x["delta"])
            mag = (tau * x["Q"].abs() @ x["K"].abs().T).masked_fill(~seen, 0).amax(-1, keepdim=True)
            x["eS"] = 2.0 ** -21 * (mag + 1)
            yield x
