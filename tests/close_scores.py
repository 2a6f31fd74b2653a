"""How far fikit_token_scores may be from 64 bits, from its operations one by one: nothing but the sum's logarithm grows with the logits' size.

With away_j = |z_j - max z|, p_j the probabilities, S = sum exp(z_j - max z) and first-order terms (u = 2^-24 is half a step of 32 bits):

  d_j = (x_j - m) c     a difference, a product, and c, itself a rounded product of a rounded log2(e): 4 u |d_j|, so 4 u away_j in exp's argument, also
                        where sums move from one largest logit to another, as the parts of a way add up to it
  exp2                  2 u, a unit in the last place; so a term is within e_j = 4 u away_j + 2 u
  S                     sums of V / 64 terms at most in a lane; then a dozen moves and 26 additions through lanes, waves and parts, and a move for each 1024
                        logits in a lane, of 3 u each: n = (V / 48 + 64) u.  S is within P + n of itself, P = sum p e
  log2 S                2 u of it, or 2 u where it is small: L = P + n + 2 u (1 + ln S)
  lse                   m scale is exact in its sum with ln 2 log2 S (two more roundings of it) until that is rounded: L + 2 u ln S + u |lse|
  log p_j               ln 2 (d_j - log2 S), three roundings: 4 u away_j + L + 3 u |log p_j|; from away_j = 2^22 ln 2 on z_j - lse, two roundings and lse's own
  T = sum 2^d d         its terms within 2 e_j + 4 u of themselves (2^d, d, and the s that a move adds), sums as S with as many roundings again in moves and
                        products: 4 n; the quotient T / S P + n and 4 u more; so the entropy is within
                        L + sum p away (2 e + 4 u) + (4 n + P + 4 u) sum p away + 2 u (ln S + sum p away)
"""
import torch

from around_model import Scores

U = 2.0 ** -24


class CloseScores(Scores):
    def __init__(self, logits, tokens, scale, top):
        super().__init__(logits, tokens, scale, top)
        x = logits.double().cpu()
        rows, v = x.shape
        if v == 0:
            return
        z = x * float(torch.tensor(scale, dtype=torch.float32))
        fine = ~(torch.isnan(x) | (x == float("inf"))).any(1) & ~(x == -float("inf")).all(1)
        z = torch.where(fine[:, None], z, 0.0)
        most = z.amax(1, keepdim=True)
        away = (z - most).abs()
        log_s = torch.logsumexp(z - most, 1)
        log_p = -away - log_s[:, None]
        p = log_p.exp()
        away = torch.where(torch.isfinite(away), away, 0.0)
        log_p = torch.where(torch.isfinite(log_p), log_p, 0.0)
        z = torch.where(torch.isfinite(z), z, 0.0)
        e, n = 4 * U * away + 2 * U, (v / 48 + 64) * U
        p_e, p_away = (p * e).sum(1), (p * away).sum(1)
        of_log = p_e + n + 2 * U * (1 + log_s)
        of_lse = of_log + 2 * U * log_s + U * (most[:, 0] + log_s).abs()
        of_token = 4 * U * away + of_log[:, None] + 3 * U * log_p.abs()
        far = U * z.abs() + of_lse[:, None] + U * log_p.abs()
        of_token = torch.where(away > 2.0 ** 21, torch.maximum(of_token, far), of_token)
        entropy = of_log + (p * away * (2 * e + 4 * U)).sum(1) + (4 * n + p_e + 4 * U) * p_away + 2 * U * (log_s + p_away)
        self.bound.update(lse=of_lse, entropy=entropy)
        if tokens is not None:
            t = tokens.long().cpu()
            self.bound["logprob"] = torch.where(t >= 0, of_token.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
        order = torch.sort(torch.where(torch.isnan(x), -float("inf"), x + 0.0), dim=1, descending=True, stable=True).indices[:, :top]
        self.bound["top_logprob"] = of_token.gather(1, torch.nn.functional.pad(order, (0, top - order.shape[1])))
