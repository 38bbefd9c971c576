"""What the tests of scores far from zero share."""
import torch

from kv_helpers import attention, score_size, scores


def check_largest(c, Q, out, lse, scale, **options):
    """A score is off by at most 2^-19 of the magnitudes in it; where the largest is ahead of the next by more than twice that and by 50, its token's value is the
    result: the others weigh 2^-72, and the weight is rounded once, as is the result."""
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    _, ref, _ = attention(c, Q, scale=scale, **options)
    off = 2.0 ** -19 * score_size(c, Q, scale)
    assert ((lse.double() - ref).abs() <= off + 2.0 ** -22 * ref.abs() + 2.0 ** -19).all()
    clear = 0
    for b, n in enumerate(c.new):
        start, _ = c.rows(b)
        x = scores(c, Q, b, scale=scale, **options)      # [heads, group, new, length]
        top = x.topk(min(2, x.shape[-1]), -1)
        ahead = top.values[..., 0] - top.values[..., 1] > 2 * off + 50 if x.shape[-1] > 1 else torch.ones_like(top.values[..., 0], dtype=torch.bool)
        v = c.V[b].permute(1, 0, 2).unsqueeze(1).expand(-1, c.G, -1, -1)   # [heads, group, length, dim]
        want = torch.gather(v, 2, top.indices[..., :1].expand(-1, -1, -1, c.D)).permute(2, 0, 1, 3).reshape(n, -1, c.D)
        err = (out[start:start + n].double() - want).abs()
        tol = (2.0 ** -8 + 2.0 ** -11) * want.abs() + 2.0 ** -35 * v.abs().sum(2).amax()
        ahead = ahead.permute(2, 0, 1).reshape(n, -1, 1)
        assert (err <= tol)[ahead.expand_as(err)].all()
        clear += int(ahead.sum())
    assert clear > out.shape[0] * out.shape[1] // 2      # most rows are such
