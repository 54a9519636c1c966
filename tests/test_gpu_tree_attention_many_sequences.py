"""Attention of many sequences of very different lengths, whose tokens are dealt out 64 sequences at a time, against the formula in 64 bits."""
import math

import pytest
import torch

from test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu


class Many(Case):
    """A case whose answer is formed a sequence at a time; every row sees some token or none, all are numbers."""

    def plain(self):
        b, n, h, d = self.q.shape
        kv, eps = self.k.shape[3], torch.finfo(self.t).eps / 2
        outs = []
        pool = [x[0].double().cuda() for x in (self.k, self.v)]
        for s in range(b):
            length = self.lens[s]
            keys, values = (torch.cat([p[self.table[s].long()].flatten(0, 1)[:length], new[s].double().cuda()]).repeat_interleave(h // kv, 1).transpose(0, 1).contiguous()
                            for p, new in zip(pool, (self.k_new, self.v_new)))               # [head][token][d]
            sees = torch.cat([torch.ones(n, length, dtype=torch.bool), self.sees[s]], 1).cuda()
            q = self.q[s].double().cuda().transpose(0, 1).contiguous()                          # [head][node][d]
            x = (torch.bmm(q, keys.transpose(1, 2).contiguous()) * self.scale).masked_fill(~sees, -math.inf)
            size = (torch.bmm(q.abs(), keys.abs().transpose(1, 2).contiguous()) * self.scale).masked_fill(~sees, 0.0).amax(2)
            p = torch.softmax(x, 2).nan_to_num(0.0)
            out, lse, total = torch.bmm(p, values), torch.logsumexp(x, 2), sees.sum(1)
            # as in Case.plain()
            score = 2.0 ** -23 * (d + 4) * size + 2.0 ** -20
            some = eps + 2 * score + 2 * total * 2.0 ** -24
            bound = some[..., None] * torch.bmm(p, values.abs()) + eps * out.abs() + torch.finfo(self.t).smallest_normal * eps
            lse_bound = score + total * 2.0 ** -24 + 2.0 ** -22 * (1 + lse.abs())
            outs.append([y.transpose(0, 1).cpu() for y in (out, lse, bound, lse_bound)])
        out, lse, self.bound, self.lse_bound = (torch.stack(y) for y in zip(*outs))
        return out, lse


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("batch", [63, 64, 65, 130, 200])
@pytest.mark.parametrize("nodes,heads,kv", [(1, 4, 4), (3, 8, 2), (20, 4, 2), (33, 8, 1)])
def test_lengths_of_many_sequences(dtype, batch, nodes, heads, kv):
    """Lengths of zero among them, the longest ones in the second and third 64; expected lengths that are short, right and long; then no context at all."""
    lens = [(0, 1, 33, 100, 64, 7, 250)[i % 7] for i in range(batch)]
    lens[batch - 1], lens[batch // 2], lens[min(70, batch - 2)] = 2999, 0, 1531
    c = Many(dtype, batch, nodes, heads, kv, 64, 64, lens, mask="tree", seed=batch)
    for max_len in (0, 300, 3000, 10 ** 6):
        c.check(max_len=max_len)
    c.lens = [0] * batch
    c.check(max_len=3000)
    c.mask, c.sees = c.mask.clone(), c.sees.clone()
    c.mask[1::2] = 0                      # and rows that see nothing
    c.sees[1::2] = False
    c.check(max_len=3000)
