"""Learn the rows of an index, and search it: the training calls and the graph together.

Items that are used together (here: items of one topic, drawn in pairs) should be near in the distance that the graph searches
by.  A step looks up a batch of pairs and their mined negatives, takes the softmax loss over squared distances and its
gradients, sums them by item and takes an AdamW step, which also writes the 16-bit copy of the table.  Every few steps a
graph is built on that copy and searched for the negatives: the items that the table now holds to be near, and that are not.

    python examples/train_rows.py [--items 100000] [--steps 300]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2310_20419_amd as rn  # noqa: E402


class Table:
    """A float32 table, its 16-bit copy, its gradient, and 8-bit moments (all zero bytes: zero)."""

    def __init__(self, items, d, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.master = torch.randn(items, d, device="cuda", generator=g) / d ** 0.5
        self.rows = self.master.bfloat16()
        self.grad = torch.empty_like(self.master)
        bytes_ = lambda n: torch.zeros(n, dtype=torch.uint8, device="cuda")  # noqa: E731
        n = items * d
        self.tensors = rn.AdamwTensors([dict(param=self.master, grad=self.grad, m=bytes_(n), v=bytes_(n), m_scale=bytes_(-(-n // 128)),
                                             v_scale=bytes_(-(-n // 128)), copy=self.rows)])
        self.steps = 0

    def step(self, query, positive, negative, scale, lr):
        """One step on pairs (query[i], positive[i]) against each other's positives and the shared negatives; ids of -1 are padding."""
        B = query.shape[0]
        ids = torch.cat([query, positive, negative])
        found = rn.rnnd_embed(self.rows, ids)
        target = torch.arange(B, dtype=torch.int32, device="cuda")
        weight = torch.full((B,), 1.0 / B, device="cuda")
        loss, dq, dk = rn.rnnd_contrast(found[:B], found[B:], target, scale, query_ids=query, key_ids=ids[B:], row_weight=weight)
        rn.rnnd_embed_grad(torch.cat([dq, dk]), ids, self.master.shape[0], grad=self.grad)
        self.steps += 1
        rn.rnnd_adamw(self.tensors, self.steps, lr=lr, seed=2310)
        return loss

    def index(self, S=12, R=48, T1=2, T2=6, seed=2310):
        return rn.rnnd_build(self.rows, S, R, T1, T2, seed)


def train(items=100_000, topics=2_000, d=64, batch=8_192, mined=4, steps=300, mine_every=50, scale=8.0, lr=0.01, seed=1, say=print):
    """Returns (loss of the first step, of the last, share of the 10 nearest found that are of the item's own topic)."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    topic = torch.randint(0, topics, (items,), device="cuda", generator=g)
    by_topic = torch.argsort(topic)                   # the items, topic after topic
    first = torch.searchsorted(topic[by_topic], torch.arange(topics + 1, device="cuda"))
    table = Table(items, d, seed)
    near = torch.full((items, mined), -1, dtype=torch.int32, device="cuda")

    def partner(x):
        low, high = first[topic[x]], first[topic[x] + 1]
        return by_topic[low + (torch.rand(len(x), device="cuda", generator=g) * (high - low)).long().clamp_(max=items)]

    losses = []
    for i in range(steps):
        if i and i % mine_every == 0:                 # the nearest of another topic (rows of -1 where there is none)
            graph, degree = table.index()
            found, _, _ = rn.rnnd_search(table.rows, graph, degree, table.rows, 64, 32, 2 * mined, i)
            other = (found >= 0) & (topic[found.clamp(min=0).long()] != topic[:, None])
            rank = other.int().cumsum(1)
            near.fill_(-1)
            for k in range(mined):
                at = other & (rank == k + 1)
                near[:, k] = torch.where(at.any(1), found.gather(1, at.int().argmax(1, keepdim=True))[:, 0], -1)
        q = torch.randint(0, items, (batch,), device="cuda", generator=g)
        p = partner(q)
        losses.append(table.step(q.int(), p.int(), near[q].reshape(-1), scale, lr).mean())
        if say and (i + 1) % mine_every == 0:
            say("step %4d  loss %.3f" % (i + 1, torch.stack(losses[-mine_every:]).mean().item()))
    graph, degree = table.index()
    ask = torch.randint(0, items, (2_000,), device="cuda", generator=g)
    found, _, _ = rn.rnnd_search(table.rows, graph, degree, table.rows[ask].contiguous(), 64, 32, 11, 7)
    mine = (found >= 0) & (found != ask[:, None])     # without the item itself
    share = ((topic[found.clamp(min=0).long()] == topic[ask][:, None]) & mine).sum() / mine.sum()
    return losses[0].item(), losses[-1].item(), share.item()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--items", type=int, default=100_000)
    ap.add_argument("--steps", type=int, default=300)
    a = ap.parse_args()
    start, end, share = train(items=a.items, topics=max(2, a.items // 50), steps=a.steps)
    print("loss %.3f -> %.3f; of the 10 nearest that the index finds, %.0f %% are of the item's topic" % (start, end, 100 * share))
