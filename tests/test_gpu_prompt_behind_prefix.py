"""Prompts of requests whose decode steps stand behind a shared prefix: their
rows attend to it through a copy of its entries, their K and V rows go into the
copy and into the request's own sequence."""
import numpy as np
import pytest
import torch

from gpu_util import dev, i32, say
from paper_2609_27233_amd import lib as sm
from test_gpu_e4m3_attention import assert_within, attended
from test_gpu_e4m3_write import BF, E4, by_slot, features, slots_of
from test_gpu_rotary import _rand

pytestmark = pytest.mark.gpu


def to_ints(*shape):
    return torch.empty(shape, dtype=torch.int32, device=dev())


class Layer:
    """A cache with room for the prefix (sequence 0), its copy (1) and requests (2 ..)."""

    def __init__(self, dt, Hq, H, D, bs, seqs, longest):
        pages = -(-longest // bs)
        self.Hq, self.rope = Hq, sm.rope_params(D, theta=10000.0)
        self.c = sm.PagedCache(dtype=dt, num_kv_heads=H, head_dim=D, block_size=bs, num_blocks=seqs * pages, max_seqs=seqs,
                               max_blocks_per_seq=pages)

    def room(self, seq, rows):
        offs, pos, slots = to_ints(2), to_ints(rows), to_ints(rows)
        sm.kv_reserve(self.c, i32([seq]), i32([rows]), offs, pos, slots)
        return offs, pos, slots

    def rows(self, rows, seed):
        return tuple(_rand((rows, h, self.c.D), BF, seed + i).to(dev()) for i, h in enumerate((self.Hq, self.c.H, self.c.H)))

    def copied(self, n):
        """The prefix's n entries as sequence 1's."""
        K, V = (torch.empty((n, self.c.H, self.c.D), dtype=BF, device=dev()) for _ in "KV")
        sm.kv_read(self.c, i32([0]), i32([0, n]), K, V)
        _, pos, slots = self.room(1, n)
        sm.kv_write_rotary(self.c, torch.zeros_like(pos), slots, None, K, V, self.rope, None)

    def prompt(self, seq, q, k, v):
        """Turned queries and their attention over the prefix and the prompt; the prompt's entries are sequence seq's after."""
        m = len(q)
        offs, pos, slots = self.room(1, m)
        own = self.room(seq, m)[2]
        turned, out = torch.empty_like(q), torch.empty_like(q)
        sm.kv_write_rotary(self.c, pos, slots, q, k, v, self.rope, turned)
        sm.kv_write_rotary(self.c, pos, own, None, k, v, self.rope, None)
        sm.prefill_attention(self.c, i32([1]), offs, turned, out, m)
        sm.kv_rollback(self.c, i32([1]), i32([m]))
        return turned, out


@pytest.mark.parametrize("dt", [BF, E4], ids=str)
@pytest.mark.parametrize("Hq,H,D,bs,prefix,prompts", [(32, 8, 128, 16, 333, [40, 1, 100]), (16, 4, 64, 32, 64, [17, 250, 2]),
                                                      (4, 4, 64, 16, 1, [1, 5])])
def test_prompts_attend_to_the_prefix_and_steps_follow_them(Hq, H, D, bs, prefix, prompts, dt):
    say("prompts behind a prefix", dt, Hq, H, D, bs, prefix, prompts)
    L = Layer(dt, Hq, H, D, bs, 2 + len(prompts), prefix + max(prompts) + 1)
    c, n = L.c, len(prompts)
    q, k, v = L.rows(prefix, 1)
    _, pos, slots = L.room(0, prefix)
    sm.kv_write_rotary(c, pos, slots, q, k, v, L.rope, torch.empty_like(q))
    L.copied(prefix)
    got = [L.prompt(2 + i, *L.rows(m, 10 * (i + 1))) for i, m in enumerate(prompts)]
    torch.cuda.synchronize()
    assert c.error_bits() == 0 and c.lengths.cpu().tolist() == [prefix, prefix] + prompts
    table = c.block_table.cpu().numpy()
    at = [slots_of(table, bs, s, np.arange(m)) for s, m in enumerate(c.lengths.cpu().tolist())]
    K, V = features(c)
    # the copy: bf16 as it is; e4m3 values to the last bit but those below the least normal one of a larger exponent
    assert torch.equal(V[at[1]], V[at[0]])
    if dt == BF:
        assert torch.equal(K[at[1]], K[at[0]])
    else:
        step = torch.exp2(by_slot(c)[2][at[1]].double() - 127 - 10)[..., None]
        assert bool(((K[at[1]] - K[at[0]]).abs() <= step).all())
    for i, (m, (turned, out)) in enumerate(zip(prompts, got)):
        s = np.concatenate([at[1], at[2 + i]])
        seen = torch.ones((m, prefix + m), dtype=torch.bool).tril(prefix)
        assert_within(out, *attended(turned.double().cpu(), K[s], V[s], D ** -0.5, seen))
    # a step of all requests behind the prefix
    offs, pos, slots = to_ints(n + 1), to_ints(n), to_ints(n)
    ids = i32(range(2, 2 + n))
    sm.kv_reserve(c, ids, i32([1] * n), offs, pos, slots)
    pos += prefix
    q, k, v = L.rows(n, 90)
    turned, out = torch.empty_like(q), torch.empty_like(q)
    sm.kv_write_rotary(c, pos, slots, q, k, v, L.rope, turned)
    longest = max(prompts) + 1
    ws = torch.zeros(sm.decode_shared_workspace_bytes(n, Hq, D, longest, prefix), dtype=torch.uint8, device=dev())
    sm.decode_attention_shared(c, ids, i32([0]), i32([0, n]), turned, out, ws, longest, prefix)
    torch.cuda.synchronize()
    assert c.error_bits() == 0
    K, V = features(c)
    table = c.block_table.cpu().numpy()
    for i, m in enumerate(prompts):
        s = np.concatenate([at[0], slots_of(table, bs, 2 + i, np.arange(m + 1))])
        assert_within(out[i:i + 1], *attended(turned[i:i + 1].double().cpu(), K[s], V[s], D ** -0.5))
