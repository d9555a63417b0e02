"""The plan of a batched attention call ends for many uneven batches, and covers its parts (host arithmetic only)."""
import ctypes as C
import random

from paper_2401_18079_amd import binding as B
from test_batch_refusals import cache, table


def test_plans_of_uneven_batches():
    f = B.load_library().kvq_attention_decode_batch_workspace_bytes
    rng = random.Random(1)
    for _ in range(400):
        heads = rng.choice([1, 2, 3, 8, 32, 40])
        ratio = rng.choice([1, 1, 2, 4, 8, 33, 70])
        n_seqs = rng.choice([1, 2, 7, 32, 64])
        top = rng.choice([1, 40, 2000, 9000])
        make = lambda n: cache(n_kv_heads=heads, n_q_heads=heads * ratio, cap_tokens=1 << 20, n_tokens_k=n, n_tokens_v=n)  # noqa: E731
        own = [make(rng.randrange(top + 1)) for _ in range(n_seqs)]
        prefix = rng.choice([None, make(rng.choice([1, 31, 33001, 524287]))])
        need = f(None if prefix is None else C.byref(prefix), table(own), n_seqs)
        assert need > 0
        tokens = sum(c.n_tokens_k for c in own) + (prefix.n_tokens_k if prefix is not None else 0)
        entries = sum(min(4096, c.n_tokens_k * heads * 128) for c in own + ([prefix] if prefix is not None else []))
        assert need >= 8 * entries + tokens // 32 * 8 * (heads + 1)
