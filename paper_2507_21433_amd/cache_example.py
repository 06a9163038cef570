"""A few decoding steps of one layer on the 4-bit cache, as a serving engine runs them: new tokens are written, attention reads the cache
through the block tables, blocks that are full are read back and searched for in the pool, and the tables go where the search says.

    python -m paper_2507_21433_amd.cache_example

Two requests of the same prompt; the second one's sealed blocks are found among the first one's, its table is pointed at them, and the
attention over the shared blocks gives what it gave over its own.
"""
import torch

from . import binding as rc

T, H, G, D = 16, 8, 5, 128


def main(device="cuda:0", prompt=80, steps=5, dtype=torch.float16, seed=0):
    """Returns dict(matches, tables, before, after): the search's decisions, the last tables, attention before and after sharing."""
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, generator=g, device=device).to(dtype)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=device)
    R, E = 2, -(-(prompt + steps) // T)
    NB = R * E
    cache = rc.cache_tensor(1, NB, T, H, device)
    tables = torch.arange(NB, dtype=torch.int32, device=device).reshape(1, R, E)
    refcount = torch.ones((1, NB), dtype=torch.int32, device=device)
    workspace = torch.empty(max(16, rc.rc_cache_attend_workspace_size(cache, dtype, R, E, H * G, prompt)), dtype=torch.uint8, device=device)

    def write(k, v, first):
        """k, v [tokens of a request][H][D], the same for both requests, at the positions from `first` on."""
        n = k.shape[0]
        pos = torch.arange(first, first + n, device=device)
        slots = torch.cat([tables[0, r, pos // T] * T + pos % T for r in range(R)]).to(torch.int32)
        both = lambda x: x.repeat(R, 1, 1)[None]
        rc.rc_cache_write(both(k), both(v), slots, cache)

    # the prompt: written, then attended over by all its tokens
    write(randn(prompt, H, D), randn(prompt, H, D), 0)
    q = randn(1, R * prompt, H * G, D)
    first = rc.rc_cache_attend(q, cache, tables, ints([prompt] * R), q_start=ints([0, prompt, 2 * prompt]), max_q=prompt, workspace=workspace)

    # decoding, one token of each request a step
    for s in range(steps):
        write(randn(1, H, D), randn(1, H, D), prompt + s)
        q = randn(1, 1, H * G, D).repeat(1, R, 1, 1)
        before = rc.rc_cache_attend(q, cache, tables, ints([prompt + s + 1] * R), workspace=workspace)

    # the second request's sealed blocks against the first one's
    sealed = (prompt + steps) // T
    kp, vp = rc.rc_cache_read(cache, tables[0, 0, :sealed].contiguous(), dtype)
    query_ids = tables[0, 1, :sealed].contiguous()
    kq, vq = rc.rc_cache_read(cache, query_ids, dtype)
    m = rc.rc_match_blocks(kq, vq, *rc.rc_block_norms(kq, vq), kp, vp, *rc.rc_block_norms(kp, vp), None, 0.95)
    r = rc.rc_remap_block_table(tables, query_ids, tables[0, 0, :sealed].contiguous(), m["match_idx"], sealed, NB, refcount)
    after = rc.rc_cache_attend(q, cache, r["tables"], ints([prompt + steps] * R), workspace=workspace)
    return dict(matches=m["match_idx"], tables=r["tables"], freed=r["freed"], prompt=first, before=before, after=after)


if __name__ == "__main__":
    out = main()
    torch.cuda.synchronize()
    print("blocks of the second request found among the first one's:", out["matches"][0].tolist())
    print("its table:", out["tables"][0, 1].tolist(), "  blocks freed:", int(out["freed"].sum()))
    print("attention over shared blocks as before:", torch.equal(out["before"]["out"], out["after"]["out"]))
