"""The operators beside the products on the GPU, against their definitions in 64 bits."""
import numpy as np
import pytest

from paper_2605_11582_amd import binding as egt, synth
import gpu_common as G
import serve_reference as R

pytestmark = pytest.mark.gpu


def dev(a):
    """numpy -> device, FP16 and unsigned words included."""
    torch = G.torch_mod()
    a = np.ascontiguousarray(a)
    if a.dtype in (np.uint64, np.uint32):
        a = a.view({8: np.int64, 4: np.int32}[a.dtype.itemsize])
    return torch.from_numpy(a).cuda()


def f16(rng, *shape, scale=1.0):
    return (rng.standard_normal(shape) * scale).astype(np.float16)


def guarded(shape, dtype, fill, guard=64):
    """(buffer, the tensor inside it with `guard` elements of `fill` on both sides)."""
    torch = G.torch_mod()
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * guard,), fill, dtype=dtype, device="cuda")
    return buf, buf[guard:guard + n].view(shape)


def untouched(buf, fill, guard=64):
    host = buf.cpu().numpy()
    assert (host[:guard] == fill).all() and (host[len(host) - guard:] == fill).all(), "write outside the output"


# ---------------------------------------------------------------- block tables and slot maps
def slots_case(rng, n, most, context, page, share, spare=0):
    lens, counts = rng.integers(0, context + 1, n).astype(np.int32), rng.integers(0, most + 1, n).astype(np.int32)
    width = -(-(context + most) // page)
    ids = rng.permutation(n * width + 5).astype(np.int32)
    have = -(-lens // page)
    table = np.where(np.arange(width) < have[:, None], ids[:n * width].reshape(n, width), -7).astype(np.int32)
    need = int((-(-(lens + counts) // page) - have).sum())
    free = np.setdiff1d(ids, table)[:max(1, int(share * need) + 2)].astype(np.int32)
    return lens, counts, table, free, len(ids), n * most + spare


def check_slots(lens, counts, table, page, blocks, free, head, n_slots, pad=0):
    torch = G.torch_mod()
    want = R.kv_slots(lens, counts, table, page, blocks, free, head, n_slots)
    n, width = table.shape
    wide = torch.full((n, width + pad), -99, dtype=torch.int32, device="cuda")
    wide[:, :width] = dev(table)
    got_table = wide[:, :width]
    b1, slots = guarded((n_slots,), torch.int32, -55)
    b2, cu = guarded((n + 1,), torch.int32, -55)
    b3, new = guarded((n,), torch.int32, -55)
    b4, new_head = guarded((1,), torch.int32, -55)
    for _ in range(2):                                   # (again: the same answer, the old lengths are still there)
        egt.kv_slots(dev(lens), dev(counts), got_table, page, blocks, dev(free), dev(np.array([head], np.int32)), slots, cu, new, new_head)
        torch.cuda.synchronize()
        for name, g, w in zip(("slots", "cu_tokens", "new_lens", "new_head", "block_table"), (slots, cu, new, new_head, got_table), want):
            assert np.array_equal(g.cpu().numpy(), w), name
    for b in (b1, b2, b3, b4):
        untouched(b, -55)
    assert (wide[:, width:] == -99).all()


@pytest.mark.parametrize("n,most,context,page,share,pad", [
    (1, 1, 1, 1, 1, 0), (1, 64, 300, 16, 1, 3), (3, 5, 40, 8, 1, 1), (64, 16, 900, 16, 1, 0), (255, 3, 50, 4, 1, 0), (256, 40, 64, 32, 0.5, 0), (257, 7, 129, 64, 0.3, 5),
    (1000, 9, 33, 2, 1, 0), (2049, 30, 100, 16, 0.9, 0), (7, 5000, 1000, 128, 1, 0), (5, 700, 2000, 1, 0.6, 0), (egt.MAX_REQUESTS, 2, 9, 4, 0.7, 0)])
def test_slots(n, most, context, page, share, pad):
    rng = np.random.default_rng(n * 7919 + most)
    lens, counts, table, free, blocks, n_slots = slots_case(rng, n, most, context, page, share, spare=n % 5)
    check_slots(lens, counts, table, page, blocks, free, 0, n_slots, pad)


def test_slots_that_cannot_be_had():
    rng = np.random.default_rng(5)
    lens, counts, table, free, blocks, n_slots = slots_case(rng, 40, 20, 100, 8, 1)
    lens[3], counts[5], counts[7], lens[9], counts[11], lens[12] = -4, -1, 10000, 2 ** 31 - 1, 0, 0
    check_slots(lens, counts, table, 8, blocks, free, 2, n_slots)
    check_slots(lens, counts, table, 8, blocks, free, -1, n_slots)              # a head outside the list: no page to be had
    check_slots(lens, counts, table, 8, blocks, free, len(free) + 3, n_slots)
    counts[7] = 2
    check_slots(lens, counts, table, 8, blocks, free, 0, int(counts.clip(0).sum()) // 2)     # fewer slots than tokens
    check_slots(lens, counts, table, 8, blocks // 2, free, 0, n_slots)          # pages that are not the cache's
    check_slots(lens, np.zeros(40, np.int32), table, 8, blocks, free, 0, 3)     # nothing new
    check_slots(lens, counts, table, 8, blocks, free, 0, 0)                     # no slots at all


@pytest.mark.parametrize("n,most,context,page,share", [(300, 4096, 500, 16, 0.97), (64, 20000, 3000, 64, 0.9), (1, 1100003, 7, 128, 1), (2000, 600, 40, 8, 0.95)])
def test_slots_past_a_million(n, most, context, page, share):
    """More slots than the workgroups take at once, not a multiple of four; pages that run out among the last."""
    rng = np.random.default_rng(n + most)
    lens, counts, table, free, blocks, n_slots = slots_case(rng, n, most, context, page, share, spare=3)
    assert n_slots > 1 << 20
    check_slots(lens, counts if n > 1 else np.array([most], np.int32), table, page, blocks, free if n > 1 else np.arange(blocks, dtype=np.int32)[::-1].copy(), 0, n_slots)


# ---------------------------------------------------------------- rows into the cache
def paged(rng, blocks, heads, page, dim, order):
    """A cache tensor (blocks, heads, page, dim) whose axes lie in memory as `order` says."""
    shape = (blocks, heads, page, dim)
    base = dev(f16(rng, *[shape[a] for a in order], dim))
    return base.permute(*[order.index(a) for a in range(3)], 3)


@pytest.mark.parametrize("n,heads,dim,page,order,picked", [
    (1, 1, 8, 1, (0, 1, 2), False), (5, 2, 64, 16, (0, 1, 2), True), (64, 8, 128, 16, (0, 2, 1), True), (33, 3, 80, 8, (0, 1, 2), False),
    (300, 32, 128, 64, (1, 0, 2), False), (17, 5, 256, 4, (0, 2, 1), True), (1025, 1, 40, 32, (2, 0, 1), False)])
def test_append(n, heads, dim, page, order, picked):
    torch = G.torch_mod()
    rng = np.random.default_rng(n + heads)
    blocks = -(-2 * n // page) + 1
    kc, vc = paged(rng, blocks, heads, page, dim, order), paged(rng, blocks, heads, page, dim, order[::-1])
    kv = dev(f16(rng, n, 2 * heads + 1, dim))
    k, v = kv[:, :heads], kv[:, heads + 1:]
    slots = rng.permutation(blocks * page)[:n].astype(np.int32)
    slots[::7] = [-1, blocks * page, -2 ** 31, 2 ** 31 - 1][n % 4]
    rows = rng.integers(0, n, n).astype(np.int32) if picked else None
    if picked:
        rows[1::5] = [-1, n][n % 2]
    want = []
    for cache, new in ((kc, k), (vc, v)):
        c, x = cache.cpu().numpy().copy(), new.cpu().numpy()
        for i, s in enumerate(slots.tolist()):
            row = int(rows[i]) if picked else i
            if 0 <= s < blocks * page and 0 <= row < n:
                c[s // page, :, s % page] = x[row]
        want.append(c)
    egt.kv_append(k, v, dev(slots), kc, vc, None if rows is None else dev(rows))
    torch.cuda.synchronize()
    assert np.array_equal(kc.cpu().numpy().view(np.uint16), want[0].view(np.uint16)) and np.array_equal(vc.cpu().numpy().view(np.uint16), want[1].view(np.uint16))


# ---------------------------------------------------------------- attention
def tree_case(rng, lens, counts, heads, kv_heads, dim, page, order=(0, 1, 2), spare=2, scale=1.0):
    torch = G.torch_mod()
    n, width = len(lens), max(1, -(-max(lens) // page)) + 1
    blocks = n * width + 3
    cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    N = int(cu[-1]) + spare
    qkv = dev(f16(rng, N, heads + 2 * kv_heads, dim, scale=scale))
    c = dict(q=qkv[:, :heads], k=qkv[:, heads:heads + kv_heads], v=qkv[:, heads + kv_heads:], k_cache=paged(rng, blocks, kv_heads, page, dim, order),
             v_cache=paged(rng, blocks, kv_heads, page, dim, order), table=rng.permutation(blocks)[:n * width].reshape(n, width).astype(np.int32),
             lens=np.array(lens, np.int32), cu=cu, mask=R.trees(rng, counts, N), scale=dim ** -0.5, max_tokens=max(max(counts), 1))
    c["buf"], c["out"] = guarded((N, heads, dim), torch.float16, 7.0)
    c["ws"] = torch.full((egt.tree_attention_ws_bytes(c["q"], c["k_cache"], dev(c["table"]), dev(c["lens"]), c["max_tokens"]),), 255, dtype=torch.uint8, device="cuda")
    return c


def run_tree(c, stream=None):
    egt.tree_attention(c["q"], c["k"], c["v"], c["k_cache"], c["v_cache"], dev(c["table"]), dev(c["lens"]), dev(c["cu"]), dev(c["mask"]), c["out"], c["scale"],
                       c["max_tokens"], c["ws"], stream)
    G.torch_mod().cuda.synchronize()
    return c["out"].cpu().numpy()


def want_tree(c):
    f = lambda t: t.cpu().numpy().astype(np.float64)  # noqa: E731
    return R.tree_attention(f(c["q"]), f(c["k"]), f(c["v"]), f(c["k_cache"]), f(c["v_cache"]), c["table"], c["lens"], c["cu"], c["mask"], c["scale"])


def check_tree(c, what=""):
    print("case", what, c["lens"].tolist(), c["cu"].tolist(), tuple(c["q"].shape), tuple(c["k_cache"].shape), flush=True)
    got = run_tree(c)
    want, bound = want_tree(c)
    used = int(c["cu"][-1])
    R.close(got[:used], want[:used], bound[:used], what)
    assert (got[used:] == 7).all(), "rows behind the last request"
    untouched(c["buf"], 7)


CASES = [
    ([0], [1], 1, 1, 8, 1), ([1], [1], 1, 1, 64, 16), ([37], [1], 4, 4, 128, 16), ([777], [1], 32, 32, 128, 16), ([64, 0, 1], [1, 1, 1], 8, 2, 64, 8),
    ([31, 32, 33, 63, 64, 65], [1, 2, 3, 15, 16, 17], 4, 2, 128, 32), ([100, 0, 300], [33, 64, 7], 14, 2, 80, 8), ([513], [64], 8, 1, 96, 64),
    ([129, 5], [20, 0], 6, 3, 32, 128), ([1000], [48], 8, 8, 256, 16), ([700, 90], [5, 31], 10, 5, 40, 2), ([260], [40], 24, 3, 192, 4), ([2500, 3], [3, 9], 16, 2, 128, 1),
    ([4097], [64], 16, 2, 128, 64), ([127, 128], [64, 1], 2, 1, 224, 16), ([90, 17, 200], [64, 63, 2], 12, 1, 72, 16), ([300], [2], 128, 1, 16, 32)]


@pytest.mark.parametrize("lens,counts,heads,kv_heads,dim,page", CASES)
def test_attention(lens, counts, heads, kv_heads, dim, page):
    rng = np.random.default_rng(sum(lens) + dim)
    check_tree(tree_case(rng, lens, counts, heads, kv_heads, dim, page, [(0, 1, 2), (0, 2, 1), (1, 0, 2)][dim % 3]))


# Every kernel of the attention, in one span and in several (test_serve_host.py asks the library which kernels these are):
# (head size, key heads, query heads a key head, drafted tokens of the largest request, context of the largest)
FORMS = [(dim, kv, group, tokens, context) for dim in (40, 64, 72, 96, 128, 160, 192, 200, 256) for context in (77, 1500)
         for kv, group, tokens in ((3, 1, 1), (2, 1, 20), (1, 4, 8), (2, 1, 50), (2, 2, 50), (2, 4, 50))]


def form_case(dim, kv, group, tokens, context):
    """Three requests: the largest; one that has no context and whose first token sees nothing; a short one."""
    rng = np.random.default_rng(dim * 1000 + kv * group * tokens + context)
    c = tree_case(rng, [context, 0, 33], [tokens, max(1, tokens // 3), min(tokens, 2)], kv * group, kv, dim, (16, 1, 64)[(dim // 8) % 3], [(0, 1, 2), (0, 2, 1), (1, 0, 2)][group % 3])
    c["mask"][tokens] = 0
    return c


@pytest.mark.parametrize("dim,kv,group,tokens,context", FORMS)
def test_every_form_of_the_attention(dim, kv, group, tokens, context):
    c = form_case(dim, kv, group, tokens, context)
    check_tree(c)
    assert (c["out"][tokens] == 0).all()
    if tokens > 1:                                        # the last token of a tree is nobody's ancestor
        want, bound = want_tree(c)
        c["k"][tokens - 1], c["v"][tokens - 1] = float("nan"), float("inf")
        others = np.arange(int(c["cu"][-1])) != tokens - 1
        R.close(run_tree(c)[:len(others)][others], want[:len(others)][others], bound[:len(others)][others])


@pytest.mark.parametrize("dim,tokens,context", [(128, 1, 2000), (128, 50, 900), (256, 1, 700), (192, 20, 1200), (64, 1, 3000)])
def test_captured_attention_of_large_tiles(dim, tokens, context):
    torch = G.torch_mod()
    c = form_case(dim, 2, 1, tokens, context)
    table, lens, cu, mask = dev(c["table"]), dev(c["lens"]), dev(c["cu"]), dev(c["mask"])
    step = lambda: egt.tree_attention(c["q"], c["k"], c["v"], c["k_cache"], c["v_cache"], table, lens, cu, mask, c["out"], c["scale"], c["max_tokens"], c["ws"])  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        lens.copy_(torch.tensor([[context, 0, 33], [5, 1, 0], [context // 2, context, context - 1], [context, 31, 32]][k], dtype=torch.int32))
        step()
        torch.cuda.synchronize()
        want = c["out"].clone()
        c["out"].fill_(3)
        c["ws"].fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        used = int(c["cu"][-1])
        assert torch.equal(c["out"][:used], want[:used]) and bool((c["out"][used:] == 3).all())


def test_attention_over_a_long_context():
    check_tree(tree_case(np.random.default_rng(3), [40001, 11, 0, 9000], [2, 1, 4, 3], 4, 2, 64, 16))


def test_attention_of_many_requests():
    rng = np.random.default_rng(4)
    n = 150
    check_tree(tree_case(rng, rng.integers(0, 400, n).tolist(), rng.integers(0, 6, n).tolist(), 4, 2, 64, 16))


def test_attention_of_large_scores():
    # scores of some hundreds: one key takes nearly all the weight
    check_tree(tree_case(np.random.default_rng(5), [300, 20], [9, 40], 8, 2, 128, 16, scale=6.0))


@pytest.mark.parametrize("scale", [0.05, 0.3, 1.0, -7.0, 1e3, -1e6])
def test_attention_of_scores_past_whole_numbers(scale):
    """Scores from 2^20 on, up to 2^50: still weights between 0 and 1 that sum to 1."""
    for lens, counts, heads, kv_heads, dim in (([70, 0, 301], [5, 40, 1], 4, 2, 128), ([900], [2], 2, 2, 64), ([33], [64], 16, 4, 128), ([6000], [3], 4, 2, 96)):
        c = tree_case(np.random.default_rng(31), lens, counts, heads, kv_heads, dim, 16, scale=3000.0)
        c["k_cache"].mul_(3000)
        c["v"].copy_(c["v"] / 3000)
        c["scale"] = scale
        check_tree(c, scale)
        got, seen = c["out"][:int(c["cu"][-1])].float(), max(float(c["v"].abs().max()), float(c["v_cache"].abs().max()))
        assert float(got.abs().max()) <= seen and bool((got != 0).any(-1).all())


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-40, -0.125, -3.0])
def test_attention_of_other_scales(scale):
    """Every visible key weighs the same where the scale is zero, and what is masked still does not enter."""
    c = tree_case(np.random.default_rng(30), [0, 45, 300], [7, 40, 3], 4, 2, 64, 16)
    c["scale"] = scale
    c["mask"][3] = 0
    check_tree(c, scale)


def test_attention_rows_that_see_nothing_and_other_masks():
    rng = np.random.default_rng(6)
    c = tree_case(rng, [0, 70, 0], [40, 20, 64], 6, 2, 64, 16)
    c["mask"][:5] = 0                                     # no context, no token
    c["mask"][5] = (1 << 64) - 1                          # bits past the request's tokens do not count
    c["mask"][6] = 1 << 39
    c["mask"][45:50] = 0                                  # the context alone
    c["mask"][60:124] = [(1 << (j + 1)) - 1 for j in range(64)]      # a chain
    c["mask"][70] = 0
    c["mask"] = c["mask"].astype(np.uint64)
    check_tree(c)
    got = c["out"].cpu().numpy()
    assert (got[:5] == 0).all() and (got[70] == 0).all()


def test_attention_does_not_see_what_is_masked():
    """NaN and infinities behind the context, in pages past it, in masked tokens and in rows of other requests."""
    torch = G.torch_mod()
    rng = np.random.default_rng(7)
    for dim, heads in ((64, 8), (128, 2)):
        c = tree_case(rng, [37, 64, 0, 5], [30, 12, 40, 1], heads, 2, dim, 16)
        want, bound = want_tree(c)
        for cache in (c["k_cache"], c["v_cache"]):
            used = torch.zeros(cache.shape[0], cache.shape[2], dtype=torch.bool)
            for r, n in enumerate(c["lens"].tolist()):
                for p in range(n):
                    used[c["table"][r, p // 16], p % 16] = True
            cache.permute(0, 2, 1, 3)[~used.cuda()] = float("nan")
        hidden = [7, 33, 50]                              # tokens of requests 0, 1 and 2 that only they themselves see
        for t, bad in zip(hidden, (float("nan"), float("inf"), float("-inf"))):
            r = int(np.searchsorted(c["cu"], t, side="right")) - 1
            bit = np.uint64(1 << (t - c["cu"][r]))
            rows = slice(c["cu"][r], c["cu"][r + 1])
            c["mask"][rows] &= ~bit
            c["mask"][t] |= bit
        want, bound = want_tree({**c, "k_cache": c["k_cache"].nan_to_num(0), "v_cache": c["v_cache"].nan_to_num(0)})
        for t, bad in zip(hidden, (float("nan"), float("inf"), float("-inf"))):
            c["k"][t] = bad
            c["v"][t, :, 3::5] = bad
        c["q"][83:] = float("nan")
        got = run_tree(c)
        fine = [i for i in range(83) if i not in hidden]
        R.close(got[fine], want[fine], bound[fine], f"dim {dim}")


def test_attention_passes_on_what_a_row_sees():
    """A NaN or an infinite value that a row does see is in its result, there and nowhere else."""
    rng = np.random.default_rng(8)
    c = tree_case(rng, [40, 70], [20, 33], 4, 2, 64, 16)
    c["mask"][:20] |= np.uint64(1 << 4)
    c["mask"][20:53] |= np.uint64(1 << 32)
    want, bound = want_tree(c)
    c["v"][4, 0, 5] = float("nan")
    c["v"][52, 1, 9] = float("inf")
    c["v_cache"][int(c["table"][1, 2]), 0, 3, 7] = float("-inf")
    want[:20, :2, 5] = np.nan
    want[20:53, 2:, 9] = np.inf
    want[20:53, :2, 7] = -np.inf
    R.close(run_tree(c)[:53], want[:53], bound[:53])


def test_attention_of_what_it_cannot_trust():
    """NaN for bad pages, lengths and counts, in the rows of that request; other requests as ever."""
    rng = np.random.default_rng(9)
    base = tree_case(rng, [40, 70, 33, 90], [3, 20, 5, 7], 4, 2, 64, 16)
    want, bound = want_tree(base)
    rows = [slice(int(a), int(b)) for a, b in zip(base["cu"], base["cu"][1:])]
    for what, change in {"page": lambda c: c["table"].__setitem__((1, 2), -1), "page past the cache": lambda c: c["table"].__setitem__((1, 4), c["k_cache"].shape[0]),
                         "negative length": lambda c: c["lens"].__setitem__(1, -1), "length past the table": lambda c: c["lens"].__setitem__(1, 10 ** 6),
                         "more tokens than said": lambda c: c.__setitem__("max_tokens", 19)}.items():
        c = {**base, "table": base["table"].copy(), "lens": base["lens"].copy()}
        change(c)
        c["out"].fill_(7.0)
        got = run_tree(c)
        assert np.isnan(got[rows[1]]).all(), what
        for r in (0, 2, 3):
            R.close(got[rows[r]], want[rows[r]], bound[rows[r]], what)
        assert (got[35:] == 7).all()
    c = {**base, "table": base["table"].copy()}
    c["table"][0, 3:] = -5                                # pages past the length are not looked at
    R.close(run_tree(c)[rows[0]], want[rows[0]], bound[rows[0]])
    c = {**base, "cu": np.array([0, 3, 2, 30, 60], np.int32)}       # requests 1 and 3 are none: their rows stay
    c["out"].fill_(7.0)
    c["max_tokens"] = 64
    got = run_tree({**c, "ws": tree_case(rng, [40, 70, 33, 90], [3, 64, 5, 7], 4, 2, 64, 16)["ws"]})
    R.close(got[:2], want[:2], bound[:2])
    assert (got[30:] == 7).all()


def test_attention_is_the_same_on_every_run_and_with_any_workspace():
    rng = np.random.default_rng(10)
    for lens, counts in (([9000], [3]), ([700, 3000, 11], [20, 1, 9])):
        c = tree_case(rng, lens, counts, 8, 2, 128, 32)
        a = run_tree(c).copy()
        c["ws"].zero_()
        assert np.array_equal(run_tree(c), a)
        c["ws"] = G.torch_mod().full((c["ws"].numel() + 512,), 127, dtype=G.torch_mod().uint8, device="cuda")[256:]
        assert np.array_equal(run_tree(c), a)


def test_attention_far_into_a_cache():
    """Offsets past 32 bits: pages beyond 4 GB of a cache of 5 GB, and a token stride that is a page's."""
    torch = G.torch_mod()
    rng = np.random.default_rng(11)
    c = tree_case(rng, [200], [5], 4, 2, 128, 16)
    blocks = (5 << 30) // (2 * 16 * 128 * 2)
    width = c["table"].shape[1]
    for name in ("k_cache", "v_cache"):
        big = torch.empty((blocks, 2, 16, 128), dtype=torch.float16, device="cuda")
        big[-width:] = c[name][torch.from_numpy(c["table"][0]).long().cuda()]
        c[name] = big
    small = {**c, "k_cache": c["k_cache"][-width:], "v_cache": c["v_cache"][-width:], "table": np.arange(width, dtype=np.int32)[None]}
    c["table"] = np.arange(blocks - width, blocks, dtype=np.int32)[None]
    want, bound = want_tree(small)
    R.close(run_tree(c)[:5], want[:5], bound[:5])
    slots = np.array([blocks * 16 - 1, (blocks - 2) * 16 + 3], np.int32)
    egt.kv_append(c["k"][:2], c["v"][:2], dev(slots), c["k_cache"], c["v_cache"])
    assert torch.equal(c["k_cache"][-1, :, 15], c["k"][0]) and torch.equal(c["v_cache"][-2, :, 3], c["v"][1])


def test_attention_refuses_on_the_host():
    c = tree_case(np.random.default_rng(12), [20], [3], 4, 2, 64, 16)
    call = lambda **k: egt.tree_attention(**{**dict(q=c["q"], k=c["k"], v=c["v"], k_cache=c["k_cache"], v_cache=c["v_cache"], block_table=dev(c["table"]),  # noqa: E731
                                                    lens=dev(c["lens"]), cu_tokens=dev(c["cu"]), mask=dev(c["mask"]), out=c["out"], scale=1.0, max_tokens=3, workspace=c["ws"]), **k})
    for wrong in (dict(q=c["q"].float()), dict(k=c["k"][:, :1]), dict(v=c["v"][:-1]), dict(lens=dev(np.array([20], np.int64))), dict(mask=dev(c["mask"])[:2]),
                  dict(out=c["q"]), dict(out=c["out"][:1].expand(5, -1, -1)), dict(q=c["q"].transpose(1, 2)), dict(v_cache=c["v_cache"][:1]), dict(cu_tokens=dev(c["cu"])[:1]),
                  dict(scale="1"), dict(max_tokens=3.0), dict(workspace=c["ws"].cpu()), dict(stream=3)):
        with pytest.raises(ValueError):
            call(**wrong)
    for wrong, status in ((dict(workspace=None), 1), (dict(max_tokens=65), 2), (dict(workspace=c["ws"][:8]), 2), (dict(scale=float("nan")), 2)):
        with pytest.raises(egt.EgtError) as e:
            call(**wrong)
        assert e.value.status == status
    call()


# ---------------------------------------------------------------- adapters
def lora_case(rng, M, cols, rows, rank, n, index=None, pad=0, scale=0.02):
    torch = G.torch_mod()
    c = dict(X=dev(f16(rng, M, cols + 8 * pad))[:, :cols], A=dev(f16(rng, n, rank, cols, scale=scale)), B=dev(f16(rng, n, rows, rank, scale=scale)),
             base=dev(f16(rng, M, rows + pad))[:, :rows], index=np.array(rng.integers(-1, n, M) if index is None else index, np.int32),
             scale=rng.uniform(0.25, 2, n).astype(np.float32))
    c["buf"], wide = guarded((M, rows + pad), torch.float16, 9.0)
    c["wide"], c["Y"] = wide, wide[:, :rows]
    c["ws"] = torch.full((egt.lora_smallm_ws_bytes(c["X"], c["A"]),), 255, dtype=torch.uint8, device="cuda")
    return c


def check_lora(c, base=True, scale=True, what=""):
    torch = G.torch_mod()
    print("case lora", tuple(c["X"].shape), tuple(c["B"].shape), flush=True)
    egt.lora_smallm(c["X"], c["A"], c["B"], dev(c["index"]), c["Y"], c["ws"], base=c["base"] if base else None, scale=dev(c["scale"]) if scale else None)
    torch.cuda.synchronize()
    f = lambda t: t.cpu().numpy().astype(np.float64)  # noqa: E731
    want, bound = R.lora(f(c["X"]), f(c["A"]), f(c["B"]), c["index"], f(c["base"]) if base else np.zeros(c["Y"].shape),
                         c["scale"].astype(np.float64) if scale else np.ones(len(c["scale"])))
    R.close(c["Y"].cpu().numpy(), want, bound, what)
    untouched(c["buf"], 9)
    assert (c["wide"][:, c["Y"].shape[1]:] == 9).all()


@pytest.mark.parametrize("M,cols,rows,rank,n,pad", [
    (1, 8, 1, 8, 1, 0), (1, 4096, 4096, 16, 3, 0), (2, 512, 333, 8, 2, 1), (5, 1000, 129, 24, 4, 3), (16, 4096, 1024, 16, 4, 0), (17, 264, 4097, 40, 9, 0),
    (33, 2048, 700, 64, 2, 1), (64, 4096, 2048, 32, 64, 0), (64, 1032, 500, 128, 3, 2), (64, 11008, 260, 8, 1, 0), (48, 96, 64, 120, 100, 0), (64, 16384, 64, 56, 5, 0)])
def test_adapters(M, cols, rows, rank, n, pad):
    check_lora(lora_case(np.random.default_rng(M * 1000 + cols), M, cols, rows, rank, n, pad=pad))


@pytest.mark.parametrize("rows,rank,pad", [(4096, 32, 0), (4100, 64, 1), (8192, 128, 0), (4099, 16, 0)])
def test_adapters_of_many_tokens_and_rows(rows, rank, pad):
    rng = np.random.default_rng(rows)
    index = rng.integers(-1, 65, 64)                      # none, one past the last, and tokens that share one
    index[40:60] = 7
    c = lora_case(rng, 64, 64, rows, rank, 64, index.tolist(), pad=pad)
    check_lora(c)
    check_lora(c, base=False)


# Every kernel of the adapters' second product (test_serve_host.py asks the library), with rows that do not fill the last workgroup
ADAPTER_FORMS = [(rows, rank, pad) for rank in (16, 32, 40, 64, 72, 128) for rows, pad in ((60, 0), (4100, 0), (4100, 4), (2100, 0), (2099, 1))]


@pytest.mark.parametrize("rows,rank,pad", ADAPTER_FORMS)
def test_every_form_of_the_adapters(rows, rank, pad):
    rng = np.random.default_rng(rows + rank)
    index = rng.integers(-1, 65, 64)
    index[40:60] = 7
    c = lora_case(rng, 64, 72, rows, rank, 64, index.tolist(), pad=pad)
    check_lora(c)
    check_lora(c, base=False)


def test_adapters_one_for_all_none_for_all_and_without_options():
    rng = np.random.default_rng(20)
    for index in ([2] * 64, [-1] * 64, list(range(64)), [-5, 3] * 32):
        c = lora_case(rng, 64, 512, 300, 16, 64, index)
        check_lora(c)
        check_lora(c, base=False)
        check_lora(c, scale=False)
        if index[0] == -1:
            check_lora(c)
            assert np.array_equal(c["Y"].cpu().numpy(), c["base"].cpu().numpy())


def test_adapters_in_place_and_out_of_a_pool():
    torch = G.torch_mod()
    rng = np.random.default_rng(21)
    c = lora_case(rng, 20, 640, 500, 24, 6)
    c["A"] = torch.stack([c["A"], c["A"] * 2], 1)[:, 1]   # every second matrix of a pool
    c["B"] = torch.stack([c["B"], c["B"] * 2], 1)[:, 0]
    check_lora(c)
    want = c["Y"].clone()
    Y = c["base"].clone()
    egt.lora_smallm(c["X"], c["A"], c["B"], dev(c["index"]), Y, c["ws"], base=Y, scale=dev(c["scale"]))
    assert torch.equal(Y, want)


def test_adapters_past_the_last_and_large_numbers():
    rng = np.random.default_rng(22)
    check_lora(lora_case(rng, 9, 256, 100, 16, 4, [0, 4, -1, 3, 2 ** 31 - 1, -2 ** 31, 1, 1, 100]))
    # A . x beyond the range of FP16: only the result has to fit
    c = lora_case(rng, 20, 1024, 200, 16, 3)
    c["A"] *= 5000
    c["X"] *= 100
    c["B"] *= 1e-3
    check_lora(c)
    c = lora_case(rng, 20, 1024, 200, 16, 3)              # ... and below it
    c["A"] *= 1e-2
    c["X"] *= 1e-2
    c["B"] *= 100
    check_lora(c)


def apart(c, large, small):
    """Every third rank `large`, and B zero there: the result is that of the ranks that are `small` times as large or less."""
    rank = c["A"].shape[1]
    c["A"] *= dev(np.where(np.arange(rank) % 3 == 0, large, small * 0.5 ** (np.arange(rank) % 7)).astype(np.float16))[None, :, None]
    c["B"][:, :, ::3] = 0
    c["B"] *= 2000
    c["base"].mul_(2.0 ** -10)
    return c


@pytest.mark.parametrize("large,small", [(2.0 ** 12, 2.0 ** -8), (2.0 ** 15, 2.0 ** -12)])
@pytest.mark.parametrize("M,rows,rank", [(1, 40, 8), (3, 333, 24), (20, 4100, 32), (64, 300, 64), (17, 500, 128)])
def test_adapters_whose_ranks_differ_in_size(M, rows, rank, large, small):
    c = apart(lora_case(np.random.default_rng(rank), M, 512, rows, rank, 3), large, small)
    check_lora(c)
    check_lora(c, base=False)


def test_a_token_whose_ranks_lie_far_apart_beside_others():
    """What one token needs, an infinity among it, changes no bit of the other tokens of its adapter."""
    rng = np.random.default_rng(24)
    c = lora_case(rng, 40, 512, 200, 24, 1, [0] * 40)
    c["X"][7] = 0
    c["X"][7, 0], c["A"][0, 1, 0] = 60000, 6e-8
    check_lora(c)
    alone = c["Y"].clone()
    c["X"][9, 3] = float("inf")
    egt.lora_smallm(c["X"], c["A"], c["B"], dev(c["index"]), c["Y"], c["ws"], base=c["base"], scale=dev(c["scale"]))
    ok = np.isfinite(c["Y"].cpu().numpy())
    others = np.arange(40) != 9
    assert not ok[9].any() and ok[others].all()
    assert np.array_equal(c["Y"].cpu().numpy()[others], alone.cpu().numpy()[others])


def test_adapters_of_a_small_rank_beside_a_large_one():
    torch = G.torch_mod()
    X, A, B, Y = (torch.zeros(s, dtype=torch.float16, device="cuda") for s in ((1, 8), (1, 8, 8), (1, 4, 8), (1, 4)))
    ws = torch.zeros(egt.lora_smallm_ws_bytes(X, A), dtype=torch.uint8, device="cuda")
    X[0, 0], A[0, 0, 0], A[0, 1, 1] = 30000, 1, 1
    for small, weight in ((3e-4, 1000), (0.01, 1000), (6e-8, 60000), (0.7, 1)):
        X[0, 1], B[0, :, 1] = small, weight
        egt.lora_smallm(X, A, B, dev(np.zeros(1, np.int32)), Y, ws)
        want = (X[0, 1].double() * weight).half()
        assert bool((Y == want).all()), (small, Y, want)


def test_an_infinity_stays_with_its_token():
    rng = np.random.default_rng(23)
    c = lora_case(rng, 20, 256, 100, 16, 2, [0, 1] * 10)
    c["X"][3, 5] = float("inf")
    egt.lora_smallm(c["X"], c["A"], c["B"], dev(c["index"]), c["Y"], c["ws"], base=c["base"], scale=dev(c["scale"]))
    ok = np.isfinite(c["Y"].cpu().numpy())
    assert not ok[3].any() and ok[np.arange(20) != 3].all()


# ---------------------------------------------------------------- rules on logits
def rules_case(rng, counts, vocab, length, kind, masks=3, pad=0, spare=2, n_bias=9):
    torch = G.torch_mod()
    n, cu = len(counts), np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    N = int(cu[-1]) + spare
    wide = dev((rng.standard_normal((N, vocab + pad)) * 4).astype(np.float16 if kind == "fp16" else np.float32))
    c = dict(cu=cu, history=(vocab * rng.random((n, length)) ** 3).astype(np.int32), history_len=rng.integers(0, length + 1, n).astype(np.int32),
             draft=(vocab * rng.random(N) ** 3).astype(np.int32), mask=R.trees(rng, counts, N), repetition=rng.uniform(0.8, 1.5, n).astype(np.float32),
             frequency=rng.uniform(-0.5, 1, n).astype(np.float32), presence=rng.uniform(-0.5, 1, n).astype(np.float32),
             bias_ids=rng.integers(-2, vocab + 2, (n, n_bias)).astype(np.int32), bias=rng.normal(0, 3, (n, n_bias)).astype(np.float32),
             allowed=rng.integers(0, 1 << 32, (max(masks, 1), -(-vocab // 32)), dtype=np.uint64).astype(np.uint32), allowed_row=rng.integers(-1, max(masks, 1), N).astype(np.int32))
    c["prompt_len"] = (c["history_len"] * rng.random(n)).astype(np.int32)
    if length:
        c["history"][:, ::5] = c["history"][:, :1]
        c["history"][0, -1] = vocab
        c["history"][-1, 0] = -1
    if n_bias > 4:
        c["bias_ids"][:, 4] = c["bias_ids"][:, 1]
    logits = wide[:, :vocab]
    buf, out = guarded((N, vocab + pad), logits.dtype, 5.0)
    return c, logits, buf, out


RULES = ("history", "history_len", "prompt_len", "draft", "mask", "repetition", "frequency", "presence", "bias_ids", "bias", "allowed", "allowed_row")


def check_rules(c, logits, buf, out, leave=(), what=""):
    torch = G.torch_mod()
    print("case rules", tuple(logits.shape), c["cu"].tolist()[-1], leave, flush=True)
    vocab = logits.shape[1]
    kept = {k: c[k] for k in RULES if k not in leave}
    out.fill_(5.0)
    egt.logits_rules(logits, out[:, :vocab], dev(c["cu"]), **{k: dev(v) for k, v in kept.items()})
    torch.cuda.synchronize()
    want, bound = R.rules(logits.cpu().numpy().astype(np.float64), c["cu"], logits.dtype == torch.float16, **kept)
    got, used = out.cpu().numpy(), int(c["cu"][-1])
    R.close(got[:used, :vocab], want[:used], bound[:used], what)
    assert (got[used:] == 5).all() and (got[:, vocab:] == 5).all(), "rows behind the last request, or columns behind the last id"
    untouched(buf, 5)


@pytest.mark.parametrize("counts,vocab,length,kind,pad", [
    ([1], 1, 1, "fp16", 0), ([1], 31, 7, "fp32", 0), ([1], 32003, 600, "fp16", 0), ([3, 0, 2], 1000, 40, "fp16", 1), ([64], 5000, 300, "fp32", 3), ([5, 17, 33], 4097, 0, "fp16", 0),
    ([1] * 70, 2049, 100, "fp16", 7), ([4, 4], 50257, 2000, "fp16", 0), ([2], 128000, 9000, "fp16", 0), ([2, 1], 100001, 513, "fp32", 0), ([7], 8192, 4096, "fp16", 8)])
def test_rules(counts, vocab, length, kind, pad):
    check_rules(*rules_case(np.random.default_rng(vocab + length), counts, vocab, length, kind, pad=pad))


@pytest.mark.parametrize("counts,vocab,length,kind", [
    ([1, 0, 2] * 1700, 45, 8, "fp16"), ([2] * egt.MAX_REQUESTS, 9, 3, "fp32"), ([64, 1, 0, 64, 60, 64], 100003, 5000, "fp16"), ([64, 3, 64, 61], 131072, 60, "fp32")])
def test_rules_of_many_requests_and_rows(counts, vocab, length, kind):
    """Requests by the thousand, and several rows a workgroup that change from request to request."""
    check_rules(*rules_case(np.random.default_rng(vocab), counts, vocab, length, kind, n_bias=300 if vocab > 1000 else 5))


@pytest.mark.parametrize("leave", [("history", "history_len", "prompt_len"), ("prompt_len",), ("draft", "mask"), ("repetition",), ("frequency",), ("presence",),
                                   ("bias_ids", "bias"), ("allowed", "allowed_row"), RULES])
def test_rules_left_out(leave):
    for kind in ("fp16", "fp32"):
        c, logits, buf, out = rules_case(np.random.default_rng(1), [3, 6], 9001, 200, kind)
        check_rules(c, logits, buf, out, leave)
    if leave == RULES:
        assert G.torch_mod().equal(out[:9], logits[:9])


def test_rules_masks_that_leave_nothing_and_odd_numbers():
    torch = G.torch_mod()
    for kind in ("fp16", "fp32"):
        c, logits, buf, out = rules_case(np.random.default_rng(2), [9, 5], 3001, 100, kind)
        logits[:, 5::7] = float("nan")
        logits[:, 6::7] = float("inf")
        logits[:, 7::7] = float("-inf")
        logits[:, 8::7] = torch.finfo(logits.dtype).min
        logits[:, 9::7] = -0.0
        c["allowed"][1] = 0
        c["allowed_row"][:4] = 1                          # nothing is allowed
        c["allowed_row"][4] = 3                           # past the masks
        c["allowed_row"][5] = 2 ** 31 - 1
        c["frequency"][:], c["presence"][:] = 0.5, 0.25
        vocab = logits.shape[1]
        with np.errstate(all="ignore"):
            want, bound = R.rules(logits.cpu().numpy().astype(np.float64), c["cu"], kind == "fp16", **{k: c[k] for k in RULES})
            if kind == "fp16":                            # what is beyond its range on the way out is infinite
                want = np.where(np.isfinite(want) & (np.abs(want) >= 65520), np.sign(want) * np.inf, want)
            else:
                want = want.astype(np.float32).astype(np.float64)
        egt.logits_rules(logits, out, dev(c["cu"]), **{k: dev(c[k]) for k in RULES})
        got = out.cpu().numpy()
        R.close(got[:14], want[:14], bound[:14], kind)
        assert (got[:4] == -np.inf).all() and np.isnan(got[4:6]).all()


@pytest.mark.parametrize("kind", ["fp16", "fp32"])
def test_rules_of_a_grammar_without_rows(kind):
    """Every row of it is past the last: NaN, not everything allowed."""
    c, logits, buf, out = rules_case(np.random.default_rng(6), [3, 2], 1000, 10, kind)
    c["allowed"] = c["allowed"][:0]
    c["allowed_row"] = np.array([-1, 0, 5, -7, 2 ** 31 - 1, 0, 0], np.int32)
    check_rules(c, logits, buf, out)
    got = out.cpu().numpy()
    assert np.isnan(got[[1, 2, 4]]).all() and not np.isnan(got[[0, 3]]).any()


def test_rules_in_place_and_bad_lengths():
    torch = G.torch_mod()
    c, logits, buf, out = rules_case(np.random.default_rng(3), [4, 8, 2], 6007, 64, "fp16")
    c["history_len"][:] = [-3, 1000, 20]
    c["prompt_len"][:] = [5, -1, 1000]
    check_rules(c, logits, buf, out)
    same = logits.clone()
    egt.logits_rules(same, same, dev(c["cu"]), **{k: dev(c[k]) for k in RULES})
    assert torch.equal(same[:14], out[:14]) and torch.equal(same[14:], logits[14:])
    out.fill_(5.0)
    egt.logits_rules(logits, out, dev(np.array([2, 1, 1, 40], np.int32)), **{k: dev(c[k]) for k in RULES})
    assert (out == 5).all()


def test_a_single_row_has_no_distance_to_another():
    """One token's X, Y, base and logits out of wider buffers, in place under another stride."""
    torch = G.torch_mod()
    rng = np.random.default_rng(70)
    a = lora_case(rng, 1, 64, 40, 8, 2, [1])
    a["X"] = dev(f16(rng, 1, 67))[:, :64]
    check_lora(a)
    Y = dev(f16(rng, 1, 44))[:, :40]
    want, bound = R.lora(*(t.cpu().numpy().astype(np.float64) for t in (a["X"], a["A"], a["B"])), a["index"], Y.cpu().numpy().astype(np.float64), np.ones(2))
    egt.lora_smallm(a["X"], a["A"], a["B"], dev(a["index"]), Y, a["ws"], base=Y.as_strided((1, 40), (40, 1)))
    R.close(Y.cpu().numpy(), want, bound)
    logits = dev(f16(rng, 1, 107))[:, :100]
    was = logits.cpu().numpy().astype(np.float64)
    factor = np.array([1.5], np.float32)
    history = dict(history=np.arange(0, 100, 7, dtype=np.int32)[None], history_len=np.array([9], np.int32), repetition=factor)
    egt.logits_rules(logits, logits.as_strided((1, 100), (100, 1)), dev(np.array([0, 1], np.int32)), **{k: dev(v) for k, v in history.items()})
    want, bound = R.rules(was, np.array([0, 1]), True, **history)
    R.close(logits.cpu().numpy(), want, bound)


# ---------------------------------------------------------------- together, on streams, in graphs
def test_a_verification_step():
    """Projections, adapters, attention, slots, writing and rules, twice: the second step reads what the first has written."""
    torch = G.torch_mod()
    rng = np.random.default_rng(30)
    heads, kv_heads, dim, page, hidden, vocab = 8, 2, 64, 16, 512, 2000
    rows = (heads + 2 * kv_heads) * dim
    w = synth.weights(rows, hidden, 31)
    p = egt.pack_2bitcsr(w, egt.prune_n4(w, 2), 2, 128, egt.VAL_INT4)
    dense = egt.unpack_2bitcsr(p)[0].astype(np.float64)
    wo = synth.weights(vocab, heads * dim, 32)
    po = egt.pack_2bitcsr(wo, egt.prune_n4(wo, 2), 2, 128, egt.VAL_INT4).to("cuda")
    pd = p.to("cuda")
    lens, blocks, width = np.array([30, 0, 47], np.int32), 40, 8
    ids = rng.permutation(blocks).astype(np.int32)
    table = np.full((3, width), -1, np.int32)
    table[0, :2], table[2, :3] = ids[:2], ids[2:5]
    kc, vc = dev(f16(rng, blocks, kv_heads, page, dim)), dev(f16(rng, blocks, kv_heads, page, dim))
    free, head, table_d, lens_d = dev(ids[5:]), dev(np.zeros(1, np.int32)), dev(table), dev(lens)
    A, Bm = dev(f16(rng, 3, 16, hidden, scale=0.05)), dev(f16(rng, 3, rows, 16, scale=0.05))
    for step, counts in enumerate(([7, 4, 12], [1, 20, 1])):
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        N = int(cu[-1])
        X = dev(f16(rng, N, hidden))
        Y = torch.empty((N, rows), dtype=torch.float16, device="cuda")
        index = rng.integers(-1, 3, N).astype(np.int32)
        mask = R.trees(rng, counts)
        ws = torch.empty(egt.lora_smallm_ws_bytes(X, A), dtype=torch.uint8, device="cuda")
        egt.sparse_gemm_smallm(pd, X, Y)
        egt.lora_smallm(X, A, Bm, dev(index), Y, ws, base=Y)
        f = lambda t: t.cpu().numpy().astype(np.float64)  # noqa: E731
        want, bound = R.lora(f(X), f(A), f(Bm), index, f(X) @ dense.T, np.ones(3))
        # the product before it: its own rounding to FP16, and products and sums of FP16 weights
        R.close(f(Y), want, bound + 2e-2 * (np.abs(f(X)) @ np.abs(dense).T) + 1e-3)
        qkv = Y.view(N, heads + 2 * kv_heads, dim)
        q, k, v = qkv[:, :heads], qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:]
        out = torch.empty((N, heads, dim), dtype=torch.float16, device="cuda")
        aws = torch.empty(egt.tree_attention_ws_bytes(q, kc, table_d, lens_d, max(counts)), dtype=torch.uint8, device="cuda")
        egt.tree_attention(q, k, v, kc, vc, table_d, lens_d, dev(cu), dev(mask), out, dim ** -0.5, max(counts), aws)
        want, bound = R.tree_attention(f(q), f(k), f(v), f(kc), f(vc), table_d.cpu().numpy(), lens_d.cpu().numpy(), cu, mask, dim ** -0.5)
        R.close(f(out), want, bound, f"step {step}")
        logits = torch.empty((N, vocab), dtype=torch.float16, device="cuda")
        egt.sparse_gemm_smallm(po, out.view(N, heads * dim), logits)
        draft = rng.integers(0, vocab, N).astype(np.int32)
        c = dict(draft=draft, mask=mask, frequency=np.full(3, 0.5, np.float32))
        ruled = torch.empty_like(logits)
        egt.logits_rules(logits, ruled, dev(cu), **{a: dev(b) for a, b in c.items()})
        want, bound = R.rules(f(logits), cu, True, **c)
        R.close(f(ruled), want, bound)
        # of every request the path to its last token is accepted
        accepted = [[cu[r] + j for j in range(counts[r]) if int(mask[cu[r + 1] - 1]) >> j & 1] for r in range(3)]
        n_acc = np.array([len(a) for a in accepted], np.int32)
        slots, cu2, lens2, head2 = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (40, 4, 3, 1))
        egt.kv_slots(lens_d, dev(n_acc), table_d, page, blocks, free, head, slots, cu2, lens2, head2)
        row = np.full(40, -1, np.int32)
        row[:n_acc.sum()] = np.concatenate(accepted)
        egt.kv_append(k, v, slots, kc, vc, dev(row))
        lens_d, head = lens2, head2
        assert np.array_equal(lens_d.cpu().numpy(), lens + n_acc)
        lens = lens + n_acc
        for r in range(3):
            for j, i in enumerate(accepted[r]):
                pos = int(lens[r] - n_acc[r]) + j
                assert torch.equal(kc[int(table_d[r, pos // page]), :, pos % page], k[i])


def test_captured_calls_run_again_with_other_lengths():
    torch = G.torch_mod()
    rng = np.random.default_rng(40)
    c = tree_case(rng, [700, 90, 30], [5, 9, 2], 8, 2, 64, 16)
    r, logits, buf, ruled = rules_case(rng, [5, 9, 2], 3001, 50, "fp16")
    a = lora_case(rng, 16, 512, 300, 16, 4)
    table, lens, cu, mask = dev(c["table"]), dev(c["lens"]), dev(c["cu"]), dev(c["mask"])
    rd, index = {k: dev(r[k]) for k in RULES}, dev(a["index"])
    counts, slots = dev(np.array([3, 2, 0], np.int32)), torch.zeros(8, dtype=torch.int32, device="cuda")
    free, head, cu2, lens2, head2 = (dev(np.array(v, np.int32)) for v in (range(10), [0], [0] * 4, [0] * 3, [0]))
    kc, vc = c["k_cache"].clone(), c["v_cache"].clone()

    def step():
        egt.tree_attention(c["q"], c["k"], c["v"], c["k_cache"], c["v_cache"], table, lens, cu, mask, c["out"], c["scale"], 9, c["ws"])
        egt.lora_smallm(a["X"], a["A"], a["B"], index, a["Y"], a["ws"], base=a["base"])
        egt.logits_rules(logits, ruled, cu, **rd)
        egt.kv_slots(lens, counts, table, 16, kc.shape[0], free, head, slots, cu2, lens2, head2)
        egt.kv_append(c["k"][:8], c["v"][:8], slots, kc, vc)
        return [t.clone() for t in (c["out"], a["Y"], ruled, slots, cu2, lens2, head2, kc, vc)]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        lens.copy_(torch.tensor([[700, 90, 30], [1, 0, 5], [300, 300, 300], [699, 16, 32]][k], dtype=torch.int32))
        index.copy_(torch.roll(index, 1))
        kc.copy_(c["k_cache"])
        vc.copy_(c["v_cache"])
        before = table.clone()
        want = step()
        torch.cuda.synchronize()
        for t in (c["out"], a["Y"], ruled, slots, cu2, lens2, head2):
            t.fill_(3)
        table.copy_(before)
        kc.copy_(c["k_cache"])
        vc.copy_(c["v_cache"])
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((c["out"], a["Y"], ruled, slots, cu2, lens2, head2, kc, vc), want):
            used = 16 if got is c["out"] or got is ruled else len(got)
            assert torch.equal(got[:used].view(torch.int16) if got.dtype == torch.float16 else got[:used], w[:used].view(torch.int16) if w.dtype == torch.float16 else w[:used])


def test_prepared_calls_and_other_streams():
    torch = G.torch_mod()
    rng = np.random.default_rng(50)
    c = tree_case(rng, [300, 8], [4, 6], 4, 2, 64, 16)
    a = lora_case(rng, 10, 512, 300, 16, 4)
    r, logits, buf, ruled = rules_case(rng, [4, 6], 3001, 50, "fp32")
    args = (c["q"], c["k"], c["v"], c["k_cache"], c["v_cache"], dev(c["table"]), dev(c["lens"]), dev(c["cu"]), dev(c["mask"]), c["out"], c["scale"], 6, c["ws"])
    want = [run_tree(c)[:10].copy()]
    check_lora(a, scale=False)
    want.append(a["Y"].cpu().numpy().copy())
    egt.logits_rules(logits, ruled, dev(c["cu"]), repetition=dev(r["repetition"]), draft=dev(r["draft"]), mask=dev(r["mask"]))
    want.append(ruled[:10].cpu().numpy().copy())
    kc, vc = torch.zeros_like(c["k_cache"]), torch.zeros_like(c["v_cache"])
    slots = dev(rng.permutation(50)[:12].astype(np.int32))
    head = dev(np.zeros(1, np.int32))
    o = [torch.zeros(m, dtype=torch.int32, device="cuda") for m in (5, 3, 2, 1)]
    calls = [egt.prepared_tree_attention(*args), egt.prepared_lora_smallm(a["X"], a["A"], a["B"], dev(a["index"]), a["Y"], a["ws"], base=a["base"]),
             egt.prepared_logits_rules(logits, ruled, dev(c["cu"]), repetition=dev(r["repetition"]), draft=dev(r["draft"]), mask=dev(r["mask"])),
             egt.prepared_kv_append(c["k"], c["v"], slots, kc, vc),
             egt.prepared_kv_slots(dev(np.array([3, 4], np.int32)), dev(np.array([2, 1], np.int32)), dev(np.array([[3, 0], [1, 2]], np.int32)), 4, 9, slots, head, *o)]
    del args, head, slots                                  # (the calls keep what they need)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream_ptr in (None, int(side.cuda_stream)):
        for t in (c["out"], a["Y"], ruled, kc, vc, *o):
            t.zero_()
        torch.cuda.synchronize()
        for call in calls:
            call() if stream_ptr is None else call(stream_ptr)
        torch.cuda.synchronize()
        for t, w in zip((c["out"][:10], a["Y"], ruled[:10]), want):
            assert np.array_equal(t.cpu().numpy(), w)
        assert o[2].tolist() == [5, 5] and int((kc != 0).any(3).any(1).sum()) == 12
    # the current stream, and one that is named
    for t in (c["out"], ruled):
        t.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        run_tree(c)
    egt.logits_rules(logits, ruled, dev(c["cu"]), repetition=dev(r["repetition"]), draft=dev(r["draft"]), mask=dev(r["mask"]), stream=side)
    torch.cuda.synchronize()
    assert np.array_equal(c["out"][:10].cpu().numpy(), want[0]) and np.array_equal(ruled[:10].cpu().numpy(), want[2])


def test_empty_batches():
    torch = G.torch_mod()
    z = lambda *s, t=torch.float16: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    i = lambda *s: z(*s, t=torch.int32)  # noqa: E731
    ws = z(64, t=torch.uint8)
    egt.tree_attention(z(0, 4, 64), z(0, 2, 64), z(0, 2, 64), z(3, 2, 16, 64), z(3, 2, 16, 64), i(2, 1), i(2), i(3), z(0, t=torch.int64), z(0, 4, 64), 1.0, 1, ws)
    egt.tree_attention(z(2, 4, 64), z(2, 2, 64), z(2, 2, 64), z(3, 2, 16, 64), z(3, 2, 16, 64), i(0, 1), i(0), i(1), z(2, t=torch.int64), z(2, 4, 64), 1.0, 1, ws)
    out = z(1, 4, 64) + 3
    egt.tree_attention(z(1, 4, 64), z(1, 2, 64), z(1, 2, 64), z(0, 2, 16, 64), z(0, 2, 16, 64), i(1, 0), i(1), i(2) + torch.tensor([0, 1], device="cuda", dtype=torch.int32),
                       z(1, t=torch.int64) + 1, out, 1.0, 1, z(1 << 20, t=torch.uint8))
    assert (out == 0).all()                               # no cache at all, one token that sees itself: its value
    egt.kv_append(z(0, 2, 64), z(0, 2, 64), i(0), z(3, 2, 16, 64), z(3, 2, 16, 64))
    egt.logits_rules(z(0, 100), z(0, 100), i(1))
    egt.logits_rules(z(3, 0), z(3, 0), i(2))
    torch.cuda.synchronize()


def test_an_error_of_the_hip_runtime_is_raised_by_the_call_that_meets_it():
    """Entry points that fail with a HIP error: one call, one exception, plain and prepared."""
    import ctypes as C
    rng = np.random.default_rng(60)
    calls = []
    types = {"egt_kv_slots": 2, "egt_kv_append": 3, "egt_tree_attention": 5, "egt_tree_attention_ws_bytes": 3, "egt_lora_smallm": 4, "egt_logits_rules": 2}

    def failing(name):
        def entry(*a):
            calls.append(name)
            return 7
        return C.CFUNCTYPE(C.c_int, *[C.c_size_t if (name, k) in (("egt_tree_attention", 3), ("egt_lora_smallm", 2)) else C.c_void_p for k in range(types[name])])(entry)
    c = tree_case(rng, [20], [3], 4, 2, 64, 16)
    a = lora_case(rng, 4, 64, 40, 8, 2)
    i = dev(np.zeros(4, np.int32))
    fns = [failing(name) for name in egt._batches]
    native = egt._native()
    native.bind_batches(*[C.cast(f, C.c_void_p).value for f in fns])
    tree = (c["q"], c["k"], c["v"], c["k_cache"], c["v_cache"], dev(c["table"]), dev(c["lens"]), dev(c["cu"]), dev(c["mask"]), c["out"], 1.0, 3, c["ws"])
    slots = (i[:2], i[:2], i.view(2, 2), 16, 4, i, i[:1], i, i[:3], i[:2], i[:1])
    try:
        for name, args in (("kv_slots", slots), ("kv_append", (c["k"], c["v"], dev(np.zeros(5, np.int32)), c["k_cache"], c["v_cache"])), ("tree_attention", tree),
                           ("lora_smallm", (a["X"], a["A"], a["B"], dev(a["index"]), a["Y"], a["ws"])), ("logits_rules", (a["Y"], a["Y"], dev(np.array([0, 4], np.int32))))):
            for call in (lambda: getattr(egt, name)(*args), lambda: getattr(egt, "prepared_" + name)(*args)()):
                with pytest.raises(egt.EgtError) as e:
                    call()
                assert e.value.status == 7 and calls == ["egt_" + name]
                calls.clear()
    finally:
        egt._call = None
        egt._native()
    run_tree(c)


def test_refused_calls_write_nothing():
    torch = G.torch_mod()
    rng = np.random.default_rng(61)
    a = lora_case(rng, 4, 64, 40, 8, 2)
    call = lambda **k: egt.lora_smallm(**{**dict(X=a["X"], A=a["A"], B=a["B"], index=dev(a["index"]), Y=a["Y"], workspace=a["ws"], base=a["base"], scale=dev(a["scale"])), **k})  # noqa: E731
    a["wide"].fill_(9.0)
    for wrong in (dict(X=a["X"][:, :56]), dict(A=a["A"].float()), dict(B=a["B"][:1]), dict(B=a["B"].transpose(0, 1)), dict(index=dev(np.zeros(3, np.int32))), dict(Y=a["Y"][:3]),
                  dict(base=a["base"][:, :39]), dict(scale=dev(np.ones(3, np.float32))), dict(Y=a["Y"][:1].expand(4, -1)), dict(workspace=a["ws"].cpu())):
        with pytest.raises(ValueError):
            call(**wrong)
    for wrong, status in ((dict(workspace=None), 1), (dict(workspace=a["ws"][:4]), 2), (dict(X=a["X"].repeat(17, 1), Y=a["Y"].repeat(17, 1), base=None, index=dev(np.zeros(68, np.int32))), 2)):
        with pytest.raises(egt.EgtError) as e:
            call(**wrong)
        assert e.value.status == status
    r, logits, buf, out = rules_case(rng, [3, 1], 1000, 20, "fp16")
    rules = lambda **k: egt.logits_rules(**{**dict(logits=logits, out=out, cu_tokens=dev(r["cu"]), history=dev(r["history"]), history_len=dev(r["history_len"])), **k})  # noqa: E731
    for wrong in (dict(out=out.float()), dict(out=out[:, :999]), dict(history_len=None), dict(history=dev(r["history"][:1])), dict(draft=dev(r["draft"])), dict(mask=dev(r["mask"])),
                  dict(allowed=dev(r["allowed"])), dict(allowed=dev(r["allowed"])[:, :31], allowed_row=dev(r["allowed_row"])), dict(bias_ids=dev(r["bias_ids"])), dict(repetition=dev(r["repetition"])[:1]),
                  dict(logits=logits.bfloat16()), dict(out=out.t()), dict(cu_tokens=dev(r["cu"])[:0])):
        with pytest.raises(ValueError):
            rules(**wrong)
    k = dev(f16(rng, 4, 2, 64))
    cache = dev(f16(rng, 3, 2, 16, 64))
    append = lambda **o: egt.kv_append(**{**dict(k=k, v=k, slots=dev(np.zeros(4, np.int32)), k_cache=cache, v_cache=cache), **o})  # noqa: E731
    before = cache.clone()
    for wrong in (dict(slots=dev(np.zeros(3, np.int32))), dict(v=k[:3]), dict(k=k[:, :1]), dict(k_cache=cache[:, :, :, :56]), dict(v_cache=cache[:2]), dict(k_cache=cache[:1].expand(3, -1, -1, -1)),
                  dict(rows=dev(np.zeros(3, np.int32))), dict(slots=dev(np.zeros(4, np.int64)))):
        with pytest.raises(ValueError):
            append(**wrong)
    with pytest.raises(egt.EgtError) as e:                # (a page of 12 tokens)
        append(k_cache=cache[:, :, :12], v_cache=cache[:, :, :12])
    assert e.value.status == 2
    i = dev(np.zeros(8, np.int32))
    for wrong in (dict(counts=i[:3]), dict(block_table=i.view(4, 2)), dict(cu_tokens=i[:2]), dict(new_head=i[:2]), dict(page=16.0), dict(slots=i.long()), dict(block_table=i[:2].view(2, 1).expand(2, 3))):
        with pytest.raises(ValueError):
            egt.kv_slots(**{**dict(lens=i[:2], counts=i[2:4], block_table=i.view(2, 4), page=16, blocks=4, free_blocks=i, free_head=i[:1], slots=i, cu_tokens=i[:3], new_lens=i[4:6], new_head=i[7:]), **wrong})
    torch.cuda.synchronize()
    assert (a["wide"] == 9).all() and (out == 5).all() and torch.equal(cache, before)
