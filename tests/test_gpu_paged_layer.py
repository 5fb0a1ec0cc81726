"""The sparsified attention on a cache in pages (dv_sparse_attn_paged) on the GPU against the fp64 oracle and against
dv_sparse_attn on a cache without pages, at the tolerance of the other layer tests (REL_TOL: relative L2 error)."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2310_17157_amd import binding as B
from paper_2310_17157_amd.workload import layer_objects
from synth import get_config, make_layer
from tests.gpu_util import REL_TOL, host, oracle_attn, rel_l2

pytestmark = pytest.mark.gpu


def setup(pos, n_heads, cfg="small_f16", seq=None, shared=0, page=16, biases=True, seed=3, rot=None, layout="half", **kw):
    """A layer, a pool with the attended rows filled and everything else NaN, and what the oracle needs of them."""
    rng = np.random.default_rng(seed)
    cfg = get_config(cfg).with_(**kw) if kw else get_config(cfg)
    t = make_layer(cfg, seed, device="cuda", biases=biases)
    pos = np.asarray(pos, dtype=np.int32)
    seq = np.arange(len(pos), dtype=np.int32) if seq is None else np.asarray(seq, dtype=np.int32)
    n_seq = int(seq.max()) + 1
    lens = [max([int(p) + 1 for p, s in zip(pos, seq) if s == i] + [0]) for i in range(n_seq)]
    width = max([shared] + [-(-n // page) for n in lens]) + 1
    n_pages = shared + n_seq * width
    perm = rng.permutation(n_pages)
    table = perm[shared:].reshape(n_seq, width).astype(np.int32)
    table[:, :shared] = perm[:shared]
    dt = torch.float16 if cfg.kvdtype == "f16" else torch.float32
    K, V = (torch.full((n_pages, cfg.H, page, cfg.dh), float("nan"), dtype=dt, device="cuda") for _ in range(2))
    for i, n in enumerate(lens):
        for p in range(n):
            for c in (K, V):
                c[int(table[i, p // page]), :, p % page] = torch.from_numpy(rng.normal(size=(cfg.H, cfg.dh)) * 0.7).to(dt).cuda()
    heads = np.stack([np.sort(rng.permutation(cfg.H)[:n_heads]) for _ in pos]).astype(np.int32).reshape(len(pos), n_heads)
    x = torch.from_numpy(rng.normal(size=(len(pos), cfg.d)).astype(np.float32)).cuda()
    freq = P.freqs(rot) if rot else None
    rotary = B.Rotary(torch.from_numpy(freq).cuda(), {"half": B.DV_ROPE_HALF, "interleaved": B.DV_ROPE_INTERLEAVED}[layout],
                      1.25) if rot else None
    i32 = lambda v: torch.from_numpy(np.ascontiguousarray(v)).cuda()
    return dict(cfg=cfg, t=t, attn=layer_objects(t, cfg.H, biases=biases)[0], K=K, V=V, kv=B.PagedKV(K, V, i32(table)), table=table,
                seq=seq, pos=pos, heads=heads, x=x, freq=freq, layout=layout, rotary=rotary, shared=shared, page=page,
                biases=biases, max_len=max([1, shared * page] + lens), dseq=i32(seq), dpos=i32(pos), dheads=i32(heads))


def run(c, **kw):
    kw = dict(dict(rotary=c["rotary"], seq=c["dseq"], shared_pages=c["shared"]), **kw)
    return B.dv_sparse_attn_paged(c["attn"], c["x"], c["kv"], c["dpos"], c["max_len"], c["dheads"], c["cfg"].dh ** -0.5, **kw)


def oracle(c, K, V):
    return P.layer(host(c["x"]), oracle_attn(c["t"], c["biases"]), K.astype(np.float64), V.astype(np.float64), c["table"], c["seq"],
                   c["pos"], c["heads"], c["cfg"].dh ** -0.5, c["freq"], c["layout"], 1.25)


def check(c, **kw):
    K0, V0 = host(c["K"]).copy(), host(c["V"]).copy()
    out = run(c, **kw)
    torch.cuda.synchronize()
    want, K1, V1 = oracle(c, K0, V0)
    got = host(out)
    for b in range(len(got)):
        assert rel_l2(got[b], want[b]) < REL_TOL, (b, rel_l2(got[b], want[b]))
    # only the tokens' rows of their heads changed, and hold the keys and values
    mine = np.zeros(K0.shape, dtype=bool)
    for s, p, hs in zip(c["seq"], c["pos"], c["heads"]):
        if p >= 0:
            mine[c["table"][s, p // c["page"]], hs, p % c["page"]] = True
    for new, old, w in ((host(c["K"]), K0, K1), (host(c["V"]), V0, V1)):
        assert np.array_equal(np.where(mine, 0, new), np.where(mine, 0, old), equal_nan=True)
        if mine.any():
            assert rel_l2(new[mine], w[mine]) < REL_TOL
    return out


@pytest.mark.parametrize("cfg,pos,n_heads,kw", [
    ("small_f16", [0], 3, {}),
    ("small_f16", [70], 10, dict(rot=32)),
    ("small_f16", [200], 3, dict(rot=64, layout="interleaved", page=7)),
    ("small_f32", [33], 4, dict(rot=16)),
    ("small_f16", [130], 3, dict(kvdtype="f32", rot=32, biases=False)),
    ("small_f16", [90], 2, dict(shared=3)),
    ("opt125m_b1", [127], 6, dict(rot=64)),
    ("small_b8", [0, 5, 70, 33], 4, dict(rot=32)),
    ("small_b8", [100, 64, 80, 90, 66, 70, 99, 65, 77], 5, dict(shared=4, rot=64, layout="interleaved")),
    ("small_b8", [40, 17], 10, dict(kvdtype="f32", biases=False)),
    ("small_b8", [30, 31, 32, 50, 51], 4, dict(seq=[0, 0, 0, 1, 1], rot=32)),
    ("small_b8", list(range(20, 52)), 3, dict(rot=16, page=10)),
], ids=str)
def test_against_the_oracle(cfg, pos, n_heads, kw):
    check(setup(pos, n_heads, cfg, **kw))


@pytest.mark.parametrize("cfg,pos", [("small_f16", [-1]), ("small_b8", [9, -1, 40, -5])])
def test_idle_slots(cfg, pos):
    """An idle slot writes nothing and gives bo; the others do not see it."""
    c = setup(pos, 3, cfg, rot=32)
    out = check(c, flags=B.DV_VALIDATE)
    for b, p in enumerate(pos):
        if p < 0:
            assert np.array_equal(host(out)[b], host(c["t"]["bo"]))


@pytest.mark.parametrize("cfg,pos", [("small_f16", [4]), ("small_b8", [4, 20, 3])])
def test_no_heads_is_the_bias(cfg, pos):
    c = setup(pos, 0, cfg)
    K0 = c["K"].clone()
    out = run(c)
    torch.cuda.synchronize()
    for b in range(len(pos)):
        assert np.array_equal(host(out)[b], host(c["t"]["bo"]))
    assert torch.equal(K0.view(torch.int16), c["K"].view(torch.int16))


@pytest.mark.parametrize("cfg,pos", [("small_f16", [60]), ("small_b8", [60, 3, 41, 0])])
def test_as_on_a_cache_without_pages(cfg, pos):
    """Without rotation the layer is dv_sparse_attn with its rows elsewhere: both project, append and attend the same
    values; the sums are ordered otherwise."""
    c = setup(pos, 4, cfg)
    H, dh, page = c["cfg"].H, c["cfg"].dh, c["page"]
    flat = [torch.zeros(len(pos), H, 80, dh, dtype=c["K"].dtype, device="cuda") for _ in range(2)]
    for f, pool in zip(flat, (c["K"], c["V"])):
        for b, p in enumerate(pos):
            for i in range(p):
                f[b, :, i] = pool[int(c["table"][b, i // page]), :, i % page]
    want = B.dv_sparse_attn(c["attn"], c["x"], B.KVCache(flat[0], flat[1], pos), c["dheads"], dh ** -0.5)
    out = run(c)
    torch.cuda.synchronize()
    for b in range(len(pos)):
        assert rel_l2(host(out)[b], host(want)[b]) < REL_TOL
        for h in c["heads"][b]:
            row = c["K"][int(c["table"][b, pos[b] // page]), int(h), pos[b] % page]
            assert torch.equal(row, flat[0][b, int(h), pos[b]])


def test_refused_sets_and_pages():
    for cfg, pos in (("small_f16", [20]), ("small_b8", [20, 9])):
        c = setup(pos, 3, cfg)
        for bad in ([2, 1, 3], [0, 0, 1], [0, 1, c["cfg"].H]):
            d = dict(c, dheads=torch.tensor([bad] * len(pos), dtype=torch.int32, device="cuda"))
            with pytest.raises(B.DvError) as e:
                run(d, flags=B.DV_VALIDATE)
            assert e.value.status == B.DV_ERR_INDEX
        d = dict(c, kv=B.PagedKV(c["K"], c["V"], torch.full_like(c["kv"].table, 10 ** 6)))
        with pytest.raises(B.DvError) as e:
            run(d, flags=B.DV_VALIDATE)
        assert e.value.status == B.DV_ERR_INDEX


@pytest.mark.parametrize("cfg,B_", [("small_f16", 1), ("small_b8", 6)])
def test_captured_steps_and_other_stream(cfg, B_):
    """A captured step replayed over positions that the device holds, with eager steps between, equals eager steps on a
    pool of its own and steps on another stream."""
    base = [10 + 9 * b for b in range(B_)]
    c = setup([p + 6 for p in base], 3, cfg, rot=32)
    for pool in (c["K"], c["V"]):
        pool.nan_to_num_(0.25)
    c["max_len"] = 96 if c["kv"].table.shape[1] * c["page"] >= 96 else c["kv"].table.shape[1] * c["page"]
    pools = [(c["K"].clone(), c["V"].clone()) for _ in range(3)]
    kvs = [B.PagedKV(k, v, c["kv"].table) for k, v in pools]
    need = B.sparse_attn_paged_workspace_bytes(c["attn"], kvs[0], B_, 3, c["max_len"])
    wss = [torch.zeros(need, dtype=torch.uint8, device="cuda") for _ in range(3)]
    outs = [torch.empty_like(c["x"]) for _ in range(3)]
    c["dpos"].copy_(torch.tensor(base, dtype=torch.int32))

    def step(i, **kw):
        run(dict(c, kv=kvs[i]), out=outs[i], ws=wss[i], **kw)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    for i in range(3):
        step(i)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(0)
    for i in range(5):
        c["dpos"].copy_(torch.tensor([p + i for p in base], dtype=torch.int32))
        c["x"].mul_(0.9)
        graph.replay()
        step(1)
        torch.cuda.synchronize()
        side.wait_stream(torch.cuda.current_stream())
        step(2, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2]), i
        for a in (0, 1):
            assert torch.equal(pools[0][a], pools[1][a]) and torch.equal(pools[0][a], pools[2][a])
