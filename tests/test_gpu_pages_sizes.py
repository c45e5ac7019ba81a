"""The paged cache and the rotary positions at sizes that test_gpu_pages.py and test_gpu_rotary.py do not reach: pages that are copied in
several pieces, more granted pages than fit the list in LDS, splits over more (layer, sequence) pairs than a wavefront has lanes, heads of 64
in wide pages, accesses of two elements and of one in every type and pairing."""
import numpy as np
import pytest
import torch

import test_gpu_pages as G
import test_gpu_rotary as R
from oracle import pages_oracle as P
from paper_2412_14838_amd.pages import PagedCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("Hkv,d,page_rows,n_seqs", [(8, 128, 64, 3), (8, 128, 128, 4), (5, 64, 64, 3), (1, 64, 16, 5)])
def test_copies_of_pages_of_any_size(dkv, Hkv, d, page_rows, n_seqs):
    """Beams that share a partial last page all grow: its codes and scales go to a page for each, in pieces of 16 KiB (64 and 128 KiB pages,
    20 KiB with a piece that is not full, 1 KiB)."""
    rng = np.random.RandomState(Hkv + page_rows)
    desc = G._desc(dkv, n_seqs, 2, Hkv, Hkv, d)
    cache, p = G._fresh(dkv, desc, 12 * n_seqs, page_rows, 4 * page_rows)
    p.k[:], p.v[:] = rng.randint(0, 256, p.k.shape), rng.randint(0, 256, p.v.shape)
    p.k_exp, p.v_exp = rng.randint(-9, 9, p.k_exp.shape), rng.randint(-9, 9, p.v_exp.shape)
    G._load(cache, p)
    base = np.zeros((n_seqs, 2), np.int32)
    base[0] = page_rows + 3, 2 * page_rows - 1
    for step, (parents, extra) in enumerate((([0] * n_seqs, 1), (list(range(n_seqs)), 1), ([n_seqs - 1] * n_seqs, page_rows), ([0] * n_seqs, -2), (None, 3))):
        if step == 0:
            cache.resize(torch.from_numpy(base).cuda())
            p.resize(base.tolist(), range(2))
        if parents is not None:
            cache.fork(torch.tensor(parents, dtype=torch.int32, device="cuda"))
            p.fork(parents)
        cache.resize(cache.rows, extra)
        p.resize((p.rows + extra).tolist(), range(2))
        assert p.missing == 0
        G._same(cache, p, step)


def test_a_growth_of_more_pages_than_the_list_in_lds(dkv):
    """1320 (sequence, layer) pairs of 5 pages each at once, and of 6 after some have shrunk: the granted pages go through the workspace."""
    n_seqs, L = 40, 33
    cache, p = G._fresh(dkv, G._desc(dkv, n_seqs, L, 1, 1, 64), 8000, 16, 96)
    p.k_exp[:], p.v_exp[:] = 0, 0
    rng = np.random.RandomState(1)
    for base, granted in ((np.full((n_seqs, L), 75), 6600), (rng.randint(0, 2, (n_seqs, L)) * 75, None), (np.full((n_seqs, L), 96), None)):
        before = int((p.refs > 0).sum())
        cache.resize(torch.from_numpy(base.astype(np.int32)).cuda())
        p.resize(base.tolist(), range(L))
        assert p.missing == 0 and (granted is None or int((p.refs > 0).sum()) - before == granted)
        G._same(cache, p, granted)
    # past the end of every table
    cache.resize(torch.full((n_seqs, L), 96, dtype=torch.int32, device="cuda"), 1)
    p.resize([[97] * L] * n_seqs, range(L))
    assert p.missing == n_seqs * L
    G._same(cache, p, "missing")


@pytest.mark.parametrize("dtype,d,page_rows,L", [("bf16", 128, 64, 2), ("f32", 64, 16, 1), ("bf16", 64, 128, 1)])
def test_rows_split_over_many_sequences(dkv, dtype, d, page_rows, L):
    """130 and 260 (layer, sequence) pairs, empty, short and long ones, and so more than a turn of a wavefront's lanes to find a piece."""
    rng = np.random.RandomState(d + L)
    n_seqs, Hkv, Gq = 130, 1, 3
    rows = rng.randint(1, 200, (n_seqs, L))
    rows[rng.rand(n_seqs, L) < 0.3] = 0
    rows[(0, 1, 63, 64, 65, 100, 127, 128, 129), 0] = (0, 4500, 640, 4100, 0, 1, 1025, 2000, 4300)
    rows[-1, -1] = 4301
    desc = G._desc(dkv, n_seqs, L, Hkv * Gq, Hkv, d, dtype, w=1)
    cache, p = G._fresh(dkv, desc, int((-(-rows // page_rows)).sum()) + 1, page_rows, 4608)
    G._fill(rng, p, rows, 1)
    G._load(cache, p)
    q = (torch.from_numpy(rng.standard_normal((L, n_seqs, Hkv * Gq, d)).astype(np.float32)) * 2).to(cache.tdtype).cuda()
    q_np = q.double().cpu().numpy()
    for expected in (0, 200):                             # in pieces (4608 rows to expect), and a workgroup each
        out, lse = torch.full((L, n_seqs, Hkv * Gq, d), 7.0, device="cuda"), torch.full((L, n_seqs, Hkv * Gq), 7.0, device="cuda")
        cache.attention_layers(0, L, q, out, lse, expected_rows=expected)
        got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        for l in range(L):
            for s in range(n_seqs):
                k, v = p.held(s, l)
                want, want_lse = P.attention(q_np[l, s], k, v, d ** -0.5)
                most, most_lse = G._bounds(q_np[l, s], k, v, d ** -0.5)
                assert (np.abs(got[l, s] - want) <= most).all(), (expected, l, s, rows[s, l])
                assert np.isneginf(got_lse[l, s]).all() if rows[s, l] == 0 else (np.abs(got_lse[l, s] - want_lse) <= most_lse).all(), (expected, l, s)


@pytest.mark.parametrize("dtype,d,Hkv,Gq,page_rows,n_seqs,L", [("bf16", 64, 2, 4, 64, 5, 5), ("bf16", 64, 1, 16, 128, 4, 6), ("f32", 64, 1, 3, 64, 4, 6),
                                                               ("bf16", 128, 1, 5, 32, 4, 6), ("f32", 128, 2, 2, 16, 3, 8)])
def test_attention_over_every_kind_of_page(dkv, dtype, d, Hkv, Gq, page_rows, n_seqs, L):
    """Eight wavefronts to a workgroup, and pieces."""
    G.test_attention(dkv, dtype, d, Hkv, Gq, page_rows, n_seqs, L)


@pytest.mark.parametrize("dtype,d,page_rows", [("bf16", 64, 64), ("bf16", 64, 128), ("bf16", 128, 16), ("f32", 128, 64), ("f32", 64, 32)])
def test_short_sequences_over_every_kind_of_page(dkv, dtype, d, page_rows):
    """One, two and four wavefronts to a workgroup."""
    G.test_attention_many_short_sequences(dkv, dtype, d, page_rows)


@pytest.mark.parametrize("dtype,d,r,interleaved,n_seqs,tokens,Hq,Hkv", [
    ("f32", 64, 20, False, 2, 17, 3, 1), ("f32", 64, 22, True, 3, 9, 2, 2), ("bf16", 64, 20, True, 2, 17, 3, 1),          # two elements
    ("bf16", 7, 6, True, 2, 33, 2, 1), ("bf16", 9, 4, False, 3, 7, 2, 3), ("f32", 9, 6, False, 2, 5, 4, 1),               # one
    ("bf16", 128, 96, True, 1, 70, 4, 2), ("f32", 128, 128, True, 2, 40, 2, 1),                                           # 16 bytes
])
def test_rotation_by_every_access(dkv, dtype, d, r, interleaved, n_seqs, tokens, Hq, Hkv):
    R.test_rotation(dkv, dtype, d, r, interleaved, n_seqs, tokens, Hq, Hkv)


def test_a_full_layer_takes_a_new_token_by_default(dkv):
    """A cache made without max_rows: window and layer_max rows, filling their last page, then a row more."""
    rng = np.random.RandomState(3)
    desc = G._desc(dkv, 2, 1, 4, 2, 64, w=16, layer_max=48, tokens=200, longest=100)
    cache = PagedCache(desc, n_pages=6)
    p = P.Pages(2, 1, 2, 64, 6, 64, cache.table.shape[2])
    cu = torch.tensor([0, 100, 200], dtype=torch.int32, device="cuda")
    (k, k_np), (v, v_np) = (G._values(rng, (2, 200, 64), "bf16") for _ in range(2))
    idx = np.stack([[rng.permutation(84)[:48] for _ in range(2)] for _ in range(2)]).astype(np.int32)
    counts = torch.tensor([[48], [48]], dtype=torch.int32, device="cuda")
    cache.resize(counts, cu_seqlens=cu)
    cache.store(0, k, v, cu, torch.from_numpy(idx).cuda(), counts)
    p.resize([[64], [64]], range(1))
    for s in range(2):
        at = np.stack([np.concatenate([np.arange(84, 100), idx[s, h]]) + 100 * s for h in range(2)])
        p.write(s, 0, 0, *(np.stack([x[h, at[h]] for h in range(2)]) for x in (k_np, v_np)), True)
    G._same(cache, p, "prompt")
    (k, k_np), (v, v_np) = (G._values(rng, (2, 2, 64), "bf16") for _ in range(2))
    cache.resize(cache.rows, 1)
    cache.append(0, k, v)
    p.resize([[65], [65]], range(1))
    for s in range(2):
        p.write(s, 0, 64, k_np[s][:, None], v_np[s][:, None], False)
    assert p.missing == 0
    G._same(cache, p, "token")
    q, out = torch.randn(2, 4, 64, device="cuda").to(torch.bfloat16), torch.zeros(2, 4, 64, device="cuda")
    cache.attention(0, q, out)
    for s in range(2):
        kk, vv = p.held(s, 0)
        q_np = q[s].double().cpu().numpy()
        want, _ = P.attention(q_np, kk, vv, 0.125)
        assert (np.abs(out[s].double().cpu().numpy() - want) <= G._bounds(q_np, kk, vv, 0.125)[0]).all()
