"""Pages shared with forks, copied, given back and moved to the front, on the GPU against their definition."""
import numpy as np
import pytest
import torch

import paper_2512_23966_amd as loza
from tests import beside_reference as N

pytestmark = pytest.mark.gpu
BF, I32 = torch.bfloat16, torch.int32


def _dev(x, dev):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(dev)


class Pool:
    """Requests on a pool whose pages are all held by one request or free."""

    def __init__(self, rng, B, page, most, spare=5, empty=0.4):
        self.B, self.page, self.most = B, page, most
        lens = rng.integers(0, most * page + 1, size=B).astype(np.int32)
        lens = np.where(rng.random(B) < 0.3, lens // page * page, lens)             # (some end on a page border)
        lens[rng.random(B) < empty] = 0
        self.lens = lens.astype(np.int32)
        need = -(-self.lens // page)
        self.held = np.where(self.lens > 0, np.minimum(most, need + rng.integers(0, 2, size=B)), 0).astype(np.int32)
        self.held[rng.random(B) < 0.2] = 0                                          # (fewer than the rows need: taken as that many)
        count = np.maximum(self.held, need)
        self.pages = int(count.sum()) + spare + B
        perm = rng.permutation(self.pages).astype(np.int32)
        self.table = rng.integers(-3, self.pages + 3, size=(B, most)).astype(np.int32)
        at = 0
        for b in range(B):
            self.table[b, :count[b]] = perm[at:at + count[b]]
            at += int(count[b])
        self.free = np.full(self.pages, -7, dtype=np.int32)
        self.free[:self.pages - at] = perm[at:]
        self.count = self.pages - at
        self.shared = np.zeros(self.pages, np.int32)
        self.trimmed = np.zeros(B, np.int32)


def _fork(dev, p, source, sink_blocks, block, count=None, trimmed=True):
    B = p.B
    i32 = dict(dtype=I32, device=dev)
    o = {k: torch.full((B,), -77, **i32) for k in ("forked", "lens", "held", "trimmed", "copy_from", "copy_to", "copy_rows")}
    o["left"], o["shared"], o["table"] = torch.full((1,), -77, **i32), torch.full((p.pages,), -77, **i32), _dev(p.table, dev)
    ins = [_dev(x, dev) for x in (source, p.lens, p.held)]
    loza.loza_ssa_pages_fork(*ins, _dev(p.trimmed, dev) if trimmed else None, _dev(p.free, dev), torch.tensor([p.count if count is None else count], **i32), _dev(p.shared, dev),
                             o["table"], p.pages, p.page, sink_blocks, block, o["forked"], o["lens"], o["held"], o["trimmed"] if trimmed else None, o["copy_from"],
                             o["copy_to"], o["copy_rows"], o["left"], o["shared"])
    return {k: v.cpu().numpy() for k, v in o.items()}


@pytest.mark.parametrize("B,page,most", [(1, 32, 3), (2, 32, 1), (7, 64, 9), (40, 32, 300), (300, 128, 5), (1025, 32, 4)])
def test_fork(gpu_device, B, page, most):
    rng = np.random.default_rng(B + most)
    p = Pool(rng, B, page, most)
    p.trimmed = np.where(rng.random(B) < 0.4, np.maximum(0, p.lens // page - 1), 0).astype(np.int32)
    p.shared = rng.integers(0, 3, size=p.pages).astype(np.int32)
    source = rng.integers(-1, B + 1, size=B).astype(np.int32)
    if B > 30:
        p.lens[3], p.lens[4], p.table[5, 0] = -4, most * page + 1, p.pages + 9     # sources that are none, and a page that is none
        source[[0, 8, 9]] = [3, 4, 5]
    for count in {p.count, 0, 1, 3, p.count + 100, -2}:
        for sink, block in ((0, 1), (1, page), (page + 1, 1)):
            got, ref = _fork(gpu_device, p, source, sink, block, count), N.pages_fork(source, p.lens, p.held, p.trimmed, p.free, count, p.shared, p.table, page, -(-sink * block // page))
            for k in ref:
                assert np.array_equal(got[k], ref[k]), (k, count, sink)
    q = N.pages_fork(source, p.lens, p.held, np.zeros(B, np.int32), p.free, p.count, p.shared, p.table, page, 0)
    got = _fork(gpu_device, p, source, 4, 1, trimmed=False)
    for k in q:
        assert k == "trimmed" or np.array_equal(got[k], q[k]), k


def _free(dev, p, ending, sink, window, block, count=None, trimmed=True, shared=True):
    B = p.B
    i32 = dict(dtype=I32, device=dev)
    o = {"lens": torch.full((B,), -77, **i32), "held": torch.full((B,), -77, **i32), "trimmed": torch.full((B,), -77, **i32) if trimmed else None, "count": torch.full((1,), -77, **i32),
         "shared": torch.full((p.pages,), -77, **i32) if shared else None, "free": _dev(p.free, dev)}
    loza.loza_ssa_pages_free(_dev(ending, dev), _dev(p.lens, dev), _dev(p.held, dev), _dev(p.trimmed, dev) if trimmed else None, _dev(p.table, dev),
                             _dev(p.shared, dev) if shared else None, o["free"], torch.tensor([p.count if count is None else count], **i32), p.pages, p.page, sink, window, block,
                             o["lens"], o["held"], o["trimmed"], o["count"], o["shared"])
    return {k: None if v is None else v.cpu().numpy() for k, v in o.items()}


def _same(got, ref):
    for k in ref:
        assert (ref[k] is None) == (got[k] is None) and (ref[k] is None or np.array_equal(got[k], ref[k])), k


@pytest.mark.parametrize("B,page,most", [(1, 32, 3), (2, 32, 1), (7, 64, 9), (40, 32, 300), (300, 128, 5), (20, 32, 1500)])
def test_free(gpu_device, B, page, most):
    rng = np.random.default_rng(B + most)
    p = Pool(rng, B, page, most, empty=0.2)
    p.shared = np.where(rng.random(p.pages) < 0.3, rng.integers(1, 3, size=p.pages), 0).astype(np.int32)
    p.table[0, 0] = p.table[B - 1, 0]                                               # (pages that two rows name, shared or not)
    p.trimmed = np.where(rng.random(B) < 0.4, p.lens // page // 2, 0).astype(np.int32)
    if B > 30:
        p.lens[3], p.lens[4], p.held[5], p.held[6], p.trimmed[7], p.trimmed[8] = -4, most * page + 1, -1, most + 1, -9, most + 4
        p.table[9, 0] = p.pages + 9
    ending = (rng.random(B) < 0.3).astype(np.int32) * 5
    for sink, window, block in ((0, 1, 1), (33, 70, 1), (1, 7, 128), (0, 1 << 62, 1), (1 << 40, 1, 1 << 40), (2, 2, page), (0, 1, 1 << 50)):
        for end in (ending, None):
            _same(_free(gpu_device, p, end, sink, window, block), N.pages_free(end, p.lens, p.held, p.trimmed, p.table, p.shared, p.free, p.count, page, sink, window, block))
    for count in (0, p.pages - 1, p.pages + 5, -3):
        _same(_free(gpu_device, p, ending, 0, 64, 1, count), N.pages_free(ending, p.lens, p.held, p.trimmed, p.table, p.shared, p.free, count, page, 0, 64, 1))
    _same(_free(gpu_device, p, ending, 9, 64, 1, trimmed=False, shared=False), N.pages_free(ending, p.lens, p.held, None, p.table, None, p.free, p.count, page, 9, 64, 1))


@pytest.mark.parametrize("pages", [2, 3, 31, 33, 4095, 4096, 4097, 9000, 70_001])
@pytest.mark.parametrize("share", [0.0, 0.3, 0.97, 1.0])
def test_compact(gpu_device, pages, share):
    rng = np.random.default_rng(pages)
    B, most = 11, max(1, pages // 9)
    perm = rng.permutation(pages).astype(np.int32)
    count = int(share * pages)
    free = np.full(pages + 3, 5, dtype=np.int32)
    free[:count] = perm[:count]
    table = rng.integers(-2, pages + 2, size=(B, most)).astype(np.int32)
    shared = rng.integers(0, 4, size=pages).astype(np.int32)
    if count > 4:
        free[0], free[1] = free[2], pages + 7                                       # twice the same, and none
    for sh in (shared, None):
        i32 = dict(dtype=I32, device=gpu_device)
        o = {"table": torch.empty(B, most, **i32), "free": torch.full((pages + 3,), -77, **i32), "count": torch.empty(1, **i32),
             "shared": torch.full((pages,), -77, **i32) if sh is not None else None, "copy_from": torch.full((pages // 2,), -77, **i32),
             "copy_to": torch.full((pages // 2,), -77, **i32), "copies": torch.empty(1, **i32)}
        loza.loza_ssa_pages_compact(_dev(table, gpu_device), _dev(free, gpu_device), torch.tensor([count], **i32), _dev(sh, gpu_device), pages, o["table"], o["free"], o["count"],
                                    o["shared"], o["copy_from"], o["copy_to"], o["copies"])
        ref = N.pages_compact(table, free, count, sh, pages)
        for k in ref:
            assert o[k] is None or np.array_equal(o[k].cpu().numpy(), ref[k]), k


@pytest.mark.parametrize("dtype,Hkv,dk,dv,page,layers", [(BF, 1, 576, 0, 32, 3), (BF, 2, 128, 128, 64, 1), (torch.float32, 3, 4, 20, 32, 2), (torch.uint8, 1, 16, 16, 128, 1),
                                                         (torch.int64, 1, 2048, 6, 64, 1)])
def test_copy(gpu_device, dtype, Hkv, dk, dv, page, layers):
    rng = np.random.default_rng(dk)
    pages, n = 40, 17
    k = torch.from_numpy(rng.integers(0, 100, size=(layers, pages, page, Hkv, dk))).to(dtype).to(gpu_device)
    v = torch.from_numpy(rng.integers(0, 100, size=(layers, pages, page, Hkv, dv))).to(dtype).to(gpu_device) if dv else None
    perm = rng.permutation(pages).astype(np.int32)
    src, dst = perm[:n].copy(), perm[20:20 + n].copy()
    src[1], src[2], dst[3], dst[4], src[5] = src[0], -1, -1, pages, pages              # one page to two, and entries that are none
    src[6] = dst[6]
    for rows, count in ((None, None), (rng.integers(-1, page + 2, size=n).astype(np.int32), None), (None, 9), (None, -1), (None, 99)):
        ka, va = k.clone(), None if v is None else v.clone()
        loza.loza_ssa_pages_copy(ka, va, _dev(src, gpu_device), _dev(dst, gpu_device), rows=_dev(rows, gpu_device),
                                 count=None if count is None else torch.tensor([count], dtype=I32, device=gpu_device))
        for new, old in ((ka, k), (va, v)):
            if old is None:
                continue
            ref = old.clone()
            for i in range(n if count is None else min(max(0, count), n)):
                if 0 <= src[i] < pages and 0 <= dst[i] < pages:
                    r = page if rows is None else min(max(0, int(rows[i])), page)
                    ref[:, dst[i], :r] = old[:, src[i], :r]
            assert torch.equal(new, ref)


def test_copies_beyond_2_32_bytes(gpu_device):
    pages, page = 130_000, 32                                                      # 4.8 GB a layer
    k = torch.zeros(2, pages, page, 1, 576, dtype=BF, device=gpu_device)
    g = torch.Generator(device=gpu_device).manual_seed(1)
    k[:, 5] = torch.randn(2, page, 1, 576, generator=g, device=gpu_device).to(BF)
    i32 = lambda *x: torch.tensor(x, dtype=I32, device=gpu_device)
    loza.loza_ssa_pages_copy(k, None, i32(5), i32(pages - 1))
    loza.loza_ssa_pages_copy(k, None, i32(pages - 1), i32(pages - 2), rows=i32(7))
    assert torch.equal(k[:, -1], k[:, 5]) and torch.equal(k[:, -2, :7], k[:, 5, :7]) and not bool(k[:, -2, 7:].any()) and not bool(k[:, 6:-2].any())
    del k
    torch.cuda.empty_cache()


@pytest.mark.parametrize("spare", [5, 9000])
def test_calls_are_repeatable_also_in_a_graph(gpu_device, spare):
    rng = np.random.default_rng(3)
    p = Pool(rng, 50, 32, 40, spare=spare)
    source = rng.integers(-1, 50, size=50).astype(np.int32)
    i32 = dict(dtype=I32, device=gpu_device)
    ins = {k: _dev(x, gpu_device) for k, x in (("source", source), ("lens", p.lens), ("held", p.held), ("trimmed", p.trimmed), ("free", p.free), ("shared", p.shared), ("table", p.table),
                                               ("ending", (rng.random(50) < 0.3).astype(np.int32)))}
    count = torch.tensor([p.count], **i32)
    o = {k: torch.empty(50, **i32) for k in ("forked", "lens1", "held1", "trimmed1", "cf", "ct", "cr", "lens2", "held2", "trimmed2")}
    o.update(left=torch.empty(1, **i32), count2=torch.empty(1, **i32), shared1=torch.empty(p.pages, **i32), shared2=torch.empty(p.pages, **i32), free2=ins["free"].clone(),
             table3=torch.empty_like(ins["table"]), free3=torch.empty(p.pages, **i32), count3=torch.empty(1, **i32), shared3=torch.empty(p.pages, **i32),
             f3=torch.empty(p.pages // 2, **i32), t3=torch.empty(p.pages // 2, **i32), n3=torch.empty(1, **i32))
    ws = torch.empty(loza.loza_ssa_pages_compact_workspace_bytes(p.pages), dtype=torch.uint8, device=gpu_device)
    ws2 = torch.empty(loza.loza_ssa_pages_free_workspace_bytes(p.pages), dtype=torch.uint8, device=gpu_device)

    def calls(**kw):
        loza.loza_ssa_pages_fork(ins["source"], ins["lens"], ins["held"], ins["trimmed"], ins["free"], count, ins["shared"], ins["table"], p.pages, 32, 16, 1, o["forked"],
                                 o["lens1"], o["held1"], o["trimmed1"], o["cf"], o["ct"], o["cr"], o["left"], o["shared1"], **kw)
        loza.loza_ssa_pages_free(ins["ending"], o["lens1"], o["held1"], o["trimmed1"], ins["table"], o["shared1"], o["free2"], o["left"], p.pages, 32, 16, 200, 1, o["lens2"],
                                 o["held2"], o["trimmed2"], o["count2"], o["shared2"], ws2, **kw)
        loza.loza_ssa_pages_compact(ins["table"], o["free2"], o["count2"], o["shared2"], p.pages, o["table3"], o["free3"], o["count3"], o["shared3"], o["f3"], o["t3"], o["n3"], ws, **kw)
    calls()
    torch.cuda.synchronize()
    ref = {k: v.clone() for k, v in o.items()}
    assert int(o["forked"].sum()) > 3 and int(o["n3"]) > 3
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    s = torch.cuda.Stream()
    for k in range(3):
        for name, v in o.items():
            if name != "free2":
                v.fill_(-5)
        torch.cuda.synchronize()
        graph.replay() if k < 2 else calls(stream=s)
        torch.cuda.synchronize()
        for name in o:
            assert torch.equal(o[name], ref[name]), (k, name)


# ---- a pool small enough for one workgroup, and just not -----------------------------------------------------------------

@pytest.mark.parametrize("B,page,most", [(128, 32, 100), (129, 32, 30), (20, 32, 512), (20, 32, 513), (31, 32, 400)])
def test_forks_and_frees_around_one_workgroup(gpu_device, B, page, most):
    test_fork(gpu_device, B, page, most)
    test_free(gpu_device, B, page, most)


@pytest.mark.parametrize("pages,B,most,extra", [(8191, 8, 40, 0), (8192, 1, 32_768, 3), (8192, 1, 32_769, 0), (8193, 8, 40, 0), (100, 1000, 33, 0), (50, 3, 20, 32_718), (50, 3, 20, 32_719)])
def test_compact_around_one_workgroup(gpu_device, pages, B, most, extra):
    rng = np.random.default_rng(pages + most)
    perm = rng.permutation(pages).astype(np.int32)
    for count in (0, 1, pages // 3, pages - 1, pages):
        free = np.full(pages + extra, 5, dtype=np.int32)
        free[:count] = perm[:count]
        table, shared = rng.integers(-2, pages + 2, size=(B, most)).astype(np.int32), rng.integers(0, 4, size=pages).astype(np.int32)
        i32 = dict(dtype=I32, device=gpu_device)
        o = {"table": torch.empty(B, most, **i32), "free": torch.full((pages + extra,), -77, **i32), "count": torch.empty(1, **i32), "shared": torch.full((pages,), -77, **i32),
             "copy_from": torch.full((pages // 2,), -77, **i32), "copy_to": torch.full((pages // 2,), -77, **i32), "copies": torch.empty(1, **i32)}
        loza.loza_ssa_pages_compact(_dev(table, gpu_device), _dev(free, gpu_device), torch.tensor([count], **i32), _dev(shared, gpu_device), pages, o["table"], o["free"], o["count"],
                                    o["shared"], o["copy_from"], o["copy_to"], o["copies"])
        ref = N.pages_compact(table, free, count, shared, pages)
        for k in ref:
            assert np.array_equal(o[k].cpu().numpy(), ref[k]), (count, k)
