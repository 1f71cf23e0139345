"""Host-only checks of the paged cache's operators: what the header refuses is refused before a device is touched, the
workspace's size goes by the same rules, and no launch is larger than a grid may be."""
import os

import pytest

import paper_2511_03586_amd as perf
from tests import launches as L

FAKE = 0x10000  # a non-null, 16-byte aligned device address; never dereferenced
NULL, SHAPE, DTYPE, ALIGN, UNSUPPORTED = (perf.PERF_ERR_NULL, perf.PERF_ERR_SHAPE, perf.PERF_ERR_DTYPE, perf.PERF_ERR_ALIGN,
                                          perf.PERF_ERR_UNSUPPORTED)
F32, BF16, E4M3 = perf.PERF_F32, perf.PERF_BF16, perf.PERF_E4M3
HUGE = 1 << 60

APPEND = dict(q=FAKE, k=FAKE, v=FAKE, rotation=FAKE, q_out=FAKE, k_pages=FAKE, v_pages=FAKE, k_scales=FAKE, v_scales=FAKE, table=FAKE,
              lengths=FAKE, cu=FAKE, tokens=40, sequences=3, q_heads=8, kv_heads=2, head_dim=64, ldq=512, ldk=128, ldv=128, ldq_out=512,
              pages=50, page_size=16, table_pages=9, ldt=9, rotary_dim=64, positions=200, interleaved=0, x_dt=BF16)
ATTENTION = dict(q=FAKE, k_pages=FAKE, v_pages=FAKE, k_scales=FAKE, v_scales=FAKE, table=FAKE, lengths=FAKE, cu=FAKE, o=FAKE, lse=FAKE,
                 workspace=FAKE, tokens=40, sequences=3, max_tokens=30, q_heads=8, kv_heads=2, head_dim=64, ldq=512, ldo=512, pages=50,
                 page_size=16, table_pages=9, ldt=9, window=0, scale=0.125, x_dt=BF16)
SHARED = [(dict(table=None), NULL), (dict(lengths=None), NULL), (dict(cu=None), NULL), (dict(k_pages=None), NULL), (dict(v_pages=None), NULL),
          (dict(k_scales=None), NULL), (dict(v_scales=None), NULL),
          (dict(tokens=0), SHAPE), (dict(tokens=(1 << 28) + 1), SHAPE), (dict(sequences=0), SHAPE), (dict(sequences=(1 << 24) + 1), SHAPE),
          (dict(q_heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(q_heads=7), SHAPE), (dict(q_heads=1026, ldq=1 << 20, ldo=1 << 20), SHAPE),
          (dict(kv_heads=16), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=-64), SHAPE), (dict(head_dim=1 << 40), SHAPE),
          (dict(pages=0), SHAPE), (dict(pages=(1 << 30) + 1), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=-16), SHAPE),
          (dict(page_size=1 << 31), SHAPE), (dict(table_pages=0), SHAPE), (dict(table_pages=(1 << 26) + 1, ldt=1 << 27), SHAPE),
          (dict(ldt=8), SHAPE), (dict(ldt=HUGE), SHAPE), (dict(ldq=511), SHAPE), (dict(ldq=HUGE), SHAPE),
          (dict(x_dt=E4M3), DTYPE), (dict(x_dt=9), DTYPE), (dict(x_dt=-1), DTYPE),
          (dict(q=FAKE + 1), ALIGN), (dict(x_dt=F32, q=FAKE + 2), ALIGN), (dict(k_pages=FAKE + 8), ALIGN), (dict(v_pages=FAKE + 8), ALIGN),
          (dict(table=FAKE + 2), ALIGN), (dict(lengths=FAKE + 2), ALIGN), (dict(cu=FAKE + 2), ALIGN),
          (dict(head_dim=32, rotary_dim=32), UNSUPPORTED), (dict(head_dim=96, ldq=768, ldk=192, ldv=192, ldq_out=768, ldo=768), UNSUPPORTED),
          (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED)]


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(perf.LIB_PATH):
        from paper_2511_03586_amd import build
        build.build(verbose=False)


def _refuses(call, base, cases):
    for changes, status in cases:
        assert call(**{**base, **{k: v for k, v in changes.items() if k in base}}, check=False) == status, changes


def test_append_refuses():
    _refuses(perf.perf_cache_append_fp8, APPEND, SHARED + [
        (dict(q=None), NULL), (dict(q_out=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(rotation=None), NULL),
        (dict(ldk=127), SHAPE), (dict(ldv=127), SHAPE), (dict(ldk=HUGE), SHAPE), (dict(ldv=HUGE), SHAPE), (dict(ldq_out=511), SHAPE),
        (dict(ldq_out=HUGE), SHAPE), (dict(rotary_dim=-16), SHAPE), (dict(rotary_dim=80), SHAPE), (dict(rotary_dim=15), SHAPE),
        (dict(positions=0), SHAPE), (dict(positions=(1 << 30) + 1), SHAPE), (dict(interleaved=2), SHAPE), (dict(interleaved=-1), SHAPE),
        (dict(k=FAKE + 1), ALIGN), (dict(v=FAKE + 1), ALIGN), (dict(q_out=FAKE + 1), ALIGN), (dict(rotation=FAKE + 2), ALIGN),
        (dict(rotary_dim=24), UNSUPPORTED)])


def test_attention_refuses():
    _refuses(perf.perf_cache_attention_fp8, ATTENTION, SHARED + [
        (dict(q=None), NULL), (dict(o=None), NULL), (dict(workspace=None), NULL), (dict(max_tokens=0), SHAPE), (dict(window=-1), SHAPE),
        (dict(window=(1 << 30) + 1), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(ldo=511), SHAPE),
        (dict(ldo=HUGE), SHAPE), (dict(o=FAKE + 1), ALIGN), (dict(lse=FAKE + 2), ALIGN), (dict(workspace=FAKE + 8), ALIGN)])


def test_workspace_size_goes_by_the_same_rules():
    base = {k: ATTENTION[k] for k in ("tokens", "sequences", "max_tokens", "q_heads", "kv_heads", "head_dim", "page_size", "table_pages")}
    size = perf.perf_cache_attention_fp8_workspace_bytes
    assert size(**base) >= 0
    for changes, status in SHARED + [(dict(max_tokens=0), SHAPE)]:
        if status in (SHAPE, UNSUPPORTED) and set(changes) - {"ldq", "ldk", "ldv", "ldo", "ldq_out", "ldt", "pages", "rotary_dim"}:
            assert size(**{**base, **{k: v for k, v in changes.items() if k in base}}) == -1, changes


def test_attention_refuses_more_rows_than_it_counts():
    wide = dict(q_heads=1024, kv_heads=1, ldq=1 << 16, ldo=1 << 16)
    sizes = ("tokens", "sequences", "max_tokens", "q_heads", "kv_heads", "head_dim", "page_size", "table_pages")
    big = {**ATTENTION, **wide, "tokens": (1 << 20) + 1}
    assert perf.perf_cache_attention_fp8(**big, check=False) == UNSUPPORTED
    assert perf.perf_cache_attention_fp8_workspace_bytes(**{k: big[k] for k in sizes}) == -1
    assert perf.perf_cache_attention_fp8_workspace_bytes(**{k: {**big, "tokens": 1 << 20}[k] for k in sizes}) > 0


@pytest.fixture(scope="module")
def recorder(tmp_path_factory):
    return L.build_recorder(str(tmp_path_factory.mktemp("recorder")))


def _check_grids(calls, results):
    refused = 0
    for (_, a), r in zip(calls, results):
        if r["status"] == UNSUPPORTED:
            assert not r["launches"] and a["tokens"] + a["sequences"] >= 1 << 16, a
            refused += 1
            continue
        assert r["status"] == perf.PERF_OK and r["launches"], a
        for launch in r["launches"]:
            for n, threads in zip(launch["grid"], launch["block"]):
                assert 0 < n * threads < 1 << 32, (a, launch)
            assert launch["grid"][1] <= 65535 and launch["grid"][2] <= 65535, launch
    assert 3 * refused < 2 * len(calls)


SIZES = [(tokens, sequences, heads, dim, page) for tokens in (1, 17, 3000, 1 << 20, 1 << 28) for sequences in (1, 100, 1 << 16, 1 << 24)
         for heads in ((1, 1), (32, 8), (1024, 1), (1024, 1024)) for dim, page in ((64, 16), (128, 64), (256, 256))]


def test_append_grids(recorder):
    calls = []
    for tokens, sequences, (hq, kv), dim, page in SIZES:
        for x_dt in (F32, BF16):
            calls.append(("perf_cache_append_fp8", {**APPEND, "tokens": tokens, "sequences": sequences, "q_heads": hq, "kv_heads": kv,
                                                    "head_dim": dim, "page_size": page, "ldq": hq * dim, "ldq_out": hq * dim, "ldk": kv * dim,
                                                    "ldv": kv * dim, "x_dt": x_dt, "rotary_dim": dim}))
    _check_grids(calls, L.record(recorder, calls))


def test_attention_grids(recorder):
    calls = []
    for tokens, sequences, (hq, kv), dim, page in SIZES:
        for x_dt, most, columns in ((F32, 1, 9), (BF16, 1, 1 << 20), (BF16, tokens, 1 << 15)):
            calls.append(("perf_cache_attention_fp8", {**ATTENTION, "tokens": tokens, "sequences": sequences, "max_tokens": most, "q_heads": hq,
                                                       "kv_heads": kv, "head_dim": dim, "page_size": page, "ldq": hq * dim, "ldo": hq * dim,
                                                       "table_pages": columns, "ldt": columns, "x_dt": x_dt}))
    _check_grids(calls, L.record(recorder, calls))
