"""The paged cache's entry points on the host: what they refuse, and that no number of a batch, however wrong,
becomes a row or a page outside the tensors (the device's own checks, run on the CPU)."""
import ctypes
import os
import subprocess

import pytest

import paper_2608_15665_amd as zo
from paper_2608_15665_amd import _build
from paper_2608_15665_amd._lib import KvBatchDesc, KvCacheDesc

FAKE = 1 << 20  # never dereferenced: the calls refuse first, or have nothing to do


def _descs(**kw):
    c = dict(num_pages=10, page_size=16, kv_heads=2, dh=128, dtype=1, K=FAKE, V=FAKE, k_scale=None, v_scale=None)
    b = dict(nseq=3, rows=8, max_q=4, max_pages=5, q_start=FAKE, kv_len=FAKE, page_table=FAKE, bad_flag=None)
    for k, v in kw.items():
        (c if k in c else b)[k] = v
    return KvCacheDesc(*c.values()), KvBatchDesc(*b.values())


def _detail():
    return zo.lib().zo_last_error_detail().decode()


def _append(heads=4, dtype=1, Q=FAKE, ldq=512, Qo=FAKE, ldqo=512, K=FAKE, ldk=256, V=FAKE, ldv=256, base=1e4, **kw):
    c, b = _descs(**kw)
    return zo.lib().zo_kv_append(c, b, heads, dtype, Q, ldq, Qo, ldqo, K, ldk, V, ldv, base, None)


def _attend(heads=4, dtype=1, Q=FAKE, ldq=512, O=FAKE, ldo=512, ws=FAKE, n=1 << 40, **kw):
    c, b = _descs(**kw)
    return zo.lib().zo_paged_attention(c, b, heads, dtype, Q, ldq, O, ldo, ws, n, None)


def test_struct_layouts():
    assert ctypes.sizeof(KvCacheDesc) == 5 * 4 + 4 + 4 * 8 and ctypes.sizeof(KvBatchDesc) == 4 * 4 + 4 * 8


SHARED = [
    (dict(nseq=-1), 1, "nseq"), (dict(rows=-1), 1, "rows"), (dict(max_q=-1), 1, "max_q"), (dict(max_pages=0), 1, "max_pages"),
    (dict(num_pages=0), 1, "num_pages"), (dict(kv_heads=0), 1, "kv_heads"), (dict(rows=(1 << 30) + 1), 1, "too many"),
    (dict(dtype=0), 2, "dtype 0"), (dict(dtype=3), 2, "dtype 3"), (dict(dtype=2), 2, "a cache of dtype 1"),
    (dict(dh=96), 2, "head dim 96"), (dict(page_size=8), 2, "page_size 8"), (dict(page_size=48), 2, "page_size 48"),
    (dict(page_size=512), 2, "page_size 512"), (dict(page_size=0), 2, "page_size 0"), (dict(max_pages=1 << 27), 1, "2^31"),
    (dict(q_start=None, rows=2), 1, "without q_start"), (dict(q_start=None, max_q=0), 1, "without q_start"),
    (dict(kv_len=None), 1, "NULL"), (dict(page_table=None), 1, "NULL"), (dict(kv_len=FAKE + 2), 1, "4-byte"),
    (dict(bad_flag=FAKE + 1), 1, "4-byte"), (dict(q_start=FAKE + 2), 1, "4-byte"),
]


@pytest.mark.parametrize("call", [_append, _attend])
@pytest.mark.parametrize("kw,status,needle", SHARED + [
    (dict(K=None), 1, "NULL"), (dict(V=FAKE + 8), 1, "16-byte"),
])
def test_shared_refusals(call, kw, status, needle):
    if call is _append and ("K" in kw or "V" in kw):
        c, b = _descs(**kw)
        st = zo.lib().zo_kv_append(c, b, 4, 1, FAKE, 512, FAKE, 512, FAKE, 256, FAKE, 256, 1e4, None)
    elif "dtype" in kw and kw["dtype"] != 2:
        st = call(dtype=kw["dtype"])  # the rows' type
    elif "dtype" in kw:
        st = call(dtype=2)
    else:
        st = call(**kw)
    assert st == status and needle in _detail(), (st, _detail())


def test_8_bit_caches_need_their_scales():
    c, b = _descs(dtype=3)
    for k, v in ((None, None), (FAKE, None), (None, FAKE), (FAKE, FAKE + 2)):
        c.k_scale, c.v_scale = k, v
        assert zo.lib().zo_kv_append(c, b, 0, 1, None, 0, None, 0, FAKE, 256, FAKE, 256, 0.0, None) == 1
        assert "k_scale" in _detail()
        assert zo.lib().zo_paged_attention(c, b, 4, 1, FAKE, 512, FAKE, 512, FAKE, 1 << 40, None) == 1


@pytest.mark.parametrize("kw,needle", [
    (dict(base=1.0), "rope_base"), (dict(base=-2.0), "rope_base"), (dict(base=float("nan")), "rope_base"),
    (dict(base=float("inf")), "rope_base"), (dict(base=0.0), "without a rotation"), (dict(Qo=None), "go together"),
    (dict(Q=None), "go together"), (dict(heads=0), "heads"), (dict(ldq=504), "rows of Q"), (dict(ldq=516), "rows of Q"),
    (dict(ldqo=520), "row distance"), (dict(ldk=248), "rows of K"), (dict(ldv=260), "rows of V"), (dict(K=None), "K is NULL"),
    (dict(V=FAKE + 4), "V is NULL or not"), (dict(ldv=1 << 31), "rows of V"),
])
def test_append_refusals(kw, needle):
    assert _append(**kw) == 1 and needle in _detail(), _detail()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(heads=3), 1, "multiple of kv_heads"), (dict(heads=0), 1, "multiple of kv_heads"), (dict(ldq=504), 1, "rows of Q"),
    (dict(ldo=520), 1, "row distance"), (dict(O=None), 1, "O is NULL"), (dict(Q=FAKE + 2), 1, "Q is NULL or not"),
    (dict(max_pages=4000, ws=None), 6, "workspace"), (dict(max_pages=4000, n=1), 6, "workspace"),
    (dict(max_pages=4000, ws=FAKE + 16), 1, "256-byte"),
])
def test_attention_refusals(kw, status, needle):
    assert _attend(**kw) == status and needle in _detail(), _detail()


@pytest.mark.parametrize("nseq,rows,heads,kvh", [(1 << 26, 1 << 30, 1 << 15, 1), (1 << 30, 1 << 30, 1 << 15, 1 << 15),
                                                 (3, 1 << 30, 1 << 15, 1), (1 << 17, 1 << 14, 1 << 15, 1 << 15)])
def test_more_work_than_a_launch_holds(nseq, rows, heads, kvh):
    """Numbers whose products leave 32 or 64 bits are refused; nothing wraps to a small launch, or to 0."""
    kw = dict(nseq=nseq, rows=rows, max_q=rows, kv_heads=kvh)
    ld = 1 << 22
    for cache in (1, 3):
        c, b = _descs(**kw)
        c.dtype = cache
        if cache == 3:
            c.k_scale = c.v_scale = FAKE
        assert zo.lib().zo_paged_attention_workspace(c, b, heads, 1) == 0
        assert zo.lib().zo_paged_attention(c, b, heads, 1, FAKE, ld, FAKE, ld, FAKE, 1 << 62, None) == 2, _detail()
        assert "too many" in _detail()
        assert zo.lib().zo_kv_append(c, b, heads, 1, FAKE, ld, FAKE, ld, FAKE, ld, FAKE, ld, 1e4, None) == 2, _detail()
        assert "too many" in _detail()


def test_nothing_to_do():
    for kw in (dict(nseq=0), dict(rows=0), dict(max_q=0)):
        assert _append(**kw) == 0 and _attend(**kw) == 0
    assert _attend(nseq=0, kv_len=None, page_table=None, Q=None, O=None, ws=None, n=0) == 0


def test_workspace_goes_by_host_arguments():
    ws = lambda heads=4, **kw: zo.lib().zo_paged_attention_workspace(*_descs(**kw), heads, 1)  # noqa: E731
    assert ws(max_pages=1) == 0 and ws(nseq=0) == 0 and ws(heads=3) == 0
    one = ws(nseq=1, rows=1, max_q=1, q_start=None, max_pages=1000)
    assert 0 < one <= 1 << 20
    assert ws(nseq=1, rows=1, max_q=1, q_start=None, max_pages=1000, kv_len=None) == 0  # refused


CHECK = r"""
#include "zo_kv.h"
#include <stdio.h>
#include <random>
#include <vector>
void zo_set_error(const char*, ...) {}
int main() {
  std::mt19937 r(1);
  const int odd[] = {0, 1, -1, 2147483647, -2147483647 - 1, 1 << 30, -(1 << 30), 17, 40, 100};
  long long seen = 0, bad = 0;
  for (int it = 0; it < 200000; ++it) {
    KvArgs a = {};
    int flag = 0, q[3], len, table[4];
    a.nseq = 2; a.rows = r() % 50; a.max_q = r() % 60; a.max_pages = 4; a.num_pages = 1 + r() % 5; a.log2ps = 4 + r() % 5;
    for (int& x : q) x = r() % 3 ? (int)(r() % 60) - 5 : odd[r() % 10];
    for (int& x : table) x = r() % 3 ? (int)(r() % 7) - 1 : odd[r() % 10];
    len = r() % 2 ? (int)(r() % 300) - 20 : odd[r() % 10];
    a.q_start = r() % 4 ? q : nullptr; a.kv_len = &len; a.table = table; a.bad_flag = &flag;
    if (!a.q_start && a.rows < 1) continue;
    const KvSpan sp = kv_span(a, 0);
    if (sp.r0 < 0 || sp.n < 0 || (long long)sp.r0 + sp.n > a.rows) return printf("rows %d %d of %d\n", sp.r0, sp.n, a.rows), 1;
    if (a.q_start && !flag && (sp.r0 != q[0] || sp.n != q[1] - q[0] || sp.n > a.max_q)) return printf("unflagged\n"), 1;
    for (int i = 0; i < sp.n; ++i) {
      const long long p = (long long)sp.len - sp.n + i;
      if (p != (long long)(sp.len - sp.n + i)) return printf("wraps\n"), 1;
      if (p < 0) continue;
      const int page = kv_page(a, 0, (int)p >> a.log2ps);
      const bool fine = p < kv_cap(a) && table[p >> a.log2ps] >= 0 && table[p >> a.log2ps] < a.num_pages;
      if ((page >= 0) != fine || page >= a.num_pages) return printf("page %d\n", page), 1;
      ++(fine ? seen : bad);
    }
  }
  printf("%lld %lld\n", seen, bad);
  return seen > 10000 && bad > 10000 ? 0 : 1;
}
"""


def test_no_number_leaves_the_tensors(tmp_path):
    try:
        cc = _build.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    src, exe = tmp_path / "check.hip", str(tmp_path / "check")
    src.write_text(CHECK)
    p = subprocess.run([cc, "--offload-host-only", "-O1", "-std=c++17", f"-I{_build.INCLUDE}", f"-I{_build.CSRC}", str(src), "-o", exe],
                       capture_output=True, text=True)
    assert p.returncode == 0, p.stderr[-2000:]
    p = subprocess.run([exe], capture_output=True, text=True, env={**os.environ}, timeout=60)
    assert p.returncode == 0, p.stdout
