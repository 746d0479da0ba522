"""What the calls on a paged cache need and launch at sizes that no GPU test has, on the recording stand-in of the HIP
runtime (host_stub.py); needs no GPU."""
import host_stub

CACHE = '''
import paper_2605_29707_amd.binding as bd
lib, F = bd.load(), h.FAKE
def cache(**kw):
    c = dict(k=F, v=F, weights=F, page_table=F, layer_stride=1 << 40, page_stride=1 << 30, slot_stride=1 << 14, head_stride=128,
             n_layers=1, n_pages=9, page_size=64, n_kv_heads=8, head_dim=128, batch=64, max_pages=256, dtype=1)
    c.update(kw)
    return C.byref(bd.domino_paged_cache(**c))
'''


def test_a_workspace_is_for_the_very_call(tmp_path):
    """As the header says: a prompt's call needs less than a decoding step, which its workspace does not serve; the greatest of
    both sizes serves both, and rows that no sequence has cost a call nothing but their place."""
    host_stub.run(CACHE + '''
def need(*a):
    return lib.domino_paged_attention_workspace_bytes(cache(), a[0], 32, a[1], 16384, a[2])
def attend(tokens, new, acc, n):
    return lib.domino_paged_attention(cache(), 0, tokens, 32, new, 16384, F, 4096, F + 8192, 4096, F, F, 0.1, None, 0, None, acc, F, n, None)
for acc, kinds in ((1, [(4096, 4096), (64, 1), (256, 4)]), (0, [(4096, 4096), (64, 1)])):
    sizes = [need(*k, acc) for k in kinds]
    assert sizes[0] < 1 << 20 and all(s > 16 << 20 for s in sizes[1:]), sizes
    assert attend(*kinds[0], acc, sizes[0]) == 0 and attend(*kinds[1], acc, sizes[0]) == -2
    assert str(sizes[1]) in bd.last_error()
    for k in kinds:
        assert attend(*k, acc, max(sizes)) == 0
assert [round(need(*k, 1) / 1e5) for k in ((4096, 4096), (64, 1), (256, 4))] == [5, 1513, 6051]   # the header's figures, in 0.1 MB
''', tmp_path)


def test_the_most_heads_fit_a_grid(tmp_path):
    """Eviction over as many heads as are accepted, in place and to new pages: no grid of 2^32 threads or more; what would need one
    is refused."""
    host_stub.run(CACHE + '''
def check(st):
    """Launched within the limits, or refused before any launch."""
    out = [r for r in h.log() if r[0] == "launch"]
    for r in out:
        assert int(r[2]) * int(r[3]) * int(r[4]) * int(r[5]) < 2**32 and int(r[3]) <= 65535, r
    assert (len(out) > 0) == (st == 0) and st in (0, -3), (st, out, bd.last_error())
    return st == 0
h.log()
took = {}
for dtype in (0, 1):
    for dh in (64, 128):
        for layers in (1, 16, 32, 60, 61, 63, 64):
            for table in (None, F):
                c = cache(n_layers=layers, batch=2048, max_pages=15, dtype=dtype, head_dim=dh)
                n = lib.domino_paged_evict_workspace_bytes(c, 960, 100)
                took[dtype, dh, layers, table] = check(lib.domino_paged_evict(c, F, F + 64, 960, 100, 0, 0, table, 1 << 10, None, F, n, None))
assert took[0, 128, 60, None] and not took[0, 128, 61, None] and not took[0, 128, 64, None]
assert all(v for k, v in took.items() if k[:2] != (0, 128) or k[3] or k[2] <= 60)
''', tmp_path)


def test_an_append_of_many_heads_fits_a_grid(tmp_path):
    host_stub.run(CACHE + '''
h.log()
for tokens in (1, 600, 1023):
    for heads in (8, 1 << 19):
        c = cache(n_kv_heads=heads, max_pages=1)
        assert lib.domino_paged_append(c, 0, tokens, heads, F, heads * 128, F, heads * 128, F, heads * 128, F, heads * 128, F, F, None,
                                       None, 0, 0, 1.0, None, None, 0.0, F, 16, None) == 0, bd.last_error()
        (r,) = [r for r in h.log() if r[0] == "launch"]
        assert int(r[2]) > tokens and int(r[3]) <= 65535 and int(r[2]) * int(r[3]) * int(r[5]) < 2**32, r
''', tmp_path)


def test_commit_writes_no_array_that_it_reads(tmp_path):
    host_stub.run(CACHE + '''
for ctx, acc, path, new in ((1, 2, 3, 1), (1, 2, 3, 2), (1, 2, 3, 3), (1, 2, 3, 4)):
    h.log()
    st = lib.domino_paged_commit(cache(), 61, 15, F * ctx, F * acc, F * path, F * new, F, 16, None)
    assert (st, len(h.log())) == ((0, 1) if new == 4 else (-1, 0)), (new, st)
''', tmp_path)
