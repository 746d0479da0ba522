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
