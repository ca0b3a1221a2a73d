"""Sizes of the paged cache's calls that no launch could hold are refused as shapes, before the device is touched."""
import paper_2502_15779_amd as rcp

FAKE = 0x1000   # never dereferenced


def test_attention_of_more_tiles_than_a_grid_holds():
    L = rcp.lib()

    def f(rows, H, H_q, sequences=2):
        c = rcp._Kv8Cache(k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE, n_pages=8, H=H, page=16, D=64)
        b = rcp._Kv8Batch(starts=FAKE, lengths=FAKE, table=FAKE, rows=rows, sequences=sequences, width=4)
        return L.rcp_kv8_attn(c, b, FAKE, 0, H_q, 1.0, FAKE, 0, FAKE, 0, None)
    assert f(1 << 20, 2048, 2048) == -2 and b"too many" in L.rcp_last_error()   # 8194 tiles of 128 rows, 2048 heads: 2^24 workgroups of 256 threads and more
    assert f(1 << 20, 1024, 4096) == -2
    assert f(8190 * 128, 2048, 2048, sequences=1) == -5                         # 8191 tiles: only the workspace is missing
