"""Which kernels an attention takes by its hints and sizes, on devices that need not be there, and how many workgroups they get."""
import re

from recording_runtime import record

SCRIPT = r"""
def batch(count, tokens, heads=32, kv_heads=8, dim=128, page=64, most=64, new=0, length=0, cus=256):
    device(cus, 1)
    ctx = sb.Context(0, 0)
    rows = kv_heads * page
    cache = sb.KvCache(fake(1), fake(1), fake(1), fake(1), 1000, rows * dim // 2, rows * sb.mx_scale_pitch(dim), page, kv_heads, dim)
    seqs = sb.Sequences(fake(1), fake(1), fake(1), most, count, most, new, length)
    import ctypes as C
    need = ctx.kv_attention_ws_bytes(cache, seqs, tokens, heads)
    log()
    rc = sb.load().sbits_kv_attention(ctx.h, C.addressof(cache), C.addressof(seqs), tokens, heads, fake(1), heads * dim, dim, 0.1, 1, 0, fake(1), heads * dim, dim, None,
                                      fake(need), need)
    assert rc == 0, rc
    lines = [line.split() for line in log() if line.startswith("launch")]
    return need, [(line[1], line[3]) for line in lines]
out = {}
out["token"] = batch(1, 1, new=1, length=1000)
out["long"] = batch(1, 1, most=2048, new=1)
out["decode"] = batch(64, 64, new=1)
out["prompt"] = batch(1, 8192, most=128)
out["mixed"] = batch(32, 1031, most=64)
out["unknown"] = batch(64, 64)
out["chunk"] = batch(1, 64, most=2048)
out["wide"] = batch(8, 8, dim=256, new=1)
out["small"] = batch(64, 64, new=1, cus=32)
out["most"] = batch(200000, 200000, new=1, most=4)
answer(out)
"""


def test_kernels_by_sizes(tmp_path):
    got = record(tmp_path, SCRIPT)

    def names(key):
        return [re.search(r"attention_(\w+?)_kernel", name).group(1) for name, _ in got[key][1]]

    def grid(key, nth):
        return [int(n) for n in got[key][1][nth][1].split(",")]

    assert names("token") == ["few"] and got["token"][0] == 0 and grid("token", 0) == [16, 1, 1]             # too short to be cut
    assert names("long") == ["few", "join"] and grid("long", 0) == [512, 1, 1] and grid("long", 1) == [4, 8, 1]
    assert names("decode") == ["few", "join"] and grid("decode", 0) == [512, 1, 1] and grid("decode", 1) == [1, 8, 64]
    assert got["decode"][0] == 512 * 2 * 16 * 130 * 4
    assert names("prompt") == ["many"] and grid("prompt", 0) == [8, 1, 257] and got["prompt"][0] == 0
    assert names("mixed") == ["many", "few", "join"]
    assert names("unknown") == ["many", "few", "join"]                                                       # up to 64 new tokens of one sequence
    assert names("chunk") == ["many", "join"] and grid("chunk", 0)[1] > 1
    assert grid("wide", 0) == [256, 1, 1] and grid("small", 0) == [64, 1, 1]
    places = sum(int(g.split(",")[2]) for n, g in got["most"][1] if "join" in n)
    assert places in (0, 200000)
