"""What the calls of the 8-bit cache refuse, before anything is launched."""
import ctypes as C

import pytest
import torch

import paper_2406_00059_amd as ld

FAKE = 1 << 20     # an aligned non-null "device address" that is never dereferenced on the CPU
NAN, INF = float("nan"), float("inf")


def _call(name, args, **change):
    """Status of a C entry point with these named arguments, some of them changed."""
    unknown = set(change) - set(args)
    assert not unknown, unknown
    return getattr(ld.lib(), name)(*{**args, **change}.values())


TABLE = dict(pos=FAKE, T=3, rot=64, base=10000.0, scaling=None, cos_sin=FAKE, stream=None)


@pytest.mark.parametrize("bad", [dict(T=-1), dict(rot=0), dict(rot=63), dict(rot=-2), dict(base=0.0), dict(base=-1.0), dict(base=NAN), dict(base=INF),
                                 dict(pos=None), dict(cos_sin=None)])
def test_angles_refuse(bad):
    assert _call("ldk_rope_table_scaled", TABLE, T=0) == ld.LD_OK
    assert _call("ldk_rope_table_scaled", TABLE, **bad) == ld.LD_E_INVAL and "ldk_rope_table_scaled" in ld.ld_last_error()


@pytest.mark.parametrize("bad", [(0.0, 0, 0, 0, 1), (-1.0, 0, 0, 0, 1), (NAN, 0, 0, 0, 1), (INF, 0, 0, 0, 1), (8.0, 1.0, 1.0, 100, 1), (8.0, 4.0, 1.0, 100, 1),
                                 (8.0, NAN, 1.0, 100, 1), (8.0, 0.0, INF, 100, 1), (8.0, 0, 0, -1, 1), (1.0, 0, 0, 0, NAN), (1.0, 0, 0, 0, INF)])
def test_angles_refuse_scalings(bad):
    s = ld.ld_rope_scaling(*bad)
    assert _call("ldk_rope_table_scaled", TABLE, scaling=C.addressof(s)) == ld.LD_E_INVAL


WRITE = dict(qkv=FAKE, qkv_stride=12 * 64, q_gain=FAKE, k_gain=FAKE, eps=1e-5, cos_sin=FAKE, rot=64, interleaved=0, pos=FAKE, seq_slot=FAKE, table=FAKE,
             table_stride=4, codes=FAKE, expo=FAKE, T=2, H=8, Hkv=2, hd=64, q_out=2 * FAKE, q_out_stride=8 * 64, stream=None)


@pytest.mark.parametrize("bad", [dict(qkv=None), dict(qkv_stride=12 * 64 - 1), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(cos_sin=None), dict(rot=63),
                                 dict(rot=66), dict(rot=-2), dict(pos=None), dict(seq_slot=None), dict(table=None), dict(table_stride=-1), dict(codes=None),
                                 dict(codes=FAKE + 8), dict(expo=None), dict(expo=FAKE + 4), dict(T=-1), dict(H=0), dict(H=7), dict(Hkv=0), dict(hd=96),
                                 dict(hd=0), dict(q_out=None), dict(q_out_stride=511), dict(q_out=FAKE)])
def test_append_refuses(bad):
    assert _call("ldk_rope_kv_write_q8", WRITE, T=0) == ld.LD_OK
    assert _call("ldk_rope_kv_write_q8", WRITE, **bad) == ld.LD_E_INVAL and "ldk_rope_kv_write_q8" in ld.ld_last_error()


def test_append_refuses_more_heads_than_a_launch_has():
    assert _call("ldk_rope_kv_write_q8", WRITE, H=1 << 24, Hkv=1, qkv_stride=(1 << 31) - 1, q_out_stride=(1 << 31) - 1) in (ld.LD_E_INVAL, ld.LD_E_RANGE)
    assert _call("ldk_rope_kv_write_q8", WRITE, H=32768, Hkv=32768, qkv_stride=3 * 32768 * 64, q_out_stride=32768 * 64) == ld.LD_E_RANGE


TO = dict(pool=FAKE, dtype=ld.LD_BF16, table=FAKE, table_stride=4, codes=FAKE, expo=FAKE, q8_table=FAKE, q8_table_stride=4, ranges=FAKE, n_ranges=1, max_len=9,
          Hkv=2, hd=128, stream=None)
FROM = dict(codes=FAKE, expo=FAKE, q8_table=FAKE, q8_table_stride=4, pool=FAKE, dtype=ld.LD_BF16, table=FAKE, table_stride=4, ranges=FAKE, n_ranges=1, max_len=9,
            Hkv=2, hd=128, stream=None)


@pytest.mark.parametrize("name,args", [("ldk_kv_to_q8", TO), ("ldk_kv_from_q8", FROM)])
@pytest.mark.parametrize("bad", [dict(pool=None), dict(pool=FAKE + 8), dict(dtype=2), dict(table=None), dict(table_stride=-1), dict(codes=None), dict(codes=FAKE + 1),
                                 dict(expo=None), dict(expo=FAKE + 8), dict(q8_table=None), dict(q8_table_stride=-1), dict(ranges=None), dict(n_ranges=-1),
                                 dict(max_len=-1), dict(Hkv=0), dict(hd=32)])
def test_moves_refuse(name, args, bad):
    assert _call(name, args, n_ranges=0) == ld.LD_OK and _call(name, args, max_len=0) == ld.LD_OK
    assert _call(name, args, **bad) == ld.LD_E_INVAL and name in ld.ld_last_error()
    assert _call(name, args, n_ranges=65536) == ld.LD_E_RANGE and _call(name, args, Hkv=32768) == ld.LD_E_RANGE


DECODE = dict(q=FAKE, q_stride=512, codes=FAKE, expo=FAKE, table=FAKE, table_stride=100, seq_slot=FAKE, first=None, ctx_len=FAKE, max_ctx=1000, T=2, H=8, Hkv=2, hd=64,
              window=0, softcap=0.0, slopes=None, out=FAKE, scratch=FAKE, scratch_bytes=1 << 40, stream=None)
PREFILL = dict(q=FAKE, q_stride=512, codes=FAKE, expo=FAKE, table=FAKE, table_stride=100, tiles=FAKE, n_tiles=2, H=8, Hkv=2, hd=64, window=0, softcap=0.0, slopes=None,
               max_pos=999, out=FAKE, scratch=FAKE, scratch_bytes=1 << 40, stream=None)
BOTH = [dict(q=None), dict(q_stride=511), dict(codes=None), dict(codes=FAKE + 8), dict(expo=None), dict(expo=FAKE + 2), dict(table=None), dict(table_stride=-1), dict(H=0),
        dict(H=9), dict(Hkv=0), dict(hd=96), dict(window=-1), dict(softcap=-1.0), dict(softcap=NAN), dict(softcap=INF), dict(out=None)]


@pytest.mark.parametrize("bad", BOTH + [dict(seq_slot=None), dict(ctx_len=None), dict(max_ctx=-1), dict(T=-1)])
def test_decode_refuses(bad):
    assert _call("ldk_paged_attention_q8", DECODE, T=0) == ld.LD_OK
    assert _call("ldk_paged_attention_q8", DECODE, **bad) == ld.LD_E_INVAL and "ldk_paged_attention_q8" in ld.ld_last_error()


@pytest.mark.parametrize("bad", BOTH + [dict(tiles=None), dict(max_pos=-1), dict(n_tiles=-1)])
def test_prefill_refuses(bad):
    assert _call("ldk_prefill_attention_q8", PREFILL, n_tiles=0) == ld.LD_OK
    assert _call("ldk_prefill_attention_q8", PREFILL, **bad) == ld.LD_E_INVAL and "ldk_prefill_attention_q8" in ld.ld_last_error()


@pytest.mark.parametrize("name,args", [("ldk_paged_attention_q8", DECODE), ("ldk_prefill_attention_q8", PREFILL)])
def test_attention_refuses_caps_next_to_zero(name, args):
    assert _call(name, args, softcap=1e-39) == ld.LD_E_INVAL and _call(name, args, softcap=9e-31) == ld.LD_E_INVAL


def test_attention_refuses_scratch_that_is_too_small():
    L = ld.lib()
    n = L.ldk_attention_q8_scratch_bytes(1, 8, 2, 64, 100000, 0)
    if n:
        args = dict(DECODE, T=1, max_ctx=100000)
        assert _call("ldk_paged_attention_q8", args, scratch_bytes=n - 1) == ld.LD_E_INVAL and "scratch" in ld.ld_last_error()
        assert _call("ldk_paged_attention_q8", args, scratch=None) == ld.LD_E_INVAL
        assert _call("ldk_paged_attention_q8", args, scratch=FAKE + 4) == ld.LD_E_INVAL
    n = L.ldk_prefill_attention_q8_scratch_bytes(1, 8, 2, 64, 100000, 0)
    if n:
        args = dict(PREFILL, n_tiles=1, max_pos=100000)
        assert _call("ldk_prefill_attention_q8", args, scratch_bytes=n - 1) == ld.LD_E_INVAL and "scratch" in ld.ld_last_error()
        assert _call("ldk_prefill_attention_q8", args, scratch=None) == ld.LD_E_INVAL
    for bad in ((0, 8, 2, 64, 100, 0), (1, 0, 2, 64, 100, 0), (1, 7, 2, 64, 100, 0), (1, 8, 2, 96, 100, 0), (1, 8, 2, 64, -1, 0), (1, 8, 2, 64, 100, -1)):
        assert L.ldk_attention_q8_scratch_bytes(*bad) == 0 and L.ldk_prefill_attention_q8_scratch_bytes(*bad) == 0


@pytest.mark.parametrize("T", [1, 3, 32])
@pytest.mark.parametrize("H,Hkv", [(4, 4), (32, 8), (48, 1)])
def test_a_buffer_for_more_serves_less(T, H, Hkv):
    L = ld.lib()
    for fn in (L.ldk_attention_q8_scratch_bytes, L.ldk_prefill_attention_q8_scratch_bytes):
        for hd in (64, 128):
            most = fn(T, H, Hkv, hd, 70000, 0)
            assert all(fn(t, H, Hkv, hd, n, w) <= most for t in range(1, T + 1) for n in (0, 1, 64, 65, 777, 5000, 33333, 70000) for w in (0, 100, 5000))


# ---------------------------------------------------------------- the binding's own checks (sizes that C cannot see)

def _z(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


I32, I8 = torch.int32, torch.int8
H, HKV, HD = 4, 2, 64
CODES, EXPO = _z(3, 2, HKV, 16, HD, dtype=I8), _z(3, 2, HKV, 16, dtype=I8)


def _refused(fn, *args, **kw):
    with pytest.raises(ld.LdError) as e:
        fn(*args, stream=0, **kw)
    assert e.value.status == ld.LD_E_INVAL


def test_binding_refuses_append_tensors_that_do_not_fit():
    good = dict(qkv=_z(5, 8 * HD), cos_sin=_z(5, HD // 2, 2), pos=_z(5, dtype=I32), seq_slot=_z(5, dtype=I32), table=_z(1, 3, dtype=I32), codes=CODES, expo=EXPO, H=H,
                Hkv=HKV, hd=HD, q_out=_z(5, H * HD))
    for bad in (dict(qkv=_z(4, 8 * HD)), dict(qkv=_z(5, 8 * HD - 1)), dict(qkv=_z(5, 8 * HD).double()), dict(cos_sin=_z(5, HD // 2)), dict(cos_sin=None),
                dict(pos=_z(5, dtype=torch.int64)), dict(seq_slot=_z(4, dtype=I32)), dict(table=_z(3, dtype=I32)), dict(table=_z(1, 3)), dict(codes=CODES[:2]),
                dict(codes=CODES.to(torch.uint8)), dict(expo=EXPO[:, :1]), dict(expo=EXPO.float()), dict(q_out=_z(5, H * HD - 1)), dict(q_out=_z(4, H * HD)),
                dict(q_gain=_z(HD - 1)), dict(k_gain=_z(HD).half()), dict(qkv=_z(8 * HD, 5).t()), dict(hd=128), dict(Hkv=0), dict(H=3)):
        _refused(ld.ldk_rope_kv_write_q8, **{**good, **bad})


def test_binding_refuses_moves_that_do_not_fit():
    good = dict(pool_layer=_z(4, 2, HKV, 16, HD), table=_z(1, 3, dtype=I32), codes=CODES, expo=EXPO, q8_table=_z(1, 3, dtype=I32), ranges=_z(2, 3, dtype=I32), max_len=5,
                Hkv=HKV, hd=HD)
    for bad in (dict(pool_layer=_z(4, 2, HKV, 16, HD).half()), dict(pool_layer=_z(2 * HKV * 16 * HD - 1)), dict(table=_z(3, dtype=I32)), dict(ranges=_z(6, dtype=I32)),
                dict(ranges=_z(2, 3)), dict(expo=EXPO[:1]), dict(q8_table=_z(1, 3)), dict(Hkv=0)):
        _refused(ld.ldk_kv_to_q8, **{**good, **bad})
        _refused(ld.ldk_kv_from_q8, **{**good, **bad})


def test_binding_refuses_attention_tensors_that_do_not_fit():
    good = dict(q=_z(3, H * HD), q_stride=H * HD, codes=CODES, expo=EXPO, table=_z(3, 4, dtype=I32), seq_slot=_z(3, dtype=I32), ctx_len=_z(3, dtype=I32), max_ctx=64, H=H,
                Hkv=HKV, hd=HD, out=_z(3, H, HD), scratch=_z(1 << 20))
    for bad in (dict(q=_z(2, H * HD)), dict(q=_z(3, H * HD).half()), dict(q_stride=H * HD - 1), dict(codes=CODES[:1]), dict(seq_slot=_z(2, dtype=I32)),
                dict(ctx_len=_z(4, dtype=I32)), dict(first=_z(3)), dict(slopes=_z(H - 1)), dict(out=_z(3, H, HD).double()), dict(out=_z(2, H, HD)), dict(table=_z(12, dtype=I32)),
                dict(Hkv=0), dict(softcap=-1.0)):
        _refused(ld.ldk_paged_attention_q8, **{**good, **bad})
    good = dict(q=_z(3, H * HD), q_stride=H * HD, codes=CODES, expo=EXPO, table=_z(3, 4, dtype=I32), tiles=_z(1, 6, dtype=I32), H=H, Hkv=HKV, hd=HD, out=_z(3, H, HD),
                max_pos=63, scratch=_z(1 << 20))
    for bad in (dict(q=_z(2, H * HD)), dict(q_stride=0), dict(tiles=_z(1, 4, dtype=I32)), dict(tiles=_z(1, 6)), dict(expo=EXPO[:1]), dict(out=_z(3, H, HD - 1)), dict(H=0),
                dict(slopes=_z(H + 1)), dict(max_pos=-1)):
        _refused(ld.ldk_prefill_attention_q8, **{**good, **bad})


# ---------------------------------------------------------------- calls of more threads than a launch has

@pytest.mark.parametrize("name,args", [("ldk_rope_table_scaled", dict(TABLE, T=1 << 26, rot=128)), ("ldk_rope_table_scaled", dict(TABLE, T=(1 << 31) - 1, rot=64)),
                                       ("ldk_rope_kv_write_q8", dict(WRITE, T=1 << 26, rot=22)), ("ldk_rope_kv_write_q8", dict(WRITE, T=(1 << 29) + 1)),
                                       ("ldk_rope_kv_write_q8", dict(WRITE, T=1 << 28, hd=128, qkv_stride=12 * 128, q_out_stride=8 * 128)),
                                       ("ldk_kv_to_q8", dict(TO, max_len=1 << 28)), ("ldk_kv_from_q8", dict(FROM, max_len=1 << 24, Hkv=32)),
                                       ("ldk_paged_attention_q8", dict(DECODE, T=1 << 23, scratch_bytes=1 << 60)),
                                       ("ldk_paged_attention_q8", dict(DECODE, T=8192, max_ctx=131072, H=32, Hkv=32, q_stride=2048, scratch_bytes=1 << 60)),
                                       ("ldk_prefill_attention_q8", dict(PREFILL, n_tiles=1 << 21, scratch_bytes=1 << 60))])
def test_calls_of_more_threads_than_a_launch_has_are_refused(name, args):
    assert _call(name, args) == ld.LD_E_RANGE and name in ld.ld_last_error()
