"""attention_only of a z2z_encoder: any value but 0 and Z2Z_ENC_GATED is the attention layer alone, and nothing behind such a struct is read (stub_hip.cpp)."""
from test_scratch_refused import without_a_device  # noqa: F401  (the fixture)


def test_plain_encoders_are_not_read_past_their_end(without_a_device):
    without_a_device("""
import mmap
libc = ctypes.CDLL(None)
libc.mmap.restype = ctypes.c_void_p
libc.mmap.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_long]
libc.mprotect.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
page = mmap.PAGESIZE
base = libc.mmap(None, 2 * page, 3, 0x22, -1, 0)                        # (read and write, private, anonymous)
assert libc.mprotect(base + page, page, 0) == 0                         # nothing can be read from here on
at = base + page - ctypes.sizeof(api.EncoderDesc)
c = context(B=2, V=100, M=3, cap=50, d=512)

def calls(value):
    e = encoder(512, 2)
    for lay in e.keep:                                                  # (an attention layer has none of these)
        lay.ln2_g = lay.ln2_b = lay.w_1 = lay.b_1 = lay.w_2 = lay.b_2 = None
    e.attention_only = value
    ctypes.memmove(at, ctypes.addressof(e), ctypes.sizeof(e))
    p = ctypes.cast(ctypes.c_void_p(at), ctypes.POINTER(api.EncoderDesc))
    assert lib.z2z_hyper_encode(c, P, p, P, None, 0, None) == 0
    log = launches()
    assert lib.z2z_hyper_encode_keep(c, P, p, P, None) == 0 and lib.z2z_hyper_encode_backward(c, P, p, P, p, P, 0, None) == 0
    return log + launches()

one = calls(1)
assert api.ENC_GATED not in (1, 2, 3, -1)
for value in (2, 3, -1, 1 << 30):
    assert calls(value) == one, value
clean()
""")


def test_a_gradients_own_flag_is_not_read(without_a_device):
    without_a_device("""
c = context(B=2, V=100, M=3, cap=50, d=512)

def back(kind, grads, null=()):
    e, g = encoder(512, 2), encoder(512, 2)
    e.attention_only, g.attention_only = kind, grads
    for lay in g.keep:
        for name in null:
            setattr(lay, name, None)
    rc = lib.z2z_hyper_encode_backward(c, P, ctypes.byref(e), P, ctypes.byref(g), P, 0, None)
    return rc, launches()

block = ("ln2_g", "ln2_b", "w_1", "b_1", "w_2", "b_2")
for kind in (0, 1):
    rc, log = back(kind, kind)
    assert rc == 0
    for value in (0, 1, 2, 7, api.ENC_GATED):
        assert back(kind, value) == (0, log), (kind, value)
# a gradient names what its encoder has
for value in (0, 1, api.ENC_GATED):
    assert back(0, value, ("w_1",)) == (api.E_INVAL, []) and back(0, value, block) == (api.E_INVAL, [])
    assert back(1, value, block)[0] == 0
clean()
""")
