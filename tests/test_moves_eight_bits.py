"""What ttc_pages_write leaves in an 8-bit cache, byte by byte, signs of zeros among them: quotients in 32 bits, cut at +-448, rounded to nearest even; for scales of
every size and sign."""
import numpy as np
import pytest
import torch

import moves_reference as ref
import paper_1603_02297_amd as ttc

gpu = pytest.mark.gpu
DEV = "cuda"
EDGE = [np.float32(2.0 ** -60), np.float32(2.0 ** 60)]            # beyond these the kernel divides, up to them it multiplies and corrects
SCALES = [None, 1.0, 0.0078125, 0.013, -0.013, -1.0, 3.0, 0.1, *EDGE, -EDGE[0], -EDGE[1], np.nextafter(EDGE[0], np.float32(0)), np.nextafter(EDGE[1], np.float32(1e30)),
          -np.nextafter(EDGE[0], np.float32(0)), 2.0 ** -70, -(2.0 ** -100), 2.0 ** 70, -3.0 * 2.0 ** 99, 0.0, -0.0, np.inf, -np.inf, np.nan]


def encode(q):
    """The format's byte for a quotient; every NaN is 0x7f."""
    table = ref.f8_values()[:127]                                 # ascending
    v = ref.to_f8(q)
    code = np.searchsorted(table, np.abs(np.where(np.isnan(v), 0.0, v)))
    assert np.array_equal(table[code], np.abs(np.where(np.isnan(v), 0.0, v)))
    return np.where(np.isnan(v), 0x7f, code | np.where(np.signbit(q), 0x80, 0)).astype(np.uint8)


def numbers():
    """The format's values, the middles between them and their neighbours in 32 bits, and what lies beyond."""
    table = ref.f8_values()
    finite = np.sort(np.unique(table[np.isfinite(table)]))
    middles = ((finite[1:] + finite[:-1]) / 2).astype(np.float32)
    return np.concatenate([[0.0, -0.0], finite, middles, np.nextafter(middles, np.float32(1e9)), np.nextafter(middles, np.float32(-1e9)),
                           [1e-30, -1e-30, 449.0, -464.0, 511.0, -513.0, 1e9, -1e30, np.inf, -np.inf, np.nan, -0.0, 0.0]]).astype(np.float64)


@gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cut", [0, 1, 3])
def test_every_byte(kind, cut):
    """All numbers times the scale as one head's vector; cut: without the first few, so that the last vector of the head is moved back."""
    code, dtype = ref.TYPES[kind]
    plain = numbers()[cut:]
    for scale in SCALES:
        by = 1.0 if scale is None else float(np.float32(scale))
        size = by if np.isfinite(by) and by != 0 else 1.0
        with np.errstate(over="ignore", under="ignore", invalid="ignore"):
            x = torch.from_numpy((plain * size).astype(np.float32)).to(dtype)
        x32 = x.float().numpy()
        with np.errstate(divide="ignore", invalid="ignore", over="ignore", under="ignore"):
            want = encode(x32 / np.float32(by))
        pages = ttc.ttc_pages_create(code, ttc.TTC_F8, 1, len(plain), 1, 1)
        cache = torch.full((len(plain),), 0x55, dtype=torch.uint8, device=DEV)
        slot, d_x = torch.zeros(1, dtype=torch.int32, device=DEV), x.to(DEV)
        d_scale = None if scale is None else torch.tensor([scale], dtype=torch.float32, device=DEV)
        ttc.ttc_pages_write(pages, 1, slot.data_ptr(), d_x.data_ptr(), len(plain), 0, 0, cache.data_ptr(), 0, 0 if scale is None else d_scale.data_ptr(), 0,
                            torch.cuda.current_stream().cuda_stream)
        got = cache.cpu().numpy()
        ttc.ttc_pages_destroy(pages)
        got = np.where((got & 0x7f) == 0x7f, 0x7f, got)
        wrong = np.nonzero(got != want)[0]
        assert wrong.size == 0, (scale, [(float(x32[i]), int(got[i]), int(want[i])) for i in wrong[:5]])


@gpu
@pytest.mark.parametrize("dim", [1, 2, 3, 7])
def test_short_heads(dim):
    """Heads shorter than a vector go element by element: the same bytes, a scale for each head."""
    plain = numbers()
    heads = len(plain) // dim
    plain = plain[:heads * dim].reshape(heads, dim)
    by = np.array([s for s in SCALES if s is not None], np.float32)
    scale = by[np.arange(heads) % len(by)]
    size = np.where(np.isfinite(scale) & (scale != 0), scale, 1.0).astype(np.float64)
    with np.errstate(all="ignore"):
        x = torch.from_numpy((plain * size[:, None]).astype(np.float32))
        want = encode(x.numpy() / scale[:, None])
    pages = ttc.ttc_pages_create(ttc.TTC_F32, ttc.TTC_F8, heads, dim, 1, 1)
    cache, slot = torch.full((heads * dim,), 0x55, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    d_x, d_scale = x.to(DEV), torch.from_numpy(scale).to(DEV)
    ttc.ttc_pages_write(pages, 1, slot.data_ptr(), d_x.data_ptr(), heads * dim, 0, 0, cache.data_ptr(), 0, d_scale.data_ptr(), 0, torch.cuda.current_stream().cuda_stream)
    got = cache.cpu().numpy()
    ttc.ttc_pages_destroy(pages)
    got = np.where((got & 0x7f) == 0x7f, 0x7f, got)
    assert np.array_equal(got, want.reshape(-1))


def test_the_encoding_here_is_the_formats():
    """All 256 bytes through their values and back, and torch's rounding for what it does not cut."""
    table = ref.f8_values()
    codes = np.arange(256)
    assert np.array_equal(encode(table)[~np.isnan(table)], codes[~np.isnan(table)]) and (encode(table)[np.isnan(table)] == 0x7f).all()
    q = numbers()
    q = q[np.abs(q) <= 448].astype(np.float32)
    assert np.array_equal(encode(q), torch.from_numpy(q).to(torch.float8_e4m3fn).view(torch.uint8).numpy())
