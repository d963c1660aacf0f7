"""More than two groups of 32 heads on the matrix-core path, with batches that are and are not a multiple of eight rows."""
import numpy as np
import pytest

import elitekv_synth as synth
import paper_2503_01586_amd as ekv
from oracle import elitekv_oracle as orc

from gpu_util import TOL, dev, gpu_decode, host64, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_h", [72, 100])
@pytest.mark.parametrize("B", [1, 7, 8, 16])
def test_every_head_of_every_group(n_h, B):
    rng = np.random.default_rng(n_h + B)
    d_h, r, d_c = 64, 8, 256
    lens = [int(n) for n in rng.integers(1, 90, B)]
    stride = max(lens)
    idx = synth.draw_elite_idx(rng, n_h, d_h, r)
    _, _, W_uk, W_uv = synth.draw_weights(rng, 64, n_h, d_h, r, d_c)
    ke64, c64 = synth.draw_cache_planes(rng, B * stride, n_h, r, d_c)
    q = synth.draw_query(rng, B, n_h, d_h)
    dims = ekv.make_dims(64, n_h, d_h, r, d_c, "bf16", 10000.0)
    assert ekv.elitekv_decode_path(dims) == ekv.PATH_MATRIX_CORE
    ked, cd, qd, Wukd, Wuvd = (dev(a, "bf16") for a in (ke64, c64, q, W_uk, W_uv))
    q_pos = np.array(lens) - 1
    out = host64(gpu_decode(dims, qd, i32(q_pos), i32(lens), stride, stride, Wukd, Wuvd, i32(idx), ked, cd))
    ref = orc.decode_attn(host64(qd), q_pos, host64(ked).reshape(B, stride, n_h, -1), host64(cd).reshape(B, stride, -1),
                          lens, host64(Wukd), host64(Wuvd), idx, d_h, 10000.0)
    assert np.all(np.isfinite(out))
    assert orc.max_abs_rel(out, ref) <= TOL["bf16"]
