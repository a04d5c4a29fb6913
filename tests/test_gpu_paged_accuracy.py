"""How exact the single-token attention is, against the plainest computation in 32 bits: every sum one running sum.

The worst-case tolerance of paged_util.decode_tolerance is some hundred times what 32-bit arithmetic is off by as a rule, since it lets every
rounding of a score count in full.  Here the error itself is measured against 64 bits, and so is the plain computation's on the same inputs.
The kernels sum a score in four runs of d / 4 (f32) or inside the matrix instruction, the values in runs of a tile's tokens by wave and workgroup:
shorter sums, so smaller errors.  What the kernels do in addition is one more rounding of a score's difference to the maximum (the factor log2 e /
sqrt(d)) and of the partial sums when they are joined.  So the root of the mean square is allowed twice the plain one's, the largest error three
times the plain one's largest: both are largest ones of some thousand errors of one distribution."""
import math

import numpy as np
import pytest
import torch

from paged_util import HALF_STEP, attention64, rows_of
from test_gpu_paged import BF, F32, _decode_case, ints
from paper_2605_19726_amd import binding as bd

pytestmark = pytest.mark.gpu


def _plain32(q, k, v):
    """One query over k and v [n, d] (numpy, fp32), every sum one after the other: (out, lse)."""
    f, (n, d) = np.float32, k.shape
    s = np.zeros(n, dtype=f)
    for i in range(d):
        s = s + q[i] * k[:, i]
    s = s / f(math.sqrt(d))
    m = s.max()
    p = np.exp(s - m)
    z, o = f(0), np.zeros(d, dtype=f)
    for t in range(n):
        z = z + p[t]
        o = o + p[t] * v[t]
    return o / z, m + np.log(z)


def _errors(dtype, d, lens, width):
    """(kernel's errors, plain errors, kernel's lse errors, plain lse errors, what bf16 outputs may be off by beyond half a step)"""
    hq, hk, page = 4, 2, 16
    q, k, v, table = _decode_case(dtype, d, hq, hk, page, lens, 77, width=width)
    out, lse = bd.basa_decode_attn(q, bd.PagedCache(k, v), ints(table), ints(lens), want_lse=True)
    got, plain, got_lse, plain_lse, room = [], [], [], [], []
    for i, n in enumerate(lens):
        at, off = (x.to(q.device) for x in rows_of(table[i], n, page))
        ks, vs = k[at, :, off], v[at, :, off]
        ref, ref_lse, _ = attention64(q[i], ks, vs)
        for h in range(hq):
            g = h // (hq // hk)
            o, l = _plain32(*(x.float().cpu().numpy() for x in (q[i, h], ks[:, g], vs[:, g])))
            w, w_lse = ref[h].cpu().numpy(), float(ref_lse[h])
            plain.append(o.astype(np.float64) - w)
            plain_lse.append(float(l) - w_lse)
            got_lse.append(float(lse[i, h]) - w_lse)
            err = out[i, h].double().cpu().numpy() - w
            if dtype == BF:
                err = np.sign(err) * np.maximum(np.abs(err) - HALF_STEP[BF] * np.abs(w), 0.0)
                s = torch.mv(ks[:, g].double(), q[i, h].double()) / math.sqrt(d)
                pv = torch.exp(s - ref_lse[h])[:, None] * vs[:, g].double()
                room.append(pv.square().sum(0).sqrt().cpu().numpy())
            got.append(err)
    cat = lambda x: np.concatenate(x) if x else None
    return cat(got), cat(plain), np.array(got_lse), np.array(plain_lse), cat(room)


rms = lambda x: float(np.sqrt(np.mean(np.square(x))))
CASES = [([700, 333, 90], 44), ([5000, 900, 129], 313), ([40, 60, 9] + [30] * 61, 4)]         # one launch, cut by runs, small workgroups


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,width", CASES)
def test_f32_is_as_exact_as_32_bits(d, lens, width):
    got, plain, got_lse, plain_lse, _ = _errors(F32, d, lens, width)
    assert rms(got) <= 2 * rms(plain) and np.abs(got).max() <= 3 * np.abs(plain).max(), (rms(got), rms(plain), np.abs(got).max(), np.abs(plain).max())
    assert rms(got_lse) <= 2 * rms(plain_lse) and np.abs(got_lse).max() <= 3 * np.abs(plain_lse).max(), (rms(got_lse), rms(plain_lse))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,width", CASES)
def test_bf16_rounds_its_output_alone(d, lens, width):
    """lse, which is fp32, as for f32; outputs, beyond half a step of their type: what the weights' 2^-17 adds up to (each evenly spread within that, of
    either sign: 2^-17 / sqrt 3 times the root of sum (p v)^2, six times which no one of some thousand passes), and the error of 32 bits."""
    got, plain, got_lse, plain_lse, room = _errors(BF, d, lens, width)
    assert rms(got_lse) <= 2 * rms(plain_lse) and np.abs(got_lse).max() <= 3 * np.abs(plain_lse).max(), (rms(got_lse), rms(plain_lse))
    over = np.abs(got) - 6 * 2.0 ** -17 / math.sqrt(3) * room - 3 * np.abs(plain).max()
    assert over.max() <= 0, (float(over.max()), float(np.abs(got).max()))
