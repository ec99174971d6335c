"""The host rules of the layer's operators on the CPU, compiled from the headers
that the kernels are built from."""
import paper_2601_18999_amd as K
from test_layer_abi_cpu import product
from test_serve_rules_cpu import compiled

HEAD = """
#include <cstdio>
#include "kvr_layer.h"
"""


def tiles(tmp_path, sizes):
    """(channels, tokens, groups, threads, workgroups) of the tiles for each (tokens, channels)."""
    out = compiled(tmp_path, HEAD + """
int main() {
  const long long sizes[][2] = {%s};
  for (const auto& s : sizes) {
    const kvr::ProductTile t = kvr::product_tile(s[0], s[1]);
    std::printf("%%d %%d %%d %%d %%lld\\n", t.channels, t.tokens, t.groups, t.threads,
                (long long)kvr::product_tiles(s[0], s[1], t.tokens, t.channels));
  }
}
""" % ", ".join("{%dll, %dll}" % s for s in sizes), "-x", "hip", "--offload-arch=gfx950")
    v = list(map(int, out))
    return [tuple(v[i:i + 5]) for i in range(0, len(v), 5)]


def accepted(tokens, channels):
    try:
        K.kvr_product_workspace(product(num_tokens=tokens, channels=channels, dim=16, x_token=16, w_channel=16))
    except K.KvrError:
        return False
    return True


def test_a_product_that_is_accepted_fits_a_launch(tmp_path):
    # around every power of two, the last accepted number of tokens for few channels, and of channels for few tokens
    around = sorted({n + d for p in range(32) for n in (1 << p,) for d in (-256, -65, -1, 0, 1, 63, 64, 65, 128, 200)
                     if 1 <= n + d < 1 << 31} | {(1 << 30) - 129, (1 << 30) - 128})
    sizes = [(t, c) for t in around for c in around if c <= 1 << 24 and accepted(t, c)]
    assert (1 << 29, 64) in sizes and ((1 << 30) - 129, 1) in sizes and (65, 1 << 24) in sizes
    got = tiles(tmp_path, sizes)
    over = [(s, t) for s, t in zip(sizes, got) if t[3] * t[4] >= 1 << 32]
    assert not over, over[:4]
    # (64-wide tiles are left only where they would not fit)
    assert dict(zip(sizes, got))[((1 << 29) - 65, 64)][:2] == (64, 64)


def test_the_tiles_that_were_measured_are_taken(tmp_path):
    sizes = {(128, 8192): (64, 64, 2), (200, 1024): (64, 64, 2), (512, 4096): (128, 64, 2), (256, 16384): (128, 128, 2),
             (1024, 8192): (128, 128, 1), (2048, 8192): (256, 256, 1), (9216, 16384): (256, 256, 1)}
    got = tiles(tmp_path, list(sizes))
    assert [t[:3] for t in got] == list(sizes.values())
