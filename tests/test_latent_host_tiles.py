"""The cases of test_gpu_latent_row_tiles.py are what they say: entries of several row tiles, cut along the keys or whole, with the launch or uploaded."""
import os
import subprocess

from test_gpu_latent_row_tiles import CASES
from test_latent_host import CSRC, ROOT

DRIVER = r'''
#include <cstdio>
#include <vector>
#include "latent_plan.h"
using namespace mc;
using namespace mc::host;
// heads R head_dim batch, prefixes, new tokens -> entries, row tiles, most row tiles of an entry, cut row tiles
int main() {
  mc_latent_params p = {0, 0, 64, 0, 16, MC_DTYPE_BF16, 1 << 20, 0.f};
  int batch;
  while (std::scanf("%d %d %d %d", &p.num_heads, &p.latent_dim, &p.head_dim, &batch) == 4) {
    std::vector<int32_t> prefix((size_t)batch), fresh((size_t)batch);
    for (int32_t& x : prefix) if (std::scanf("%d", &x) != 1) return 1;
    for (int32_t& x : fresh) if (std::scanf("%d", &x) != 1) return 1;
    const LatentPrefillLayout l = latent_prefill_layout(&p, prefix.data(), fresh.data(), batch);
    std::vector<LatentReq> reqs((size_t)latent_entries(fresh.data(), batch));
    fill_latent_entries(&p, prefix.data(), fresh.data(), batch, reqs.data());
    int tiles = 0, most = 0;
    for (const LatentReq& r : reqs) tiles += latent_row_tiles(r.chunk), most = latent_row_tiles(r.chunk) > most ? latent_row_tiles(r.chunk) : most;
    std::printf("%zu %d %d %d\n", reqs.size(), tiles, most, l.most_tiles > 0 ? (int)l.cut_tiles : 0);
  }
}
'''


def test_entries_of_several_row_tiles(tmp_path):
    src, exe = tmp_path / "tiles.cpp", tmp_path / "tiles"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", str(exe), str(src),
                    os.path.join(CSRC, "latent_plan.cpp"), os.path.join(CSRC, "host_plan.cpp"), "-lpthread"], check=True)
    text = "\n".join(" ".join(map(str, (h, R, D, len(prefix), *prefix, *new))) for h, R, D, prefix, new, _ in CASES.values())
    res = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, timeout=60)
    lines = [[int(x) for x in line.split()] for line in res.stdout.splitlines()]
    assert len(lines) == len(CASES)
    for (name, (*_, new, cut)), (entries, tiles, most, cut_tiles) in zip(CASES.items(), lines):
        assert entries == len(new) and entries != tiles and most >= 2, (name, entries, tiles, most)
        assert (cut_tiles >= 2) == cut and (cut or cut_tiles == 0), (name, cut_tiles)
        assert (entries > 64) == name.startswith("uploaded"), name
