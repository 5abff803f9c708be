"""Latent operators on a batch whose block table is widened, by columns that hold no pages, until the attention takes a given number of query rows at a time."""
import numpy as np

import latent_util as U

BEGINS = {16: 0, 32: 3001, 64: 6001, 128: 12001}         # groups of 16 rows x 64 tokens


class Device(U.Device):
    def __init__(self, c, at_a_time, **more):
        groups = len(c["ctx"]) * -(-int(c["n"].max()) * c["H"] // 16)
        columns = 4 * -(-BEGINS[at_a_time] // groups)
        spare = np.full((len(c["ctx"]), max(0, columns - c["table"].shape[1])), -1, dtype=np.int32)
        super().__init__(dict(c, table=np.concatenate([c["table"], spare], 1)), **more)
        assert f": {at_a_time} query rows" in self.sv.spec_describe_attn_latent_plan(self.desc)
