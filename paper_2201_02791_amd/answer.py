"""Answers of a trained model: (s, r, ?) and (?, r, t) from an embedding table of 4 bits.

Holds the table and the relations' diagonals on the device and issues the library calls of a batch of questions on one stream:
rows of the asked entities -> scores against every entity -> draws.  No arithmetic of the method happens in Python or torch.
"""
from __future__ import annotations

from . import binding as kb


class Answers:
    """H: embeddings [n_entities][d] (float32 or bfloat16) as the encoder leaves them, M: [n_relations][d] float32, device tensors.  The table
    is made of H; H itself is not kept unless full_rows, where questions take the asked entity's embedding from H instead of the
    table."""

    def __init__(self, H, M, full_rows: bool = False, stream=None):
        self.table = kb.table4_encode(H, stream=stream)
        self.M = M
        self.H = H if full_rows else None

    def scores(self, entity, rel, out=None, stream=None):
        """float32 [questions][n_entities]: DistMult is symmetric in its entities, so entity (int32, device) may be head or tail."""
        if self.H is not None:
            return kb.table4_scores(self.table, self.H, fixed=entity, M=self.M, rel=rel, out=out, stream=stream)
        X = kb.table4_decode(self.table, rows=entity, stream=stream)
        return kb.table4_scores(self.table, X, M=self.M, rel=rel, out=out, stream=stream)

    def ask(self, entity, rel, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, known=None, stream=None):
        """(answers int32 [questions][draws], their shares): drawn from each question's scores by the random numbers u
        ([questions][draws] in [0, 1)); temperature 0 gives the best answer.  known: (questions, entities), two int64 tensors of
        pairs that are no answers, such as the known triples and the asked entity itself.  -1: no entity is left."""
        import torch
        if stream is not None and not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(stream, self.M.device) if stream else torch.cuda.default_stream(self.M.device)
        with torch.cuda.stream(stream):
            S = self.scores(entity, rel, stream=stream)
            if known is not None:
                S[known[0], known[1]] = float("-inf")
            return kb.sample_scores(S, u, temperature, top_k, top_p, min_p, want_prob=True, stream=stream)
