"""Shapes (n, M, N) that between them reach every form of orthogonalize, with remainders: the tiles of the symmetric
products and of X, and the shares that X X^T's sum is split into."""
FORMS = {(1, 7, 5): (64, 64, 1), (1, 64, 4000): (64, 64, 7), (2, 2100, 130): (64, 64, 4), (3, 250, 260): (64, 64, 1),
         (43, 512, 600): (64, 128, 1), (1, 500, 8200): (64, 128, 14), (1, 1530, 6140): (64, 256, 1), (2, 2040, 2030): (128, 128, 1),
         (1, 2040, 8180): (128, 256, 3), (1, 8180, 2040): (128, 256, 3), (1, 4090, 8100): (256, 256, 3)}
